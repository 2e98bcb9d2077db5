"""Combinations of rows that are wider than a launch takes at most of shorter ones."""
import subprocess
import sys

import pytest
import torch

import paper_2509_24416_amd as clq


def test_the_launches_of_very_wide_rows_end():
    """In a process without a GPU every launch is an error: what is left is the host's loop."""
    if torch.cuda.is_available():
        pytest.skip("addresses that are not real")
    code = f"""
import ctypes
L, p, i = ctypes.CDLL({clq.LIB_PATH!r}), ctypes.c_void_p, ctypes.c_int64
f = L.clq_expert_combine
f.argtypes = [p, ctypes.c_int32, i, p, p, i, i, i, i, p, ctypes.c_int32, i, p]
for N in (2 ** 30 + 1, 2 ** 31 - 1):
    ld = (N + 7) // 8 * 8
    print(f(0x10000, 0, ld, 0x10000, 0x10000, 2, 1, 4, N, 0x10000, 0, ld, None))
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=60)
    assert r.stdout.split() == [str(clq.CLQ_ERR_HIP)] * 2, r.stderr[-2000:]


@pytest.mark.gpu
def test_very_wide_rows():
    T, N = 3, 2 ** 30 + 1
    ld = (N + 7) // 8 * 8
    y = torch.empty(1, ld, dtype=torch.float16, device="cuda")
    for part in y[0].split(1 << 26):
        part.copy_(torch.arange(len(part), device="cuda") % 1021)
    y[0, N - 1] = 7
    rows, w = torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.tensor([[1.0], [2.0], [-1.0]], device="cuda")
    rows[1] = -1
    out = torch.full((T, ld), 5.0, dtype=torch.float16, device="cuda")
    s = clq.lib().clq_expert_combine(y.data_ptr(), 0, ld, rows.data_ptr(), w.data_ptr(), T, 1, 1, N, out.data_ptr(), 0, ld,
                                     torch.cuda.current_stream().cuda_stream)
    assert s == clq.CLQ_OK
    assert torch.equal(out[0, :N], y[0, :N]) and (out[1, :N] == 0).all()
    assert torch.equal(out[2, :N], 0 - y[0, :N])
    assert (out[:, N:] == 5).all()


def test_a_plan_holds_the_tables_that_products_read():
    """Counts, and the tiles before each expert for tiles of 32, 128 and 256 rows."""
    for E in (1, 64, 512):
        assert clq.clq_expert_plan_ints(E) == E + 3 * (E + 1)
