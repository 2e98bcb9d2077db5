"""Heads given for the results of rotary positions: refused where they meet the input's, and only there."""
import itertools

import pytest
import torch

from paper_2509_24416_amd.block import _heads_meet


def places(at, M, ld, H, lh, D):
    return {at + i * ld + j * lh + k for i in range(M) for j in range(H) for k in range(D)}


@pytest.mark.parametrize("M,ld,H,lh,D", [(3, 96, 2, 24, 8), (4, 72, 3, 24, 8), (3, 16, 2, 64, 8), (5, 8, 2, 40, 8), (1, 64, 4, 16, 16),
                                         (4, 40, 1, 8, 8), (2, 50, 3, 16, 8)])
def test_heads_of_one_spacing(M, ld, H, lh, D):
    """Against the places themselves, at every distance up to past both ends."""
    first = places(0, M, ld, H, lh, D)
    end = (M - 1) * ld + (H - 1) * lh + D
    for at in range(-end - 3, end + 4):
        assert _heads_meet(at, M, ld, H, lh, D) == bool(first & places(at, M, ld, H, lh, D)), at


@pytest.mark.gpu
def test_heads_beside_each_other():
    """Queries, keys and values of a head side by side: one third turned into another, in itself, and into a third that it
    meets."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2509_24416_amd as clq
    M, H, D = 33, 4, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    pos, freqs = torch.arange(M, dtype=torch.int32, device="cuda").unsqueeze(1), clq.clq_rope_freqs((D,))
    for order in itertools.permutations(range(3), 2):
        for dims in ((M, H, 3, D), (H, M, 3, D)):
            wide = torch.randn(*dims, device="cuda", generator=g).half()
            x, y, rest = (wide[..., i, :] for i in (*order, 3 - sum(order)))
            x, y, rest = (t if dims[0] == M else t.transpose(0, 1) for t in (x, y, rest))
            want, kept = clq.clq_rope_axes(x, pos, freqs, (D,)), (x.clone(), rest.clone())
            assert clq.clq_rope_axes(x, pos, freqs, (D,), out=y) is y
            assert torch.equal(y, want) and torch.equal(x, kept[0]) and torch.equal(rest, kept[1])
            assert torch.equal(clq.clq_rope_axes(x, pos, freqs, (D,), out=x), want)
    flat = torch.zeros(M * H * 3 * D + 8, dtype=torch.float16, device="cuda")
    for shift, bad in ((8, True), (D - 8, True), (D, False), (2 * D, False), (2 * D + 8, True), (3 * D, True)):
        x = flat.as_strided((M, H - 1, D), (3 * H * D, 3 * D, 1))
        y = flat.as_strided((M, H - 1, D), (3 * H * D, 3 * D, 1), shift)
        if bad:
            with pytest.raises(ValueError, match="overlaps"):
                clq.clq_rope_axes(x, pos, freqs, (D,), out=y)
        else:
            clq.clq_rope_axes(x, pos, freqs, (D,), out=y)
    still = flat[:D].expand(M, H, D)   # (no places of their own: refused as before)
    for x, y in ((still, still), (still, flat[8:D + 8].expand(M, H, D))):
        with pytest.raises((ValueError, clq.ClqError)):
            clq.clq_rope_axes(x, pos, freqs, (D,), out=y)
