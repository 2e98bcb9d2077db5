"""An expert MLP on the MX4 products, optionally replayed as one HIP graph.

A transformer block's MLP with `experts` experts of which each token takes top_k:

    ids, weights = route(x . W_router^T)
    y = sum over the token's experts of weight * (act(x . W1^T + b1) . W2^T + b2)

All products but the router's (a T x experts one, left in fp32) run on MX4 codes with the
paper's block-Hadamard rotation (CLQ, arXiv 2509.24416, Sec. 3.3) in front of both layers'
quantizers; the activation, the second rotation and quantizer are part of the first product's
launch.  Tokens are sorted by expert on the GPU, so nothing waits for the host, and a captured
graph replays with other tokens, experts and tile counts.
"""
import torch

from . import (clq_expert_combine, clq_expert_plan, clq_expert_route, clq_mx4_dispatch, clq_mx4_experts,
               clq_mx4_experts_mx4, clq_mx4_quantize_weights)


class ExpertMLP:
    """router: [experts, hidden]; w1: [experts, mlp, hidden] (swiglu: 2 * mlp rows, the gates
    first), b1: [experts, rows of w1]; w2: [experts, hidden, mlp], b2: [experts, hidden]; fp16 or
    bf16 device tensors, biases of the inputs' type or None.  block: Hadamard block size of both
    layers (swiglu: 64 at most).  results: type of the experts' results ahead of their sum (fp32:
    the layer rounds once; fp16 and bf16 are quicker on many tokens).  route: further arguments of
    clq_expert_route."""

    def __init__(self, router, w1, b1, w2, b2, top_k, act="gelu", block=64, results=torch.float32, **route):
        self.router = router.float()
        self.experts, self.top_k, self.act, self.block, self.route = router.shape[0], top_k, act, block, route
        # weights are rotated and quantized once
        self.w1 = clq_mx4_quantize_weights(w1, block, gated=act == "swiglu")
        self.w2 = clq_mx4_quantize_weights(w2, block)
        self.b1, self.b2, self.results = b1, b2, results
        self.graph = None

    def forward(self, x):
        """x: fp16 or bf16 [tokens, hidden] -> the same shape and type.  No tokens (a process that was
        sent none) give none."""
        if x.shape[0] == 0 and x.dtype in (torch.float16, torch.bfloat16) and x.shape[1:] == self.router.shape[1:]:
            return torch.empty_like(x)   # (the operators take one token or more)
        ids, weights = clq_expert_route(x.float() @ self.router.t(), self.top_k, **self.route)
        plan = clq_expert_plan(ids, self.experts)
        q = clq_mx4_dispatch(x, plan, self.block)
        h = clq_mx4_experts_mx4(q, plan, self.w1, self.b1, act=self.act, block=self.block)
        y = clq_mx4_experts(h, plan, self.w2, self.b2, dtype=self.results)
        return clq_expert_combine(y, plan, weights, dtype=x.dtype)

    def capture(self, tokens, dtype=torch.float16):
        """Captures forward for `tokens` tokens as one graph."""
        dev = self.router.device
        x = torch.zeros(tokens, self.router.shape[1], dtype=dtype, device=dev)
        self.forward(x)   # every kernel loaded first
        torch.cuda.synchronize(dev)
        graph = torch.cuda.CUDAGraph()
        # (on a stream of this device: by itself it takes one of the device that is current, or was when
        # it was first used)
        with torch.cuda.device(dev), torch.cuda.graph(graph, stream=torch.cuda.Stream(dev)):
            y = self.forward(x)
        # (together, and only now: a capture that fails leaves the one before as it was)
        self.x_in, self.x_out, self.graph = x, y, graph
        return graph

    def replay(self, x):
        """x: as many tokens as were captured, of the same type.  The result is overwritten by the
        next replay."""
        if x.shape != self.x_in.shape or x.dtype != self.x_in.dtype:
            raise ValueError(f"x is {x.dtype} {tuple(x.shape)}, captured was {self.x_in.dtype} {tuple(self.x_in.shape)}")
        self.x_in.copy_(x)
        self.graph.replay()
        return self.x_out
