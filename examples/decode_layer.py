"""A decode step of one decoder layer on 4-bit weights in which every row picks weights of its own.

    python examples/decode_layer.py [--batch 32] [--hidden 4096] [--inter 11008] [--experts 8] [--top-k 2]
                                    [--adapters 16] [--rank 16] [--steps 50]

Each row is a request with a low-rank adapter of its own (or none) on the attention projections, and each token is sent
to ``top_k`` of the layer's experts.  The step is

    qkv  = gptq_w4a16_gemm_lora(norm(x))          shared 4-bit projection + the rows' adapters
    x   += gptq_w4a16_gemm_lora(attention)        the same for the output projection
    x   += gptq_w4a16_moe(norm(x), router)        routing and the experts' 4-bit products

with random weights.  Attention itself is the serving program's; here a request has one token, whose attention output
is its value.  The step is run once eagerly, which is when the library allocates its scratch, then captured into a HIP
graph and replayed, as a serving loop does.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2511_19438_amd import serving  # noqa: E402

GROUP = 128


def packed(gen, K, N, *lead):
    """Random packed weights in the format of the library: codes, zero points, scales."""
    words = lambda *s: torch.randint(-2 ** 31, 2 ** 31, s, dtype=torch.int32, device="cuda", generator=gen)  # noqa: E731
    scales = torch.empty(*lead, K // GROUP, N, device="cuda").uniform_(0.0005, 0.001, generator=gen)
    return words(*lead, K // 8, N), words(*lead, K // GROUP, N // 8), scales.half()


def adapters(gen, count, rank, K, N):
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    return (normal(count, rank, K) / K ** 0.5).half(), (0.02 * normal(count, N, rank)).half(), torch.ones(count, device="cuda")


def norm(x):
    return (x * torch.rsqrt(x.float().square().mean(1, keepdim=True) + 1e-5)).half()


class Layer:
    def __init__(self, batch, hidden, inter, experts, top_k, count, rank, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.top_k, self.hidden = top_k, hidden
        self.qkv, self.o = packed(gen, hidden, 3 * hidden), packed(gen, hidden, hidden)
        self.qkv_adapters = adapters(gen, count, rank, hidden, 3 * hidden)
        self.o_adapters = adapters(gen, count, rank, hidden, hidden)
        self.router = torch.randn(hidden, experts, device="cuda", generator=gen).half()
        self.gate_up = packed(gen, hidden, 2 * inter, experts)
        self.down = packed(gen, inter, hidden, experts)
        half = dict(dtype=torch.float16, device="cuda")
        self.qkv_out, self.o_out = torch.empty(batch, 3 * hidden, **half), torch.empty(batch, hidden, **half)
        self.moe_out = torch.empty(batch, hidden, **half)

    def step(self, x, adapter):
        """x [batch, hidden] fp16, adapter [batch] int32 (-1: none) -> x after the layer."""
        serving.gptq_w4a16_gemm_lora(norm(x), *self.qkv, *self.qkv_adapters, adapter, self.qkv_out, GROUP)
        attention = self.qkv_out[:, 2 * self.hidden:].contiguous()  # one token: its value
        serving.gptq_w4a16_gemm_lora(attention, *self.o, *self.o_adapters, adapter, self.o_out, GROUP)
        x = x + self.o_out
        h = norm(x)
        serving.gptq_w4a16_moe(h, h @ self.router, self.gate_up, self.down, self.moe_out, self.top_k, GROUP)
        return x + self.moe_out


def run(batch=32, hidden=4096, inter=11008, experts=8, top_k=2, count=16, rank=16, steps=50):
    layer = Layer(batch, hidden, inter, experts, top_k, count, rank)
    x = torch.randn(batch, hidden, device="cuda").half()
    adapter = torch.randint(-1, count, (batch,), dtype=torch.int32, device="cuda")
    eager = layer.step(x, adapter).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.step(x, adapter)
    graph.replay()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    return eager, out, begin.elapsed_time(end) * 1000 / steps


def main():
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in [("batch", 32), ("hidden", 4096), ("inter", 11008), ("experts", 8), ("top-k", 2), ("adapters", 16),
                        ("rank", 16), ("steps", 50)]:
        parser.add_argument("--" + name, type=int, default=value)
    a = parser.parse_args()
    eager, out, us = run(a.batch, a.hidden, a.inter, a.experts, a.top_k, a.adapters, a.rank, a.steps)
    same = torch.equal(eager, out)
    print(f"{a.batch} rows, {us:.1f} us a step, graph and eager step {'agree' if same else 'DIFFER'}, "
          f"mean square {out.float().square().mean():.3f}")
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
