"""A decoder layer's attention sublayer with PIFA projections, served: prompts, then decode steps.

    python examples/attention_block.py [--width 4096] [--heads 32] [--requests 8] [--prompt 700] [--steps 32] [--cache-bits 16]

q, k and v are one grouped call (three layers of one shape that share their input), the output projection another;
between them the step's page tables, the rotation with the cache write, and the attention over the pages. The
prompts run as one ragged step; the decode step is captured once into a CUDA graph that updates lengths and
the free list's head in place, and replayed. Layers are random (drawn like compressed ones); the last
step's output is checked against the same sublayer computed densely in float64. With --cache-bits 8 keys and values are
held as e4m3 numbers with a scale for each block of 16 tokens and head.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2501_19090_gb300 import pifa as P  # noqa: E402

DEV = "cuda"
BF16 = torch.bfloat16


def random_layers(gen, groups, width, rank):
    """`groups` PIFA layers (width x width, rank `rank`) stacked as pifa_forward_grouped takes them."""
    piv, nonp = [], []
    for g in range(groups):
        order = torch.randperm(width, device=DEV, generator=gen)
        piv.append(order[:rank].sort().values + g * width)
        nonp.append(order[rank:].sort().values + g * width)
    Wp = (torch.randn((groups * rank, width), device=DEV, generator=gen) * width ** -0.5).to(BF16)
    C = (torch.randn((groups * (width - rank), rank), device=DEV, generator=gen) * 0.7 * rank ** -0.5).to(BF16)
    return {"groups": groups, "Wp": Wp, "C": C, "piv": torch.cat(piv).int(), "nonp": torch.cat(nonp).int()}


def project(layers, X, Y=None):
    if layers["groups"] > 1:
        return P.pifa_forward_grouped(layers["groups"], X, layers["Wp"], layers["C"], layers["piv"], layers["nonp"], Y=Y)
    return P.pifa_forward(X, layers["Wp"], layers["C"], layers["piv"], layers["nonp"], Y=Y)


class Block:
    """The sublayer's weights and cache, and the state of the requests that it serves."""

    def __init__(self, width, heads, requests, longest, page=16, rank=None, seed=0, cache_bits=16):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        rank = width // 2 if rank is None else rank
        self.heads, self.dim, self.page = heads, width // heads, page
        self.qkv, self.out = random_layers(gen, 3, width, rank), random_layers(gen, 1, width, rank)
        cols = -(-longest // page)
        pages = requests * cols
        held = torch.float8_e4m3fn if cache_bits == 8 else BF16
        self.cache = [torch.empty((pages, page, heads, self.dim), dtype=held, device=DEV) for _ in range(2)]
        if cache_bits == 8:  # keys, values, and the scales of each
            self.cache += [torch.empty((pages, page // P.PIFA_Q8_BLOCK, heads), dtype=torch.float8_e8m0fnu, device=DEV) for _ in range(2)]
        self.write = P.pifa_rope_cache_q8 if cache_bits == 8 else P.pifa_rope_cache
        self.attend = P.pifa_paged_attention_q8 if cache_bits == 8 else P.pifa_paged_attention
        self.free_pages = torch.randperm(pages, device=DEV, generator=gen).int()
        self.free_first = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.table = torch.full((requests, cols), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(requests, dtype=torch.int32, device=DEV)
        self.freq = P.pifa_rope_frequencies(self.dim, device=DEV)

    def step_buffers(self, tokens):
        i32 = dict(dtype=torch.int32, device=DEV)
        return {"tables": (torch.empty(self.lens.numel() + 1, **i32), self.lens, torch.empty(tokens, **i32),
                           torch.empty(tokens, dtype=torch.int64, device=DEV), self.free_first),
                "q": torch.empty((tokens, self.heads, self.dim), dtype=BF16, device=DEV),
                "o": torch.zeros((tokens, self.heads, self.dim), dtype=BF16, device=DEV)}

    def step(self, X, new_len, max_q, buf):
        """One step of every request: X holds the new tokens' inputs, request after request."""
        T = X.shape[0]
        q_start, kv_len, positions, slots, _ = P.pifa_page_tables(self.lens, new_len, self.page, self.free_pages, self.free_first,
                                                                  self.table, T, out=buf["tables"])
        q, k, v = project(self.qkv, X).view(T, 3, self.heads, self.dim).unbind(1)
        self.write(q, k, v, positions, slots, self.freq, *self.cache, Qr=buf["q"])
        self.attend(buf["q"], *self.cache, self.table, q_start, kv_len, max_q, O=buf["o"])
        return project(self.out, buf["o"].view(T, -1))


def dense(layers, X):
    """The layers' output in float64, from the same weights."""
    G = layers["groups"]
    r, w = layers["Wp"].shape[0] // G, X.shape[1]
    Y = torch.empty((X.shape[0], G * w), dtype=torch.float64, device=DEV)
    for g in range(G):
        Yp = X.double() @ layers["Wp"][g * r:(g + 1) * r].double().t()
        n = layers["C"].shape[0] // G
        Y[:, layers["piv"][g * r:(g + 1) * r].long()] = Yp
        Y[:, layers["nonp"][g * n:(g + 1) * n].long()] = Yp @ layers["C"][g * n:(g + 1) * n].double().t()
    return Y


def dense_last(block, X):
    """The last token's output of one request whose inputs are X, in float64."""
    T, H, d = X.shape[0], block.heads, block.dim
    q, k, v = dense(block.qkv, X).view(T, 3, H, d).unbind(1)
    a = 2.0 * torch.pi * torch.arange(T, device=DEV, dtype=torch.float64)[:, None] * block.freq.double()[None] / 2.0 ** 64
    c, s = a.cos()[:, None], a.sin()[:, None]
    turn = lambda x: torch.cat([x[..., :d // 2] * c - x[..., d // 2:] * s, x[..., d // 2:] * c + x[..., :d // 2] * s], -1)
    q, k = turn(q)[-1:], turn(k)
    p = torch.softmax(torch.einsum("qhd,khd->hqk", q, k) * d ** -0.5, -1)
    return dense(block.out, torch.einsum("hqk,khd->qhd", p, v).reshape(1, H * d))[0]


def serve(width=4096, heads=32, requests=8, prompt=700, steps=32, seed=0, cache_bits=16):
    """Runs the loop; returns (largest error of the last step over the outputs' rms, prompt us, decode us a step)."""
    block = Block(width, heads, requests, prompt + steps + 1, seed=seed, cache_bits=cache_bits)
    gen = torch.Generator(device=DEV).manual_seed(seed + 1)
    lens = [max(1, prompt * (b + 1) // requests) for b in range(requests)]
    X = torch.randn((sum(lens), width), device=DEV, generator=gen).to(BF16)
    seen = list(X.split(lens))  # every request's inputs, for the check
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)

    begin.record()
    block.step(X, torch.tensor(lens, dtype=torch.int32, device=DEV), max(lens), block.step_buffers(sum(lens)))
    end.record()
    torch.cuda.synchronize()
    prompt_us = begin.elapsed_time(end) * 1e3

    # Decode: one token each. The first step runs eagerly (workspaces), the rest as replays of one graph.
    ones, buf = torch.ones(requests, dtype=torch.int32, device=DEV), block.step_buffers(requests)
    x, stream = torch.empty((requests, width), dtype=BF16, device=DEV), torch.cuda.Stream()

    def feed():
        x.copy_(torch.randn((requests, width), device=DEV, generator=gen))
        for b in range(requests):
            seen[b] = torch.cat([seen[b], x[b:b + 1]])

    feed()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        Y = block.step(x, ones, 1, buf)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            Y = block.step(x, ones, 1, buf)
    decode_us = 0.0
    for _ in range(steps):
        feed()
        begin.record()
        graph.replay()
        end.record()
        torch.cuda.synchronize()
        decode_us += begin.elapsed_time(end) * 1e3 / steps
    status = P.pifa_device_status()
    if status != P.PIFA_OK:
        raise RuntimeError(f"device status {P.pifa_status_string(status)}")
    assert block.lens.tolist() == [n + 1 + steps for n in lens]
    want = torch.stack([dense_last(block, s) for s in seen])
    error = float((Y.double() - want).abs().max() / want.square().mean().sqrt())
    return error, prompt_us, decode_us


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("width", 4096), ("heads", 32), ("requests", 8), ("prompt", 700), ("steps", 32)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache-bits", type=int, default=16, choices=(8, 16))
    a = vars(ap.parse_args())
    error, prompt_us, decode_us = serve(**a)
    print(f"{a['requests']} requests, width {a['width']}, {a['heads']} heads, cache in {a['cache_bits']} bits: prompts {prompt_us:.0f} us, decode step "
          f"{decode_us:.1f} us, largest error of the last step {error:.3g} of the outputs' rms")
