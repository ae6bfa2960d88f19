"""An attention block of a Llama3-8B-shaped layer: nested weights, a paged 8-bit cache, prompts and decoding.

Prompts of unequal length go through the block at once (`grinqh_prefill`), decode steps one token per sequence
(`grinqh_vmm_threshold`).  Both write their keys and values into the same cache (`grinqh_kv_write`) and attend over it
(`grinqh_attend`).  The decode step is captured once as a HIP graph, which advances the sequences itself.  Rotary
embedding and the MLP are left out.

    python examples/attention_block.py [--window 256 --sinks 4]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_23419_amd import grinqh as g  # noqa: E402
from synth import inputs  # noqa: E402

HIDDEN, HEADS, KV_HEADS, HEAD_DIM, PAGE = 4096, 32, 8, 128, 64
LEVELS, BUDGET = inputs.LEVELS_B, 4


class Linear:
    """Packed nested weights with the thresholds that meet the budget on calibration activations."""

    def __init__(self, K, N, calibration, gen):
        W = (torch.randn(N, K, device="cuda", generator=gen) * K ** -0.5).half()
        self.desc = g.grinqh_resolve_desc(g.make_desc(K, N, LEVELS))
        self.codes, self.scales = g.grinqh_pack(self.desc, W=W)
        self.theta = g.grinqh_calibrate(self.desc, calibration, inputs.BUDGETS[LEVELS][BUDGET]).cpu().tolist()

    def __call__(self, x, prompt):
        if prompt:
            return g.grinqh_prefill(self.desc, self.codes, self.scales, x)
        return g.grinqh_vmm_threshold(self.desc, self.codes, self.scales, x, self.theta)


def normed(x):
    return (x / x.float().pow(2).mean(-1, keepdim=True).sqrt()).half()


class Block:
    def __init__(self, sequences, max_len, window=0, sinks=0, seed=0):
        gen = torch.Generator("cuda").manual_seed(seed)
        sample = torch.randn(64, HIDDEN, device="cuda", generator=gen).half()
        self.qkv = Linear(HIDDEN, (HEADS + 2 * KV_HEADS) * HEAD_DIM, sample, gen)
        self.o = Linear(HEADS * HEAD_DIM, HIDDEN, sample, gen)
        self.window, self.sinks, self.max_len = window, sinks, max_len
        # pages in any order: a serving loop hands them out as sequences grow
        width = (max_len + PAGE - 1) // PAGE
        self.kv = g.make_kv_desc(g.GRINQH_KV_I8, KV_HEADS, HEAD_DIM, PAGE, sequences * width)
        self.cache = g.kv_cache(self.kv)
        self.table = torch.randperm(sequences * width, device="cuda", generator=gen).int().view(sequences, width)
        self.lens = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.each = g.KvBatch(self.table, self.lens, torch.arange(sequences + 1, dtype=torch.int32, device="cuda"))
        n = g.grinqh_attend_workspace_bytes(self.kv, HEADS, sequences, sequences, 1, max_len, window, sinks)
        self.workspace = torch.empty(n, dtype=torch.uint8, device="cuda")

    def forward(self, x, batch, prompt, max_rows):
        """x [rows, HIDDEN] fp16 -> (y, qkv, attention's rows)"""
        qkv = self.qkv(normed(x), prompt).view(-1, HEADS + 2 * KV_HEADS, HEAD_DIM)
        g.grinqh_kv_write(self.kv, self.cache, batch, qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:])
        a = g.grinqh_attend(self.kv, self.cache, batch, qkv[:, :HEADS].half(), window=self.window, sinks=self.sinks,
                            max_rows=max_rows, max_len=self.max_len, workspace=None if prompt else self.workspace)
        y = x + self.o(a.view(-1, HEADS * HEAD_DIM), prompt).half()
        return y, qkv, a

    def prompts(self, x, lengths):
        """The sequences' prompts, one after the other in x."""
        self.lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        offsets = torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).int().cuda()
        return self.forward(x, g.KvBatch(self.table, self.lens, offsets), True, max(lengths))

    def step(self, x):
        """One token of every sequence; runs inside a graph."""
        self.lens += 1
        return self.forward(x, self.each, False, 1)


def plain(q, k, v, window, sinks):
    """Attention of the last rows q over k and v in float32."""
    n, L = q.shape[0], k.shape[0]
    q, k, v = q.half().float(), k.repeat_interleave(HEADS // KV_HEADS, 1), v.repeat_interleave(HEADS // KV_HEADS, 1)
    s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0).contiguous()) * HEAD_DIM ** -0.5
    at, t = torch.arange(L - n, L, device=q.device)[:, None], torch.arange(L, device=q.device)[None]
    sees = t <= at
    if window:
        sees &= (t > at - window) | (t < sinks)
    return torch.matmul(s.masked_fill(~sees, float("-inf")).softmax(-1), v.transpose(0, 1).contiguous()).transpose(0, 1)


def run(lengths=(300, 77, 1), steps=16, window=0, sinks=0):
    """Largest relative error (2-norm) of attention against float32 over unquantised keys and values, µs per step."""
    lengths = list(lengths)
    block = Block(len(lengths), max(lengths) + steps + 3, window, sinks)
    x = torch.randn(sum(lengths), HIDDEN, device="cuda").half()
    worst, kept = 0.0, [[] for _ in lengths]

    def check(s, qkv, a):
        nonlocal worst
        kept[s].append(qkv[:, HEADS:].clone())
        kv = torch.cat(kept[s])
        ref = plain(qkv[:, :HEADS], kv[:, :KV_HEADS], kv[:, KV_HEADS:], window, sinks)
        error = ((a.float() - ref).norm() / ref.norm()).item()
        if not math.isfinite(error):     # max() would pass over a NaN
            raise FloatingPointError(f"attention of sequence {s}, {kv.shape[0]} tokens, is not finite")
        worst = max(worst, error)

    y, qkv, a = block.prompts(x, lengths)
    for s, (rows, att) in enumerate(zip(qkv.split(lengths), a.split(lengths))):
        check(s, rows, att)

    x = torch.cat([rows[-1:] for rows in y.split(lengths)])
    ends = block.lens.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):       # once before the capture
        block.step(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, qkv, a = block.step(x)
    block.lens.copy_(ends)              # the rows written so far past the ends are written again
    for _ in range(steps):
        graph.replay()
        for s in range(len(lengths)):
            check(s, qkv[s:s + 1], a[s:s + 1])
        x.copy_(y)

    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    block.lens.copy_(ends)
    start.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    end.synchronize()
    return worst, start.elapsed_time(end) / steps * 1e3


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--lengths", type=int, nargs="+", default=[300, 77, 1], help="the prompts' lengths, up to 4 sequences")
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    args = ap.parse_args()
    error, us = run(args.lengths, args.steps, args.window, args.sinks)
    print(f"{len(args.lengths)} sequences, {args.steps} decode steps: attention within {error:.1e} of float32 over unquantised "
          f"keys and values, {us:.0f} us per decode step of the block")
