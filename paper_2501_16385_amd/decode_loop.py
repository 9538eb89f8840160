"""Token-by-token decode over a stack of decoder layers whose seven linear layers (q, k, v, o, gate, up,
down) are fused sub-branched quantized linears, replayed from one HIP graph per token.

    python -m paper_2501_16385_amd.decode_loop --layers 32 --hidden 4096 --inter 11008 --r 128 --bits 4

The paper reports whole-model decode speed for this configuration (Sec. 5.3: batch 1, rank 128);
--batch B decodes B independent sequences per step (B rows through every linear: from three rows on
the matrix-core kernel streams the weights once for all of them).  Only
the linear layers are the paper's method, so only they are real here; the glue between them is the
least that keeps the data flow of a decoder layer and the values bounded:

    q, k, v = x Wq, x Wk, x Wv        one grouped launch (they share x)
    a       = v                        attention over a single position returns v; q and k are computed and dropped
    h       = (x + a Wo) / 2           residual, halved instead of normalised (no reduction kernels in the graph)
    g, u    = h Wg, h Wu               one grouped launch
    x'      = (h + (silu(g) * u) Wd) / 2

With a cache (DecoderStack(cache=..)) attention is real: k and v go into the cache's pages and a = softmax(q k^T / sqrt(d)) v over what the sequences hold, in
the same graph (see batch_decode.py for a batch of samples of one prompt).

Five launches per layer: four fused ones, two of which write the averages as well, and silu(g) * u.  Weights are random packed words (speed
does not depend on the values) unless a list of quantized layers is passed in.  Prints one JSON line.
"""
from __future__ import annotations

import argparse
import ctypes
import json
import os
import sys
from dataclasses import dataclass

import torch

from . import cache as kv
from . import fbq
from .random_layers import random_layer

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import fbq_synth  # noqa: E402  (byte accounting)

NAMES = ("q", "k", "v", "o", "gate", "up", "down")


def layer_shapes(hidden: int, inter: int, kv_hidden: int = 0):
    """(N, K) of the seven linears of one decoder layer; kv_hidden: rows of k and v where heads share them (0: hidden)."""
    kv_rows = kv_hidden or hidden
    return {"q": (hidden, hidden), "k": (kv_rows, hidden), "v": (kv_rows, hidden), "o": (hidden, hidden),
            "gate": (inter, hidden), "up": (inter, hidden), "down": (hidden, inter)}


@dataclass(frozen=True)
class Budget:
    """What the rows of a cache may hold: at most `keep` tokens, the first `first` and the last `recent` ones among them, and those of the others that were attended to most; what a token
    was given counts `decay` times as much a step later."""
    keep: int
    first: int = 0
    recent: int = 1
    decay: float = 1.0

    def __post_init__(self):
        if self.first < 0 or self.recent < 0 or self.first + self.recent > self.keep or not 0 <= self.decay <= 1:
            raise ValueError("budget: first and recent tokens, 0 or more, within the ones to keep; decay 0 .. 1")      # (else no row would ever be cut back)


class DecoderStack:
    """layers: list (one per decoder layer) of dicts name -> fbq.DeviceLayer.

    cache: a kv.Cache with a layer for each of them; `batch` is then the number of tokens of a step, and a step appends them to the cache's rows and attends over what
    these hold.  counts [rows]: tokens of each row in a step (None: one); shared: the pages that all rows begin with (a view of a row of the table stays
    right when pages move).  A row that no pages are left for, in the pool or in its row of the table, is not written in that step, and what the step makes of it means
    nothing.  `lacking` [1]: the pages that the last step lacked, `most_lacking` [1] that any has; `lowest_start` [rows]: -1 where a step has left a row out.

    The cache may be one of 4 bits.  budget: a Budget; then every step adds up the attention weights in `weights` [layers, rows, kv_heads, tokens] and ends with the rows cut back
    (a row that begins with another's tokens, as a forked one does, wants that one's weights copied there; the weights of a row that a step leaves out, or has a `count` of 0 for, stay as they are); `evicted` [2]: rows cut back by the last step, and rows that could not be;
    `most_skipped` [1]: the most of these that any step has had.
    """

    def __init__(self, layers, hidden: int, inter: int, keep_per_layer_buffers: bool = False, batch: int = 1,
                 share_workspaces: bool = False, cache=None, counts=None, shared=None, budget=None):
        self.layers, self.hidden, self.inter, self.batch = layers, hidden, inter, batch
        self.cache, self.shared, self.budget = cache, shared, budget
        if cache is not None:
            self._attend_over(cache, counts)
        elif budget is not None:
            raise ValueError("budget: of a cache's rows")
        kv_hidden = hidden if cache is None else cache.heads * cache.head_dim
        self.lib = fbq.load()
        dev = "cuda"
        f16 = lambda n: torch.zeros((batch, n), dtype=torch.float16, device=dev)
        self.x = f16(hidden)
        n_buf = len(layers) if keep_per_layer_buffers else 1
        self.buf = [{"q": f16(hidden), "k": f16(kv_hidden), "v": f16(kv_hidden), "a": f16(hidden) if cache is not None else None, "o": f16(hidden), "h": f16(hidden),
                     "gate": f16(inter), "up": f16(inter), "act": f16(inter), "down": f16(hidden), "x_in": f16(hidden)}
                    for _ in range(n_buf)]
        # one zero-filled workspace per linear: launches of one token never share one.  A prompt pass of hundreds of rows
        # needs megabytes per linear (the re-ordered activations): its layers, which run one after the other, share a set.
        if share_workspaces:
            one = {n: self._workspace(layers[0][n].desc) for n in NAMES}
            self.ws = [one for _ in layers]
        else:
            self.ws = [{n: self._workspace(l[n].desc) for n in NAMES} for l in layers]
        self.graph = None

    def _attend_over(self, cache, counts):
        """What the steps' calls of the cache need, once: tokens a row, their places, attention's workspace."""
        rows, ints = cache.lengths.numel(), lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        counts = [1] * rows if counts is None else list(counts)
        if len(counts) != rows or sum(counts) != self.batch or cache.dtype != torch.float16 or self.hidden % cache.head_dim:
            raise ValueError("cache: an fp16 cache of whole heads, with a row for every count; counts: as many tokens as the batch")
        edges = [0]
        for c in counts:
            edges.append(edges[-1] + c)
        self.count, self.start, self.lacking = ints(counts), ints([0] * rows), ints([0])
        self.lowest_start, self.most_lacking = ints([0] * rows), ints([0])
        self.max_q = max(counts)
        self.q_start = None if counts == [1] * rows else ints(edges)
        q = torch.empty((self.batch, self.hidden // cache.head_dim, cache.head_dim), dtype=torch.float16, device="cuda")
        self.attend_ws = kv.attention_workspace(cache, q, q_start=self.q_start, max_q=self.max_q, shared=self.shared)
        if self.budget is not None:
            width = cache.table.shape[1] * cache.page_size
            self.lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
            self.weights = torch.zeros((cache.pool.shape[0], rows, cache.heads, width), dtype=torch.float32, device="cuda")
            self.keep, self.evicted, self.most_skipped = ints([self.budget.keep] * rows), ints([0, 0]), ints([0])
            self.evict_ws = kv.cache_evict_workspace(cache, self.weights)
            self.added = torch.zeros_like(cache.lengths)        # the rows' lengths, 0 where a step has appended nothing: what `weights` counts
            self.appended = torch.zeros_like(cache.lengths, dtype=torch.bool)
            self.added_to = kv.Cache(cache.pool, cache.table, self.added, cache.refs, cache.dtype, cache.dim)

    def _attend(self, li, b, stream):
        """a = attention of this step's tokens over the cache, this layer's k and v in their pages first."""
        c = self.cache
        heads = lambda t, n: t.view(self.batch, n, c.head_dim)
        kv.cache_append(c, li, heads(b["k"], c.heads), heads(b["v"], c.heads), self.start, q_start=self.q_start, stream=stream)
        n = self.hidden // c.head_dim
        q, lse = heads(b["q"], n), None if self.budget is None else self.lse
        kv.attention(c, li, q, q_start=self.q_start, max_q=self.max_q, shared=self.shared, out=heads(b["a"], n), lse=lse, workspace=self.attend_ws, stream=stream)
        if lse is not None:
            kv.attention_weights(self.added_to, li, q, lse, self.weights[li], q_start=self.q_start, max_q=self.max_q, decay=self.budget.decay, stream=stream)
        return b["a"]

    def _workspace(self, desc):
        need = fbq.workspace_bytes(desc, self.batch)
        return torch.zeros(need, dtype=torch.uint8, device="cuda") if need else None

    def _group(self, li, names, xs, ys, stream_ptr, mix=None):
        """One grouped call; mix = (with, out): the last layer's result averaged with another tensor."""
        l, ws = self.layers[li], self.ws[li]
        arr = fbq.make_group([l[n] for n in names], xs, ys, [ws[n] for n in names])
        if mix is None:
            rc = self.lib.fbq_linear_group(arr, len(names), self.batch, stream_ptr)
        else:
            none = [None] * (len(names) - 1)
            rc = self.lib.fbq_linear_group_mix(arr, fbq.make_mix(none + [mix[0]], none + [mix[1]]), len(names), self.batch, stream_ptr)
        if rc:
            raise RuntimeError(f"fbq_linear_group: {fbq.status_string(rc)}")

    def step(self, stream=None):
        """One token through all layers: reads and overwrites self.x."""
        stream = stream or torch.cuda.current_stream()
        sp = ctypes.c_void_p(stream.cuda_stream)
        x = self.x
        if self.cache is not None:
            kv.cache_reserve(self.cache, self.count, start=self.start, info=self.lacking, stream=stream)
            with fbq._on(stream):                       # (every step writes its own: these two stay, over the replays of a graph)
                torch.minimum(self.lowest_start, self.start, out=self.lowest_start)
                torch.maximum(self.most_lacking, self.lacking, out=self.most_lacking)
                if self.budget is not None:             # (a last token held is no new one: its sums would begin anew, and a query that means nothing would count)
                    torch.bitwise_and(self.start, 0x7fffffff, out=self.added)                    # (-1: beyond every length)
                    torch.lt(self.added, self.cache.lengths, out=self.appended)
                    torch.mul(self.cache.lengths, self.appended, out=self.added)
        for li in range(len(self.layers)):
            b = self.buf[li % len(self.buf)]
            if len(self.buf) > 1:
                with fbq._on(stream):
                    b["x_in"].copy_(x)                  # kept for inspection only
            self._group(li, ("q", "k", "v"), [x, x, x], [b["q"], b["k"], b["v"]], sp)
            a = b["v"] if self.cache is None else self._attend(li, b, stream)
            self._group(li, ("o",), [a], [b["o"]], sp, mix=(x, b["h"]))                      # h = (x + o) / 2
            self._group(li, ("gate", "up"), [b["h"], b["h"]], [b["gate"], b["up"]], sp)
            fbq.silu_mul(b["gate"], b["up"], b["act"], stream)
            self._group(li, ("down",), [b["act"]], [b["down"]], sp, mix=(b["h"], x))         # x = (h + down) / 2
        if self.budget is not None:
            kv.cache_evict(self.cache, self.weights, self.keep, first=self.budget.first, recent=self.budget.recent, info=self.evicted, workspace=self.evict_ws, stream=stream)
            with fbq._on(stream):
                torch.maximum(self.most_skipped, self.evicted[1:], out=self.most_skipped)
        return x

    def capture(self):
        """Records step() into a HIP graph (after one eager step on a side stream, as capture requires).  With a cache that step is one of the sequences' own."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step(side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph, stream=side):
            self.step(side)
        return self.graph


def random_stack(n_layers, hidden, inter, r, bits, seed=1, kv_hidden=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    shapes = layer_shapes(hidden, inter, kv_hidden)
    return [{n: random_layer(fbq.Desc(shapes[n][0], shapes[n][1], r, bits), gen, gain=0.5) for n in NAMES} for _ in range(n_layers)]


def prompt_then_decode(layers, hidden, inter, prompt=256, new_tokens=64, warmup=2):
    """The shape of the paper's end-to-end measurement (Sec. 5.3: batch 1, a prompt of 256 tokens, then 64 generated):
    one pass of `prompt` rows through the stack (the prefill GEMM in every linear), then `new_tokens` single-row steps
    replayed from a HIP graph.  Returns milliseconds for each leg and tokens per second over the whole run."""
    pre = DecoderStack(layers, hidden, inter, batch=prompt, share_workspaces=True)
    dec = DecoderStack(layers, hidden, inter, batch=1)
    pre.x.copy_(torch.randn(prompt, hidden, device="cuda").half())
    dec.x.copy_(torch.randn(1, hidden, device="cuda").half())
    g = dec.capture()
    e = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    best = None
    for it in range(warmup + 3):
        torch.cuda.synchronize()
        e[0].record()
        pre.step()
        e[1].record()
        for _ in range(new_tokens):
            g.replay()
        e[2].record()
        torch.cuda.synchronize()
        t = (e[0].elapsed_time(e[1]), e[1].elapsed_time(e[2]))
        if it >= warmup and (best is None or sum(t) < sum(best)):
            best = t
    total_s = sum(best) * 1e-3
    return {"prompt_tokens": prompt, "generated_tokens": new_tokens, "prompt_ms": round(best[0], 3),
            "decode_ms_per_token": round(best[1] / new_tokens, 4), "total_ms": round(sum(best), 3),
            "generated_tokens_per_s": round(new_tokens / total_s, 1),
            "all_tokens_per_s": round((prompt + new_tokens) / total_s, 1),
            "finite": bool(torch.isfinite(pre.x).all() and torch.isfinite(dec.x).all())}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=32)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--inter", type=int, default=11008)
    ap.add_argument("--r", type=int, default=128)
    ap.add_argument("--bits", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=64, help="decode steps to time")
    ap.add_argument("--batch", type=int, default=1, help="sequences decoded together (rows per step)")
    ap.add_argument("--warmup", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=0, help="run a prompt pass of this many tokens first and report the whole run (Sec. 5.3: 256)")
    a = ap.parse_args()
    if a.prompt:
        out = prompt_then_decode(random_stack(a.layers, a.hidden, a.inter, a.r, a.bits), a.hidden, a.inter, a.prompt, a.tokens)
        out.update({"layers": a.layers, "bits": a.bits, "r": a.r, "hidden": a.hidden, "inter": a.inter})
        print(json.dumps(out), flush=True)
        return
    stack = DecoderStack(random_stack(a.layers, a.hidden, a.inter, a.r, a.bits), a.hidden, a.inter, batch=a.batch)
    stack.x.copy_(torch.randn(a.batch, a.hidden, device="cuda").half())
    g = stack.capture()
    for _ in range(a.warmup):
        g.replay()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    e0.record()
    for _ in range(a.tokens):
        g.replay()
    e1.record()
    torch.cuda.synchronize()
    us = e0.elapsed_time(e1) / a.tokens * 1e3
    shapes = layer_shapes(a.hidden, a.inter)
    nbytes = a.layers * sum(fbq_synth.algorithmic_bytes(N, K, a.r, a.bits, a.batch) for N, K in shapes.values())
    print(json.dumps({"tokens_per_s": round(a.batch * 1e6 / us, 1), "us_per_step": round(us, 1), "batch": a.batch, "layers": a.layers,
                      "fused_launches_per_step": 4 * a.layers, "GBps_over_linear_layers": round(nbytes / us / 1e3, 1),
                      "bits": a.bits, "r": a.r, "hidden": a.hidden, "inter": a.inter, "tokens_timed": a.tokens,
                      "finite": bool(torch.isfinite(stack.x).all())}), flush=True)


if __name__ == "__main__":
    main()
