"""Samples of one prompt decoded together: the quantized stack of decode_loop.py with a paged key/value cache between its linears.

    python -m paper_2501_16385_amd.batch_decode --layers 4 --prompt 1024 --samples 8 --tokens 32 [--cache-bits 4] [--keep 1040]

What a server does with one prompt and several samples of it, everything but the choice of rows on the device:

    prompt    one pass of `prompt` tokens: pages are reserved, every layer's keys and values appended, attention causal over them
    fork      `samples` rows become second holders of the prompt's pages (a partial last page is copied)
    decode    `tokens` steps of one token a sample, replayed from one HIP graph: reserve, append and attention of every layer in it; the prompt's
              full pages are read once for all samples
              (--keep N: and every step ends with the samples cut back to N tokens each: the prompt's full pages, the latest ones, and those that were attended to most)
    drop      half of the samples are freed, the pool is compacted in place, and the others go on in the same graph (a freed row stays empty: count 0)

Prints one JSON line.  Weights are random packed words, as in decode_loop.py.
"""
from __future__ import annotations

import argparse
import json

import torch

from . import cache as kv
from .decode_loop import Budget, DecoderStack, random_stack


def run(layers, hidden: int, inter: int, head_dim: int, kv_heads: int, prompt: int, samples: int, tokens: int, page_size: int = 16, x0=None, cache_bits: int = 16,
        keep: int = 0):
    """Returns (record, cache, last hidden states [samples, hidden]); row 0 of the cache is the prompt's, rows 1 .. samples the samples'.  keep: tokens that a sample may hold (0: all)."""
    prompt_pages = -(-prompt // page_size)
    own_pages = -(-(prompt % page_size + 2 * tokens + 2) // page_size) + 1
    first = prompt // page_size * page_size                   # what the samples share stays
    if keep and keep <= first:
        raise ValueError(f"keep: more than the {first} tokens of the prompt's full pages")
    cache = kv.cache_create(len(layers), prompt_pages + samples * own_pages, page_size, kv_heads, head_dim, samples + 1, prompt_pages + own_pages, bits=cache_bits)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    event = [torch.cuda.Event(enable_timing=True) for _ in range(6)]

    pre = DecoderStack(layers, hidden, inter, batch=prompt, share_workspaces=True, cache=cache.rows(0, 1), counts=[prompt], budget=Budget(prompt) if keep else None)
    pre.x.copy_(torch.randn(prompt, hidden, device="cuda").half() if x0 is None else x0)
    event[0].record()
    pre.step()
    event[1].record()

    rows = list(range(1, samples + 1))
    info, compacted = ints([0, 0]), ints([0, 0])
    kv.cache_fork(cache, ints([0] * samples), ints(rows), info=info)
    full = prompt // page_size
    shared = cache.table[0, :full] if full else None          # a view: right after pages have moved, too
    dec = DecoderStack(layers, hidden, inter, batch=samples, cache=cache.rows(1, samples + 1), shared=shared,
                       budget=Budget(keep, first, max(1, (keep - first) // 2)) if keep else None)
    if keep:
        dec.weights.copy_(pre.weights.expand_as(dec.weights))
    dec.x.copy_(pre.x[-1:].expand(samples, hidden))
    graph = dec.capture()                                     # (the eager step before it is the first token)
    event[2].record()
    for _ in range(tokens - 1):
        graph.replay()
    event[3].record()

    gone = rows[samples // 2:] if samples > 1 else []
    if gone:
        kv.cache_free(cache, ints(gone))
        dec.count.copy_(ints([1] * (samples - len(gone)) + [0] * len(gone)))
    kv.cache_compact(cache, info=compacted)
    event[4].record()
    for _ in range(tokens):
        graph.replay()
    event[5].record()
    torch.cuda.synchronize()
    us = lambda i, n: round(event[i].elapsed_time(event[i + 1]) / max(1, n) * 1e3, 1)
    record = {"prompt_tokens": prompt, "samples": samples, "prompt_us": us(0, 1), "us_per_step": us(2, tokens - 1), "drop_and_compact_us": us(3, 1),
              "us_per_step_after": us(4, tokens), "fork": info.tolist(), "pages_in_use_and_moved": compacted.tolist(), "pages_lacking": max(int(pre.most_lacking), int(dec.most_lacking)),
              "rows_left_out": [row for row, lowest in enumerate(pre.lowest_start.tolist() + dec.lowest_start.tolist()) if lowest < 0],
              "rows_not_cut_back": int(dec.most_skipped) if keep else 0, "lengths": cache.lengths.tolist(), "finite": bool(torch.isfinite(dec.x[:samples - len(gone)]).all())}
    return record, cache, dec.x


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--inter", type=int, default=11008)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--kv-heads", type=int, default=0, help="0: as many as query heads")
    ap.add_argument("--r", type=int, default=64)
    ap.add_argument("--bits", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=1024)
    ap.add_argument("--samples", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=32, help="decode steps before, and after, half of the samples are dropped")
    ap.add_argument("--page-size", type=int, default=16)
    ap.add_argument("--cache-bits", type=int, default=16, choices=(16, 4))
    ap.add_argument("--keep", type=int, default=0, help="tokens that a sample may hold; 0: all")
    a = ap.parse_args()
    kv_heads = a.kv_heads or a.hidden // a.head_dim
    stack = random_stack(a.layers, a.hidden, a.inter, a.r, a.bits, kv_hidden=kv_heads * a.head_dim)
    record, _, _ = run(stack, a.hidden, a.inter, a.head_dim, kv_heads, a.prompt, a.samples, a.tokens, a.page_size, cache_bits=a.cache_bits, keep=a.keep)
    record.update({"cache_bits": a.cache_bits, "keep": a.keep, "layers": a.layers, "hidden": a.hidden, "kv_heads": kv_heads, "bits": a.bits, "r": a.r})
    print(json.dumps(record), flush=True)


if __name__ == "__main__":
    main()
