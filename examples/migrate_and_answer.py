"""Prompts are answered, packed, migrated and decoded from on the other side: the paged cache operators around the engine.

One layer's keys and values of a few requests.  The prefill side appends the prompts to 16-bit pages and attends over them,
packs the pages to 4 bits and lets the engine move these (declare, plan, execute) into the decode side's pools, at page
numbers of its own.  The decode side then appends a token to every request and attends, step by step, over 4-bit pages.

    python examples/migrate_and_answer.py [--prompts 700 1331 64] [--steps 8]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_00368_amd import binding as T, kv, workloads as W  # noqa: E402

HEADS, Q_HEADS, DIM, PAGE_TOKENS, DTYPE = 8, 32, 128, 16, torch.bfloat16


def tables(tokens, room, n_pages, rng):
    """A page table with room for `room` more tokens a request, pages in any order."""
    pages = [-(-(t + room) // PAGE_TOKENS) for t in tokens]
    order = rng.permutation(n_pages)[:sum(pages)].astype(np.int32)
    table = np.zeros((len(tokens), max(pages)), np.int32)
    for i, part in enumerate(np.split(order, np.cumsum(pages)[:-1])):
        table[i, :len(part)] = part
    return table


def batch_of(table, lengths, rows):
    """A batch of the last `rows` tokens of each request."""
    start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    on = [torch.from_numpy(np.asarray(x, np.int32)).cuda() for x in (table, lengths, start)]
    return kv.Batch(*on, n_rows=int(start[-1]), max_rows=max(rows), max_kv=max(lengths))


def extents(segment, pools, page_bytes, table, lengths):
    """Extents of every request's K pages, then its V pages; a pool of K, and one of V behind it, in one segment."""
    rows = []
    for i, n in enumerate(lengths):
        pages = table[i, :-(-n // PAGE_TOKENS)].astype(np.uint64)
        for which in range(2):
            e = np.zeros(len(pages), W.EXTENT_DTYPE)
            e["seg"], e["len"], e["off"] = segment, page_bytes, np.uint64(which * pools) + pages * np.uint64(page_bytes)
            rows.append(e)
    return np.cumsum([0] + [len(r) for r in rows]), np.concatenate(rows)


def migrate(src, dst, page_bytes, src_table, dst_table, lengths, slice_bytes=64 << 10):
    """Moves the pages of all requests from the pools `src` [2, pages, bytes] to `dst` through the engine."""
    src_ptr, src_ext = extents(0, src[0].numel(), page_bytes, src_table, lengths)
    dst_ptr, dst_ext = extents(1, dst[0].numel(), page_bytes, dst_table, lengths)
    rails = W.make_rails([50000] * 4)
    total = int(src_ext["len"].sum(dtype=np.uint64))
    arena = torch.empty(total + (len(rails) + 1) * 256, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream()
    ctx = T.tent_create(slice_bytes, arena.data_ptr(), arena.numel())
    try:
        T.tent_register_segment(ctx, src.data_ptr(), src.numel())
        T.tent_register_segment(ctx, dst.data_ptr(), dst.numel())
        b = T.tent_declare(ctx, src_ptr.astype(np.uint32), src_ext, dst_ptr.astype(np.uint32), dst_ext)
        status, _ = T.tent_plan(ctx, b, rails, want_info=True, stream=stream)
        if status != T.TENT_OK:
            raise T.TentError(status, "tent_plan")
        T.tent_execute(ctx, b, stream)
        if T.tent_poll(ctx, b, stream) != 0:
            raise RuntimeError("slices are left")
    finally:
        T.tent_destroy(ctx)
    return total


def run(prompts, steps, seed=0):
    """Attention outputs of the prompts [tokens, heads, dim], and of every decode step [requests, heads, dim]; bytes that were
    moved, and what they would have been in 16 bits."""
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda")
    g.manual_seed(seed)

    def rows(n, heads, size=1.0):
        return (size * torch.randn(n, heads, DIM, generator=g, device="cuda")).to(DTYPE)

    q_weight, k_weight = ((1 + 0.1 * torch.randn(DIM, generator=g, device="cuda")).to(DTYPE) for _ in "qk")
    rope = kv.rope_table(max(prompts) + steps, DIM, 500000.0)
    turn = dict(q_weight=q_weight, k_weight=k_weight, rope=rope)
    n_pages = sum(-(-(t + steps) // PAGE_TOKENS) for t in prompts) + 5

    # prefill: prompts into 16-bit pages, attention over them
    pools16 = torch.zeros(2, n_pages, PAGE_TOKENS, HEADS, DIM, dtype=DTYPE, device="cuda")
    cache16 = kv.Cache(*pools16)
    table16 = tables(prompts, 0, n_pages, rng)
    batch = batch_of(table16, prompts, prompts)
    n = sum(prompts)
    q = kv.append(cache16, batch, rows(n, HEADS, 1.5), rows(n, HEADS), q=rows(n, Q_HEADS, 2.0), **turn)
    answers = kv.attend(cache16, batch, q)

    # packed, and moved
    page_bytes = kv.packed_page_bytes(PAGE_TOKENS, HEADS, DIM)
    shape = dict(dtype=DTYPE, page_tokens=PAGE_TOKENS, kv_heads=HEADS, head_dim=DIM)
    packed, arrived = (torch.zeros(2, n_pages, page_bytes, dtype=torch.uint8, device="cuda") for _ in range(2))
    used = torch.from_numpy(np.concatenate([table16[i, :-(-t // PAGE_TOKENS)] for i, t in enumerate(prompts)])).cuda()
    kv.pack(cache16, kv.Cache(*packed, **shape), used, used, errors=batch.errors)
    table4 = tables(prompts, steps, n_pages, rng)
    moved = migrate(packed, arrived, page_bytes, table16, table4, prompts)

    # decode: a token of every request a step
    cache4 = kv.Cache(*arrived, **shape)
    outs = []
    for i in range(1, steps + 1):
        step = batch_of(table4, [t + i for t in prompts], [1] * len(prompts))
        q = kv.append(cache4, step, rows(len(prompts), HEADS, 1.5), rows(len(prompts), HEADS), q=rows(len(prompts), Q_HEADS, 2.0), **turn)
        outs.append(kv.attend(cache4, step, q))
        batch.errors |= step.errors
    if int(batch.errors):
        raise RuntimeError(f"pages, lengths or positions were wrong: {int(batch.errors)}")
    return dict(answers=answers, outs=outs, moved=moved, moved16=moved * cache16.page_bytes // page_bytes, cache16=cache16, table16=table16,
                cache4=cache4, table4=table4, last_q=q)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompts", type=int, nargs="+", default=[700, 1331, 64])
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    r = run(a.prompts, a.steps)
    print(f"{len(a.prompts)} prompts of {sum(a.prompts)} tokens answered; {r['moved']} bytes moved instead of {r['moved16']}; "
          f"{len(r['outs'])} steps decoded from the 4-bit pages that arrived")


if __name__ == "__main__":
    main()
