"""Weights onto the tokens of a cache, the choice of those that stay, and the move that makes them the sequence, on a GPU; and the
operators together, as a step of speculative decoding and an eviction use them."""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv_tree_reference as TR  # noqa: E402
from paper_2604_00368_amd import binding as T  # noqa: E402
from test_gpu_kv import Setup, kv, same  # noqa: E402,F401

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16
I32 = dict(dtype=torch.int32, device="cuda")


# ---- weigh ---------------------------------------------------------------------------------------
def lse_of(s, window, causal, scale):
    """What attention says, of the definition."""
    out = np.full((s.n_rows, s.q_heads), -math.inf)
    for i, n in enumerate(s.rows):
        if n:
            at = slice(s.starts[i], s.starts[i] + n)
            out[at] = TR.attend(s.q[at].double().numpy(), s.held(s.k_pool, i), s.held(s.v_pool, i), TR.spans(n, s.tokens[i], window, causal), scale)[1]
    return torch.from_numpy(out).float()


def check_weights(s, lse, got, before, per_head, window=0, causal=True, scale=None, skip=()):
    scale = 1 / math.sqrt(s.dim) if scale is None else scale
    got, before = got.cpu().double().numpy(), before.double().numpy()
    for i, n in enumerate(s.rows):
        if i in skip:
            continue
        at, t = slice(s.starts[i], s.starts[i] + n), s.tokens[i]
        want, off = TR.weigh(s.q[at].double().numpy(), s.held(s.k_pool, i), lse[at].double().numpy(), TR.spans(n, t, window, causal), scale)
        if not per_head:
            off = off.sum(0) + 2.0 ** -24 * s.heads * want.sum(0)
            want = want.sum(0)
        have = before[i, ..., :t]
        want, off = want + have, off + 2.0 ** -24 * (want + np.abs(have))
        d = np.abs(got[i, ..., :t] - want)
        assert (d <= off).all(), (i, float((d / np.maximum(off, 1e-300)).max()), np.unravel_index((d / np.maximum(off, 1e-300)).argmax(), d.shape))
        same(got[i, ..., t:], before[i, ..., t:])


WEIGH = [(BF16, 128, 2, 8, 16, [1, 4, 3, 0, 2], [9, 21, 500, 40, 33]), (FP16, 64, 1, 3, 8, [70, 10, 1], [0, 77, 130]), (BF16, 64, 3, 3, 1, [40, 64, 5], [0, 31, 97]),
         (FP16, 256, 2, 4, 64, [33, 16], [0, 4]), (BF16, 256, 1, 1, 128, [1, 1], [300, 256]), (FP16, 128, 2, 10, 32, [129, 31], [0, 128])]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("case", range(len(WEIGH)))
def test_weigh(kv, case, per_head, bits):
    dtype, dim, heads, q_heads, page_tokens, rows, before = WEIGH[case]
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], dtype, bits, q_heads, heads, dim, page_tokens, seed=case, spare_bytes=32)
    q, most = s.q.cuda(), max(s.tokens)
    shape = (len(rows), heads, most) if per_head else (len(rows), most)
    held = torch.rand(shape, generator=s.g)
    for window, causal, scale in ((0, True, None), (7, True, 0.2), (0, False, None), (40, False, None)):
        lse = lse_of(s, window, causal, 1 / math.sqrt(dim) if scale is None else scale)
        how = dict(per_head=per_head, window=window, causal=causal, scale=scale)
        fresh = kv.weigh(s.cache, s.batch, q, lse.cuda(), **how)
        assert fresh.shape == shape
        check_weights(s, lse, fresh, torch.zeros(shape), **how)
        mine = held.cuda()
        more = kv.weigh(s.cache, s.batch, q, lse.cuda(), weights=mine, **how)
        check_weights(s, lse, more, held, **how)
        assert torch.equal(mine.cpu(), held)
        assert kv.weigh(s.cache, s.batch, q, lse.cuda(), weights=mine, out=mine, **how) is mine and torch.equal(mine, more)
    assert int(s.batch.errors) == 0


def test_weigh_after_attend_adds_up_to_the_rows(kv):
    s = Setup(kv, [5, 1, 33], [2005, 1, 33], BF16, 4, 8, 2, 128, 16, seed=3)
    q = s.q.cuda()
    _, lse = kv.attend(s.cache, s.batch, q, want_lse=True)
    w = kv.weigh(s.cache, s.batch, q, lse).cpu().double()
    for i, n in enumerate(s.rows):                                       # every row and query head has a weight of 1 in all
        assert (w[i].sum(-1) - 4 * n).abs().max() < 4 * n * 1e-4
        assert not w[i, :, s.tokens[i]:].any()


def test_weigh_wide_lists_and_their_tails(kv):
    s = Setup(kv, [3, 4], [30, 50], BF16, 16, 4, 2, 64, 16, seed=4)
    q, lse = s.q.cuda(), lse_of(s, 0, True, 1 / 8)
    room = torch.rand(2, 2, 80, generator=s.g)
    got = kv.weigh(s.cache, s.batch, q, lse.cuda(), weights=room.cuda())
    assert got.shape == room.shape and torch.equal(got[..., 50:].cpu(), room[..., 50:])
    check_weights(s, lse, got, room, True)
    part = room.cuda()[..., :60]
    got = kv.weigh(s.cache, s.batch, q, lse.cuda(), weights=part)
    assert got.stride() == part.stride() and torch.equal(got[..., 50:], part[..., 50:])
    check_weights(s, lse, got, room[..., :60], True)


def test_weigh_rows_without_a_sum_add_nothing(kv):
    s = Setup(kv, [4, 40], [44, 40], BF16, 16, 4, 2, 64, 16, seed=5)
    lse = lse_of(s, 0, True, 1 / 8)
    lse[1], lse[2, 1], lse[9] = math.nan, math.inf, -math.inf
    s.q[1] = math.nan
    s.q[2, 1] = math.inf
    for per_head in (True, False):
        got = kv.weigh(s.cache, s.batch, s.q.cuda(), lse.cuda(), per_head=per_head)
        check_weights(s, lse, got, torch.zeros(got.shape), per_head)


@pytest.mark.parametrize("bits", [16, 4])
def test_weigh_tokens_that_are_not_seen(kv, bits):
    # what lies behind a sequence's last token, in its page, and behind a window
    s = Setup(kv, [3, 2], [37, 60], BF16, bits, 4, 2, 64, 16, seed=6)
    lse = lse_of(s, 9, True, 1 / 8)
    want = kv.weigh(s.cache, s.batch, s.q.cuda(), lse.cuda(), window=9)
    page = int(s.table[0, 2])
    if bits == 16:
        s.k_pool[page, 5:] = math.nan
    else:
        s.k_pool[page, 16 * 2 * 32 + 5 * 4:] = 255
    s.k_pool[int(s.table[1, 0])] = math.nan if bits == 16 else 255
    assert torch.equal(kv.weigh(s.cache, s.batch, s.q.cuda(), lse.cuda(), window=9), want)
    check_weights(s, lse, want, torch.zeros(want.shape), True, window=9, skip=(1,))


def test_weigh_rows_in_front_of_the_sequence_pages_and_sequences_that_are_wrong(kv):
    s = Setup(kv, [10, 3, 5], [4, 50, 30], BF16, 16, 4, 2, 64, 16, seed=7)
    lse = lse_of(s, 0, True, 1 / 8)
    got = kv.weigh(s.cache, s.batch, s.q.cuda(), lse.cuda())
    check_weights(s, lse, got, torch.zeros(got.shape), True)
    s.batch.page_table[1, 1] = -1
    s.batch.kv_len[2] = -3
    held = torch.rand(3, 2, 50, generator=s.g)
    again = kv.weigh(s.cache, s.batch, s.q.cuda(), lse.cuda(), weights=held.cuda()).cpu()
    assert int(s.batch.errors) == T.TENT_KV_BAD_PAGE | T.TENT_KV_BAD_SEQUENCE
    assert torch.equal(again[2], held[2]) and torch.equal(again[1, :, 16:32], held[1, :, 16:32])
    here = torch.cat([again[1, :, :16] - held[1, :, :16], again[1, :, 32:] - held[1, :, 32:]], -1)
    assert (here - torch.cat([got[1, :, :16], got[1, :, 32:]], -1).cpu()).abs().max() < 1e-6


def test_weigh_no_rows(kv):
    s = Setup(kv, [0, 0], [20, 30], BF16, 16, 4, 2, 64, 16, seed=8)
    held = torch.rand(2, 2, 30, generator=s.g).cuda()
    q, lse = s.q.cuda(), torch.zeros(0, 4, device="cuda")
    assert torch.equal(kv.weigh(s.cache, s.batch, q, lse, weights=held), held)
    assert not kv.weigh(s.cache, s.batch, q, lse).any()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("n_seqs,dtype,dim", [(64, BF16, 128), (256, FP16, 64), (64, BF16, 256), (256, BF16, 128)])
def test_weigh_several_tiles_to_a_wave(kv, n_seqs, dtype, dim, bits):
    """Eight heads over up to 1,000 tokens: 64 sequences have runs of two tiles, 256 of four.  Lengths end in any tile of a run."""
    rng = random.Random(n_seqs + dim)
    rows = [rng.choice([0, 1, 1, 2, 8]) for _ in range(n_seqs)]
    tokens = [r + rng.choice([0, rng.randint(0, 70), rng.randint(0, 300)]) for r in rows]
    rows[:4], tokens[:4] = [1, 8, 2, 1], [1000, 999, 513, 512]
    check_many(kv, rows, tokens, dtype, bits, 16, 8, dim, True, left_out=(5, n_seqs - 1))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("heads,dtype,dim", [(5, BF16, 128), (8, FP16, 64), (9, BF16, 256), (8, BF16, 128)])
def test_weigh_one_list_for_many_heads(kv, heads, dtype, dim, bits):
    """Four waves share the heads: they take two or three each, or some none."""
    check_many(kv, [1, 0, 3, 10, 2, 1], [300, 20, 35, 10, 129, 31], dtype, bits, 2 * heads, heads, dim, False, left_out=(4,))


class Coded(Setup):
    """4-bit pages of any codes, and scales of 2^-3 to 2^3: quicker than packing values."""

    def packed(self, values):
        n, count = values.shape[0], self.page_tokens * self.heads
        out = torch.randint(0, 256, (n, self.kv.packed_page_bytes(self.page_tokens, self.heads, self.dim)), generator=self.g).to(torch.uint8)
        scales = torch.randint(124, 131, (n, count * self.dim // 32), generator=self.g).to(torch.uint8)
        out[:, count * self.dim // 2:count * self.dim // 2 + scales.shape[1]] = scales
        return out


def check_many(kv, rows, tokens, dtype, bits, q_heads, heads, dim, per_head, left_out=()):
    """As check_weights, with a window and without; the pages' values are looked up once."""
    s = Coded(kv, rows, tokens, dtype, bits, q_heads, heads, dim, 16, seed=heads + dim)
    for i in left_out:
        s.batch.kv_len[i] = -1
    values, scale, n, most = s.values(s.k_pool), 1 / math.sqrt(dim), len(rows), max(tokens)
    keys = [values[s.table[i, :-(-t // 16)].long().numpy()].reshape(-1, heads, dim)[:t] for i, t in enumerate(tokens)]
    held = torch.rand((n, heads, most) if per_head else (n, most), generator=s.g)
    for window in (0, 40):
        seen = [TR.spans(r, t, window) for r, t in zip(rows, tokens)]
        lse = torch.full((s.n_rows, q_heads), -math.inf)
        for i, r in enumerate(rows):
            for j in range(r):
                at = seen[i][j]
                x = np.einsum("hd,thd->ht", s.q[s.starts[i] + j].double().numpy(), np.repeat(keys[i][at], q_heads // heads, 1)) * scale
                if x.shape[1]:
                    lse[s.starts[i] + j] = torch.from_numpy(np.logaddexp.reduce(x, 1))
        got = kv.weigh(s.cache, s.batch, s.q.cuda(), lse.cuda(), weights=held.cuda(), per_head=per_head, window=window)
        fresh = kv.weigh(s.cache, s.batch, s.q.cuda(), lse.cuda(), per_head=per_head, window=window)
        sides = [(x.cpu().double().numpy(), y.double().numpy()) for x, y in ((got, held), (fresh, torch.zeros(held.shape)))]
        for i, (r, t) in enumerate(zip(rows, tokens)):
            if i in left_out or r == 0:
                for result, before in sides:
                    same(result[i], before[i])
                continue
            at = slice(s.starts[i], s.starts[i] + r)
            want, off = TR.weigh(s.q[at].double().numpy(), keys[i], lse[at].double().numpy(), seen[i], scale)
            if not per_head:
                off, want = off.sum(0) + 2.0 ** -24 * heads * want.sum(0), want.sum(0)
            for result, before in sides:
                have = before[i, ..., :t]
                d = np.abs(result[i, ..., :t] - want - have)
                assert (d <= off + 2.0 ** -24 * (want + 2 * have)).all(), (window, i)
                same(result[i, ..., t:], before[i, ..., t:])
        assert int(s.batch.errors) == (T.TENT_KV_BAD_SEQUENCE if left_out else 0)


# ---- choose --------------------------------------------------------------------------------------
def a_batch(kv, tokens, most=None):
    n = len(tokens)
    return kv.Batch(torch.zeros(n, 1 + max(tokens), **I32), torch.tensor(tokens, **I32), torch.zeros(n + 1, **I32), 0, 0, max(tokens) if most is None else most)


def check_choice(kv, w, tokens, budget, first=0, recent=0, spare=0):
    batch = a_batch(kv, tokens)
    x = w.cuda()
    if spare:
        x = torch.cat([x, torch.full((*x.shape[:-1], spare), 1e30, device="cuda")], -1)
    lists, counts = kv.choose(batch, x, budget, first, recent)
    assert counts.tolist() == [min(t, budget) for t in tokens] and lists.shape == (*w.shape[:-1], budget)
    a, lists = w.numpy().reshape(len(tokens), -1, w.shape[-1]), lists.cpu().numpy().reshape(len(tokens), -1, budget)
    for i, t in enumerate(tokens):
        for h in range(a.shape[1]):
            want = TR.choose(a[i, h, :t], budget, first, recent)
            assert lists[i, h].tolist() == want + [-1] * (budget - len(want)), (i, h)
    assert int(batch.errors) == 0


@pytest.mark.parametrize("tokens", [[1], [5, 0, 64], [1000, 1023, 1024, 1025, 1, 7], [4096, 16383, 16384, 16385], [40001]])
@pytest.mark.parametrize("per_head", [True, False])
def test_choose(kv, tokens, per_head):
    g = torch.Generator().manual_seed(len(tokens))
    shape = (len(tokens), 3, max(tokens)) if per_head else (len(tokens), max(tokens))
    w = torch.empty(shape).exponential_(generator=g)
    for budget, first, recent in ((1, 0, 0), (1, 1, 0), (2, 1, 1), (7, 2, 3), (64, 4, 60), (700, 4, 100), (1024, 0, 0), (5000, 0, 4999)):
        check_choice(kv, w, tokens, budget, first, recent, spare=budget % 3)


def test_choose_equal_weights(kv):
    g = torch.Generator().manual_seed(2)
    tokens = [3000, 2500, 17, 1]
    for w in (torch.zeros(4, 2, 3000), torch.randint(0, 4, (4, 2, 3000), generator=g).float(), torch.randint(-2, 2, (4, 2, 3000), generator=g).float() * 0.0,
              torch.randint(0, 50, (4, 2, 3000), generator=g).float().mul_(2.0 ** -140), torch.full((4, 2, 3000), math.inf), torch.full((4, 2, 3000), -math.inf)):
        for budget, first, recent in ((1, 0, 0), (100, 4, 20), (1200, 0, 0), (2999, 1, 1)):
            check_choice(kv, w, tokens, budget, first, recent)


def test_choose_weights_that_are_negative_infinite_or_nan(kv):
    g = torch.Generator().manual_seed(3)
    w = torch.randn(3, 2, 2200, generator=g)
    w[:, :, 5::7] = math.inf
    w[:, :, 6::11] = -math.inf
    w[0, :, 4::3] = math.nan
    w[1, :, 4::3] = -math.nan
    w[2] = math.nan
    for budget in (1, 50, 400, 1500, 2100):
        check_choice(kv, w, [2200, 2100, 2000], budget, min(3, budget), 0)


@pytest.mark.parametrize("tokens", [[16385, 100, 70001, 32768, 0], [49152, 49153], [1050001]])
@pytest.mark.parametrize("kind", ["any", "equal", "few", "odd"])
def test_choose_from_long_lists(kv, tokens, kind):
    """Several workgroups to a list: borders at the ends of their tokens, equal weights on both sides, a workgroup that is behind the last token."""
    g = torch.Generator().manual_seed(len(tokens))
    n = max(tokens)
    shape = (len(tokens), 2, n) if n < 100000 else (1, n)
    w = torch.zeros(shape) if kind == "equal" else torch.randint(0, 5, shape, generator=g).float() if kind == "few" else torch.randn(shape, generator=g)
    if kind == "odd":
        w[..., 3::5] = math.nan
        w[..., 4::9] = math.inf
        w[..., 5::9] = -math.inf
    for budget, first, recent in ((1, 0, 0), (3, 1, 2), (4096, 0, 0), (20000, 16390, 5), (33000, 4, 16390), (n - 1, 2, 3), (40, 30, 10)):
        check_choice(kv, w, tokens, budget, first, recent, spare=budget % 2)


def test_choose_takes_a_workspace_of_any_contents(kv):
    batch, w = a_batch(kv, [40000, 20000]), torch.randn(2, 3, 40000, generator=torch.Generator().manual_seed(9)).cuda()
    need = kv.choose_workspace(batch, 3)
    assert need > 0 and kv.choose_workspace(a_batch(kv, [16384]), 3) == 0
    want = kv.choose(batch, w, 5000, 4, 100)
    for byte in (0, 1, 255):
        work = torch.full((need + 64,), byte, dtype=torch.uint8, device="cuda")
        got = kv.choose(batch, w, 5000, 4, 100, workspace=work[:need])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool((work[need:] == byte).all())


def low_weights(kind, shape, g):
    """Weights of which more than 128 share their leading 22 bits, so that the last ten decide."""
    if kind == "near one":
        return 1 + 1e-3 * torch.randn(shape, generator=g)
    if kind == "bit 10":                                                 # two values, of four in five places the smaller one
        bits = (torch.rand(shape, generator=g) < 0.2).int() << 10
    else:
        bits = torch.randint(0, 4096, shape, generator=g).int()
    return (bits + 0x3F800000 + (-0x80000000 if kind == "negative" else 0)).int().view(torch.float32)


# one list a workgroup, held whole; more lists than workgroups share, several rounds each; lists that workgroups share
@pytest.mark.parametrize("tokens,heads", [([1000, 16384, 1025], 2), ([20000, 16385], 65), ([33000, 20000], 1)])
@pytest.mark.parametrize("kind", ["any", "negative", "bit 10", "near one"])
def test_choose_weights_that_differ_in_their_last_bits(kv, tokens, heads, kind):
    g = torch.Generator().manual_seed(heads)
    n = max(tokens)
    w = low_weights(kind, (len(tokens), heads, n), g)
    batch, x = a_batch(kv, tokens), w.cuda()
    sorted_once = {}
    for share in (0.05, 0.15, 0.3, 0.5, 0.7, 0.95):                      # borders with bit 10 set and not, in each of the groups
        budget, first, recent = int(share * min(tokens)), 4, 32
        lists = torch.full((len(tokens), heads, budget + 3), -77, **I32)  # whatever is not written shows
        counts = torch.full((len(tokens),), -77, **I32)
        a = T.tent_kv_choose_args(x.data_ptr(), lists.data_ptr(), counts.data_ptr(), n, budget + 3, None, 0, heads, budget, first, recent)
        need = T.tent_kv_choose_workspace(batch.c, a)
        assert (need > 0) == (n > T.TENT_KV_CHOOSE_WHOLE and heads == 1)
        work = torch.full((max(need, 1),), 0xA5, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = work.data_ptr() if need else None, need
        T.tent_kv_choose(batch.c, a)
        assert counts.tolist() == [budget] * len(tokens) and bool((lists[..., budget:] == -77).all()) and int(batch.errors) == 0
        got = lists[..., :budget].cpu().numpy()
        for i, t in enumerate(tokens):
            for h in range(heads):                                       # as TR.choose, sorted once for all budgets
                if (i, h) not in sorted_once:
                    order = np.lexsort((np.arange(t), -w[i, h, :t].numpy()))
                    sorted_once[i, h] = order[(order >= first) & (order < t - recent)]
                want = np.sort(np.concatenate([np.arange(first), np.arange(t - recent, t), sorted_once[i, h][:budget - first - recent]]))
                assert (got[i, h] == want).all(), (budget, i, h, int((got[i, h] == -77).sum()))


def test_choose_sequences_that_are_left_out(kv):
    batch = a_batch(kv, [50, 60, 70], most=65)
    w = torch.rand(3, 65, generator=torch.Generator().manual_seed(4))
    lists, counts = kv.choose(batch, w.cuda(), 10)
    assert counts.tolist() == [10, 10, 0] and bool((lists[2] == -1).all()) and int(batch.errors) == T.TENT_KV_BAD_SEQUENCE
    assert lists[1].tolist() == TR.choose(w[1, :60].numpy(), 10, 0, 0)


# ---- keep ----------------------------------------------------------------------------------------
def raw(s, pool, i, n=None, table=None):
    """Tokens of a sequence as bytes [tokens, heads, bytes of a head], the scales behind the codes."""
    n = s.tokens[i] if n is None else n
    pages = (s.table if table is None else table)[i, :-(-n // s.page_tokens)].long()
    x = pool.cpu()[pages]
    if s.bits == 16:
        return x.view(torch.uint8).reshape(-1, s.heads, 2 * s.dim)[:n].numpy()
    half, count = s.dim // 2, s.page_tokens * s.heads
    codes = x[:, :count * half].reshape(-1, s.heads, half)
    return torch.cat([codes, x[:, count * half:count * (half + s.dim // 32)].reshape(-1, s.heads, s.dim // 32)], -1)[:n].numpy()


KEEP = [(BF16, 128, 2, 16, 16, [300, 0, 129, 16, 1]), (FP16, 64, 1, 8, 4, [77, 512]), (BF16, 256, 3, 1, 16, [40, 9]), (FP16, 128, 8, 32, 4, [1000, 257, 33]),
        (BF16, 64, 2, 128, 16, [130]), (FP16, 256, 1, 64, 4, [200, 64])]


@pytest.mark.parametrize("case", range(len(KEEP)))
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("elsewhere", [True, False])
def test_keep(kv, case, per_head, elsewhere):
    dtype, dim, heads, page_tokens, bits, tokens = KEEP[case]
    rng = random.Random(case)
    s = Setup(kv, [0] * len(tokens), [t + (t + 40 if elsewhere else 0) for t in tokens], dtype, bits, heads, heads, dim, page_tokens, seed=case, spare_bytes=16 * (case % 2))
    table, s.tokens = s.table.clone(), list(tokens)
    s.batch.kv_len.copy_(torch.tensor(tokens))
    to = None
    if elsewhere:                                                        # the pages behind the sequence's own
        width = -(-(max(tokens) + 20) // page_tokens)
        to = torch.full((len(tokens), width), 7 << 24, dtype=torch.int32)
        for i, t in enumerate(tokens):
            own = -(-t // page_tokens)
            left = table[i, own:-(-(2 * t + 40) // page_tokens)][:width]
            to[i, :len(left)] = left
    counts = [rng.randint(0, t) for t in tokens]
    n_lists, most = heads if per_head else 1, max(max(counts), 1) + 3
    entries = np.full((len(tokens), n_lists, most), -9, np.int32)
    for i, (t, c) in enumerate(zip(tokens, counts)):
        for h in range(n_lists):
            entries[i, h, :c] = [rng.randrange(0 if elsewhere else j, t) for j in range(c)] if h % 2 else sorted(rng.sample(range(t), c))
    weights = torch.rand(len(tokens), heads, max(s.batch.max_kv, 1), generator=s.g)
    before = [[raw(s, p, i) for p in (s.k_pool, s.v_pool)] for i in range(len(tokens))]
    others = [p.clone() for p in (s.k_pool, s.v_pool)]
    w = weights.cuda()
    lists = torch.from_numpy(entries if per_head else entries[:, 0]).cuda()
    length, moved = kv.keep(s.cache, s.batch, lists, torch.tensor(counts, **I32), to_table=None if to is None else to.cuda(), weights=w)
    assert length.tolist() == counts and int(s.batch.errors) == 0 and (moved is w) == (not elsewhere)
    written = torch.zeros(s.k_pool.shape[0], page_tokens, heads, dtype=torch.bool)
    for i, c in enumerate(counts):
        for pool, old in zip((s.k_pool, s.v_pool), before[i]):
            got = raw(s, pool, i, c, to)
            for h in range(heads):
                assert (got[:, h] == old[entries[i, h if per_head else 0, :c], h]).all(), (i, h)
        for h in range(heads):
            e = entries[i, h if per_head else 0, :c]
            assert torch.equal(moved[i, h, :c].cpu(), weights[i, h][torch.from_numpy(e).long()]) and not moved[i, h, c:].any()
        j = torch.arange(c)
        written[(table if to is None else to)[i, j // page_tokens].long(), j % page_tokens] = True
    for pool, old in zip((s.k_pool, s.v_pool), others):                  # and nothing else is touched
        if bits == 16:
            assert torch.equal(pool.cpu()[~written], old.cpu()[~written])
        else:
            half = dim // 2
            a, b = pool.cpu(), old.cpu()
            n = page_tokens * heads
            for lo, size in ((0, half), (n * half, dim // 32)):
                at = slice(lo, lo + n * size)
                assert torch.equal(a[:, at].reshape(-1, page_tokens, heads, size)[~written], b[:, at].reshape(-1, page_tokens, heads, size)[~written])
            assert torch.equal(a[:, n * (half + dim // 32):], b[:, n * (half + dim // 32):])


@pytest.mark.parametrize("bits", [16, 4])
def test_keep_long_lists_in_place(kv, bits):
    # many batches of entries, columns of rows, places read that later ones write to
    tokens = [5000, 3111]
    for heads, per_head in ((1, True), (8, False)):
        s = Setup(kv, [0, 0], tokens, BF16, bits, heads, heads, 128, 16, seed=20 + heads)
        rng = np.random.RandomState(heads)
        for kind in range(3):
            counts = [t - rng.randint(1, 50) if kind else t for t in tokens]
            lists = torch.full((2, max(counts)), -1, dtype=torch.int32)
            for i, (t, c) in enumerate(zip(tokens, counts)):
                j = np.arange(c)
                e = np.minimum(j + 1, t - 1) if kind == 0 else np.sort(rng.permutation(t)[:c]) if kind == 1 else j + (rng.rand(c) * (t - j)).astype(int)
                lists[i, :c] = torch.from_numpy(e.astype(np.int32))
            before = [[raw(s, p, i) for p in (s.k_pool, s.v_pool)] for i in range(2)]
            kv.keep(s.cache, s.batch, lists.cuda(), torch.tensor(counts, **I32))
            for i, c in enumerate(counts):
                for pool, old in zip((s.k_pool, s.v_pool), before[i]):
                    assert (raw(s, pool, i, c) == old[lists[i, :c].numpy()]).all(), (kind, i)


@pytest.mark.parametrize("bits,dim", [(16, 64), (16, 128), (16, 256), (4, 128)])
def test_keep_many_lists_in_place(kv, bits, dim):
    # as many lists as fill the card: a workgroup moves whole rows of its head
    rng = np.random.RandomState(dim)
    tokens = [int(t) for t in rng.randint(0, 200, 64)]
    s = Setup(kv, [0] * 64, tokens, BF16, bits, 8, 8, dim, 16, seed=dim)
    counts = [int(rng.randint(0, t + 1)) for t in tokens]
    entries = np.full((64, 8, max(counts) + 1), -1, np.int32)
    for i, (t, c) in enumerate(zip(tokens, counts)):
        for h in range(8):
            entries[i, h, :c] = np.sort(rng.permutation(t)[:c]) if h % 2 else np.arange(c) + (rng.rand(c) * (t - np.arange(c))).astype(int)
    before = [[raw(s, p, i) for p in (s.k_pool, s.v_pool)] for i in range(64)]
    weights = torch.rand(64, 8, s.batch.max_kv, generator=s.g)
    w = weights.cuda()
    length, _ = kv.keep(s.cache, s.batch, torch.from_numpy(entries).cuda(), torch.tensor(counts, **I32), weights=w)
    assert length.tolist() == counts and int(s.batch.errors) == 0
    w = w.cpu()
    for i, (t, c) in enumerate(zip(tokens, counts)):
        for pool, old in zip((s.k_pool, s.v_pool), before[i]):
            got = raw(s, pool, i)
            assert (got[c:] == old[c:]).all()
            for h in range(8):
                assert (got[:c, h] == old[entries[i, h, :c], h]).all(), (i, h)
        for h in range(8):
            assert torch.equal(w[i, h, :c], weights[i, h][torch.from_numpy(entries[i, h, :c]).long()]) and not w[i, h, c:].any()


@pytest.mark.parametrize("elsewhere", [True, False])
def test_keep_rows(kv, elsewhere):
    rows, before = [9, 1, 0, 70, 4], [100, 0, 30, 33, 64]
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], FP16, 16, 4, 2, 64, 16, seed=30)
    rng = random.Random(5)
    paths = [sorted(rng.sample(range(n), rng.randint(0, n))) for n in rows]
    lists = torch.tensor([p + [-1] * (70 - len(p)) for p in paths], **I32)
    counts = torch.tensor([len(p) for p in paths], **I32)
    weights = torch.rand(5, 2, s.batch.max_kv, generator=s.g)
    old = [raw(s, s.k_pool, i) for i in range(5)]
    to = None
    if elsewhere:                                                        # the pages of the last sequences' table, which only they use
        pool = torch.cat([s.k_pool, torch.zeros(40, 16, 2, 64, dtype=FP16, device="cuda")])
        s.k_pool, s.v_pool = pool, pool.clone()
        s.cache = kv.Cache(s.k_pool, s.v_pool)
        to = (torch.arange(5 * 8) + pool.shape[0] - 40).reshape(5, 8).int()
    length, moved = kv.keep(s.cache, s.batch, lists, counts, rows=True, to_table=None if to is None else to.cuda(), weights=weights.cuda())
    assert length.tolist() == [b + len(p) for b, p in zip(before, paths)] and int(s.batch.errors) == 0
    for i, (b, p) in enumerate(zip(before, paths)):
        n = b + len(p)
        got = raw(s, s.k_pool, i, n, to)
        assert (got[b:] == old[i][b + np.array(p, dtype=int)]).all()
        if not elsewhere:
            assert (got[:b] == old[i][:b]).all()
        assert torch.equal(moved[i, :, :n].cpu(), weights[i][:, torch.tensor(list(range(b)) + [b + x for x in p], dtype=torch.long)])
        assert not moved[i, :, n:].any()


def test_keep_what_is_wrong_is_left_out(kv):
    s = Setup(kv, [0] * 5, [40] * 5, BF16, 16, 2, 2, 64, 16, seed=31)
    old = [raw(s, s.k_pool, i) for i in range(5)]
    lists = torch.arange(5, 5 + 20, dtype=torch.int32).repeat(5, 1)
    lists[0, 3], lists[0, 7], lists[0, 9] = 2, 40, -1                    # in front of its place, behind the last token, below 0
    counts = torch.tensor([20, 41, -1, 20, 20], **I32)
    s.batch.page_table[3, 0] = 1 << 25
    s.batch.kv_len[4] = 99
    weights = torch.rand(5, 2, 40, generator=s.g)
    length, moved = kv.keep(s.cache, s.batch, lists.cuda(), counts, weights=weights.cuda())
    assert length.tolist() == [20, 40, 40, 20, 99]
    assert int(s.batch.errors) == T.TENT_KV_BAD_SEQUENCE | T.TENT_KV_BAD_POSITION | T.TENT_KV_BAD_PAGE
    e = lists[0].tolist()
    for j in (3, 7, 9):
        e[j] = j
    assert (raw(s, s.k_pool, 0, 20) == old[0][e]).all() and torch.equal(moved[0, :, :20].cpu(), weights[0][:, e])
    for i in (1, 2, 4):
        assert (raw(s, s.k_pool, i) == old[i]).all() and torch.equal(moved[i].cpu(), weights[i])
    assert (raw(s, s.k_pool, 3)[16:20] == old[3][21:25]).all()           # tokens 16 to 19 are in the second page, which is there


def test_keep_refuses_a_table_that_is_too_short_entry_by_entry(kv):
    s = Setup(kv, [0, 0], [64, 64], BF16, 16, 2, 2, 64, 16, seed=32)
    pool = torch.cat([s.k_pool, torch.zeros(4, 16, 2, 64, dtype=BF16, device="cuda")])
    cache = kv.Cache(pool, pool.clone())
    old = [raw(s, pool, i) for i in range(2)]
    to = torch.arange(4).reshape(2, 2).int() + pool.shape[0] - 4         # room for 32 tokens each
    lists = torch.arange(63, 23, -1, dtype=torch.int32).repeat(2, 1)     # in any order
    length = kv.keep(cache, s.batch, lists.cuda(), torch.tensor([40, 32], **I32), to_table=to.cuda())
    assert length.tolist() == [40, 32] and int(s.batch.errors) == T.TENT_KV_BAD_PAGE
    for i in range(2):
        assert (raw(s, pool, i, 32, to) == old[i][63:31:-1]).all()


def test_keep_writes_to_no_page_between_the_rows_of_a_table(kv):
    # the table's rows lie behind the sequences' own in one tensor: behind the first row's end are the second sequence's pages
    s = Setup(kv, [0, 0], [64, 64], BF16, 16, 2, 2, 64, 16, seed=34)
    pool = torch.cat([s.k_pool, torch.zeros(4, 16, 2, 64, dtype=BF16, device="cuda")])
    cache = kv.Cache(pool, pool.clone())
    both = torch.cat([s.table, torch.arange(4).reshape(2, 2).int() + pool.shape[0] - 4], 1).cuda()
    batch = kv.Batch(both[:, :4], s.batch.kv_len, s.batch.row_start, 0, 0, 64)
    old = pool.clone()
    lists = torch.arange(63, 13, -1, dtype=torch.int32).repeat(2, 1)
    length = kv.keep(cache, batch, lists.cuda(), torch.tensor([50, 33], **I32), to_table=both[:, 4:])
    assert length.tolist() == [50, 33] and int(batch.errors) == T.TENT_KV_BAD_PAGE
    assert torch.equal(pool[:-4], old[:-4])
    for i in range(2):
        assert (raw(s, pool, i, 32, both[:, 4:].cpu()) == raw(s, old, i)[63:31:-1]).all()


def test_empty_lists_and_empty_sequences(kv):
    s = Setup(kv, [0, 0], [20, 30], BF16, 16, 2, 2, 64, 16, seed=33)
    old = s.k_pool.clone()
    length = kv.keep(s.cache, s.batch, torch.zeros(2, 0, **I32), torch.zeros(2, **I32))
    assert length.tolist() == [0, 0] and torch.equal(s.k_pool, old)
    batch = kv.Batch(torch.zeros(2, 1, **I32), torch.zeros(2, **I32), torch.zeros(3, **I32), 0, 0, 0)
    none = torch.zeros(2, 2, 0, device="cuda")
    lists, counts = kv.choose(batch, none, 5)
    assert bool((lists == -1).all()) and counts.tolist() == [0, 0]
    length, moved = kv.keep(s.cache, batch, lists, counts, weights=none)
    assert length.tolist() == [0, 0] and moved.shape == (2, 2, 0)
    q = torch.zeros(0, 2, 64, dtype=BF16, device="cuda")
    assert kv.weigh(s.cache, batch, q, torch.zeros(0, 2, device="cuda")).shape == (2, 2, 0)
    nobody = kv.Batch(torch.zeros(0, 2, **I32), torch.zeros(0, **I32), torch.zeros(1, **I32), 0, 0, 30)
    lists, counts = kv.choose(nobody, torch.zeros(0, 2, 30, device="cuda"), 5)
    assert lists.shape == (0, 2, 5) and kv.keep(s.cache, nobody, lists, counts).shape == (0,)
    assert kv.weigh(s.cache, nobody, q, torch.zeros(0, 2, device="cuda")).shape == (0, 2, 30)
    assert int(s.batch.errors) == 0 and int(batch.errors) == 0


# ---- together ------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [16, 4])
def test_a_run_of_speculation_and_eviction(kv, bits):
    """Steps of drafting, appending, attending, verifying and keeping, with an eviction in between: the cache holds what a list of tokens
    held on the host says, and attention over it is that of the definition."""
    n, H, HQ, D, PT, vocab, most = 3, 2, 4, 64, 16, 300, 8
    g, rng = torch.Generator().manual_seed(40), random.Random(40)
    start = [50, 7, 120]
    s = Setup(kv, [0] * n, [200] * n, BF16, bits, HQ, H, D, PT, seed=41)
    s.tokens = list(start)
    held = [[raw(s, p, i)[:t] for p in (s.k_pool, s.v_pool)] for i, t in enumerate(start)]
    kv_len = torch.tensor(start, **I32)
    weights = torch.zeros(n, H, 200, device="cuda")
    want_w = [np.zeros((H, t)) for t in start]
    for step in range(6):
        rows = [rng.randint(1, most) for _ in range(n)]
        starts = torch.tensor([sum(rows[:i]) for i in range(n + 1)], **I32)
        trees = [[i - 1 if i == 0 or rng.random() < 0.4 else rng.randrange(i) for i in range(r)] for r in rows]
        parents = torch.tensor([p for t in trees for p in t], **I32)
        total = sum(rows)
        batch = kv.Batch(s.batch.page_table, kv_len + torch.tensor(rows, **I32), starts, total, most, 200)
        q, k, v = (torch.randn(total, h, D, generator=g).to(BF16).cuda() for h in (HQ, H, H))
        masks, deep = kv.tree_masks(parents, starts, most)
        positions = (kv_len[torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(rows, device="cuda"))] + deep).int()
        q = kv.append(s.cache, batch, k, v, q=q, rope=kv.rope_table(256, D), positions=positions)
        out, lse = kv.attend(s.cache, batch, q, tree=masks, want_lse=True)
        s.rows, s.starts, s.q = rows, starts.tolist(), q.cpu()
        base = list(s.tokens)
        s.tokens = [b + r for b, r in zip(base, rows)]
        from test_gpu_kv_tree import check_tree
        check_tree(s, [TR.ancestors(t) for t in trees], out, lse)
        now = [[raw(s, p, i) for p in (s.k_pool, s.v_pool)] for i in range(n)]
        for i in range(n):
            for a, b in zip(now[i], held[i]):
                assert (a[:base[i]] == b).all()
        target = torch.softmax(2 * torch.randn(total, vocab, generator=g), -1)
        tokens = torch.multinomial(target, 1, generator=g)[:, 0].int()
        tokens = torch.cat([target[b + max(p, 0)].topk(3).indices[i % 3:i % 3 + 1].int() for t, b in zip(trees, s.starts) for i, p in enumerate(t)]) if step % 2 else tokens
        accept, chance = torch.rand(total, generator=g) * 0.05, torch.rand(n, generator=g)
        path, counts, token = kv.verify(batch, target.cuda(), tokens.cuda(), accept.cuda(), chance.cuda(), parents=parents)
        kv_len = kv.keep(s.cache, batch, path, counts, rows=True)
        for i in range(n):
            at = slice(s.starts[i], s.starts[i] + rows[i])
            way, x = TR.verify(target[at].double().numpy(), None, tokens[at].tolist(), trees[i], accept[at].double().tolist(), float(chance[i].double()))
            assert path[i, :len(way)].tolist() == way and counts[i] == len(way) and token[i] == x
            held[i] = [np.concatenate([a[:base[i]], a[base[i] + np.array(way)]]) for a in now[i]]
            s.tokens[i] = base[i] + len(way)
        assert kv_len.tolist() == s.tokens
        # the last token that stands looks at the sequence, and what it looked at is added up
        one = kv.Batch(s.batch.page_table, kv_len, torch.arange(n + 1, **I32), n, 1, 200)
        q1 = torch.randn(n, HQ, D, generator=g).to(BF16)
        _, lse = kv.attend(s.cache, one, q1.cuda(), want_lse=True)
        weights = kv.weigh(s.cache, one, q1.cuda(), lse, weights=weights, out=weights)
        for i in range(n):
            add, _ = TR.weigh(q1[i:i + 1].double().numpy(), s.held(s.k_pool, i), lse[i:i + 1].cpu().double().numpy(), TR.spans(1, s.tokens[i]), 1 / 8)
            want_w[i] = np.pad(want_w[i], ((0, 0), (0, s.tokens[i] - want_w[i].shape[1]))) + add
            assert np.abs(weights[i, :, :s.tokens[i]].cpu().numpy() - want_w[i]).max() < 1e-4 and not weights[i, :, s.tokens[i]:].any()
        if step in (2, 4):
            lists, counts = kv.choose(one, weights, 30, first=2, recent=10)
            w = weights.cpu().numpy()
            kv_len, weights = kv.keep(s.cache, one, lists, counts, weights=weights)
            for i in range(n):
                e = [TR.choose(w[i, h, :s.tokens[i]], 30, 2, 10) for h in range(H)]
                held[i] = [np.stack([a[e[h], h] for h in range(H)], 1) for a in held[i]]
                want_w[i] = np.stack([want_w[i][h][e[h]] for h in range(H)])
                s.tokens[i] = len(e[0])
            assert kv_len.tolist() == s.tokens
        for i in range(n):
            for p, b in zip((s.k_pool, s.v_pool), held[i]):
                assert (raw(s, p, i) == b).all(), (step, i)
        assert int(batch.errors) == 0 and int(one.errors) == 0


def test_steps_in_a_graph(kv):
    """A step of all five, captured and replayed with other inputs in the same tensors, between eager steps and synchronizations."""
    rows, before = [5, 1, 9], [3000, 40, 511]
    n, total, vocab = 3, 15, 140001
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], BF16, 16, 8, 2, 128, 16, seed=50)
    trees = [[i - 1 if i % 2 else max(0, i - 2) - (i == 0) for i in range(r)] for r in rows]
    parents = torch.tensor([p for t in trees for p in t], **I32)
    masks, _ = kv.tree_masks(parents, s.batch.row_start, 9)
    one = kv.Batch(s.batch.page_table, s.batch.kv_len, torch.arange(n + 1, **I32), n, 1, s.batch.max_kv)
    ins = dict(q=s.q.cuda(), k=torch.zeros(total, 2, 128, dtype=BF16, device="cuda"), v=torch.zeros(total, 2, 128, dtype=BF16, device="cuda"),
               target=torch.zeros(total, vocab, device="cuda"), draft=torch.zeros(total, vocab, device="cuda"), tokens=torch.zeros(total, **I32),
               accept=torch.zeros(total, device="cuda"), next=torch.zeros(n, device="cuda"), q1=torch.zeros(n, 8, 128, dtype=BF16, device="cuda"))
    first = [p.clone() for p in (s.k_pool, s.v_pool)]

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for name in ("q", "k", "v", "q1"):
            ins[name].copy_(torch.randn(ins[name].shape, device="cuda", generator=g))
        x = 3 * torch.randn(total, vocab, device="cuda", generator=g)
        ins["target"].copy_(torch.softmax(x, -1))
        ins["draft"].copy_(torch.softmax(x + 0.5 * torch.randn(total, vocab, device="cuda", generator=g), -1))
        after = torch.tensor([b + max(p, 0) for t, b in zip(trees, s.starts) for p in t], device="cuda")
        ins["tokens"].copy_(ins["draft"][after].multinomial(1, generator=g)[:, 0])
        ins["accept"].copy_(torch.rand(total, device="cuda", generator=g))
        ins["next"].copy_(torch.rand(n, device="cuda", generator=g))
        for p, f in zip((s.k_pool, s.v_pool), first):
            p.copy_(f)

    def step():
        kv.append(s.cache, s.batch, ins["k"], ins["v"])
        out, lse = kv.attend(s.cache, s.batch, ins["q"], tree=masks, want_lse=True)
        path, counts, token = kv.verify(s.batch, ins["target"], ins["tokens"], ins["accept"], ins["next"], parents=parents, draft=ins["draft"])
        length = kv.keep(s.cache, s.batch, path, counts, rows=True)
        _, lse1 = kv.attend(s.cache, one, ins["q1"], want_lse=True)
        weights = kv.weigh(s.cache, one, ins["q1"], lse1)
        lists, kept = kv.choose(one, weights, 300, 4, 20)
        after, weights = kv.keep(s.cache, one, lists, kept, weights=weights)
        return out, lse, path, counts, token, length, weights, lists, kept, after, s.k_pool, s.v_pool

    fill(1)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (2, 3, 2, 5):
        fill(seed)
        want = [x.clone() for x in step()]
        fill(seed)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (seed, i)
        fill(seed)
        graph.replay()
        graph_again = [x.clone() for x in got]
        assert all(torch.equal(a, b) for a, b in zip(graph_again, want))
    assert int(s.batch.errors) == 0


def test_calls_on_several_streams_do_not_share_their_workspaces(kv):
    from test_gpu_kv_tree import Drafts
    sets = [Drafts(kv, [9, 17, 5], 140001, torch.float32, True, seed=60 + i) for i in range(3)]
    ins = [(d.target.cuda(), d.tokens.cuda(), d.accept.cuda(), d.next.cuda(), d.parents.cuda(), d.draft.cuda()) for d in sets]
    want = [kv.verify(d.batch, *x) for d, x in zip(sets, ins)]
    for d, w in zip(sets, want):
        d.check(*w)
    need = kv.verify_workspace(sets[0].batch, 140001, parents=True, draft=True)
    assert need > 0
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(6):
        got = []
        for d, x, stream in zip(sets, ins, streams):
            got.append(kv.verify(d.batch, *x, stream=stream))
            torch.full((need,), 0x7F, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


@pytest.mark.parametrize("bits", [16, 4])
def test_pools_beyond_four_gib(kv, bits):
    """Pages 256 MiB apart give what pages side by side give."""
    results = []
    for spare in (0, 1 << 28):
        s = Setup(kv, [9, 17], [150, 170], BF16, bits, 8, 2, 128, 16, seed=70, spare_bytes=spare)
        parents = torch.tensor([max(i - 2, 0) - (i == 0) for n in s.rows for i in range(n)], **I32)
        out = list(kv.attend(s.cache, s.batch, s.q.cuda(), tree=kv.tree_masks(parents, s.batch.row_start, 17)[0], want_lse=True))
        lse = kv.attend(s.cache, s.batch, s.q.cuda(), want_lse=True)[1]
        weights = kv.weigh(s.cache, s.batch, s.q.cuda(), lse)
        many = kv.weigh(s.cache, s.batch, s.q.cuda(), lse, per_head=False)
        lists, counts = kv.choose(s.batch, weights, 16, 2, 5)
        used = set(s.table.flatten().tolist())
        free = [p for p in range(s.k16.shape[0]) if p not in used]
        table = torch.tensor(free, **I32)[:, None]
        out += [weights, many, lists, kv.keep(s.cache, s.batch, lists, counts, to_table=table)]
        out += [raw(s, p, i, 16, table.cpu()) for p in (s.k_pool, s.v_pool) for i in (0, 1)]
        out += kv.keep(s.cache, s.batch, lists, counts, weights=weights)
        out += [raw(s, p, i) for p in (s.k_pool, s.v_pool) for i in (0, 1)]
        assert int(s.batch.errors) == 0
        results.append([x.cpu() if isinstance(x, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(x)) for x in out])
        assert spare * s.k16.shape[0] == 0 or s.k_pool.stride(0) * s.k_pool.element_size() * (s.k16.shape[0] - 1) > 1 << 32
        del s
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*results))


def test_rows_and_lists_beyond_four_gib(kv):
    """Rows of probabilities and lists of weights 4.8 GB apart."""
    apart, vocab = 1_200_000_000, 30011
    store = torch.empty(apart + 200000, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(71)
    target = torch.softmax(2 * torch.randn(2, vocab, device="cuda", generator=g), -1)
    far = store.as_strided((2, vocab), (apart, 1))
    far.copy_(target)
    batch = kv.Batch(torch.zeros(1, 20, **I32), torch.tensor([20], **I32), torch.tensor([0, 2], **I32), 2, 2, 20)
    best = int(target[0].argmax())
    args = (torch.tensor([0, best], **I32), torch.zeros(2, device="cuda"), torch.tensor([0.7], device="cuda"))
    got, want = kv.verify(batch, far, *args), kv.verify(batch, target, *args)
    assert got[1].tolist() == [2] and all(torch.equal(a, b) for a, b in zip(got, want))
    for tokens in (5000, 100000):
        w = torch.randn(2, tokens, device="cuda", generator=g)
        far = store.as_strided((2, tokens), (apart, 1))
        far.copy_(w)
        batch = a_batch(kv, [tokens, tokens - 7])
        got, want = kv.choose(batch, far, 700, 3, 40), kv.choose(batch, w, 700, 3, 40)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[0][1, 699] == tokens - 8
