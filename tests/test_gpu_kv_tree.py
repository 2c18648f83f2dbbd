"""Attention of trees of drafted tokens, and their verification, on a GPU against their definitions in 64 bits."""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv_reference as R  # noqa: E402
import kv_tree_reference as TR  # noqa: E402
from test_gpu_kv import Setup, kv  # noqa: E402,F401

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16
I32 = dict(dtype=torch.int32, device="cuda")


def some_tree(rng, n):
    return [i - 1 if i == 0 or rng.random() < 0.5 else rng.randrange(i) for i in range(n)]


def check_tree(s, seen, out, lse, window=0, scale=None, skip=()):
    """`seen`: for every sequence what its rows see of each other."""
    scale = 1 / math.sqrt(s.dim) if scale is None else scale
    for i, n in enumerate(s.rows):
        if i in skip or n == 0:
            continue
        at = slice(s.starts[i], s.starts[i] + n)
        see = TR.visible(seen[i], s.tokens[i], window)
        want, want_lse, mass, size = TR.attend(s.q[at].double().numpy(), s.held(s.k_pool, i), s.held(s.v_pool, i), see, scale)
        bound, lse_bound = R.attend_bounds(want, mass, size, max(s.tokens[i], 1), s.dim, s.dtype)
        off = np.abs(out[at].double().cpu().numpy() - want)
        assert (off <= bound).all(), (i, float((off / bound).max()), np.unravel_index((off / bound).argmax(), off.shape))
        got_lse = lse[at].double().cpu().numpy()
        none = want_lse == -math.inf
        assert (got_lse[none] == -math.inf).all() and not out[at].cpu()[torch.from_numpy(none)].any()
        off = np.abs(np.where(none, 0, got_lse) - np.where(none, 0, want_lse))
        assert (off <= lse_bound + 2.0 ** -23 * np.where(none, 0, np.abs(want_lse))).all(), (i, float(off.max()))


def masks_of(seen, stride=None, rng=None):
    stride = stride or max(1, -(-max(x.shape[0] for x in seen) // 64))
    out = []
    for x in seen:                                                       # bits behind the last row mean nothing
        junk = np.random.RandomState(rng.randrange(1 << 30)).randint(0, 2, (x.shape[0], stride * 64 - x.shape[1])).astype(np.uint64) if rng else None
        out.append(TR.words(x, stride, junk) if x.shape[0] else np.zeros((0, stride), np.int64))
    return torch.from_numpy(np.concatenate(out)).cuda()


# rows by group: up to 16, 32 and 64 lines in a wave's registers, and tiles of 128
SHAPES = [(BF16, 128, 2, 8, 16, [1, 4, 3, 0, 2], [9, 21, 500, 0, 33]), (FP16, 64, 1, 3, 8, [7, 10, 1], [7, 77, 130]), (BF16, 64, 3, 3, 1, [40, 64, 5], [0, 31, 97]),
          (FP16, 128, 2, 6, 32, [17, 9, 21], [64, 0, 255]), (BF16, 128, 1, 4, 16, [30, 70, 129], [100, 63, 0]), (FP16, 256, 2, 4, 64, [5, 16], [300, 4]),
          (BF16, 256, 1, 2, 16, [65, 20], [64, 513]), (FP16, 64, 2, 2, 128, [200, 66], [130, 1]), (BF16, 128, 1, 1, 16, [64, 60], [700, 3])]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_trees(kv, case, bits):
    dtype, dim, heads, q_heads, page_tokens, rows, before = SHAPES[case]
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], dtype, bits, q_heads, heads, dim, page_tokens, seed=case, spare_width=1, spare_bytes=32)
    rng = random.Random(case)
    seen = [TR.ancestors(some_tree(rng, n)) for n in rows]
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen, rng=rng), want_lse=True)
    check_tree(s, seen, out, lse)
    assert int(s.batch.errors) == 0


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_any_masks_windows_and_wide_words(kv, case, bits):
    dtype, dim, heads, q_heads, page_tokens, rows, before = SHAPES[case]
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], dtype, bits, q_heads, heads, dim, page_tokens, seed=50 + case)
    rng = random.Random(100 + case)
    seen = [np.random.RandomState(case * 10 + i).rand(n, n) < rng.choice([0.1, 0.5, 0.9]) for i, n in enumerate(rows)]
    for x in seen:
        if len(x):
            x[0] = False                                                 # rows that see none of the rows, not even themselves
            x[-1] = True
    stride = -(-max(rows) // 64) + 2
    for window in (0, max(rows), max(rows) + 37):
        out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen, stride, rng), window=window, want_lse=True, scale=0.11)
        check_tree(s, seen, out, lse, window, 0.11)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("rows,q_heads", [([3, 8], 4), ([30, 32], 4), ([64, 40], 8), ([150, 10], 4)])
def test_long_contexts_are_split_and_joined(kv, rows, q_heads, bits):
    s = Setup(kv, rows, [9003, 4446], BF16, bits, q_heads, 2, 128, 16, seed=len(rows) + q_heads)
    rng = random.Random(q_heads)
    seen = [TR.ancestors(some_tree(rng, n)) for n in rows]
    for window in (0, 4096):
        assert kv.attend_workspace(s.cache, s.batch, q_heads, window, tree=True) > 0
        got = [kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen, rng=rng), window=window, want_lse=True) for _ in range(2)]
        check_tree(s, seen, *got[0], window)
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_rows_in_front_of_the_sequence(kv):
    # fewer tokens than rows: the first rows have none, and masks that name them name nothing
    rows, tokens = [10, 100, 3], [4, 37, 0]
    for q_heads in (2, 8):
        s = Setup(kv, rows, tokens, BF16, 16, q_heads, 2, 64, 16, seed=9)
        seen = [np.random.RandomState(i).rand(n, n) < 0.4 for i, n in enumerate(rows)]
        out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen), want_lse=True)
        check_tree(s, seen, out, lse)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("rows", [[9, 12], [70, 90]])
def test_rows_that_are_not_seen_have_no_influence(kv, rows, bits):
    # one branch's keys and values are infinities and NaN; rows of the other branches are as with values of zero in their place
    s = Setup(kv, rows, [rows[0] + 50, rows[1] + 7], BF16, bits, 4, 2, 128, 16, seed=11)
    rng = random.Random(4)
    trees = [some_tree(rng, n) for n in rows]
    seen = [TR.ancestors(t) for t in trees]
    q, masks = s.q.cuda(), masks_of(seen)
    base = kv.attend(s.cache, s.batch, q, tree=masks, want_lse=True)
    for i, n in enumerate(rows):
        place = s.tokens[i] - n + 3                                      # row 3
        page, slot = int(s.table[i, place // 16]), place % 16
        for pool, bad in ((s.k_pool, math.nan), (s.v_pool, math.inf)):
            if bits == 16:
                pool[page, slot] = bad
            else:
                n_codes = 16 * 2 * 64
                pool[page, n_codes + slot * 2 * 4:n_codes + (slot + 1) * 2 * 4] = 255
    out, lse = kv.attend(s.cache, s.batch, q, tree=masks, want_lse=True)
    blind = torch.from_numpy(np.concatenate([~x[:, 3] for x in seen]))
    assert torch.equal(out.cpu()[blind], base[0].cpu()[blind]) and torch.equal(lse.cpu()[blind], base[1].cpu()[blind])
    assert bool(out.cpu()[~blind].isnan().all()) and bool(lse.cpu()[~blind].isnan().all())


@pytest.mark.parametrize("rows", [[6, 9], [80, 70]])
def test_infinite_values_reach_the_rows_that_see_them(kv, rows):
    s = Setup(kv, rows, [rows[0] + 20, rows[1] + 100], BF16, 16, 4, 2, 128, 16, seed=12)
    seen = [TR.ancestors(some_tree(random.Random(8), n)) for n in rows]
    q, masks = s.q.cuda(), masks_of(seen)
    base = kv.attend(s.cache, s.batch, q, tree=masks)
    for i, n in enumerate(rows):
        place = s.tokens[i] - n + 2
        s.v_pool[int(s.table[i, place // 16]), place % 16, :, 5] = -math.inf
    out = kv.attend(s.cache, s.batch, q, tree=masks).cpu()
    sees = torch.from_numpy(np.concatenate([x[:, 2] for x in seen]))
    assert bool((out[sees][:, :, 5] == -math.inf).all())
    out[sees, :, 5] = 0
    want = base.cpu()
    want[sees, :, 5] = 0
    assert torch.equal(out, want)


@pytest.mark.parametrize("rows", [[6, 9], [80, 70]])
@pytest.mark.parametrize("long", [False, True])
def test_values_near_the_largest(kv, rows, long):
    # sums of weights times values pass 32 bits; outputs do not
    s = Setup(kv, rows, [rows[0] + (6000 if long else 20), rows[1] + 100], BF16, 16, 4, 2, 64, 16, seed=13)
    s.v_pool.mul_(2.0 ** 125)
    seen = [TR.ancestors(some_tree(random.Random(9), n)) for n in rows]
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen), want_lse=True)
    check_tree(s, seen, out, lse)


def test_a_chain_is_causal_attention(kv):
    s = Setup(kv, [5, 1, 64, 30], [305, 1, 64, 900], FP16, 4, 4, 2, 128, 16, seed=14)
    parents = torch.tensor([i - 1 for n in s.rows for i in range(n)], **I32)
    masks, deep = kv.tree_masks(parents, s.batch.row_start, 64)
    assert deep.tolist() == [i for n in s.rows for i in range(n)]
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks, want_lse=True)
    s.check_attend(out, lse)


def test_wrong_pages_and_sequences(kv):
    s = Setup(kv, [4, 6, 5], [70, 40, 90], BF16, 16, 4, 2, 64, 16, seed=15)
    seen = [TR.ancestors(some_tree(random.Random(2), n)) for n in s.rows]
    table = s.batch.page_table
    table[0, 1] = 1 << 30                                                # tokens 16 .. 31 of the first
    s.batch.kv_len[1] = 10_000                                           # and the second is left out
    held = torch.zeros(15, 4, 64, dtype=BF16, device="cuda").fill_(7)
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen), want_lse=True, out=held)
    from paper_2604_00368_amd import binding as T
    assert int(s.batch.errors) == T.TENT_KV_BAD_SEQUENCE | T.TENT_KV_BAD_PAGE
    assert bool((out[4:10] == 7).all())
    see = TR.visible(seen[0], 70)
    see[:, 16:32] = False
    k, v = (s.values(p)[np.where(s.table[0, :5].numpy() < len(p), s.table[0, :5].numpy(), 0)].reshape(-1, 2, 64)[:70] for p in (s.k_pool, s.v_pool))
    want, _, mass, size = TR.attend(s.q[:4].double().numpy(), k, v, see, 1 / 8)
    bound, _ = R.attend_bounds(want, mass, size, 70, 64, BF16)
    assert (np.abs(out[:4].double().cpu().numpy() - want) <= bound).all()
    check_tree(s, seen, out, lse, skip=(0, 1))


# ---- 33 to 64 lines: two waves to 32 of them, each with half of a tile's tokens -------------------
HALVES = [(BF16, 64), (BF16, 128), (BF16, 256), (FP16, 128)]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype,dim", HALVES)
def test_trees_of_33_to_64_lines(kv, dtype, dim, bits):
    # tokens in the first wave's half of a tile only, in both, and (of a window) in the second's only; lines of the second 32 or none
    rows, before = [17, 32, 1, 0, 16, 20, 31], [0, 14, 700, 5, 16, 44, 129]
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], dtype, bits, 4, 2, dim, 16, seed=dim, spare_bytes=32)
    rng = random.Random(dim)
    trees = [TR.ancestors(some_tree(rng, n)) for n in rows]
    masks = [np.random.RandomState(dim + i).rand(n, n) < 0.3 for i, n in enumerate(rows)]
    for x in masks:
        if len(x):
            x[0] = False
    for seen in (trees, masks):
        for window in (0, 32, 45):
            out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen, 3, rng), window=window, want_lse=True)
            check_tree(s, seen, out, lse, window)
    assert int(s.batch.errors) == 0


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype,dim", HALVES)
def test_33_to_64_lines_over_a_split_context(kv, dtype, dim, bits):
    rows = [20, 32]
    s = Setup(kv, rows, [2600, 1031], dtype, bits, 4, 2, dim, 16, seed=2 * dim)
    seen = [TR.ancestors(some_tree(random.Random(dim), n)) for n in rows]
    for window in (0, 900):
        assert kv.attend_workspace(s.cache, s.batch, 4, window, tree=True) > 0
        got = [kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen), window=window, want_lse=True) for _ in range(2)]
        check_tree(s, seen, *got[0], window)
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_33_to_64_lines_in_front_of_the_sequence(kv):
    rows, tokens = [20, 32, 17], [4, 31, 0]
    s = Setup(kv, rows, tokens, BF16, 16, 4, 2, 64, 16, seed=9)
    seen = [np.random.RandomState(i).rand(n, n) < 0.4 for i, n in enumerate(rows)]
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen), want_lse=True)
    check_tree(s, seen, out, lse)


@pytest.mark.parametrize("bits", [16, 4])
def test_33_to_64_lines_without_influence_of_what_is_not_seen(kv, bits):
    test_rows_that_are_not_seen_have_no_influence(kv, [20, 30], bits)
    test_rows_that_are_not_seen_have_no_influence(kv, [32, 17], bits)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("place", [2, 37, 63, 64, 90])
def test_33_to_64_lines_and_infinite_values(kv, dim, place):
    # a token of either wave's half, of a tile that every line sees whole or of one that is masked
    rows, before = [20, 32], [100, 3]
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], BF16, 16, 4, 2, dim, 16, seed=12)
    seen = [TR.ancestors(some_tree(random.Random(8), n)) for n in rows]
    q, masks = s.q.cuda(), masks_of(seen)
    base, base_lse = kv.attend(s.cache, s.batch, q, tree=masks, want_lse=True)
    at = [place, 3 + place % 32]
    for i in range(2):
        s.v_pool[int(s.table[i, at[i] // 16]), at[i] % 16, :, 5] = -math.inf
    out, lse = kv.attend(s.cache, s.batch, q, tree=masks, want_lse=True)
    sees = torch.from_numpy(np.concatenate([TR.visible(x, t)[:, a] for x, t, a in zip(seen, s.tokens, at)]))
    assert torch.equal(lse, base_lse)
    out, want = out.cpu(), base.cpu()
    assert bool(sees.any()) and bool((out[sees][:, :, 5] == -math.inf).all())
    out[sees, :, 5] = want[sees, :, 5] = 0
    assert torch.equal(out, want)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("before", [(20, 100), (6000, 100), (0, 44)])
def test_33_to_64_lines_and_values_near_the_largest(kv, dim, before):
    rows = [20, 32]
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], BF16, 16, 4, 2, dim, 16, seed=13)
    s.v_pool.mul_(2.0 ** 125)
    seen = [TR.ancestors(some_tree(random.Random(9), n)) for n in rows]
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen), want_lse=True)
    check_tree(s, seen, out, lse)


@pytest.mark.parametrize("bits", [16, 4])
def test_33_to_64_lines_wrong_pages_and_sequences(kv, bits):
    from paper_2604_00368_amd import binding as T
    s = Setup(kv, [20, 32, 17], [90, 40, 130], BF16, bits, 4, 2, 64, 16, seed=15)
    seen = [TR.ancestors(some_tree(random.Random(2), n)) for n in s.rows]
    s.batch.page_table[0, 2] = 1 << 30                                   # tokens 32 .. 47 of the first: the second wave's
    s.batch.kv_len[1] = 10_000                                           # and the second is left out
    held = torch.zeros(69, 4, 64, dtype=BF16, device="cuda").fill_(7)
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), tree=masks_of(seen), want_lse=True, out=held)
    assert int(s.batch.errors) == T.TENT_KV_BAD_SEQUENCE | T.TENT_KV_BAD_PAGE
    assert bool((out[20:52] == 7).all())
    see = TR.visible(seen[0], 90)
    see[:, 32:48] = False
    want, _, mass, size = TR.attend(s.q[:20].double().numpy(), s.held(s.k_pool, 0), s.held(s.v_pool, 0), see, 1 / 8)
    bound, _ = R.attend_bounds(want, mass, size, 90, 64, BF16)
    assert (np.abs(out[:20].double().cpu().numpy() - want) <= bound).all()
    check_tree(s, seen, out, lse, skip=(0, 1))


# ---- verify --------------------------------------------------------------------------------------
def probabilities(rng, rows, vocab, dtype, sharp=3.0):
    x = rng.randn(rows, vocab) * sharp
    x = np.exp(x - x.max(1, keepdims=True))
    return torch.from_numpy(x / x.sum(1, keepdims=True)).to(dtype)


class Drafts:
    """Sequences of drafted tokens, and two models that agree for the most part."""

    def __init__(self, kv, rows, vocab, dtype=torch.float32, drawn=True, chain=False, seed=0, spare=0):
        self.kv, self.rows, self.vocab = kv, rows, vocab
        rng, pick = np.random.RandomState(seed), random.Random(seed)
        n = sum(rows)
        self.starts = [sum(rows[:i]) for i in range(len(rows) + 1)]
        self.trees = [[i - 1 if i == 0 or chain or pick.random() < 0.4 else pick.randrange(i) for i in range(r)] for r in rows]
        self.parents = torch.tensor([p for t in self.trees for p in t], dtype=torch.int32)
        self.target = probabilities(rng, n, vocab, dtype)
        near = self.target.double().numpy() ** 0.8 * np.exp(0.5 * rng.randn(n, vocab))
        self.draft = torch.from_numpy(near / near.sum(1, keepdims=True)).to(dtype) if drawn else None
        self.tokens = torch.zeros(n, dtype=torch.int32)
        near = torch.from_numpy(near)
        for t, b in zip(self.trees, self.starts):
            for i, p in enumerate(t):
                q = near[b + max(p, 0)]
                self.tokens[b + i] = int(q.multinomial(1, generator=torch.Generator().manual_seed(seed + b + i))) if drawn or pick.random() < 0.3 else int(q.topk(min(vocab, 4)).indices[i % min(vocab, 4)])
        self.accept, self.next = torch.from_numpy(rng.rand(n)).float().clamp(max=1 - 2 ** -24), torch.from_numpy(rng.rand(len(rows))).float().clamp(max=1 - 2 ** -24)
        z = torch.zeros(len(rows), **I32)
        self.batch = kv.Batch(torch.zeros(len(rows), 1, **I32), z, torch.tensor(self.starts, **I32), n, max(max(rows), 1) if n else 0, 0)
        self.spare = spare

    def on_gpu(self, x):
        if x is None or not self.spare:
            return None if x is None else x.cuda()
        wide = torch.full((x.shape[0], x.shape[1] + self.spare), 0.5, dtype=x.dtype, device="cuda")
        wide[:, :x.shape[1]] = x
        return wide[:, :x.shape[1]]

    def run(self, parents=True, **more):
        return self.kv.verify(self.batch, self.on_gpu(self.target), self.tokens.cuda(), self.accept.cuda(), self.next.cuda(),
                              parents=self.parents.cuda() if parents else None, draft=self.on_gpu(self.draft), **more)

    def want(self, i):
        at = slice(self.starts[i], self.starts[i + 1])
        f = lambda t: None if t is None else t[at].double().numpy()  # noqa: E731
        return TR.verify(f(self.target), f(self.draft), self.tokens[at].tolist(), self.trees[i], self.accept[at].double().tolist(), float(self.next[i].double()))

    def check(self, path, counts, token):
        path, counts, token = path.cpu().numpy(), counts.tolist(), token.tolist()
        lengths = []
        for i, n in enumerate(self.rows):
            want, x = ([], -1) if n == 0 else self.want(i)
            assert (counts[i], token[i]) == (len(want), x), (i, counts[i], token[i], want, x)
            assert path[i].tolist() == want + [-1] * (path.shape[1] - len(want)), i
            lengths.append(len(want))
        return lengths


VOCABS = [1, 2, 63, 1000, 2047, 2048, 2049, 8191, 8192, 8193, 16385, 50257, 131072, 131073, 200003]


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("vocab", VOCABS)
def test_verify(kv, vocab, drawn):
    d = Drafts(kv, [1, 5, 0, 9, 2, 17, 33, 8], vocab, torch.float32, drawn, seed=vocab)
    lengths = d.check(*d.run())
    assert int(d.batch.errors) == 0 and (vocab < 3 or not drawn or max(lengths) > 1)


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("dtype", [BF16, FP16, torch.float32])
@pytest.mark.parametrize("spare", [0, 1, 3, 8])
@pytest.mark.parametrize("vocab", [20011, 131075])
def test_verify_types_and_strides(kv, dtype, drawn, spare, vocab):
    d = Drafts(kv, [6, 12, 3, 7], vocab, dtype, drawn, seed=spare + 1, spare=spare)
    d.check(*d.run())


def test_verify_rows_one_after_the_other(kv):
    for seed in range(4):
        d = Drafts(kv, [8] * 20 + [1, 70], 9001, torch.float32, seed % 2 == 0, chain=True, seed=seed)
        assert max(d.check(*d.run(parents=False))) > 2 or seed % 2
        d.check(*d.run(parents=True))


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_trees_of_many_rows(kv, drawn):
    # several words of rows, and many rows behind one
    for seed, wide in ((1, False), (2, True)):
        d = Drafts(kv, [150, 70, 300], 700, torch.float32, drawn, seed=seed)
        if wide:
            d.trees = [[-1] + [0] * (n - 1) for n in d.rows]
            d.parents = torch.tensor([p for t in d.trees for p in t], dtype=torch.int32)
            d.accept.mul_(0.3).add_(0.7).clamp_(max=1 - 2 ** -24)        # mostly refused
        d.check(*d.run())


@pytest.mark.parametrize("vocab", [30000, 140001])
def test_verify_where_every_row_is_refused(kv, vocab):
    # sums for up to 24 refusals of a sequence, the first of them ahead or not
    d = Drafts(kv, [25, 25, 3], vocab, torch.float32, True, seed=3)
    d.trees = [[-1] + [0] * (n - 1) for n in d.rows]
    d.parents = torch.tensor([p for t in d.trees for p in t], dtype=torch.int32)
    least = d.target.argmin(1).to(torch.int32)
    for b, n in zip(d.starts, d.rows):
        d.tokens[b:b + n] = least[b]
    d.draft[:, :] = 0.9 * d.draft
    for b in d.starts[:-1]:
        d.draft[b, least[b].item()] = 0.1
    d.accept.fill_(0.9)
    assert d.check(*d.run()) == [1, 1, 1]


def test_verify_numbers_at_their_ends_and_borders(kv):
    vocab = 8200
    for drawn in (True, False):
        for accept, next_ in ((0.0, 0.0), (1 - 2 ** -24, 1 - 2 ** -24), (0.0, 1 - 2 ** -24)):
            d = Drafts(kv, [4, 6, 5], vocab, torch.float32, drawn, seed=4)
            d.accept.fill_(accept)
            d.next.fill_(next_)
            d.check(*d.run())
    # probabilities that are powers of two: sums are exact, and a number falls on a token's border
    d = Drafts(kv, [1] * 9, vocab, torch.float32, False, seed=5)
    d.target.zero_()
    d.target[:, 100] = 0.25
    d.target[:, 8191] = 0.25
    d.target[:, 8192] = 0.5
    d.next = torch.tensor([0.0, 0.25 - 2 ** -26, 0.25, 0.5 - 2 ** -25, 0.5, 0.5 + 2 ** -24, 0.75, 1 - 2 ** -24, 0.1])
    assert d.run()[2].tolist() == [100, 100, 8191, 8191, 8192, 8192, 8192, 8192, 100]


def test_verify_certain_targets(kv):
    # a target of one token each: what is accepted is what it says
    d = Drafts(kv, [6, 9, 12], 9000, torch.float32, False, seed=6)
    best = d.target.argmax(1)
    d.target.zero_()
    d.target[torch.arange(len(best)), best] = 1.0
    for t, b in zip(d.trees, d.starts):
        for i, p in enumerate(t):
            if p >= 0 and i % 3:
                d.tokens[b + i] = int(best[b + p])
    lengths = d.check(*d.run())
    assert max(lengths) > 1


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_what_is_no_probability_counts_as_nothing(kv, drawn):
    d = Drafts(kv, [5, 7, 9, 2], 12000, torch.float32, drawn, seed=7)
    for x in (d.target, d.draft) if drawn else (d.target,):
        x[:, 3::97] = math.nan
        x[:, 5::89] = math.inf
        x[:, 7::83] = -0.25
    d.target[0] = 0                                                      # nothing is left: -1 where the way ends there
    d.target[d.starts[3]:] = math.nan
    d.check(*d.run())


def test_verify_equal_models_leave_nothing(kv):
    # what was refused (by a number that is not below 1) leaves a residual of zeros: the target's own probabilities stand in
    d = Drafts(kv, [3, 4], 9000, torch.float32, True, seed=8)
    d.draft = d.target.clone()
    d.accept.fill_(1.0)
    assert d.check(*d.run()) == [1, 1]


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_tokens_outside_the_vocabulary(kv, drawn):
    from paper_2604_00368_amd import binding as T
    d = Drafts(kv, [5, 7, 9], 8500, torch.float32, drawn, seed=9)
    d.tokens[2], d.tokens[7], d.tokens[14] = 8500, -1, 1 << 30
    d.check(*d.run())
    assert int(d.batch.errors) == T.TENT_KV_BAD_TOKEN
    d = Drafts(kv, [1, 1], 50, torch.float32, drawn, seed=9)
    d.tokens.fill_(-5)                                                   # the first row's is not read
    d.check(*d.run())
    assert int(d.batch.errors) == 0


def test_verify_rows_behind_none(kv):
    d = Drafts(kv, [6, 70], 300, torch.float32, False, seed=10)
    for t in d.trees:
        t[2], t[3], t[4] = 2, 5, -7
    d.trees[1][66] = 1 << 20
    d.parents = torch.tensor([p for t in d.trees for p in t], dtype=torch.int32)
    d.check(*d.run())


def test_verify_sequences_that_are_left_out(kv):
    from paper_2604_00368_amd import binding as T
    d = Drafts(kv, [3, 4, 5], 9000, torch.float32, True, seed=11)
    d.batch.kv_len[1] = 5                                                # more than max_kv
    path, counts, token = d.run()
    assert counts.tolist()[1] == 0 and token.tolist()[1] == -1 and bool((path[1] == -1).all())
    assert int(d.batch.errors) == T.TENT_KV_BAD_SEQUENCE
    for i in (0, 2):
        want, x = d.want(i)
        assert (counts[i], token[i]) == (len(want), x)


def test_verify_no_rows(kv):
    z = torch.zeros(2, **I32)
    batch = kv.Batch(torch.zeros(2, 1, **I32), z, torch.zeros(3, **I32), 0, 0, 0)
    e = torch.zeros(0, device="cuda")
    path, counts, token = kv.verify(batch, e.reshape(0, 30), e.int(), e, z.float())
    assert path.shape == (2, 0) and counts.tolist() == [0, 0] and token.tolist() == [-1, -1]


@pytest.mark.parametrize("drawn", [True, False])
def test_tokens_are_distributed_as_the_target_says(kv, drawn):
    # two tokens behind the first row, drawn each by itself (or always the same two): the first token that comes out is the target's
    n, vocab, g = 60000, 5, torch.Generator().manual_seed(1)
    p, q = torch.tensor([0.1, 0.35, 0.05, 0.3, 0.2]), torch.tensor([0.4, 0.1, 0.2, 0.05, 0.25])
    tokens = torch.zeros(n, 3, dtype=torch.int32)
    tokens[:, 1:] = q.multinomial(2 * n, True, generator=g).reshape(n, 2).int() if drawn else torch.tensor([1, 4]).int()
    z, after = torch.zeros(n, **I32), torch.tensor([-1, 0, 0], **I32).repeat(n)
    batch = kv.Batch(z[:, None], z, torch.arange(n + 1, **I32) * 3, 3 * n, 3, 0)
    rows = lambda x: x.cuda().expand(3 * n, vocab).contiguous()  # noqa: E731
    path, counts, token = kv.verify(batch, rows(p), tokens.flatten().cuda(), torch.rand(3 * n, generator=g).cuda(), torch.rand(n, generator=g).cuda(), parents=after,
                                    draft=rows(q) if drawn else None)
    first = torch.where(counts.cpu() > 1, tokens.gather(1, path.cpu()[:, 1:2].clamp(min=0).long())[:, 0], token.cpu())
    got = torch.bincount(first, minlength=vocab).double() / n
    assert (got - p).abs().max() < 5 * math.sqrt(0.25 / n)               # five standard deviations of a share at most
