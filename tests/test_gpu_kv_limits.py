"""Paged cache operators at the ends of what their types hold: infinities, NaN, the largest and the least values, and what is noted of
wrong input, on a GPU against their definitions in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv_reference as R  # noqa: E402
from test_gpu_kv import Setup, kv  # noqa: E402,F401

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


# ---- values that are not finite ------------------------------------------------------------------
class Marks:
    """Attention of a setup with values that are not finite put into V of some tokens, against the finite setup's outputs."""

    def __init__(self, s, window=0, causal=True, gone=()):
        self.s, self.window, self.causal = s, window, causal
        self.clean = s.kv.attend(s.cache, s.batch, s.q.cuda(), window=window, causal=causal)
        self.want, self.bound = (np.zeros((s.n_rows, s.q_heads, s.dim)) for _ in range(2))
        for i, n in enumerate(s.rows):
            at = slice(s.starts[i], s.starts[i] + n)
            k, v = (np.delete(s.held(p, i), list(gone) if i == 0 else [], 0) for p in (s.k_pool, s.v_pool))
            assert causal or not window                                  # tokens that are gone shift no window then
            want, _, mass, size = R.attend(s.q[at].double().numpy(), k, v, 1 / math.sqrt(s.dim), window, causal)
            self.want[at] = want
            self.bound[at] = R.attend_bounds(want, mass, size, s.tokens[i], s.dim, s.dtype)[0]

    def sees(self, row, token):
        """Whether a row of the first sequence sees a token of it."""
        n, total = self.s.rows[0], self.s.tokens[0]
        hi = total - n + row + 1 if self.causal else total
        return token < hi and (not self.window or token >= hi - self.window)

    def check(self, token, head):
        """Marks one token of the first sequence, for one head, runs, checks every output, and takes the marks back."""
        s = self.s
        page, slot = int(s.table[0, token // s.page_tokens]), token % s.page_tokens
        group = s.q_heads // s.heads
        heads = slice(head * group, (head + 1) * group)
        expect = {3: math.inf, 40: -math.inf, 61: math.nan}
        if s.bits == 16:
            row = s.v_pool[page, slot, head]
            old = row.clone()
            for d, x in expect.items():
                row[d] = x
        else:
            at = s.page_tokens * s.heads * s.dim // 2 + (slot * s.heads + head) * (s.dim // 32)
            row = s.v_pool[page, at + 1:at + 2]                          # the scale of dims 32 .. 63
            old = row.clone()
            row.fill_(255)
            expect = dict.fromkeys(range(32, 64), math.nan)
        out = s.kv.attend(s.cache, s.batch, s.q.cuda(), window=self.window, causal=self.causal)
        row.copy_(old)
        see = np.zeros(s.n_rows, bool)
        see[:s.rows[0]] = [self.sees(r, token) for r in range(s.rows[0])]
        assert see.any()
        hit = np.zeros(out.shape, bool)
        for d in expect:
            hit[see, heads, d] = True
        got = out.double().cpu().numpy()
        for d, x in expect.items():
            part = got[see, heads, d]
            assert (np.isnan(part) if math.isnan(x) else part == x).all(), (token, head, d, part.ravel()[:4])
        assert torch.equal(out[torch.from_numpy(~see).cuda()], self.clean[torch.from_numpy(~see).cuda()]), token
        assert (np.abs(got - self.want) <= self.bound)[~hit].all(), token
        return int(see.sum())


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("rows,heads,dim", [([60, 3], 1, 128), ([140, 3], 2, 64), ([60, 3], 1, 256), ([5, 3], 1, 128)])
def test_values_that_are_not_finite_in_split_and_windowed_contexts(kv, rows, heads, dim, dtype, bits):
    # A window makes lines begin at tokens of their own, so that a tile at the end of a split may be half of one that every line sees;
    # and around the first and the last tokens that lines see.
    tokens, window = [9001, 4447], 2500
    s = Setup(kv, rows, tokens, dtype, bits, 4 * heads, heads, dim, 16, seed=dim + heads)
    assert kv.attend_workspace(s.cache, s.batch, s.q_heads, window=window) > 0
    m = Marks(s, window)
    lo = tokens[0] - rows[0] + 1 - window
    some = 0
    for token in [lo, lo + 31, lo + rows[0] - 1, *range(lo + 40, lo + 700, 24), 8000, tokens[0] - rows[0], tokens[0] - 1]:
        some += m.check(token, heads - 1) < rows[0]
    assert some >= 2                                                     # tokens that some rows see and others do not, too


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("rows,dim", [(70, 128), (3, 128), (40, 256), (100, 64)])
def test_values_that_are_not_finite_beside_a_bad_page(kv, rows, dim, dtype, bits):
    s = Setup(kv, [rows, 2], [200, 9], dtype, bits, 2, 1, dim, 16, seed=dim)
    s.batch.page_table[0, 2] = -5                                        # tokens 32 .. 47 are not seen
    m = Marks(s, causal=False, gone=range(32, 48))
    for token in (0, 31, 48, 50, 63, 64, 130, 191, 199):
        m.check(token, 0)
    assert int(s.batch.errors) == 2


# ---- scores that are not finite ------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("rows,tokens", [([4, 1], [70, 40]), ([100, 30], [150, 40]), ([4, 1], [9001, 4447]), ([100, 2], [9001, 4447])])
def test_logsumexp_of_scores_that_are_not_finite(kv, rows, tokens, dtype):
    s = Setup(kv, rows, tokens, dtype, 16, 2, 1, 128, 16, seed=7)
    first = s.starts[1]
    q = s.q.cuda()
    q[:, :, 0] = 0.5
    q[first - 1, 0, 0], q[first - 1, 1, 0] = -0.5, math.nan
    page, slot = int(s.table[0, 20 // 16]), 20 % 16
    s.k_pool[page, slot, 0, 0] = math.inf                                # token 20 of the first sequence: a score of infinity
    out, lse = kv.attend(s.cache, s.batch, q, want_lse=True)
    assert bool((lse[:first - 1] == math.inf).all()) and bool(out[:first - 1].isnan().all())
    assert bool(lse[first - 1, 0].isfinite()) and bool(out[first - 1, 0].isfinite().all())     # minus infinity: not seen
    assert bool(lse[first - 1, 1].isnan()) and bool(out[first - 1, 1].isnan().all())
    s.q = q.cpu()
    s.check_attend(out, lse, skip=(0,))
    s.k_pool[page, slot, 0, 1] = math.nan                                # and now none
    _, lse = kv.attend(s.cache, s.batch, q, want_lse=True)
    assert bool(lse[:first].isnan().all())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows,tokens", [([4, 1], [70, 40]), ([100, 30], [150, 40]), ([4, 1], [9001, 4447]), ([100, 2], [9001, 4447])])
def test_rows_of_scores_of_minus_infinity_are_zeros_whatever_the_values(kv, rows, tokens, causal, dtype):
    s = Setup(kv, rows, tokens, dtype, 16, 2, 1, 64, 16, seed=7)
    q = s.q.cuda()
    q[:s.starts[1], :, 0] = 1.0
    pages = s.table[0, :-(-tokens[0] // 16)].long().cuda()
    s.k_pool[pages, :, :, 0] = -math.inf
    s.v_pool[pages, :, :, 5], s.v_pool[pages, :, :, 6] = math.inf, math.nan
    out, lse = kv.attend(s.cache, s.batch, q, causal=causal, want_lse=True)
    assert not out[:s.starts[1]].any() and bool((lse[:s.starts[1]] == -math.inf).all())
    s.check_attend(out, lse, causal=causal, skip=(0,))


# ---- the ends of the type's range ----------------------------------------------------------------
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("power", [125, -128])
@pytest.mark.parametrize("rows,tokens,q_heads,heads,dim", [
    ([1], [1], 2, 1, 128), ([1, 5], [300, 40], 8, 2, 64), ([3, 2], [65, 700], 8, 1, 256), ([100, 33], [700, 33], 4, 2, 128), ([50, 40], [300, 40], 4, 1, 256),
    ([1, 1], [9001, 4447], 8, 2, 128), ([60, 3], [9001, 4447], 4, 1, 64), ([60, 3], [9001, 4447], 4, 1, 128)])
def test_attend_values_near_the_ends_of_bfloat16(kv, rows, tokens, q_heads, heads, dim, power, bits):
    # weights times values, and their sums, pass what 32 bits hold long before the outputs do
    s = Setup(kv, rows, tokens, BF16, bits, q_heads, heads, dim, 16, seed=dim)
    s.v16 = (s.v16.double().clamp(-4, 4) * 2.0 ** power).to(BF16)
    s.v16[..., ::7] = (s.v16[..., ::7].double() * 2.0 ** (-power)).to(BF16)      # ordinary values beside them
    s.v_pool = s.pool(s.v16)
    s.cache = s.make_cache(s.k_pool, s.v_pool)
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), want_lse=True)
    assert bool(out.isfinite().all())
    s.check_attend(out, lse)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("rows,tokens,q_heads,heads,dim", [
    ([3, 2], [300, 40], 4, 2, 64), ([100, 3], [300, 40], 4, 2, 128), ([40, 3], [300, 40], 4, 1, 256), ([4, 2], [2001, 1100], 4, 2, 128), ([60, 3], [2001, 1100], 4, 1, 128)])
def test_large_values_beside_values_that_are_not_finite(kv, rows, tokens, q_heads, heads, dim, window, bits):
    # dimensions whose sums pass 32 bits in rows that see infinities or NaN in others, of a first, a middle and a last token
    s = Setup(kv, rows, tokens, BF16, bits, q_heads, heads, dim, 16, seed=dim)
    s.v16 = (s.v16.double().clamp(-4, 4) * 2.0 ** 125).to(BF16)
    s.v_pool = s.pool(s.v16)
    s.cache = s.make_cache(s.k_pool, s.v_pool)
    scale = 1 / math.sqrt(dim)
    want, bound = (np.zeros((s.n_rows, q_heads, dim)) for _ in range(2))
    for i, n in enumerate(rows):
        at = slice(s.starts[i], s.starts[i] + n)
        want[at], _, mass, size = R.attend(s.q[at].double().numpy(), s.held(s.k_pool, i), s.held(s.v_pool, i), scale, window, True)
        bound[at] = R.attend_bounds(want[at], mass, size, tokens[i], dim, BF16)[0]
    marked = [tokens[0] - rows[0] - 39, tokens[0] - rows[0] - 2, tokens[0] - 1]
    dims = slice(5, 6) if bits == 16 else slice(32, 64)
    for t in marked:
        page, slot = int(s.table[0, t // 16]), t % 16
        if bits == 16:
            s.v_pool[page, slot, 0, dims] = math.nan
        else:
            s.v_pool[page, 16 * heads * dim // 2 + slot * heads * (dim // 32) + 1] = 255
    out = kv.attend(s.cache, s.batch, s.q.cuda(), window=window).double().cpu().numpy()
    hit = np.zeros(out.shape, bool)
    for r in range(rows[0]):
        hi = tokens[0] - rows[0] + r + 1
        if any((hi - window if window else 0) <= t < hi for t in marked):
            hit[r, :q_heads // heads, dims] = True
    assert hit.any() and np.isnan(out[hit]).all()
    assert (np.abs(out - want) <= bound)[~hit].all()


@pytest.mark.parametrize("rows,tokens", [([4, 2], [300, 40]), ([100, 30], [300, 40]), ([60, 2], [9001, 4447]), ([4, 2], [9001, 4447])])
def test_rows_that_do_not_see_large_values_do_not_change(kv, rows, tokens):
    s = Setup(kv, rows, tokens, BF16, 16, 4, 2, 128, 16, seed=2)
    q = s.q.cuda()
    clean, lse = kv.attend(s.cache, s.batch, q, want_lse=True)
    seen_from = rows[0] // 2                                             # of the first sequence, by this row and those behind it
    token = tokens[0] - rows[0] + seen_from
    s.v_pool[int(s.table[0, token // 16]), token % 16] = 2.0 ** 127
    out, again = kv.attend(s.cache, s.batch, q, want_lse=True)
    see = torch.zeros(s.n_rows, dtype=torch.bool, device="cuda")
    see[seen_from:rows[0]] = True
    assert torch.equal(out[~see], clean[~see]) and torch.equal(lse[~see], again[~see])
    s.check_attend(out, again)


# ---- what is noted -------------------------------------------------------------------------------
def test_a_row_outside_the_rotations_without_a_page_notes_both(kv):
    s = Setup(kv, [1, 2], [30, 2], BF16, 16, 2, 1, 64, 16)
    x = torch.zeros(3, 1, 64, dtype=BF16, device="cuda")
    s.batch.page_table[0, 1] = 1 << 20
    for at, page, noted in ((0, 1 << 20, 2), (40, int(s.table[0, 1]), 4), (40, 1 << 20, 2 | 4)):
        s.batch.errors.zero_()
        s.batch.page_table[0, 1] = page
        positions = torch.tensor([at, 0, 1], dtype=torch.int32, device="cuda")
        kv.append(s.cache, s.batch, x, x, rope=kv.rope_table(40, 64), positions=positions)
        assert int(s.batch.errors) == noted


@pytest.mark.parametrize("n_seqs", [3, 64, 65, 300])
@pytest.mark.parametrize("wrong", ["length", "rows", "beyond"])
def test_wrong_sequences_without_rows_of_their_own_are_noted(kv, n_seqs, wrong):
    # sequence s - 1 has no rows, or rows that are no rows of the call
    rows = [2] + [0] * (n_seqs - 3) + [0, 1]
    s = Setup(kv, rows, [r + 3 for r in rows], BF16, 16, 2, 1, 64, 16)
    x = torch.zeros(3, 1, 64, dtype=BF16, device="cuda")
    calls = (lambda: kv.append(s.cache, s.batch, x, x), lambda: kv.read(s.cache, s.batch), lambda: kv.attend(s.cache, s.batch, s.q.cuda()))
    for call in calls:
        call()
        assert int(s.batch.errors) == 0
    if wrong == "length":
        s.batch.kv_len[n_seqs - 2] = 1 << 20
    elif wrong == "rows":
        s.batch.row_start[n_seqs - 1] = 1                                # it would end before it starts
    else:
        s.batch.row_start[n_seqs] = 4                                    # the last one's rows go past the call's
    for call in calls:
        s.batch.errors.zero_()
        call()
        assert int(s.batch.errors) & 1


# ---- norms ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("power,eps", [(62, 1e-6), (120, 1e-6), (-60, 0.0), (-120, 0.0), (-60, 1e-6), (10, 0.0)])
def test_norms_of_large_and_small_rows(kv, dim, pairs, power, eps, bits):
    # of queries as of keys; every second head is of ordinary size
    s = Setup(kv, [3, 2], [30, 2], BF16, bits, 4, 2, dim, 16)
    q, k, v = (torch.randn(5, h, dim, generator=s.g).to(BF16) for h in (4, 2, 2))
    for x in (q, k):
        x[:, ::2] = (x[:, ::2].double() * 2.0 ** power).to(BF16)
    weights = [(1 + 0.3 * torch.randn(dim, generator=s.g)).to(BF16) for _ in "qk"]
    table = kv.rope_table(30, dim, device="cpu")
    got = kv.append(s.cache, s.batch, k.cuda(), v.cuda(), q=q.cuda(), q_weight=weights[0].cuda(), k_weight=weights[1].cuda(), eps=eps,
                    rope=table.cuda(), rope_pairs=pairs)
    turn = table.double().numpy()[[27, 28, 29, 0, 1]]
    e = float(np.float32(eps))
    want_k = R.to_type(R.norm_rotate(k.double().numpy(), weights[1].double().numpy(), e, turn, dim, pairs), BF16)
    back, _ = kv.read(s.cache, s.batch)
    want = R.decode4(*R.encode4(want_k, BF16)) if bits == 4 else want_k
    assert np.array_equal(back.cpu().double().numpy(), want)
    want = R.norm_rotate(q.double().numpy(), weights[0].double().numpy(), e, turn, dim, pairs)
    # 32-bit arithmetic, or better: a sum of squares over `dim`, a root, a quotient, products; terms of a turn do not exceed the pair's size
    size = 2 * np.abs(want).max(-1, keepdims=True)
    off = np.abs(got.cpu().double().numpy() - want)
    assert (off <= R.half_step(BF16) * np.abs(want) * 1.01 + (dim + 32) * 2.0 ** -24 * size + 2.0 ** -133).all()
    assert int(s.batch.errors) == 0
