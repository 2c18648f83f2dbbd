"""Operators on paged key/value caches on a GPU against their definitions in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def kv():
    assert torch.cuda.is_available()
    from paper_2604_00368_amd import binding, kv as module
    binding.lib()
    return module


def same(got, want):
    """Equal values, NaN where NaN is; says where not."""
    got = got.cpu().double().numpy() if isinstance(got, torch.Tensor) else got
    off = np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))))
    assert not len(off), (len(off), off[0].tolist(), float(got[tuple(off[0])]), float(want[tuple(off[0])]))


class Setup:
    """Pools in use, shuffled page tables, and rows for sequences of `kv` tokens of which `rows` are new."""

    def __init__(self, kv, rows, tokens, dtype=BF16, bits=16, q_heads=4, heads=2, dim=64, page_tokens=16, seed=0, spare_width=0, spare_bytes=0):
        self.kv, self.rows, self.tokens, self.dtype, self.bits = kv, rows, tokens, dtype, bits
        self.q_heads, self.heads, self.dim, self.page_tokens = q_heads, heads, dim, page_tokens
        self.g = torch.Generator().manual_seed(seed)
        pages = [-(-t // page_tokens) for t in tokens]
        n_pages = sum(pages) + 2
        order = torch.randperm(n_pages, generator=self.g).to(torch.int32)
        self.table = torch.full((len(rows), max(max(pages), 1) + spare_width), 0x7FFFFFF0, dtype=torch.int32)
        at = 0
        for i, n in enumerate(pages):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.k16, self.v16 = (torch.randn(n_pages, page_tokens, heads, dim, generator=self.g).to(dtype) for _ in "kv")
        self.n_rows = sum(rows)
        self.starts = [sum(rows[:i]) for i in range(len(rows) + 1)]
        self.batch = kv.Batch(self.table.cuda()[:, :self.table.shape[1]], torch.tensor(tokens, dtype=torch.int32).cuda(),
                              torch.tensor(self.starts, dtype=torch.int32).cuda(), self.n_rows, max(max(rows), 1), max(tokens))
        self.k_pool, self.v_pool = self.pool(self.k16, spare_bytes), self.pool(self.v16, spare_bytes)
        self.cache = self.make_cache(self.k_pool, self.v_pool)
        self.q = (2 * torch.randn(self.n_rows, q_heads, dim, generator=self.g)).to(dtype)

    def packed(self, values):
        """Host bytes of 4-bit pages of 16-bit values."""
        codes, scales = R.encode4(values.double().numpy(), self.dtype)
        n = values.shape[0]
        data = np.concatenate([(codes[..., 0::2] + 16 * codes[..., 1::2]).reshape(n, -1), scales.reshape(n, -1)], 1)
        out = torch.zeros(n, self.kv.packed_page_bytes(self.page_tokens, self.heads, self.dim), dtype=torch.uint8)
        out[:, :data.shape[1]] = torch.from_numpy(data.astype(np.uint8))
        return out

    def pool(self, values, spare_bytes=0):
        data = self.packed(values) if self.bits == 4 else values
        flat = data.reshape(data.shape[0], -1).cuda()
        if spare_bytes:                                                  # pages further apart than they are long
            wide = torch.zeros(flat.shape[0], flat.shape[1] + spare_bytes // flat.element_size(), dtype=flat.dtype, device="cuda")
            wide[:, :flat.shape[1]] = flat
            flat = wide[:, :flat.shape[1]]
        return flat if self.bits == 4 else flat.unflatten(1, data.shape[1:])

    def make_cache(self, k, v):
        if self.bits == 16:
            return self.kv.Cache(k, v)
        return self.kv.Cache(k, v, dtype=self.dtype, page_tokens=self.page_tokens, kv_heads=self.heads, head_dim=self.dim)

    def values(self, pool):
        return R.page_values(pool, self.bits, self.page_tokens, self.heads, self.dim)

    def held(self, pool, i):
        """Tokens of sequence i in 64 bits."""
        pages = self.table[i, :-(-self.tokens[i] // self.page_tokens)].long().numpy()
        return self.values(pool)[pages].reshape(-1, self.heads, self.dim)[:self.tokens[i]]

    def check_attend(self, out, lse, window=0, causal=True, scale=None, skip=()):
        scale = 1 / math.sqrt(self.dim) if scale is None else scale
        for i, n in enumerate(self.rows):
            if i in skip:
                continue
            at = slice(self.starts[i], self.starts[i] + n)
            k, v = self.held(self.k_pool, i), self.held(self.v_pool, i)
            if n > self.tokens[i]:                                       # rows in front of the sequence see nothing
                lead = n - self.tokens[i]
                if causal:
                    assert not out[at][:lead].any() and bool((lse[at][:lead] == -math.inf).all())
                    at, n = slice(at.start + lead, at.stop), n - lead
            want, want_lse, mass, size = R.attend(self.q[at].double().numpy(), k, v, scale, window, causal)
            bound, lse_bound = R.attend_bounds(want, mass, size, max(self.tokens[i], 1), self.dim, self.dtype)
            got, got_lse = out[at].double().cpu().numpy(), lse[at].double().cpu().numpy()
            off = np.abs(got - want)
            assert (off <= bound).all(), (i, float((off / bound).max()), np.unravel_index((off / bound).argmax(), off.shape))
            none = want_lse == -math.inf
            assert (got_lse[none] == -math.inf).all()
            off = np.abs(got_lse - want_lse)[~none]
            assert (off <= (lse_bound + 2.0 ** -23 * np.abs(want_lse))[~none]).all(), (i, float(off.max()))


# ---- append, read, pack --------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype,dim,heads,q_heads,page_tokens,norm,rope,rope_dim", [
    (BF16, 128, 2, 6, 16, True, "half", 128), (FP16, 128, 1, 3, 8, True, "pairs", 64), (BF16, 64, 3, 3, 1, False, "half", 32),
    (FP16, 64, 2, 8, 32, True, "none", 0), (BF16, 256, 2, 2, 4, True, "pairs", 256), (FP16, 256, 1, 5, 64, False, "half", 96),
    (BF16, 128, 8, 32, 16, False, "none", 0), (FP16, 128, 4, 0, 16, True, "half", 16)])
def test_append_and_read(kv, bits, dtype, dim, heads, q_heads, page_tokens, norm, rope, rope_dim):
    rows, before = [1, 0, 37, 2, 0, 5], [0, 9, 21, 63, 0, 1]
    tokens = [r + b for r, b in zip(rows, before)]
    s = Setup(kv, rows, tokens, dtype, bits, max(q_heads, 1), heads, dim, page_tokens, seed=dim + heads, spare_bytes=48)
    n = s.n_rows
    x = torch.randn(n, q_heads + 2 * heads, dim, generator=s.g).to(dtype)          # one tensor, as a projection leaves it
    x[0, q_heads] = 0                                                    # a key of zeros
    x[1, q_heads:] *= 2 ** -12
    x[2, q_heads:] *= 2 ** 9
    f = x.cuda()
    q, k, v = f[:, :q_heads], f[:, q_heads:q_heads + heads], f[:, q_heads + heads:]
    weights = [(1 + 0.3 * torch.randn(dim, generator=s.g)).to(dtype) for _ in "qk"] if norm else [None, None]
    table = kv.rope_table(max(tokens) + 3, rope_dim, device="cpu") if rope != "none" else None
    eps = 1e-5
    before_k, before_v = s.values(s.k_pool), s.values(s.v_pool)
    got = kv.append(s.cache, s.batch, k, v, q=q if q_heads else None, q_weight=weights[0].cuda() if norm and q_heads else None,
                    k_weight=weights[1].cuda() if norm else None, eps=eps, rope=table.cuda() if table is not None else None, rope_pairs=rope == "pairs")
    back_k, back_v = kv.read(s.cache, s.batch)
    position = np.concatenate([np.arange(b, t) for b, t in zip(before, tokens)])
    turn = table.double().numpy()[position] if table is not None else None
    h = x.double().numpy()
    w = [None if y is None else y.double().numpy() for y in weights]
    want_k = R.to_type(R.norm_rotate(h[:, q_heads:q_heads + heads], w[1], np.float32(eps).astype(np.float64), turn, rope_dim, rope == "pairs"), dtype)
    want_v = h[:, q_heads + heads:]
    if bits == 4:
        want_k, want_v = (R.decode4(*R.encode4(y, dtype)) for y in (want_k, want_v))
    same(back_k, want_k)
    same(back_v, want_v)
    # the pools hold that, and nothing else changed
    seq = np.repeat(np.arange(len(rows)), rows)
    page = s.table.numpy()[seq, position // page_tokens]
    before_k[page, position % page_tokens], before_v[page, position % page_tokens] = want_k, want_v
    same(s.values(s.k_pool), before_k)
    same(s.values(s.v_pool), before_v)
    if q_heads:
        want = R.norm_rotate(h[:, :q_heads], w[0], eps, turn, rope_dim, rope == "pairs")
        # 32-bit arithmetic: a sum of squares over `dim`, a root, a quotient, products; terms of a turn do not exceed the pair's size
        size = np.sqrt((want ** 2).reshape(n, q_heads, -1).max(-1, keepdims=True) * 2)
        off = np.abs(got.cpu().double().numpy() - want)
        info = torch.finfo(dtype)
        assert (off <= R.half_step(dtype) * np.abs(want) * 1.01 + (dim + 32) * 2.0 ** -24 * size + info.tiny * info.eps).all()
    else:
        assert got is None
    assert int(s.batch.errors) == 0


@pytest.mark.parametrize("bits", [16, 4])
def test_append_and_read_many_sequences_and_many_heads(kv, bits):
    # more sequences than are looked up in one load, and rows of more heads than a workgroup has in flight at once
    rows = [i % 4 for i in range(97)]
    before = [i % 6 for i in range(97)]
    s = Setup(kv, rows, [r + b for r, b in zip(rows, before)], BF16, bits, 64, 8, 128, 4, seed=8)
    k, v = (torch.randn(s.n_rows, 8, 128, generator=s.g).to(BF16) for _ in "kv")
    table = kv.rope_table(16, 128, device="cpu")
    got = kv.append(s.cache, s.batch, k.cuda(), v.cuda(), q=s.q.cuda(), rope=table.cuda())
    back_k, back_v = kv.read(s.cache, s.batch)
    position = np.concatenate([np.arange(b, b + r) for b, r in zip(before, rows)])
    turn = table.double().numpy()[position]
    want_k, want_v = R.to_type(R.norm_rotate(k.double().numpy(), None, 0, turn, 128, False), BF16), v.double().numpy()
    if bits == 4:
        want_k, want_v = (R.decode4(*R.encode4(y, BF16)) for y in (want_k, want_v))
    same(back_k, want_k)
    same(back_v, want_v)
    want = R.norm_rotate(s.q.double().numpy(), None, 0, turn, 128, False)
    # two products and a sum in 32 bits, then the type; the terms of a turn do not exceed the pair's size
    size = np.abs(s.q.double().numpy()).max(-1, keepdims=True) * 2
    assert (np.abs(got.cpu().double().numpy() - want) <= R.half_step(BF16) * np.abs(want) * 1.01 + 4 * 2.0 ** -24 * size).all()
    assert int(s.batch.errors) == 0


def test_append_in_place_positions_and_rows_outside_the_table(kv):
    s = Setup(kv, [3, 2], [7, 2], dim=64, heads=1, q_heads=2)
    q = torch.randn(5, 2, 64, generator=s.g).to(BF16).cuda()
    k, v = (torch.randn(5, 1, 64, generator=s.g).to(BF16).cuda() for _ in "kv")
    table = kv.rope_table(40, 64)
    at = torch.tensor([30, 2, 39, 40, -1], dtype=torch.int32, device="cuda")        # the last two are outside
    old, old_k = q.clone(), s.values(s.k_pool)
    out = kv.append(s.cache, s.batch, k, v, q=q, q_out=q, rope=table, positions=at)
    assert out is q and int(s.batch.errors) == 4
    want = R.norm_rotate(old[:3].cpu().double().numpy(), None, 0, table.cpu().double().numpy()[[30, 2, 39]], 64, False)
    assert np.abs(q[:3].cpu().double().numpy() - want).max() <= 2 * R.half_step(BF16) * np.abs(want).max()
    assert torch.equal(q[3:], old[3:])
    now = s.values(s.k_pool)
    page = s.table[1, 0]
    assert np.array_equal(now[page], old_k[page])                        # nothing of the second sequence is stored
    assert np.array_equal(now[s.table[0, 0], 4], R.to_type(R.norm_rotate(k[:1].cpu().double().numpy(), None, 0, table.cpu().double().numpy()[[30]], 64, False), BF16)[0])


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim,heads,page_tokens", [(128, 8, 16), (64, 1, 1), (256, 3, 2), (64, 5, 64)])
def test_pack_of_every_kind_of_value(kv, dtype, dim, heads, page_tokens):
    n = 5
    g = torch.Generator().manual_seed(dim)
    x = torch.randn(2, n, page_tokens, heads, dim, generator=g).double()
    blocks = x.view(-1, 32)
    blocks *= 2.0 ** torch.randint(-30, 18, (blocks.shape[0], 1), generator=g)       # past both ends of float16
    lead = blocks[:, 0]
    for i, special in enumerate((0.0, -0.0, math.inf, -math.inf, math.nan, 1.75, 7.0, 6.0, 5.0, 0.25, -2.5, 3.5)):
        if i < blocks.shape[0]:
            blocks[i, :] = torch.tensor([special, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25] * 4) if i % 2 else special
    lead[-1] = torch.finfo(dtype).max
    blocks[-2] = torch.finfo(dtype).tiny * torch.finfo(dtype).eps * torch.arange(-16, 16)    # the least steps there are
    x = x.to(dtype)
    k, v = x[0].cuda(), x[1].cuda()
    src = kv.Cache(k, v)
    pools = [kv.packed_pool(n + 3, page_tokens, heads, dim) for _ in "kv"]
    dst = kv.Cache(*pools, dtype=dtype, page_tokens=page_tokens, kv_heads=heads, head_dim=dim)
    a = torch.tensor([3, 0, 4, 1, n, 2], dtype=torch.int32, device="cuda")
    b = torch.tensor([7, 2, 5, 0, 1, n + 3], dtype=torch.int32, device="cuda")        # the last two: one number outside each
    errors = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv.pack(src, dst, a, b, errors=errors)
    assert int(errors) == 2
    for pool, want in zip(pools, (x[0], x[1])):
        codes, scales = R.encode4(want.double().numpy(), dtype)
        count = page_tokens * heads * dim
        data = np.zeros((n + 3, pool.shape[1]), np.uint8)
        for i, j in ((3, 7), (0, 2), (4, 5), (1, 0)):
            data[j, :count // 2] = (codes[i].ravel()[0::2] + 16 * codes[i].ravel()[1::2])
            data[j, count // 2:count // 2 + count // 32] = scales[i].ravel()
        same(pool, data)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_packing_what_was_appended_is_appending_in_four_bits(kv, dtype):
    rows, tokens = [70, 33], [70, 50]
    s16, s4 = (Setup(kv, rows, tokens, dtype, bits, 8, 4, 128, 16, seed=3) for bits in (16, 4))
    k, v = (torch.randn(103, 4, 128, generator=s16.g).to(dtype).cuda() for _ in "kv")
    w, rope = (1 + 0.1 * torch.randn(128, generator=s16.g)).to(dtype).cuda(), kv.rope_table(70, 128, 500000.0)
    for s in (s16, s4):
        kv.append(s.cache, s.batch, k, v, k_weight=w, rope=rope)
    pools = [torch.zeros_like(s4.k_pool) for _ in "kv"]
    every = torch.arange(s16.k_pool.shape[0], dtype=torch.int32, device="cuda")
    kv.pack(s16.cache, s4.make_cache(*pools), every, every)
    assert torch.equal(pools[0], s4.k_pool) and torch.equal(pools[1], s4.v_pool)


@pytest.mark.parametrize("bits", [16, 4])
def test_read_leaves_out_what_is_wrong(kv, bits):
    s = Setup(kv, [4, 3, 2], [20, 3, 2], bits=bits, dim=128, spare_width=1)
    s.batch.page_table[0, 1] = -1                                        # tokens 16 .. 19 of the first sequence
    s.batch.kv_len[1] = 2                                                # its first row would be at position -1
    out = torch.full((9, 2, 128), 7.0, dtype=BF16, device="cuda")
    k, v = kv.read(s.cache, s.batch, k_out=out, v_out=out.clone())
    assert int(s.batch.errors) == 2 | 4
    assert not k[:4].any() and not v[:4].any() and bool((k[4] == 7).all())
    assert np.array_equal(k[7:].cpu().double().numpy(), s.held(s.k_pool, 2))
    s.batch.errors.zero_()
    s.batch.kv_len[2] = 500                                              # more than max_kv
    k, _ = kv.read(s.cache, s.batch, k_out=torch.full_like(out, 5.0), v_out=out)
    assert int(s.batch.errors) == 1 | 2 | 4 and bool((k[7:] == 5).all())


# ---- attend --------------------------------------------------------------------------------------
SHAPES = [
    # rows, tokens, q_heads, heads, dim, page_tokens
    ([1], [1], 1, 1, 64, 16), ([1, 1, 1], [5, 33, 64], 8, 2, 128, 16), ([1, 0, 1, 1], [300, 7, 0, 129], 4, 4, 128, 8),
    ([2, 1, 3], [40, 1, 31], 5, 1, 64, 32), ([4, 8, 7], [70, 8, 95], 8, 2, 128, 4), ([1, 1], [1000, 17], 64, 1, 128, 16),
    ([3, 2], [65, 200], 16, 1, 256, 16), ([1, 1], [700, 63], 2, 2, 256, 64), ([16, 5], [100, 5], 8, 2, 64, 1),
    ([65, 130, 1], [65, 200, 90], 4, 2, 128, 16), ([100, 33], [100, 33], 3, 1, 64, 16), ([50, 40], [300, 40], 6, 2, 256, 32),
    ([200], [200], 10, 2, 128, 128), ([33, 70], [20, 70], 8, 2, 128, 16), ([9, 3], [4, 3], 2, 2, 128, 16)]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attend(kv, shape, dtype, bits):
    rows, tokens, q_heads, heads, dim, page_tokens = SHAPES[shape]
    s = Setup(kv, rows, tokens, dtype, bits, q_heads, heads, dim, page_tokens, seed=shape)
    for window, causal, scale in ((0, True, None), (1, True, None), (19, True, 0.4), (0, False, None), (37, False, 0.05)):
        out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), scale=scale, window=window, causal=causal, want_lse=True)
        s.check_attend(out, lse, window, causal, scale)
        assert int(s.batch.errors) == 0


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [3, 40])
def test_attend_every_count_of_tiles(kv, dim, bits, rows):
    # one tile of 32 or 64 tokens to nine, the last one not whole: rows of tiles that are not there are not asked for
    for tokens in ([64 * i - 5 for i in range(1, 10)], [64 * i for i in range(3, 8)], [129, 192, 191, 130]):
        s = Setup(kv, [min(rows, n) for n in tokens], tokens, BF16, bits, 4, 1, dim, 16, seed=rows)
        out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), want_lse=True)
        s.check_attend(out, lse)
        assert int(s.batch.errors) == 0


@pytest.mark.parametrize("dtype,bits,rows,q_heads,heads,dim", [
    (BF16, 4, [1, 1], 8, 2, 128), (FP16, 16, [1, 1], 4, 1, 64), (BF16, 16, [4, 2], 8, 2, 128), (FP16, 4, [60, 3], 4, 1, 128),
    (BF16, 4, [6, 1], 8, 1, 256), (FP16, 4, [8, 8], 8, 1, 64)])
def test_attend_long_contexts_are_split_and_joined(kv, dtype, bits, rows, q_heads, heads, dim):
    tokens = [9001, 4447]
    s = Setup(kv, rows, tokens, dtype, bits, q_heads, heads, dim, 16, seed=dim)
    assert kv.attend_workspace(s.cache, s.batch, q_heads) > 0
    q = s.q.cuda()
    for window in (0, 2500):
        out, lse = kv.attend(s.cache, s.batch, q, window=window, want_lse=True)
        s.check_attend(out, lse, window)
        again, lse_again = kv.attend(s.cache, s.batch, q, window=window, want_lse=True)
        assert torch.equal(out, again) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("rows,tokens,q_heads", [([1, 1], [600, 40], 4), ([6, 20], [50, 20], 4), ([130, 70], [200, 70], 2)])
@pytest.mark.parametrize("bits", [16, 4])
def test_attend_large_scores_and_one_heavy_token(kv, rows, tokens, q_heads, bits):
    # rows whose maximum grows late, by a lot, and scores far below it
    s = Setup(kv, rows, tokens, FP16 if bits == 16 else BF16, bits, q_heads, 2, 64, 16, seed=1)
    ramp = torch.linspace(0.02, 6.0, s.k16.shape[0])[:, None, None, None]
    s.k16 = (s.k16.float() * ramp).to(s.dtype)
    s.k_pool = s.pool(s.k16)
    s.cache = s.make_cache(s.k_pool, s.v_pool)
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), scale=1.5, want_lse=True)
    s.check_attend(out, lse, scale=1.5)


@pytest.mark.parametrize("rows,tokens,q_heads,heads,dim", [([5, 1], [37, 50], 4, 2, 128), ([90, 3], [120, 3], 4, 2, 64), ([12, 40], [30, 40], 12, 1, 128), ([45, 6], [60, 90], 2, 1, 256)])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("window", [0, 11])
def test_attend_is_not_reached_by_what_a_row_does_not_see(kv, rows, tokens, q_heads, heads, dim, bits, window):
    s = Setup(kv, rows, tokens, BF16, bits, q_heads, heads, dim, 16, seed=5)
    clean = kv.attend(s.cache, s.batch, s.q.cuda(), window=window, want_lse=True)
    # the places behind a sequence's last token, and pages that are nobody's, hold infinities and NaN
    used = {}
    for i, n in enumerate(tokens):
        for t in range(n):
            used.setdefault(int(s.table[i, t // 16]), set()).add(t % 16)
    for page in range(s.k16.shape[0]):
        for slot in range(16):
            if slot not in used.get(page, ()):
                s.k16[page, slot], s.v16[page, slot] = math.nan, math.inf if slot % 2 else math.nan
    # and the last token of the first sequence, which only its last row sees, has some of each among its values
    page, slot = int(s.table[0, (tokens[0] - 1) // 16]), (tokens[0] - 1) % 16
    s.v16[page, slot, 0, 3], s.v16[page, slot, 0, 40], s.v16[page, slot, heads - 1, 33] = math.inf, -math.inf, math.nan
    s.k_pool, s.v_pool = s.pool(s.k16), s.pool(s.v16)
    s.cache = s.make_cache(s.k_pool, s.v_pool)
    out, lse = kv.attend(s.cache, s.batch, s.q.cuda(), window=window, want_lse=True)
    last = rows[0] - 1
    same = torch.ones(s.n_rows, dtype=torch.bool)
    same[last] = False
    assert torch.equal(out[same.cuda()], clean[0][same.cuda()]) and torch.equal(lse, clean[1])
    group = q_heads // heads
    row = out[last].float().cpu().view(heads, group, dim)
    if bits == 16:
        assert bool((row[0, :, 3] == math.inf).all()) and bool((row[0, :, 40] == -math.inf).all()) and bool(row[heads - 1, :, 33].isnan().all())
        row[0, :, 3] = row[0, :, 40] = row[heads - 1, :, 33] = 0
        assert bool(row.isfinite().all())
    else:
        assert bool(row[0, :, :64].isnan().all()) and bool(row[heads - 1, :, 32:64].isnan().all())
        assert bool(row[:, :, 64:].isfinite().all())


@pytest.mark.parametrize("rows,tokens", [([1, 1, 1], [80, 50, 20]), ([40, 50, 20], [80, 50, 20])])
@pytest.mark.parametrize("bits", [16, 4])
def test_attend_leaves_out_bad_pages_and_sequences(kv, rows, tokens, bits):
    s = Setup(kv, rows, tokens, BF16, bits, 8, 2, 128, 16, seed=2)
    q = s.q.cuda()
    s.batch.page_table[0, 2] = -5                                        # tokens 32 .. 47 are not seen
    s.batch.kv_len[2] = 1 << 20
    out = torch.full((s.n_rows, 8, 128), 9.0, dtype=BF16, device="cuda")
    out, lse = kv.attend(s.cache, s.batch, q, causal=False, out=out, want_lse=True)
    assert int(s.batch.errors) == 1 | 2
    assert bool((out[s.starts[2]:] == 9).all())
    s.check_attend(out, lse, causal=False, skip=(0, 2))
    k, v = (np.delete(s.held(p, 0), slice(32, 48), 0) for p in (s.k_pool, s.v_pool))
    want, want_lse, mass, size = R.attend(s.q[:rows[0]].double().numpy(), k, v, 1 / math.sqrt(128), 0, False)
    bound, _ = R.attend_bounds(want, mass, size, 80, 128, BF16)
    assert (np.abs(out[:rows[0]].double().cpu().numpy() - want) <= bound).all()


def test_attend_scores_of_minus_infinity(kv):
    s = Setup(kv, [2], [6], dim=64, heads=1, q_heads=1)
    s.k_pool.view(-1, 64)[:, 0] = -math.inf
    q = s.q.cuda()
    q[0, 0, 0], q[1, 0, 0] = 1.0, -1.0
    out, lse = kv.attend(s.cache, s.batch, q, want_lse=True)
    assert not out[0].any() and float(lse[0]) == -math.inf               # nothing but minus infinity
    assert bool(out[1].isnan().all())                                    # plus infinity, several times


@pytest.mark.parametrize("bits", [16, 4])
def test_pages_beyond_four_gibibytes(kv, bits):
    # the same few pages at both ends of pools whose byte offsets, and for 16 bits element offsets, pass 32 bits
    heads, dim, page_tokens = 8, 128, 16
    few = Setup(kv, [3, 70], [50, 70], BF16, bits, 8, heads, dim, page_tokens, seed=9)
    n = few.k_pool.shape[0]
    page = few.k_pool[0].numel() * few.k_pool.element_size()
    total = (9 << 30) // page if bits == 16 else (5 << 30) // page
    pools = [torch.empty((total,) + tuple(few.k_pool.shape[1:]), dtype=few.k_pool.dtype, device="cuda") for _ in "kv"]
    for big, small in zip(pools, (few.k_pool, few.v_pool)):
        big[:n], big[total - n:] = 0, small
    cache = few.make_cache(*pools)
    near = kv.attend(few.cache, few.batch, few.q.cuda(), want_lse=True)
    at = torch.where(few.batch.page_table < n, few.batch.page_table + (total - n), few.batch.page_table)
    batch = kv.Batch(at, few.batch.kv_len, few.batch.row_start, few.n_rows, 70, 70)
    far = kv.attend(cache, batch, few.q.cuda(), want_lse=True)
    assert torch.equal(near[0], far[0]) and torch.equal(near[1], far[1])
    k, v = kv.read(cache, batch)
    want_k, want_v = kv.read(few.cache, few.batch)
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    kv.append(cache, batch, v, k)
    back = kv.read(cache, batch)
    kv.append(few.cache, few.batch, want_v, want_k)
    want = kv.read(few.cache, few.batch)
    assert torch.equal(back[0], want[0]) and torch.equal(back[1], want[1])
    assert not pools[0][:n].any() and not pools[1][:n].any()


def test_strided_rows_and_a_stream_of_the_callers(kv):
    s = Setup(kv, [1, 6], [90, 30], FP16, 16, 4, 2, 128, 16, seed=4, spare_width=3, spare_bytes=128)
    want = kv.attend(s.cache, s.batch, s.q.cuda())
    wide = torch.zeros(7, 4 * 128 + 24, dtype=FP16, device="cuda")
    q, out = wide[:, 8:520].unflatten(1, (4, 128)), torch.zeros(7, 1, 4, 128, dtype=FP16, device="cuda")[:, 0]
    q.copy_(s.q)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    kv.attend(s.cache, s.batch, q, out=out, stream=stream)
    stream.synchronize()
    assert torch.equal(out, want)
    with torch.cuda.stream(stream):
        again = kv.attend(s.cache, s.batch, q)
    stream.synchronize()
    assert torch.equal(again, want)


def test_a_step_in_a_graph(kv):
    s = Setup(kv, [1, 1], [3000, 70], BF16, 4, 8, 2, 128, 16, seed=6)
    q, k, v = (torch.randn(2, h, 128, generator=s.g).to(BF16).cuda() for h in (8, 2, 2))
    rope = kv.rope_table(3000, 128)

    def step():
        turned = kv.append(s.cache, s.batch, k, v, q=q, rope=rope)
        return kv.attend(s.cache, s.batch, turned)

    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out = step()
    torch.cuda.synchronize()
    for i in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=s.g))
        s.batch.kv_len.copy_(torch.tensor([3000 - 17 * i, 70 - i], dtype=torch.int32))
        want = step()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_batches_of_nothing(kv):
    s = Setup(kv, [1], [4])
    none = kv.Batch(s.batch.page_table, s.batch.kv_len, torch.zeros(2, dtype=torch.int32, device="cuda"), 0, 0, 4)
    q = torch.empty(0, 4, 64, dtype=BF16, device="cuda")
    assert kv.attend(s.cache, none, q).shape == (0, 4, 64)
    assert kv.read(s.cache, none)[0].shape == (0, 2, 64)
    x = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    assert kv.append(s.cache, none, x, x, q=q).shape == (0, 4, 64)
    nothing = torch.empty(0, dtype=torch.int32, device="cuda")
    packed = kv.packed_pool(1, 16, 2, 64)
    kv.pack(s.cache, kv.Cache(packed, packed.clone(), dtype=BF16, page_tokens=16, kv_heads=2, head_dim=64), nothing, nothing)


def test_tensors_that_are_refused(kv):
    from paper_2604_00368_amd import binding as T
    s = Setup(kv, [1, 2], [20, 9])
    q = s.q.cuda()
    for bad in (q.float(), q[:2], q.cpu(), q.transpose(1, 2), q[..., :32], None):
        with pytest.raises(ValueError):
            kv.attend(s.cache, s.batch, bad)
    with pytest.raises(T.TentError) as e:                                # rows that do not start at whole 16 bytes
        kv.attend(s.cache, s.batch, torch.zeros(3, 4 * 64 + 4, dtype=BF16, device="cuda")[:, :256].unflatten(1, (4, 64)))
    assert e.value.status == T.TENT_ERR_INVALID
    with pytest.raises(T.TentError) as e:
        kv.attend(s.cache, s.batch, torch.zeros(3, 3, 64, dtype=BF16, device="cuda"))
    assert e.value.status == T.TENT_ERR_RANGE                            # 3 heads do not share 2
    for scale in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(T.TentError):
            kv.attend(s.cache, s.batch, q, scale=scale)
    with pytest.raises(ValueError):
        kv.Batch(s.batch.page_table, s.batch.kv_len[:1], s.batch.row_start, 3, 2, 20)
    with pytest.raises(ValueError):
        kv.attend(s.cache, kv.Batch(s.batch.page_table, s.batch.kv_len, s.batch.row_start, 3, 2, 33), q)
    x = torch.zeros(3, 2, 64, dtype=BF16, device="cuda")
    for bad in (dict(rope=kv.rope_table(8, 24)), dict(rope=kv.rope_table(8, 128)), dict(eps=-1.0)):
        with pytest.raises(T.TentError):
            kv.append(s.cache, s.batch, x, x, **bad)
    with pytest.raises(T.TentError):
        kv.pack(s.cache, s.cache, s.batch.kv_len, s.batch.kv_len)
    long = Setup(kv, [1], [5000], dim=128, heads=1, q_heads=1)
    with pytest.raises(T.TentError) as e:
        kv.attend(long.cache, long.batch, long.q.cuda(), workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == T.TENT_ERR_RANGE
