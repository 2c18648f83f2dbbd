"""Paged cache operators with more workgroups than one launch takes, on a GPU."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_kv import Setup, kv  # noqa: E402,F401

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_packing_millions_of_small_pages(kv):
    n, part = 8_600_000, 2_900_000                                       # 17 million workgroups; 6 million a part
    k = torch.randn(n, 1, 1, 64, device="cuda", dtype=BF16)
    src, shape = kv.Cache(k, k), dict(dtype=BF16, page_tokens=1, kv_heads=1, head_dim=64)
    pages = torch.arange(n, dtype=torch.int32, device="cuda")
    whole, parts = ([kv.packed_pool(n + 1, 1, 1, 64) for _ in "kv"] for _ in range(2))
    errors = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv.pack(src, kv.Cache(*whole, **shape), pages, pages.flip(0), errors=errors)
    for lo in range(0, n, part):
        kv.pack(src, kv.Cache(*parts, **shape), pages[lo:lo + part], pages.flip(0)[lo:lo + part], errors=errors)
    assert int(errors) == 0
    for a, b in zip(whole, parts):
        assert torch.equal(a, b) and bool(a[:n].any(1).all()) and not a[n].any()


def test_attention_of_one_token_each_over_many_heads(kv):
    n_seqs, heads = 65535, 512                                           # 34 million workgroups of few lines
    v = torch.randn(37, 1, heads, 64, device="cuda", dtype=BF16)
    cache = kv.Cache(torch.randn_like(v), v)
    table = torch.randint(0, 37, (n_seqs, 1), dtype=torch.int32, device="cuda")
    batch = kv.Batch(table, torch.ones(n_seqs, dtype=torch.int32, device="cuda"), torch.arange(n_seqs + 1, dtype=torch.int32, device="cuda"),
                     n_seqs, 1, 1)
    q = torch.randn(n_seqs, heads, 64, device="cuda", dtype=BF16)
    out = kv.attend(cache, batch, q)
    for lo in range(0, n_seqs, 8192):                                    # of a single token: its values
        assert torch.equal(out[lo:lo + 8192], v[table[lo:lo + 8192, 0].long(), 0])
    assert int(batch.errors) == 0


def test_attention_with_room_for_many_lines(kv):
    # 65 tiles of 128 lines by 65535 sequences by 4 heads; the lines that there are come last
    few = Setup(kv, [65, 2, 8], [100, 30, 70], BF16, 16, 4, 4, 64, 16, seed=1)
    q = few.q.cuda()
    want, want_lse = kv.attend(few.cache, few.batch, q, want_lse=True)
    n_seqs, n_rows = 65535, 8320
    at = [0, 40000, n_seqs - 1]
    table = torch.zeros(n_seqs, few.table.shape[1], dtype=torch.int32)
    length, rows = torch.zeros(n_seqs, dtype=torch.int32), torch.zeros(n_seqs, dtype=torch.int32)
    for i, s in enumerate(at):
        table[s], length[s], rows[s] = few.table[i], few.tokens[i], few.rows[i]
    start = torch.cat([torch.zeros(1, dtype=torch.int32), rows.cumsum(0).to(torch.int32)])
    batch = kv.Batch(table.cuda(), length.cuda(), start.cuda(), n_rows, n_rows, 112)
    wide = torch.zeros(n_rows, 4, 64, dtype=BF16, device="cuda")
    wide[:few.n_rows] = q
    out = torch.full_like(wide, 9.0)
    out, lse = kv.attend(few.cache, batch, wide, out=out, want_lse=True)
    assert torch.equal(out[:few.n_rows], want) and torch.equal(lse[:few.n_rows], want_lse)
    assert bool((out[few.n_rows:] == 9).all()) and int(batch.errors) == 0
