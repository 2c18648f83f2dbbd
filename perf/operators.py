"""Performance cases of the paged key/value cache operators: append, pack, read and attend.

A serving engine that migrates paged KV blocks also fills them, shrinks them for the wire and answers from them:

  append  new tokens of every sequence: queries and keys normalised per head (RMS) and rotated, keys and values written
          to the pages of the sequence, in 16 bits or in 4
  pack    whole 16-bit pages become 4-bit pages, 3.8 times fewer bytes to migrate
  read    tokens come back from the pages of a sequence as dense rows of 16 bits
  attend  softmax attention of the new tokens' queries over the pages, for single tokens and for prompts

A page holds `page_tokens` tokens of `kv_heads` heads of `head_dim` values, K and V in pools of their own.  A 16-bit page
is [token][head][dim].  A 4-bit page is the codes [token][head][dim / 2] followed by the scales [token][head][dim / 32]:
every 32 values of a head share a power of two (a byte: exponent + 127, 255 for a block with an infinity or a NaN), every
value is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, and a byte of codes has the even dimension in its low half.  The
exponent is the least at which no value of the block is off by more than half a step, within what the 16-bit type holds.
Keys that go into 4 bits are rounded to the 16-bit type first (by way of 32 bits), so that packing a page gives what
appending in 4 bits gives.

Row r of a call belongs to the sequence s with row_start[s] <= r < row_start[s + 1]; the rows of a sequence are its last
tokens.  What is held in 4 bits is returned as the values that it stands for (`read`).
"""
import math
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}
MiB = 1 << 20

# the attention shape of an 8B-class transformer, with the pages that the KV migration workload moves
_GQA = dict(type="bf16", q_heads=32, kv_heads=8, head_dim=128, page_tokens=16)
_APPEND = dict(_GQA, op="append", norm=True, rope="half", rope_dim=128)
_ATTEND = dict(_GQA, op="attend", window=0, causal=True)


def listed():
    return [
        # one user's next token in one layer: launch latency decides it
        dict(_APPEND, name="append_one_token", bits=16, n_seqs=1, rows_lo=1, rows_hi=1, kv_lo=500, kv_hi=500, shape=1),
        # a decode step of 64 requests over a 4-bit cache, and what it stored read back
        dict(_APPEND, name="append_step_fp4", bits=4, n_seqs=64, rows_lo=1, rows_hi=1, kv_lo=2048, kv_hi=8192, shape=2),
        # four prompts of the migration workload's lengths, no norms, a 16-bit cache
        dict(_APPEND, name="append_prompts", norm=False, bits=16, n_seqs=4, rows_lo=2048, rows_hi=8192, kv_lo=0, kv_hi=0, shape=3),
        # odd prompts behind what is cached, half of each head rotated in pairs, stored in 4 bits and read back
        dict(_APPEND, name="append_odd_prompts_fp4", type="fp16", rope="pairs", rope_dim=64, head_dim=128, q_heads=16, kv_heads=4,
             page_tokens=32, bits=4, n_seqs=13, rows_lo=1, rows_hi=1501, kv_lo=7, kv_hi=2345, shape=4),
        # one request's prefix is packed for its migration and read back
        dict(_GQA, name="pack_request", op="pack", n_seqs=1, rows_lo=2048, rows_hi=8192, kv_lo=0, kv_hi=0, shape=5),
        # one layer of the whole migration workload: 32 requests of 2k-8k tokens
        dict(_GQA, name="pack_requests", op="pack", n_seqs=32, rows_lo=2048, rows_hi=8192, kv_lo=0, kv_hi=0, shape=6),
        # cached prefixes of a few requests as dense 16-bit rows, for a step that wants them contiguous
        dict(_GQA, name="read_prefixes_fp4", op="read", bits=4, n_seqs=8, rows_lo=300, rows_hi=8192, kv_lo=0, kv_hi=0, shape=7),
        # one user's next token over a short context: latency again
        dict(_ATTEND, name="attend_one_token", bits=16, n_seqs=1, rows_lo=1, rows_hi=1, kv_lo=500, kv_hi=500, shape=8),
        # the decode step of the migrated requests, over what arrived in 4 bits
        dict(_ATTEND, name="attend_step_fp4", bits=4, n_seqs=32, rows_lo=1, rows_hi=1, kv_lo=2048, kv_hi=8192, shape=9),
        # two users with contexts of 128k tokens, speculating three tokens ahead
        dict(_ATTEND, name="attend_long_fp4", type="fp16", bits=4, n_seqs=2, rows_lo=4, rows_hi=4, kv_lo=100001, kv_hi=131072, shape=10),
        # prompts: every token of two sequences against the ones before it
        dict(_ATTEND, name="attend_prompts", bits=16, n_seqs=2, rows_lo=3500, rows_hi=4096, kv_lo=0, kv_hi=0, shape=11),
        # chunks of prompts behind long prefixes in 4 bits
        dict(_ATTEND, name="attend_chunks_fp4", bits=4, n_seqs=3, rows_lo=257, rows_hi=511, kv_lo=6001, kv_hi=16384, shape=12),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    n = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["append", "append", "pack", "read", "attend", "attend", "attend"])
    kv_heads = rng.choice([1, 2, 4, 8])
    head_dim = rng.choice([64, 128, 128, 128, 256])
    q_heads = kv_heads * rng.choice([1, 2, 4, 4, 5, 8, 16])
    case = dict(op=op, type=rng.choice(["bf16", "fp16"]), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                page_tokens=rng.choice([8, 16, 16, 32, 64, 128]), bits=rng.choice([4, 16]), shape=rng.randrange(1 << 20))
    kv_dim = kv_heads * head_dim
    if op == "append":
        total = _log(rng, 1, min(20000, 100 * MiB // ((q_heads + 2 * kv_heads) * head_dim)))
        case.update(norm=rng.random() < 0.6, rope=rng.choice(["half", "half", "pairs", "none"]), rope_dim=head_dim // rng.choice([1, 1, 2, 4]))
    elif op in ("pack", "read"):
        total = _log(rng, 1, min(150000, 150 * MiB // kv_dim))
        case["q_heads"] = kv_heads
        if op == "pack":
            case["bits"] = 16
    else:
        kind = rng.choice(["token", "token", "few", "chunk", "prompt"])
        case.update(window=rng.choice([0, 0, 0, _log(rng, 1, 4096)]), causal=rng.random() < 0.9)
        if kind == "prompt":
            total = _log(rng, 1, 8192)
            case["n_seqs"] = n = rng.randint(1, min(6, total))
            # the plain form holds every score of every sequence, and more than once
            most = int(math.sqrt(900 * MiB * 128 / (n * q_heads * max(128, head_dim))))
            high = max(1, min(total // n, most, 4096))
            case.update(rows_lo=max(1, high // rng.choice([1, 2, 9])), rows_hi=high, kv_lo=0, kv_hi=0)
            return case
        case["n_seqs"] = n = _log(rng, 1, 96)
        rows = {"token": 1, "few": rng.randint(2, 16), "chunk": _log(rng, 17, 512)}[kind]
        cached = 1 + 240 * MiB // (n * max(kv_dim, rows * q_heads * head_dim // 256))
        high = _log(rng, 1, max(2, min(131072, cached)))
        case.update(rows_lo=1 if kind != "few" or rng.random() < 0.5 else rows, rows_hi=rows, kv_lo=max(1, high // rng.choice([1, 2, 8, 1000])), kv_hi=high)
        return case
    n = min(total, _log(rng, 1, 256))
    high = max(1, total // n)
    high = high + 1 if high == 3072 else high
    case.update(n_seqs=n, rows_lo=rng.choice([high, max(1, high // 2), 1]), rows_hi=high, kv_lo=0, kv_hi=0)
    if op == "append" and rng.random() < 0.5:
        case.update(kv_lo=1, kv_hi=_log(rng, 1, 4096))
    return case


# ---- what follows from the case alone -----------------------------------------------------------
def _lengths(case):
    """New rows of every sequence, and the tokens that its pages hold with them."""
    rng = random.Random(case["shape"])
    rows = [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["n_seqs"])]
    before = [rng.randint(case["kv_lo"], case["kv_hi"]) for _ in range(case["n_seqs"])]
    return rows, [r + b for r, b in zip(rows, before)]


def work(case):
    rows, kv = _lengths(case)
    n, H, HQ, D = sum(rows), case["kv_heads"], case["q_heads"], case["head_dim"]
    in4, in16 = D // 2 + D // 32, 2 * D                                  # bytes of one head of one token
    stored = in4 if case.get("bits") == 4 else in16
    if case["op"] == "append":
        rope = 0 if case["rope"] == "none" else case["rope_dim"]
        back = 2 * H * in16 if case["bits"] == 4 else 0
        return {"bytes": n * (2 * HQ * in16 + 2 * H * (in16 + stored) + back + 4 * rope),
                "flops": n * (HQ + H) * ((4 * D if case["norm"] else 0) + 3 * rope)}
    if case["op"] == "pack":
        pages = sum(-(-k // case["page_tokens"]) for k in kv)
        return {"bytes": 2 * H * (pages * case["page_tokens"] * (in16 + in4) + n * in16), "flops": 0}
    if case["op"] == "read":
        return {"bytes": 2 * H * n * (stored + in16), "flops": 0}
    pairs = tokens = 0
    for r, k in zip(rows, kv):
        window = case["window"] or k
        first = k - r + 1 if case["causal"] else k                       # tokens that the first row may see, the window aside
        pairs += sum(min(t, window) for t in range(first, k + 1)) if case["causal"] else r * min(k, window)
        tokens += min(k, window + k - first)
    return {"bytes": 2 * n * HQ * in16 + 4 * n * HQ + 2 * H * tokens * stored, "flops": 4 * D * HQ * pairs}


# ---- inputs -------------------------------------------------------------------------------------
def _page_bytes(case):
    """Bytes of a 4-bit page, whole vectors of 16."""
    n = case["page_tokens"] * case["kv_heads"] * (case["head_dim"] // 2 + case["head_dim"] // 32)
    return -(-n // 16) * 16


def _pool(case, n_pages, bits, g):
    """A pool in use: every page has values of earlier tokens."""
    shape = (case["page_tokens"], case["kv_heads"], case["head_dim"])
    pool16 = bits == 16
    pool = torch.empty((n_pages,) + shape if pool16 else (n_pages, _page_bytes(case)), dtype=DTYPE[case["type"]] if pool16 else torch.uint8, device="cuda")
    step = max(1, 64 * MiB // math.prod(shape))
    for lo in range(0, n_pages, step):
        part = pool[lo:lo + step]
        if pool16:
            part.normal_(generator=g)
        else:
            part.zero_()
            _store4(case, part, (slice(None),), torch.randn((part.shape[0],) + shape, device="cuda", generator=g).to(DTYPE[case["type"]]).float())
    return pool


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + case["shape"])
    dtype, H, HQ, D, PT = DTYPE[case["type"]], case["kv_heads"], case["q_heads"], case["head_dim"], case["page_tokens"]
    rows, kv = _lengths(case)
    n_rows, n_seqs = sum(rows), len(rows)
    pages = [-(-k // PT) for k in kv]
    n_pages = sum(pages) + 3
    width = max(pages)
    ids = torch.randperm(n_pages, device="cuda", generator=g)[:sum(pages)].to(torch.int32).split(pages)
    s = {"case": case, "n_rows": n_rows, "max_rows": max(rows), "max_kv": max(kv)}
    s["table"] = torch.stack([torch.nn.functional.pad(i, (0, width - i.numel())) for i in ids])
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
    s["row_start"] = torch.tensor([sum(rows[:i]) for i in range(n_seqs + 1)], dtype=torch.int32, device="cuda")
    bits = case.get("bits", 16)
    s["k_pool"], s["v_pool"] = _pool(case, n_pages, bits, g), _pool(case, n_pages, bits, g)
    if case["op"] == "pack":
        s["src_pages"] = torch.cat(ids)
        s["dst_pages"] = torch.randperm(n_pages, device="cuda", generator=g)[:sum(pages)].to(torch.int32)
        s["k_packed"], s["v_packed"] = (torch.zeros(n_pages, _page_bytes(case), dtype=torch.uint8, device="cuda") for _ in "kv")
        s["packed_table"] = torch.stack([torch.nn.functional.pad(i, (0, width - i.numel())) for i in s["dst_pages"].split(pages)])
    if case["op"] in ("append", "attend"):
        s["q"] = torch.randn(n_rows, HQ, D, device="cuda", generator=g).mul_(2.0).to(dtype)
    if case["op"] == "append":
        s["k"] = torch.randn(n_rows, H, D, device="cuda", generator=g).mul_(1.5).to(dtype)
        s["v"] = torch.randn(n_rows, H, D, device="cuda", generator=g).to(dtype)
        s["q_weight"] = s["k_weight"] = s["rope"] = None
        if case["norm"]:
            s["q_weight"], s["k_weight"] = ((1 + 0.2 * torch.randn(D, device="cuda", generator=g)).to(dtype) for _ in "qk")
        if case["rope"] != "none":
            half = case["rope_dim"] // 2
            angle = torch.arange(max(kv), device="cuda", dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
            s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    if own:                                                              # the handles that a serving program keeps beside its pools
        from paper_2604_00368_amd import kv as ops
        s["ops"] = ops
        s["cache"] = _cache(case, s["k_pool"], s["v_pool"], ops)
        batch = dict(n_rows=n_rows, max_rows=max(rows), max_kv=max(kv))
        s["batch"] = ops.Batch(s["table"], s["kv_len"], s["row_start"], **batch)
        if case["op"] == "pack":
            s["packed"] = _cache(case, s["k_packed"], s["v_packed"], ops)
            s["packed_batch"] = ops.Batch(s["packed_table"], s["kv_len"], s["row_start"], **batch)
    return s


def _cache(case, k, v, ops):
    if k.dtype != torch.uint8:
        return ops.Cache(k, v)
    return ops.Cache(k, v, dtype=DTYPE[case["type"]], page_tokens=case["page_tokens"], kv_heads=case["kv_heads"], head_dim=case["head_dim"])


# ---- one pass -----------------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _own_append(s):
    case, ops = s["case"], s["ops"]
    q = ops.append(s["cache"], s["batch"], s["k"], s["v"], q=s["q"], q_weight=s["q_weight"], k_weight=s["k_weight"], rope=s["rope"],
                   rope_pairs=case["rope"] == "pairs")
    k, v = ops.read(s["cache"], s["batch"]) if case["bits"] == 4 else (s["k_pool"], s["v_pool"])
    return {"q": q, "k": k, "v": v}


def _own_pack(s):
    s["ops"].pack(s["cache"], s["packed"], s["src_pages"], s["dst_pages"])
    k, v = s["ops"].read(s["packed"], s["packed_batch"])
    return {"k": k, "v": v}


def _own_read(s):
    k, v = s["ops"].read(s["cache"], s["batch"])
    return {"k": k, "v": v}


def _own_attend(s):
    case = s["case"]
    out, lse = s["ops"].attend(s["cache"], s["batch"], s["q"], window=case["window"], causal=case["causal"], want_lse=True)
    return {"out": out, "lse": lse}


_own = {"append": _own_append, "pack": _own_pack, "read": _own_read, "attend": _own_attend}


# ---- the plain forms ----------------------------------------------------------------------------
def _halves(case, pool):
    """The codes and the scales of a pool of 4-bit pages, by page, token and head."""
    PT, H, D = case["page_tokens"], case["kv_heads"], case["head_dim"]
    codes, scales = pool[:, :PT * H * D // 2], pool[:, PT * H * D // 2:PT * H * (D // 2 + D // 32)]
    return codes.unflatten(1, (PT, H, D // 2)), scales.unflatten(1, (PT, H, D // 32))


def _store4(case, pool, at, x):
    """Writes 32-bit values that are whole numbers of the 16-bit type to the places `at` of a pool of 4-bit pages."""
    x = x.unflatten(-1, (-1, 32))
    size = x.abs().amax(-1)
    mantissa, exponent = torch.frexp(size)                               # size = mantissa 2^exponent, mantissa in [0.5, 1)
    low, high = (-127, 125) if case["type"] == "bf16" else (-23, 13)
    power = (exponent - 3 + (mantissa > 0.875)).clamp(low, high)
    power = torch.where(size == 0, low, power)
    good = size.isfinite()
    y = torch.ldexp(torch.where(good[..., None], x, 0.0).double(), -power[..., None])
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    code += y.signbit().to(torch.uint8) * 8
    code = code.flatten(-2)
    codes, scales = _halves(case, pool)
    codes[at] = code[..., 0::2] + code[..., 1::2] * 16
    scales[at] = torch.where(good, power + 127, 255).to(torch.uint8)


_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _load4(case, pool, at):
    """The values at the places `at` of a pool of 4-bit pages, in 32 bits."""
    codes, scales = _halves(case, pool)
    codes, scales = codes[at], scales[at].int()
    value = torch.tensor(_VALUES + [-v for v in _VALUES], device=pool.device)
    x = value[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()].unflatten(-1, (-1, 32))
    x = torch.ldexp(x, (scales - 127)[..., None])
    return torch.where((scales == 255)[..., None], math.nan, x).flatten(-2)


def _places(s, table):
    """Position of every row in its sequence, and its page and place in it."""
    PT, start, kv_len = s["case"]["page_tokens"], s["row_start"].long(), s["kv_len"].long()
    row = torch.arange(s["n_rows"], device=start.device)
    seq = torch.bucketize(row, start[1:], right=True)
    position = kv_len[seq] - start[seq + 1] + row
    return position, (table[seq, position // PT].long(), position % PT)


def _norm_and_rotate(case, x, weight, rope, position):
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.to(x.dtype)
    if rope is None:
        return x
    half = case["rope_dim"] // 2
    cos, sin = rope[position].to(x.dtype)[:, None, :].split(half, -1)
    part, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (part[..., 0::2], part[..., 1::2]) if case["rope"] == "pairs" else part.split(half, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    part = torch.stack([a, b], -1).flatten(-2) if case["rope"] == "pairs" else torch.cat([a, b], -1)
    return torch.cat([part, rest], -1)


def _plain_append(s):
    case, dtype = s["case"], DTYPE[s["case"]["type"]]
    position, at = _places(s, s["table"])
    q = _norm_and_rotate(case, s["q"].float(), s["q_weight"], s["rope"], position).to(dtype)
    # values next to a border of the 4-bit codes: 64 bits, then the roundings that the format names
    k = _norm_and_rotate(case, s["k"].double(), s["k_weight"], s["rope"], position).float().to(dtype)
    if case["bits"] == 16:
        s["k_pool"][at], s["v_pool"][at] = k, s["v"]
        return {"q": q, "k": s["k_pool"], "v": s["v_pool"]}
    _store4(case, s["k_pool"], at, k.float())
    _store4(case, s["v_pool"], at, s["v"].float())
    return {"q": q, "k": _load4(case, s["k_pool"], at).to(dtype), "v": _load4(case, s["v_pool"], at).to(dtype)}


def _plain_pack(s):
    case, dtype = s["case"], DTYPE[s["case"]["type"]]
    src, dst = s["src_pages"].long(), s["dst_pages"].long()
    _store4(case, s["k_packed"], (dst,), s["k_pool"][src].float())
    _store4(case, s["v_packed"], (dst,), s["v_pool"][src].float())
    _, at = _places(s, s["packed_table"])
    return {"k": _load4(case, s["k_packed"], at).to(dtype), "v": _load4(case, s["v_packed"], at).to(dtype)}


def _load(case, pool, at):
    return _load4(case, pool, at) if pool.dtype == torch.uint8 else pool[at].float()


def _plain_read(s):
    case, dtype = s["case"], DTYPE[s["case"]["type"]]
    _, at = _places(s, s["table"])
    return {"k": _load(case, s["k_pool"], at).to(dtype), "v": _load(case, s["v_pool"], at).to(dtype)}


def _plain_attend(s):
    case = s["case"]
    H, G, D, PT = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"], case["page_tokens"]
    start, kv_len, R = s["row_start"].long(), s["kv_len"].long(), s["max_rows"]
    row = start[:-1, None] + torch.arange(R, device=start.device)        # [sequence, row], some beyond the sequence's last
    there = row < start[1:, None]
    q = s["q"][row.clamp(max=s["n_rows"] - 1)].float().unflatten(2, (H, G)).permute(0, 2, 3, 1, 4).flatten(2, 3)
    token = torch.arange(s["max_kv"], device=start.device)
    held = token < kv_len[:, None]
    at = (s["table"][:, token // PT].long(), token % PT)
    k = torch.where(held[..., None, None], _load(case, s["k_pool"], at), 0.0).permute(0, 2, 3, 1)
    v = torch.where(held[..., None, None], _load(case, s["v_pool"], at), 0.0).permute(0, 2, 1, 3)
    last = kv_len[:, None] - start[1:, None] + row if case["causal"] else (kv_len[:, None] - 1).expand(-1, R)
    seen = held[:, None, :] & (token <= last[..., None])                 # [sequence, row, token]
    if case["window"]:
        seen &= token > last[..., None] - case["window"]
    score = torch.matmul(q, k).mul_(1.0 / math.sqrt(D)).unflatten(2, (G, R))
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top.isfinite(), top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (G, R)) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(-1)
    out, lse = out.permute(0, 3, 1, 2, 4)[there], lse.permute(0, 3, 1, 2)[there]
    return {"out": out.flatten(1, 2).to(s["q"].dtype), "lse": lse.flatten(1, 2)}


_plain = {"append": _plain_append, "pack": _plain_pack, "read": _plain_read, "attend": _plain_attend}


# ---- the definition in 64 bits, sequence by sequence --------------------------------------------
def _nearest4(case, x):
    """The values that 4 bits hold of 64-bit `x`, whose last axis is whole blocks of 32; x is rounded to the 16-bit type first."""
    x = x.float().to(DTYPE[case["type"]]).double()
    step = torch.tensor(_VALUES, dtype=torch.float64, device=x.device)
    low, high = (-127, 125) if case["type"] == "bf16" else (-23, 13)
    out = torch.empty_like(x)
    flat, to = x.reshape(-1, 32), out.view(-1, 32)
    for lo in range(0, flat.shape[0], 1 << 18):
        b = flat[lo:lo + (1 << 18)]
        size = b.abs().max(1, keepdim=True).values
        power = torch.full_like(size, low)
        for e in range(low, high):                                       # the least power of two, 6 and half a step above it reach the largest
            if not bool((size > 7 * 2.0 ** e).any()):
                break
            power = torch.where(size > 7 * 2.0 ** e, e + 1.0, power)
        unit = torch.pow(2.0, power)
        off = (b.abs()[..., None] / unit[..., None] - step).abs()
        best = off.argmin(-1)
        tie = (off.gather(-1, (best + 1).clamp(max=7)[..., None]).squeeze(-1) == off.gather(-1, best[..., None]).squeeze(-1)) & (best % 2 == 1) & (best < 7)
        value = step[best + tie.long()] * unit * torch.where(torch.signbit(b), -1.0, 1.0)
        to[lo:lo + (1 << 18)] = torch.where(size.isfinite(), value, math.nan)
    return out


def _tokens(s, pool, i, table):
    """All tokens that a pool holds of sequence i, in 64 bits."""
    case = s["case"]
    PT, H, D = case["page_tokens"], case["kv_heads"], case["head_dim"]
    n = int(s["kv_len"][i])
    page = pool[table[i, :-(-n // PT)].long()]
    if pool.dtype != torch.uint8:
        return page.double().reshape(-1, H, D)[:n]
    count = PT * H * D
    nibble = torch.stack([page[:, :count // 2] % 16, page[:, :count // 2] // 16], 2).reshape(-1, 32).long()
    scale = page[:, count // 2:count // 2 + count // 32].reshape(-1, 1).double()
    value = torch.tensor(_VALUES, dtype=torch.float64, device=pool.device)[nibble % 8] * (1 - 2 * (nibble // 8)) * torch.pow(2.0, scale - 127)
    return torch.where(scale == 255, math.nan, value).reshape(-1, H, D)[:n]


def _exact_rows(case, x, weight, rope, first):
    x = x.double()
    if weight is not None:
        x = x * (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).pow(-0.5) * weight.double()
    if rope is None:
        return x
    half = case["rope_dim"] // 2
    turn = rope[first:first + x.shape[0]].double()[:, None]
    turn = torch.complex(turn[..., :half], turn[..., half:])
    y = x.clone()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["rope"] == "pairs" else (slice(0, half), slice(half, 2 * half))
    z = torch.complex(x[..., a], x[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    rows, kv = _lengths(case)
    if case["op"] == "attend":
        return _exact_attend(s, rows, kv)
    if case["op"] == "read":
        return {n: torch.cat([_tokens(s, s[n + "_pool"], i, s["table"])[k - r:] for i, (r, k) in enumerate(zip(rows, kv))]) for n in "kv"}
    if case["op"] == "pack":
        return {n: torch.cat([_nearest4(case, _tokens(s, s[n + "_pool"], i, s["table"])) for i in range(len(rows))]) for n in "kv"}
    firsts = [k - r for r, k in zip(rows, kv)]
    q, k = (torch.cat([_exact_rows(case, x, s[n + "_weight"], s["rope"], f) for x, f in zip(s[n].split(rows), firsts)]) for n in "qk")
    if case["bits"] == 4:
        return {"q": q, "k": _nearest4(case, k), "v": _nearest4(case, s["v"].double())}
    got = {"q": q, "k": s["k_pool"].double(), "v": s["v_pool"].double()}
    for n, x in (("k", k), ("v", s["v"].double())):
        for i, (part, f) in enumerate(zip(x.split(rows), firsts)):
            t = torch.arange(f, f + part.shape[0], device=x.device)
            got[n][s["table"][i].long()[t // case["page_tokens"]], t % case["page_tokens"]] = part
    return got


def _exact_attend(s, rows, kv):
    case = s["case"]
    H, G, D = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"]
    outs, lses = [], []
    for i, (q, n, length) in enumerate(zip(s["q"].split(rows), rows, kv)):
        k, v = _tokens(s, s["k_pool"], i, s["table"]), _tokens(s, s["v_pool"], i, s["table"])
        t = torch.arange(length, device=q.device)
        last = t[length - n:, None] if case["causal"] else torch.full((n, 1), length - 1, device=q.device)
        hidden = (t > last) | (t <= last - (case["window"] or length + 1))
        out, lse = torch.empty(n, H * G, D, dtype=torch.float64, device=q.device), torch.empty(n, H * G, dtype=torch.float64, device=q.device)
        for h in range(H * G):
            score = (q[:, h].double() @ k[:, h // G].t() / math.sqrt(D)).masked_fill_(hidden, -math.inf)
            lse[:, h] = torch.logsumexp(score, 1)
            out[:, h] = torch.softmax(score, 1) @ v[:, h // G]
        outs.append(out)
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
