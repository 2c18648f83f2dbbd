"""Paged cache operators without a device: refusals, what a call enqueues (over the stand-in runtime of fake_hip.c), and the
addressing and checks that the kernels use, compiled for the host."""
import ctypes as C
import math
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LAUNCH = 1


@pytest.fixture(scope="module")
def T():
    from paper_2604_00368_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2604_00368_amd import build
        build.build()
    return binding


# addresses that are never followed
def make_cache(T, **change):
    d = dict(k=0x10000, v=0x20000, n_pages=10, page_stride=16 * 8 * 128 * 2, page_tokens=16, kv_heads=8, head_dim=128, type=0, bits=16, reserved=0)
    d.update(change)
    return T.tent_kv_cache(**d)


def make_batch(T, **change):
    d = dict(page_table=0x3000, kv_len=0x4000, row_start=0x5000, errors=0x6000, n_seqs=2, table_stride=64, n_rows=3, max_rows=2, max_kv=1000, reserved=0)
    d.update(change)
    return T.tent_kv_batch(**d)


def make_append(T, **change):
    d = dict(q=0x1000, k=0x2000, v=0x3000, q_out=0x4000, q_stride=4096, k_stride=1024, v_stride=1024, q_out_stride=4096, q_weight=0x5000,
             k_weight=0x6000, rope=0x7000, positions=0x8000, q_heads=32, rope_rows=100, rope_dim=128, flags=0, eps=1e-6, reserved=0)
    d.update(change)
    return T.tent_kv_append_args(**d)


def make_attend(T, **change):
    d = dict(q=0x1000, out=0x2000, lse=0x3000, q_stride=4096, out_stride=4096, workspace=0x40000, workspace_bytes=1 << 40, q_heads=32, window=0, flags=0, scale=0.1)
    d.update(change)
    return T.tent_kv_attend_args(**d)


INVALID, RANGE = -1, -2
BAD_CACHES = [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=0x10008), INVALID), (dict(page_stride=16 * 8 * 128 * 2 + 8), INVALID), (dict(type=2), INVALID),
    (dict(bits=8), INVALID), (dict(reserved=1), INVALID), (dict(page_tokens=12), RANGE), (dict(page_tokens=0), RANGE), (dict(page_tokens=2048), RANGE),
    (dict(kv_heads=0), RANGE), (dict(kv_heads=1025), RANGE), (dict(head_dim=96), RANGE), (dict(head_dim=512), RANGE), (dict(n_pages=0), RANGE),
    (dict(n_pages=1 << 31), RANGE), (dict(page_stride=16 * 8 * 128 * 2 - 16), RANGE), (dict(page_stride=1 << 62), RANGE)]
BAD_BATCHES = [
    (dict(page_table=None), INVALID), (dict(kv_len=None), INVALID), (dict(row_start=None), INVALID), (dict(kv_len=0x4002), INVALID), (dict(errors=0x6001), INVALID),
    (dict(reserved=5), INVALID), (dict(n_seqs=65536), RANGE), (dict(n_rows=1 << 31), RANGE), (dict(max_rows=0), RANGE), (dict(max_rows=4), RANGE),
    (dict(max_kv=1025), RANGE), (dict(max_kv=(1 << 30) + 1, table_stride=1 << 30), RANGE)]


def statuses(T, cache, batch):
    L, bytes_ = T.lib(), C.c_uint64()
    return [L.tent_kv_append(cache, batch, make_append(T), None), L.tent_kv_read(cache, batch, 0x1000, 0x2000, 1024, None),
            L.tent_kv_attend(cache, batch, make_attend(T), None), L.tent_kv_attend_workspace(cache, batch, make_attend(T), bytes_)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches_that_are_refused(T, change, status):
    assert set(statuses(T, make_cache(T, **change), make_batch(T))) == {status}
    packed = make_cache(T, bits=4)
    assert T.lib().tent_kv_pack(make_cache(T, **change), packed, 0x100, 0x200, 3, None, None) == status


@pytest.mark.parametrize("change,status", BAD_BATCHES)
def test_batches_that_are_refused(T, change, status):
    assert set(statuses(T, make_cache(T), make_batch(T, **change))) == {status}


def test_null_structures(T):
    L, c, b = T.lib(), make_cache(T), make_batch(T)
    assert set(statuses(T, None, b)) == {INVALID} and set(statuses(T, c, None)) == {INVALID}
    assert L.tent_kv_append(c, b, None, None) == INVALID and L.tent_kv_attend(c, b, None, None) == INVALID
    assert L.tent_kv_attend_workspace(c, b, make_attend(T), None) == INVALID
    assert L.tent_kv_pack(None, c, 0x100, 0x200, 3, None, None) == INVALID and L.tent_kv_pack(c, None, 0x100, 0x200, 3, None, None) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(v=0x3004), INVALID), (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(k_stride=1028), INVALID), (dict(flags=2), INVALID),
    (dict(reserved=1), INVALID), (dict(q_weight=0x5002), INVALID), (dict(k_weight=0x6008), INVALID), (dict(rope=0x7004), INVALID), (dict(positions=0x8001), INVALID),
    (dict(q_out=0x1000, q_out_stride=8192), INVALID), (dict(k_stride=1016), RANGE), (dict(q_stride=4088), RANGE), (dict(v_stride=1 << 60), RANGE),
    (dict(q_heads=1025), RANGE), (dict(eps=-1e-6), RANGE), (dict(eps=math.nan), RANGE), (dict(eps=math.inf), RANGE), (dict(rope_rows=0), RANGE), (dict(rope_dim=0), RANGE),
    (dict(rope_dim=144), RANGE), (dict(rope_dim=24), RANGE)])
def test_append_arguments_that_are_refused(T, change, status):
    assert T.lib().tent_kv_append(make_cache(T), make_batch(T), make_append(T, **change), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(q=0x1002), INVALID), (dict(lse=0x3002), INVALID), (dict(flags=2), INVALID), (dict(out_stride=4100), INVALID),
    (dict(q_heads=0), RANGE), (dict(q_heads=12), RANGE), (dict(q_heads=1032), RANGE), (dict(q_stride=4088), RANGE), (dict(scale=0.0), RANGE), (dict(scale=-1.0), RANGE),
    (dict(scale=math.nan), RANGE), (dict(scale=math.inf), RANGE), (dict(window=(1 << 30) + 1), RANGE),
    (dict(workspace=None), INVALID), (dict(workspace=0x40008), INVALID), (dict(workspace_bytes=1024), RANGE)])
def test_attend_arguments_that_are_refused(T, change, status):
    assert T.lib().tent_kv_attend(make_cache(T), make_batch(T), make_attend(T, **change), None) == status


def test_pack_and_read_arguments_that_are_refused(T):
    L, c, b = T.lib(), make_cache(T), make_batch(T)
    packed = make_cache(T, bits=4, page_stride=8704)

    def pack(src, dst, a=0x100, to=0x200, n=3, errors=None):
        return L.tent_kv_pack(src, dst, a, to, n, errors, None)

    assert pack(packed, packed) == INVALID and pack(c, c) == INVALID and pack(packed, c) == INVALID
    assert pack(c, packed, a=None) == INVALID and pack(c, packed, to=0x201) == INVALID and pack(c, packed, errors=0x302) == INVALID
    for other in (dict(type=1), dict(kv_heads=4), dict(head_dim=64), dict(page_tokens=8)):
        assert pack(c, make_cache(T, bits=4, **other)) == RANGE
    assert pack(c, packed, n=1 << 31) == RANGE and pack(c, packed, n=0) == 0
    assert L.tent_kv_read(c, b, None, 0x100, 1024, None) == INVALID and L.tent_kv_read(c, b, 0x100, 0x104, 1024, None) == INVALID
    assert L.tent_kv_read(c, b, 0x100, 0x200, 1020, None) == INVALID and L.tent_kv_read(c, b, 0x100, 0x200, 1016, None) == RANGE
    assert L.tent_kv_packed_page(16, 8, 128) == 8704 and L.tent_kv_packed_page(1, 1, 64) == 48
    assert L.tent_kv_packed_page(3, 8, 128) == 0 and L.tent_kv_packed_page(16, 8, 80) == 0


def test_nothing_to_do_needs_no_device(T):
    for change in (dict(n_seqs=0), dict(n_rows=0)):
        assert set(statuses(T, make_cache(T), make_batch(T, page_table=None, **change))) == {0}


def test_structures_are_laid_out_as_in_the_header(T, tmp_path):
    names = ["tent_kv_cache", "tent_kv_batch", "tent_kv_append_args", "tent_kv_attend_args"]
    lines = []
    for n in names:
        lines.append(f'printf("{n} %zu", sizeof({n}));')
        lines += [f'printf(" %zu", offsetof({n}, {f}));' for f, _ in getattr(T, n)._fields_]
        lines.append('printf("\\n");')
    consts = ["TENT_BF16", "TENT_FP16", "TENT_KV_BAD_SEQUENCE", "TENT_KV_BAD_PAGE", "TENT_KV_BAD_POSITION", "TENT_KV_MAX_HEADS", "TENT_KV_MAX_PAGE_TOKENS",
              "TENT_KV_ROPE_PAIRS", "TENT_KV_ATTEND_ALL"]
    lines.append('printf("consts' + " %d" * len(consts) + '\\n", ' + ", ".join(f"(int){c}" for c in consts) + ");")
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tent.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    out = {l.split()[0]: [int(x) for x in l.split()[1:]] for l in subprocess.check_output([str(exe)]).decode().splitlines()}
    for n in names:
        s = getattr(T, n)
        assert out[n] == [C.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
    assert out["consts"] == [getattr(T, c) for c in consts]


ADDRESSING = r'''
#include <assert.h>
#include <stdio.h>
#include "kv_pages.h"
using namespace tent;
int main()
{
    int32_t row_start[] = {0, 2, 2, 5, 4, 9, 9}, kv_len[] = {40, 0, 2, 8, 8, 900};
    int32_t table[6 * 4];
    for (int i = 0; i < 24; ++i) table[i] = i % 5 ? i % 10 : -1 - i;
    table[1] = 10; table[2] = 0x7FFFFFFF; table[3] = 9;
    tent_kv_batch b{};
    b.page_table = table; b.kv_len = kv_len; b.row_start = row_start; b.n_seqs = 6; b.table_stride = 4; b.n_rows = 8; b.max_rows = 3; b.max_kv = 64;
    KvSeq s = kv_sequence(b, 0);
    assert(!s.bad && s.row0 == 0 && s.rows == 2 && s.len == 40);
    s = kv_sequence(b, 1);
    assert(!s.bad && s.rows == 0 && s.len == 0);
    s = kv_sequence(b, 2);                                     // three rows, two tokens: its first row is at position -1
    assert(!s.bad && s.rows == 3 && s.len == 2);
    assert(kv_sequence(b, 3).bad && kv_sequence(b, 3).rows == 0);          // descending
    assert(kv_sequence(b, 4).bad);                             // past n_rows, and more than max_rows
    assert(kv_sequence(b, 5).bad);                             // more than max_kv
    row_start[0] = -1;
    assert(kv_sequence(b, 0).bad);
    row_start[0] = 0; kv_len[0] = -3;
    assert(kv_sequence(b, 0).bad);
    kv_len[0] = 64;
    assert(!kv_sequence(b, 0).bad);
    // pages: 16 tokens each, far apart
    tent_kv_cache c{};
    c.k = c.v = (void*)0x1000; c.n_pages = 10; c.page_stride = 1ull << 33; c.page_tokens = 16; c.kv_heads = 2; c.head_dim = 64; c.type = TENT_FP16; c.bits = 4;
    KvCache d = kv_cache_dev(c);
    assert(d.page_shift == 4 && d.heads == 2 && d.n_pages == 10);
    assert(kv_page_of(d, b, 0, 0) == -1);                      // -1
    assert(kv_page_of(d, b, 0, 16) == -1 && kv_page_of(d, b, 0, 31) == -1);    // one past the last page
    assert(kv_page_of(d, b, 0, 32) == -1);                     // 2^31 - 1
    assert(kv_page_of(d, b, 0, 63) == (int64_t)(9ull << 33));
    assert(kv_page_of(d, b, 1, 17) == -1 && kv_page_of(d, b, 1, 47) == (int64_t)(6ull << 33));
    c.page_tokens = 1;
    assert(kv_cache_dev(c).page_shift == 0);
    assert(kv_page_bytes(16, 8, 128, 16) == 32768 && kv_page_bytes(16, 8, 128, 4) == 8704 && kv_page_bytes(1024, 1024, 256, 16) == 1ull << 29);
    // what a row sees
    auto is = [](KvSpan s, int lo, int hi) { return s.lo == lo && s.hi == hi; };
    assert(is(kv_span(0, 1, 1, 0, false), 0, 1) && is(kv_span(0, 3, 10, 0, false), 0, 8) && is(kv_span(2, 3, 10, 0, false), 0, 10));
    assert(is(kv_span(2, 3, 10, 4, false), 6, 10) && is(kv_span(0, 3, 10, 1, false), 7, 8) && is(kv_span(0, 3, 10, 8, false), 0, 8));
    assert(is(kv_span(0, 3, 2, 0, false), 0, 0) && is(kv_span(1, 3, 2, 5, false), 0, 1) && is(kv_span(0, 2, 0, 3, true), 0, 0));
    assert(is(kv_span(0, 3, 10, 0, true), 0, 10) && is(kv_span(0, 3, 10, 4, true), 6, 10) && is(kv_span(0, 1, 1 << 30, 1u << 30, false), 0, 1 << 30));
    printf("ok\n");
    return 0;
}
'''


def test_addresses_and_sequences_on_the_host(tmp_path):
    src = tmp_path / "addressing.cpp"
    src.write_text(ADDRESSING)
    exe = tmp_path / "addressing"
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                           os.path.join(ROOT, "paper_2604_00368_amd", "csrc"), "-o", str(exe), str(src)])
    assert subprocess.check_output([str(exe)]).decode() == "ok\n"


# ---- what a call enqueues ------------------------------------------------------------------------
from test_host_calls import fake  # noqa: E402,F401


def run(fake, scenario):
    env = dict(os.environ)
    env["LD_LIBRARY_PATH"] = os.pathsep.join(p for p in (str(fake.parent), env.get("LD_LIBRARY_PATH")) if p)
    code = f"import sys; sys.path[:0] = [{ROOT!r}, {HERE!r}]; import test_kv_host as t; t.{scenario}()"
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def kernels_of(call, stream):
    """Names of the kernels that `call` launches; it does nothing else, and nothing on another stream."""
    hip = C.CDLL("libamdhip64.so.7")
    hip.fake_kernel_name.restype = C.c_char_p
    hip.fake_kernel_name.argtypes = [C.c_void_p]
    hip.fake_log_clear()
    assert call() == 0
    names = []
    for i in range(hip.fake_log_size()):
        where, what = C.c_void_p(), C.c_void_p()
        assert hip.fake_log_at(i, C.byref(where), C.byref(what)) == LAUNCH and where.value == stream
        names.append(hip.fake_kernel_name(what).decode())
    return names


def scenario_enqueued():
    from paper_2604_00368_amd import binding as T
    L, stream = T.lib(), 0xA0
    short, long = make_batch(T, max_kv=200), make_batch(T, max_kv=64 * 16 * 100, table_stride=6400)
    many = make_batch(T, n_rows=5000, max_rows=4000, n_seqs=40)

    def need(batch, args):
        n = C.c_uint64()
        assert L.tent_kv_attend_workspace(make_cache(T), batch, args, n) == 0
        return n.value

    for change in (dict(), dict(type=1), dict(bits=4, page_stride=8704), dict(type=1, bits=4, page_stride=8704)):
        c = make_cache(T, **change)
        assert len(kernels_of(lambda: L.tent_kv_append(c, short, make_append(T), stream), stream)) == 1
        assert len(kernels_of(lambda: L.tent_kv_read(c, many, 0x1000, 0x2000, 1024, stream), stream)) == 1
        for batch, kinds in ((short, ["narrow"]), (long, ["narrow", "join"]), (many, ["wide"])):
            names = kernels_of(lambda: L.tent_kv_attend(c, batch, make_attend(T), stream), stream)
            assert [k for k, n in zip(kinds, names) if k in n] == kinds and len(names) == len(kinds), names
            assert (need(batch, make_attend(T)) > 0) == ("join" in kinds)
        # just the workspace it asks for is enough, a byte less is not
        args = make_attend(T, workspace_bytes=need(long, make_attend(T)))
        assert L.tent_kv_attend(c, long, args, stream) == 0
        args.workspace_bytes -= 1
        assert L.tent_kv_attend(c, long, args, stream) == RANGE
    assert len(kernels_of(lambda: L.tent_kv_pack(make_cache(T), make_cache(T, bits=4, page_stride=8704), 0x100, 0x200, 7, 0x300, stream), stream)) == 1


def test_calls_enqueue_kernels_only(fake, T):  # noqa: F811
    run(fake, "scenario_enqueued")
