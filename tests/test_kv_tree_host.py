"""Trees of drafted tokens, verification and eviction without a device: refusals, what a call enqueues (over the stand-in runtime of
fake_hip.c), and what a tree's rows see, compiled for the host."""
import ctypes as C
import math
import os
import subprocess

import pytest

import test_kv_host as H
import test_kv_launches as Launches
from test_host_calls import fake  # noqa: F401
from test_kv_host import INVALID, RANGE, ROOT, T, make_attend, make_batch, make_cache  # noqa: F401


def make_tree(T, **change):  # noqa: F811
    return T.tent_kv_tree(**{**dict(masks=0x8000, mask_stride=1, reserved=0), **change})


def make_verify(T, **change):  # noqa: F811
    d = dict(target=0x1000, draft=0x2000, target_stride=50000, draft_stride=50000, tokens=0x3000, parents=0x4000, accept=0x5000, next=0x6000, path=0x7000,
             counts=0x8000, token=0x9000, workspace=0x40000, workspace_bytes=1 << 40, vocab=50000, path_stride=2, type=2, reserved=0)
    return T.tent_kv_verify_args(**{**d, **change})


def make_weigh(T, **change):  # noqa: F811
    d = dict(q=0x1000, lse=0x2000, weights=0x3000, weights_out=0x3000, q_stride=4096, weights_stride=1000, workspace=0x40000, workspace_bytes=1 << 40, q_heads=32, n_lists=8, window=0, flags=0, scale=0.1, reserved=0)
    return T.tent_kv_weigh_args(**{**d, **change})


def make_choose(T, **change):  # noqa: F811
    d = dict(weights=0x1000, lists=0x2000, counts=0x90000000, weights_stride=1000, list_stride=100, n_lists=8, budget=100, first=4, recent=20)
    return T.tent_kv_choose_args(**{**d, **change})


def make_keep(T, **change):  # noqa: F811
    d = dict(lists=0x1000, counts=0x2000, to_table=None, kv_len_out=0x90000000, weights=None, weights_out=None, list_stride=100, weights_stride=0, n_lists=8, n_weights=0,
             to_stride=0, most=100, flags=0, reserved=0)
    return T.tent_kv_keep_args(**{**d, **change})


LONG = dict(vocab=1 << 20, target_stride=1 << 20, draft_stride=1 << 20)     # a vocabulary that takes a workspace


def calls(T, cache, batch):  # noqa: F811
    L = T.lib()
    return {"tree": L.tent_kv_attend_tree(cache, batch, make_attend(T), make_tree(T), None), "verify": L.tent_kv_verify(batch, make_verify(T), None),
            "weigh": L.tent_kv_weigh(cache, batch, make_weigh(T), None), "choose": L.tent_kv_choose(batch, make_choose(T), None),
            "keep": L.tent_kv_keep(cache, batch, make_keep(T), None)}


@pytest.mark.parametrize("change,status", H.BAD_CACHES)
def test_caches_that_are_refused(T, change, status):  # noqa: F811
    got = calls(T, make_cache(T, **change), make_batch(T, n_seqs=0))
    assert {got[n] for n in ("tree", "weigh", "keep")} == {status}


@pytest.mark.parametrize("change,status", H.BAD_BATCHES)
def test_batches_that_are_refused(T, change, status):  # noqa: F811
    got = calls(T, make_cache(T), make_batch(T, **change))
    pages = [c for c in ("page_table",) if c in change] or change == dict(max_kv=1025)     # verify and choose take none
    for name, s in got.items():
        if not (pages and name in ("verify", "choose")):
            assert s == status, name


def test_null_structures(T):  # noqa: F811
    L, c, b = T.lib(), make_cache(T), make_batch(T)
    assert L.tent_kv_attend_tree(c, b, make_attend(T), None, None) == INVALID and L.tent_kv_attend_tree(c, b, None, make_tree(T), None) == INVALID
    assert L.tent_kv_verify(b, None, None) == INVALID and L.tent_kv_verify(None, make_verify(T), None) == INVALID
    assert L.tent_kv_verify_workspace(b, make_verify(T), None) == INVALID and L.tent_kv_verify_workspace(b, None, C.c_uint64()) == INVALID
    assert L.tent_kv_weigh(c, b, None, None) == INVALID and L.tent_kv_weigh(None, b, make_weigh(T), None) == INVALID
    assert L.tent_kv_choose(b, None, None) == INVALID and L.tent_kv_choose(None, make_choose(T), None) == INVALID
    assert L.tent_kv_keep(c, b, None, None) == INVALID and L.tent_kv_keep(c, None, make_keep(T), None) == INVALID


@pytest.mark.parametrize("tree,args,status", [
    (dict(masks=None), {}, INVALID), (dict(masks=0x8004), {}, INVALID), (dict(reserved=1), {}, INVALID), ({}, dict(flags=1), INVALID), (dict(mask_stride=0), {}, RANGE),
    ({}, dict(window=1), RANGE), ({}, dict(q=None), INVALID), ({}, dict(lse=0x3002), INVALID), ({}, dict(q_heads=12), RANGE), ({}, dict(scale=math.nan), RANGE)])
def test_trees_that_are_refused(T, tree, args, status):  # noqa: F811
    assert T.lib().tent_kv_attend_tree(make_cache(T), make_batch(T), make_attend(T, **args), make_tree(T, **tree), None) == status


def test_a_tree_needs_a_bit_for_every_row(T):  # noqa: F811
    call = lambda rows, words: T.lib().tent_kv_attend_tree(make_cache(T), make_batch(T, n_rows=rows, max_rows=rows), make_attend(T, q=None), make_tree(T, mask_stride=words), None)  # noqa: E731
    assert call(65, 1) == RANGE and call(64, 1) == INVALID and call(65, 2) == INVALID       # INVALID: as far as the queries


@pytest.mark.parametrize("change,status", [
    (dict(target=None), INVALID), (dict(tokens=None), INVALID), (dict(accept=None), INVALID), (dict(next=None), INVALID), (dict(path=None), INVALID), (dict(counts=None), INVALID),
    (dict(token=None), INVALID), (dict(type=3), INVALID), (dict(reserved=1), INVALID), (dict(target=0x1002), INVALID), (dict(draft=0x2001), INVALID), (dict(tokens=0x3001), INVALID),
    (dict(parents=0x4002), INVALID), (dict(token=0x9001), INVALID), (dict(vocab=0), RANGE), (dict(vocab=(1 << 20) + 1), RANGE), (dict(target_stride=49999), RANGE),
    (dict(draft_stride=49999), RANGE), (dict(target_stride=1 << 60), RANGE), (dict(path_stride=1), RANGE), (dict(workspace=None, **LONG), INVALID), (dict(workspace=0x40008, **LONG), INVALID),
    (dict(workspace_bytes=8, **LONG), RANGE)])
def test_verify_arguments_that_are_refused(T, change, status):  # noqa: F811
    assert T.lib().tent_kv_verify(make_batch(T), make_verify(T, **change), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(lse=None), INVALID), (dict(weights_out=None), INVALID), (dict(weights=0x3002), INVALID), (dict(lse=0x2001), INVALID), (dict(flags=2), INVALID),
    (dict(reserved=1), INVALID), (dict(q_stride=4100), INVALID), (dict(q_stride=4088), RANGE), (dict(q_heads=0), RANGE), (dict(q_heads=12), RANGE), (dict(n_lists=2), RANGE),
    (dict(n_lists=0), RANGE), (dict(window=(1 << 30) + 1), RANGE), (dict(scale=0.0), RANGE), (dict(scale=math.inf), RANGE), (dict(weights_stride=999), RANGE),
    (dict(weights_stride=1 << 60), RANGE), (dict(weights_out=0x3004), INVALID), (dict(weights=0x3000 + 4 * 1999), INVALID)])
def test_weigh_arguments_that_are_refused(T, change, status):  # noqa: F811
    assert T.lib().tent_kv_weigh(make_cache(T), make_batch(T), make_weigh(T, **change), None) == status


def test_weigh_refuses_more_lines_than_it_can_number(T):  # noqa: F811
    # 2^21 rows of 1024 query heads on one: 256 GiB of queries
    c = make_cache(T, kv_heads=1, head_dim=64, page_stride=2048)
    for rows, status in ((1 << 21, RANGE), ((1 << 21) - 1, RANGE), ((1 << 21) - 2, 0)):
        b, n = make_batch(T, n_rows=1 << 21, max_rows=rows, n_seqs=1), C.c_uint64()
        a = make_weigh(T, q_heads=1024, q_stride=65536, n_lists=1)
        assert T.lib().tent_kv_weigh_workspace(c, b, a, n) == status
        if status:
            assert T.lib().tent_kv_weigh(c, b, a, None) == status
    assert T.lib().tent_kv_weigh_workspace(c, make_batch(T, n_rows=0, max_rows=0xFFFFFFFF), a, n) == 0


@pytest.mark.parametrize("change,status", [
    (dict(weights=None), INVALID), (dict(lists=None), INVALID), (dict(counts=None), INVALID), (dict(lists=0x2002), INVALID), (dict(n_lists=0), RANGE), (dict(n_lists=1025), RANGE),
    (dict(budget=0, first=0, recent=0), RANGE), (dict(budget=(1 << 30) + 1, list_stride=1 << 31), RANGE), (dict(recent=97), RANGE), (dict(first=0xFFFFFFFF, recent=1), RANGE),
    (dict(weights_stride=999), RANGE), (dict(list_stride=99), RANGE), (dict(list_stride=1 << 60), RANGE), (dict(counts=0x4000), INVALID),
    (dict(counts=0x4004), INVALID), (dict(counts=0x3FFC), INVALID)])
def test_choose_arguments_that_are_refused(T, change, status):  # noqa: F811
    assert T.lib().tent_kv_choose(make_batch(T), make_choose(T, **change), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(lists=None), INVALID), (dict(counts=None), INVALID), (dict(lists=0x1002), INVALID), (dict(to_table=0x9001), INVALID), (dict(kv_len_out=0x4000), INVALID),
    (dict(kv_len_out=0x4004), INVALID), (dict(kv_len_out=0x2000), INVALID), (dict(counts=0x90000004), INVALID), (dict(kv_len_out=0x5004), INVALID),
    (dict(flags=2), INVALID), (dict(reserved=1), INVALID), (dict(weights=0x5000), INVALID), (dict(weights_out=0x5000), INVALID),
    (dict(weights=0x5000, weights_out=0x5000, n_weights=8, weights_stride=1000, to_table=0x9000, to_stride=64), INVALID), (dict(n_lists=2), RANGE), (dict(n_lists=0), RANGE),
    (dict(most=101), RANGE), (dict(list_stride=1 << 60), RANGE), (dict(weights=0x5000, weights_out=0x6000, n_weights=1, weights_stride=1000), RANGE),
    (dict(weights=0x5000, weights_out=0x6000, n_weights=4, weights_stride=1000), RANGE), (dict(weights=0x5000, weights_out=0x6000, n_weights=8, weights_stride=999), RANGE),
    (dict(weights=0x5000, weights_out=0x6000, n_weights=8, weights_stride=1000), INVALID)])
def test_keep_arguments_that_are_refused(T, change, status):  # noqa: F811
    assert T.lib().tent_kv_keep(make_cache(T), make_batch(T), make_keep(T, **change), None) == status


def test_keep_refuses_more_pages_than_lie_between_rows(T):  # noqa: F811
    for entries in (65, 0xFFFFFFFF):
        assert T.lib().tent_kv_keep(make_cache(T), make_batch(T), make_keep(T, to_table=0x9000, to_stride=64, to_entries=entries), None) == RANGE


def test_nothing_to_do_needs_no_device(T):  # noqa: F811
    assert set(calls(T, make_cache(T), make_batch(T, n_seqs=0, page_table=None)).values()) == {0}
    assert calls(T, make_cache(T), make_batch(T, n_rows=0, page_table=None))["tree"] == 0


def test_structures_are_laid_out_as_in_the_header(T, tmp_path):  # noqa: F811
    names = ["tent_kv_tree", "tent_kv_verify_args", "tent_kv_weigh_args", "tent_kv_choose_args", "tent_kv_keep_args"]
    lines = []
    for n in names:
        lines.append(f'printf("{n} %zu", sizeof({n}));')
        lines += [f'printf(" %zu", offsetof({n}, {f}));' for f, _ in getattr(T, n)._fields_]
        lines.append('printf("\\n");')
    consts = ["TENT_FP32", "TENT_KV_BAD_TOKEN", "TENT_KV_MAX_VOCAB", "TENT_KV_KEEP_ROWS", "TENT_KV_CHOOSE_WHOLE"]
    lines.append('printf("consts' + " %d" * len(consts) + '\\n", ' + ", ".join(f"(int){c}" for c in consts) + ");")
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tent.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    out = {line.split()[0]: [int(x) for x in line.split()[1:]] for line in subprocess.check_output([str(exe)]).decode().splitlines()}
    for n in names:
        s = getattr(T, n)
        assert out[n] == [C.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
    assert out["consts"] == [getattr(T, c) for c in consts]


SEEN = r'''
#include <assert.h>
#include <stdio.h>
#include <stdlib.h>
#include "kv_pages.h"
using namespace tent;
int main()
{
    srand(5);
    for (int round = 0; round < 20000; ++round) {
        const int rows = 1 + rand() % 200, len = rand() % 3 ? rows + rand() % 300 : rand() % 200, words = (rows + 63) / 64;
        uint64_t mask[4];
        for (int i = 0; i < 4; ++i) mask[i] = rand() % 4 ? (uint64_t)rand() << 40 ^ (uint64_t)rand() << 20 ^ rand() : rand() % 2 ? ~0ull : 0;
        int deep = 0;
        for (int j = 0; j < rows; ++j) deep += mask[j / 64] >> (j % 64) & 1;
        const int window = rand() % 2 ? 0 : rows + rand() % 300;
        const KvTreeSpan s = kv_tree_span(rows, len, (uint32_t)window, deep);
        assert(s.base == len - rows && s.len == len && s.words == words && s.lo >= 0);
        const int t0 = rand() % (len + 70);
        int read = 0;
        const uint64_t got = kv_tree_bits(s, t0, [&](int i) { assert(i >= 0); ++read; return i < words ? mask[i] : 0; });
        assert(read <= 2);
        for (int i = 0; i < 64; ++i) {
            const int t = t0 + i, j = t - s.base;
            if (t >= len) continue;                            // what is behind the last token is for the caller
            const bool sees = t < s.base ? !window || t >= s.base + deep - window : mask[j / 64] >> (j % 64) & 1;
            assert((got >> i & 1) == sees);
        }
    }
    printf("ok\n");
    return 0;
}
'''


def test_what_rows_of_a_tree_see_on_the_host(tmp_path):
    src = tmp_path / "seen.cpp"
    src.write_text(SEEN)
    exe = tmp_path / "seen"
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                           os.path.join(ROOT, "paper_2604_00368_amd", "csrc"), "-o", str(exe), str(src)])
    assert subprocess.check_output([str(exe)]).decode() == "ok\n"


MEET = r'''
#include <assert.h>
#include <stdio.h>
#include <stdlib.h>
#include "kv_pages.h"
using namespace tent;
int main()
{
    static float pool[400];
    srand(7);
    for (int round = 0; round < 50000; ++round) {
        const int lists = 1 + rand() % 4, width = rand() % 9, stride = width + rand() % 12 + (width == 0);
        const int a = rand() % 200, b = rand() % 3 ? rand() % 200 : a + (rand() % 5 - 2) * stride;
        if (b < 0) continue;
        bool meet = false;                                     // a value of one where one of another place is in the other
        for (int i = 0; i < lists; ++i) for (int j = 0; j < lists; ++j) for (int x = 0; x < width; ++x) {
            const int y = a + i * stride + x - b - j * stride;
            meet |= y >= 0 && y < width && a != b;
        }
        assert(kv_lists_meet(pool + a, pool + b, lists, width, stride) == meet);
        const int x_bytes = rand() % 40, y_bytes = rand() % 40;
        const char *x = (const char*)pool + a, *y = (const char*)pool + b;
        meet = x_bytes && y_bytes && x < y + y_bytes && y < x + x_bytes;
        if (x_bytes && y_bytes) assert(kv_meet(x, x_bytes, y, y_bytes) == meet);
    }
    assert(!kv_lists_meet(nullptr, pool, 2, 2, 2) && !kv_meet(nullptr, 4, pool, 4));
    printf("ok\n");
    return 0;
}
'''


def test_memory_that_two_arguments_share_is_found_on_the_host(tmp_path):
    src = tmp_path / "meet.cpp"
    src.write_text(MEET)
    exe = tmp_path / "meet"
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                           os.path.join(ROOT, "paper_2604_00368_amd", "csrc"), "-o", str(exe), str(src)])
    assert subprocess.check_output([str(exe)]).decode() == "ok\n"


KEPT = r'''
#include <assert.h>
#include <stdio.h>
#include "kv_pages.h"
using namespace tent;
int main()
{
    const int32_t most = 1 << 30;                               // the longest list, and the longest sequence
    const int32_t sizes[] = {0, 1, 255, 4096, most - 4096, most - 1, most};
    for (int32_t len : sizes) for (int32_t rows : sizes) for (int32_t count : sizes) for (int flags = 0; flags < 4; ++flags) {
        const bool by_rows = flags & 1, elsewhere = flags & 2;
        const KvKept k = kv_kept(KvSeq{0, rows, len, false}, by_rows, elsewhere, count, most);
        const int64_t base = by_rows ? (int64_t)len - rows : 0, have = by_rows ? rows : len;
        assert(k.bad == (base < 0 || (!elsewhere && count > have) || base + count > 0x7FFFFFFF));
        if (k.bad) continue;
        assert(k.length() == base + count && k.length() >= 0);
        for (int32_t room : sizes) {                             // places of weights behind the last: from here on, 256 threads
            const int64_t from = k.length_up_to(room);
            assert(from == (base + count < room ? base + count : room) && from + 255 <= 0x7FFFFFFF);
        }
    }
    assert(kv_kept(KvSeq{0, 0, most, false}, true, true, most, most).bad);
    assert(kv_kept(KvSeq{0, 0, 5, false}, false, true, -1, most).bad && kv_kept(KvSeq{0, 0, 5, false}, false, true, 8, 7).bad);
    assert(kv_kept(KvSeq{0, 0, 0, true}, false, true, 0, most).bad);
    printf("ok\n");
    return 0;
}
'''


def test_lengths_of_what_is_kept_fit_on_the_host(tmp_path):
    src = tmp_path / "kept.cpp"
    src.write_text(KEPT)
    exe = tmp_path / "kept"
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                           os.path.join(ROOT, "paper_2604_00368_amd", "csrc"), "-o", str(exe), str(src)])
    assert subprocess.check_output([str(exe)]).decode() == "ok\n"


# ---- what a call enqueues ------------------------------------------------------------------------
def scenario_enqueued():
    from paper_2604_00368_amd import binding as T
    L, stream = T.lib(), 0xA0
    short, long = make_batch(T, max_kv=200), make_batch(T, max_kv=64 * 16 * 100, table_stride=6400)
    many = make_batch(T, n_rows=5000, max_rows=4000, n_seqs=40)

    def names(call):
        return H.kernels_of(call, stream)

    def same(got, kinds):
        assert len(got) == len(kinds) and all(k in n for k, n in zip(kinds, got)), got

    for change in (dict(), dict(type=1), dict(bits=4, page_stride=8704), dict(type=1, bits=4, page_stride=8704)):
        c = make_cache(T, **change)
        sixteen = make_batch(T, n_rows=32, max_rows=16, max_kv=200)
        for batch, kinds in ((short, ["narrow"]), (long, ["narrow", "join"]), (sixteen, ["wide"]), (many, ["wide"])):
            same(names(lambda: L.tent_kv_attend_tree(c, batch, make_attend(T), make_tree(T, mask_stride=63), stream)), kinds)
        n = C.c_uint64()
        args = make_attend(T)
        assert L.tent_kv_attend_tree_workspace(c, long, args, n) == 0
        args.workspace_bytes = n.value
        assert L.tent_kv_attend_tree(c, long, args, make_tree(T), stream) == 0
        args.workspace_bytes -= 1
        assert L.tent_kv_attend_tree(c, long, args, make_tree(T), stream) == RANGE
        for n_lists in (1, 8):
            same(names(lambda: L.tent_kv_weigh(c, long, make_weigh(T, n_lists=n_lists, weights_stride=1 << 20), stream)), ["few"])
            args, n = make_weigh(T, n_lists=n_lists), C.c_uint64()
            same(names(lambda: L.tent_kv_weigh(c, many, args, stream)), ["many"] if n_lists == 8 else ["many", "weigh_join"])
            assert L.tent_kv_weigh_workspace(c, many, args, n) == 0 and n.value == (0 if n_lists == 8 else 40 * 8 * 1000 * 4)
            args.workspace_bytes = n.value
            assert L.tent_kv_weigh(c, many, args, stream) == 0
            if n.value:
                args.workspace_bytes -= 1
                assert L.tent_kv_weigh(c, many, args, stream) == RANGE
                args.workspace_bytes, args.workspace = n.value, 0x40008
                assert L.tent_kv_weigh(c, many, args, stream) == INVALID
            same(names(lambda: L.tent_kv_keep(c, short, make_keep(T, n_lists=n_lists), stream)), ["keep_kernel"])
        same(names(lambda: L.tent_kv_keep(c, short, make_keep(T, weights=0x5000, weights_out=0x5000, n_weights=8, weights_stride=200), stream)), ["keep_kernel", "keep_weights"])
        same(names(lambda: L.tent_kv_keep(c, short, make_keep(T, to_table=0x9000, to_stride=64, most=0), stream)), ["keep_copy"])
    for batch in (short, make_batch(T, n_rows=0)):                       # sequences of no rows have tokens, too
        same(names(lambda: L.tent_kv_choose(batch, make_choose(T), stream)), ["choose"])
        same(names(lambda: L.tent_kv_keep(make_cache(T), batch, make_keep(T), stream)), ["keep_kernel"])
        same(names(lambda: L.tent_kv_weigh(make_cache(T), batch, make_weigh(T), stream)), ["few"])
    n, args = C.c_uint64(), make_choose(T, weights_stride=1 << 20, workspace=0x40000, workspace_bytes=1 << 40)
    for tokens in (16384, 16385, 100000):
        batch = make_batch(T, max_kv=tokens, table_stride=6400)
        same(names(lambda: L.tent_kv_choose(batch, args, stream)), ["choose_kernel"] if tokens == 16384 else ["choose_part"] * 4)
        assert L.tent_kv_choose_workspace(batch, args, n) == 0 and (n.value == 0) == (tokens == 16384)
    args.workspace_bytes = n.value
    assert L.tent_kv_choose(batch, args, stream) == 0
    args.workspace_bytes -= 1
    assert L.tent_kv_choose(batch, args, stream) == RANGE
    args.workspace_bytes, args.workspace = n.value, 0x40008
    assert L.tent_kv_choose(batch, args, stream) == INVALID
    args.n_lists = 0
    assert L.tent_kv_choose_workspace(batch, args, n) == RANGE and L.tent_kv_choose_workspace(batch, None, n) == INVALID
    for kind in range(3):
        for change in (dict(), dict(draft=None), dict(parents=None), dict(vocab=100), dict(vocab=1 << 20, target_stride=1 << 20, draft_stride=1 << 20)):
            args, n = make_verify(T, type=kind, path_stride=4000, **change), C.c_uint64()
            for batch in (short, many):
                assert L.tent_kv_verify_workspace(batch, args, n) == 0
                got = names(lambda: L.tent_kv_verify(batch, args, stream))
                assert "verify_kernel" in got[-1] and all("ahead" in x for x in got[:-1]) and len(got) <= 2 and (len(got) == 2) == (n.value > 0)
                args.workspace_bytes = n.value
                assert L.tent_kv_verify(batch, args, stream) == 0
                if n.value:
                    args.workspace_bytes -= 1
                    assert L.tent_kv_verify(batch, args, stream) == RANGE
                args.workspace_bytes = 1 << 40
        same(names(lambda: L.tent_kv_verify(make_batch(T, n_rows=0), make_verify(T, target=None, tokens=None, accept=None, next=None), stream)), ["verify_kernel"])


def test_calls_enqueue_kernels_only(fake):  # noqa: F811
    in_child(fake, "scenario_enqueued")


def in_child(fake, scenario):  # noqa: F811
    import sys
    env = dict(os.environ)
    env["LD_LIBRARY_PATH"] = os.pathsep.join(p for p in (str(fake.parent), env.get("LD_LIBRARY_PATH")) if p)
    code = f"import sys; sys.path[:0] = [{ROOT!r}, {H.HERE!r}]; import test_kv_tree_host as t; t.{scenario}()"
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def scenario_large_calls():
    from paper_2604_00368_amd import binding as T
    L = T.lib()
    tiny = make_cache(T, page_tokens=1, kv_heads=1, head_dim=64, n_pages=1 << 30, page_stride=128)
    heads = make_cache(T, kv_heads=1024, head_dim=64, page_stride=1024 * 64 * 2, page_tokens=1)
    every = make_batch(T, n_seqs=65535, n_rows=65535, max_rows=1, max_kv=64)

    def small(call, status=0):
        got, grids = Launches.grids_of(call)
        assert got == status
        for blocks, threads in grids:
            assert blocks[0] * threads[0] < 1 << 32 and blocks[1] <= 65535 and blocks[2] == 1 and threads[1:] == (1, 1)
        return sum(b[0] for b, _ in grids)

    assert small(lambda: L.tent_kv_choose(every, make_choose(T, n_lists=1024), None)) == 65535 * 1024
    assert small(lambda: L.tent_kv_keep(heads, every, make_keep(T, n_lists=1024), None)) == 65535 * 1024
    assert small(lambda: L.tent_kv_keep(heads, every, make_keep(T, n_lists=1024, to_table=0x9000, to_stride=64, most=100000, list_stride=100000), None), RANGE) == 0
    assert small(lambda: L.tent_kv_keep(tiny, every, make_keep(T, n_lists=1, to_table=0x9000, to_stride=64, most=100000, list_stride=100000), None)) >= 65535 * 3125
    assert small(lambda: L.tent_kv_keep(heads, every, make_keep(T, n_lists=1, weights=0x5000, weights_out=0x5000, n_weights=1024, weights_stride=64), None)) == 65535 * 2048
    assert small(lambda: L.tent_kv_weigh(heads, every, make_weigh(T, q_heads=1024, q_stride=65536, n_lists=1024, weights_stride=64), None)) >= 65535 * 1024
    long = make_batch(T, n_rows=1, max_rows=1, n_seqs=1, max_kv=1 << 30, table_stride=1 << 30)
    assert small(lambda: L.tent_kv_weigh(tiny, long, make_weigh(T, q_heads=1, q_stride=64, n_lists=1, weights_stride=1 << 30), None)) > 1000
    assert small(lambda: L.tent_kv_verify(every, make_verify(T, vocab=1 << 20, target_stride=1 << 20, draft_stride=1 << 20), None)) == 65535
    assert small(lambda: L.tent_kv_choose(long, make_choose(T, n_lists=1, weights_stride=1 << 30, workspace=0x40000, workspace_bytes=1 << 40), None)) == 4 * 64
    few = make_batch(T, n_seqs=128, n_rows=1280, max_rows=10)
    assert small(lambda: L.tent_kv_verify(few, make_verify(T, path_stride=10, **LONG), None)) == 128 * (512 // 4 + 1)


def test_calls_of_any_size_stay_below_what_a_launch_takes(fake):  # noqa: F811
    in_child(fake, "scenario_large_calls")
