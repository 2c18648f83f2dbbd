"""How many workgroups the paged cache operators launch at once, over the stand-in runtime of fake_hip.c."""
import ctypes as C
import os
import subprocess
import sys

import test_kv_host as H
from test_host_calls import HERE, ROOT, fake  # noqa: F401
from test_kv_host import T  # noqa: F401


def in_child(fake, scenario):  # noqa: F811
    env = dict(os.environ)
    env["LD_LIBRARY_PATH"] = os.pathsep.join(p for p in (str(fake.parent), env.get("LD_LIBRARY_PATH")) if p)
    code = f"import sys; sys.path[:0] = [{ROOT!r}, {HERE!r}]; import test_kv_launches as t; t.{scenario}()"
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def grids_of(call):
    """Workgroups and lanes of a workgroup of each launch."""
    hip = C.CDLL("libamdhip64.so.7")
    hip.fake_log_clear()
    status = call()
    out = []
    for i in range(hip.fake_log_size()):
        blocks, threads = (C.c_uint * 3)(), (C.c_uint * 3)()
        hip.fake_log_grid(i, blocks, threads)
        out.append((tuple(blocks), tuple(threads)))
    return status, out


def check(call, total):
    status, grids = grids_of(call)
    assert status == 0 and grids
    for blocks, threads in grids:
        assert threads[1:] == (1, 1) and blocks[2] == 1 and blocks[1] <= 65535
        assert blocks[0] * threads[0] < 1 << 32 and blocks[1] * threads[1] < 1 << 32
    assert sum(blocks[0] for blocks, _ in grids) == total
    return len(grids)


def scenario_large_calls():
    from paper_2604_00368_amd import binding as T
    L = T.lib()
    tiny = dict(page_tokens=1, kv_heads=1, head_dim=64, n_pages=1 << 30)
    small, packed = H.make_cache(T, page_stride=128, **tiny), H.make_cache(T, page_stride=48, bits=4, **tiny)
    for n in (100, (1 << 22) + 1, (1 << 23) - 1, 1 << 23, 20_000_000, 1 << 29):
        many = check(lambda: L.tent_kv_pack(small, packed, 0x100, 0x200, n, None, None), 2 * n)
        assert many == -(-2 * n // (1 << 23))
    assert L.tent_kv_pack(small, packed, 0x100, 0x200, (1 << 30), None, None) == H.RANGE       # 2^31 workgroups

    # one row a workgroup, and sixteen
    wide = H.make_cache(T)
    for n in (5000, (1 << 24) - 1, 1 << 24, (1 << 31) - 1):
        rows = H.make_batch(T, n_rows=n, max_rows=n, max_kv=1000)
        check(lambda: L.tent_kv_append(wide, rows, H.make_append(T), None), n)
        narrow = H.make_append(T, q=None, q_out=None, q_weight=None, q_heads=0, k_stride=64, v_stride=64, rope=None)
        check(lambda: L.tent_kv_append(small, H.make_batch(T, n_rows=n, max_rows=n, max_kv=64), narrow, None), -(-n // 16))
        if n > 16384:
            check(lambda: L.tent_kv_read(small, H.make_batch(T, n_rows=n, max_rows=n, max_kv=64), 0x100, 0x200, 64, None), -(-n // 16))

    # attention: sequences by heads, and tiles of 128 lines by sequences by heads
    heads = H.make_cache(T, kv_heads=512, head_dim=64, page_stride=512 * 64 * 2, page_tokens=1)
    one = H.make_batch(T, n_seqs=65535, n_rows=65535, max_rows=1, max_kv=1)
    args = dict(q_heads=512, q_stride=512 * 64, out_stride=512 * 64)
    assert check(lambda: L.tent_kv_attend(heads, one, H.make_attend(T, **args), None), 65536 * 512) == 4
    mixed = H.make_batch(T, n_seqs=2048, n_rows=40000, max_rows=32768, max_kv=40000, table_stride=2500)
    assert check(lambda: L.tent_kv_attend(wide, mixed, H.make_attend(T), None), 1024 * 2048 * 8) == 2
    # more than 2^31 - 1 of them are refused
    most = H.make_batch(T, n_seqs=65535, n_rows=1 << 30, max_rows=1 << 20, max_kv=64)
    assert L.tent_kv_attend(heads, most, H.make_attend(T, **args), None) == H.RANGE


def test_calls_of_any_size_stay_below_what_a_launch_takes(fake, T):  # noqa: F811
    in_child(fake, "scenario_large_calls")


def scenario_joins():
    # every call that splits its tokens joins them in one launch that is small enough
    from paper_2604_00368_amd import binding as T
    L = T.lib()
    joined = 0
    for heads in (1, 8, 64, 1024):
        for group in (1, 4, 16):
            if heads * group > 1024:
                continue
            c = H.make_cache(T, kv_heads=heads, page_stride=16 * heads * 128 * 2)
            for n_seqs in (1, 7, 1000):
                for rows in (1, 3, 64, 500, 4000, 100000, 1 << 22):
                    b = H.make_batch(T, n_seqs=n_seqs, n_rows=rows * n_seqs, max_rows=rows, max_kv=1 << 30, table_stride=1 << 26)
                    a = H.make_attend(T, q_heads=heads * group, q_stride=heads * group * 128, out_stride=heads * group * 128, workspace_bytes=1 << 62)
                    status, grids = grids_of(lambda: L.tent_kv_attend(c, b, a, None))
                    if status == H.RANGE:
                        continue
                    assert status == 0
                    for blocks, threads in grids:
                        assert blocks[0] * threads[0] < 1 << 32 and blocks[1] <= 65535
                    joined += grids[-1][0][1] == n_seqs and n_seqs > 1
    assert joined > 20


def test_joins_stay_below_what_a_launch_takes(fake, T):  # noqa: F811
    in_child(fake, "scenario_joins")
