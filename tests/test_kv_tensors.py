"""What the tensor side of the paged cache operators (kv.py) refuses and hands on, without a device: torch's CUDA parts and the
library are replaced by stand-ins that note where each call and each allocation goes."""
import contextlib
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2604_00368_amd import binding as T, kv  # noqa: E402


class OnGpu(torch.Tensor):
    """A tensor in host memory that says it is on a GPU."""

    __torch_function__ = torch._C._disabled_torch_function_impl

    def __new__(cls, data, index, log):
        self = torch.Tensor._make_subclass(cls, data, data.requires_grad)
        self._index, self._log = index, log
        return self

    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self._index))

    def record_stream(self, stream):
        self._log.append(("record", self.data_ptr(), stream.cuda_stream))


class Stream:
    def __init__(self, device, handle):
        self.device, self.cuda_stream = torch.device("cuda", device), handle

    def __eq__(self, other):
        return self.cuda_stream == other.cuda_stream


class Gpus:
    """torch with two GPUs, of which `at` is current, and a library that notes its calls."""

    def __init__(self):
        self.at, self.streams, self.log = 0, {0: Stream(0, 0), 1: Stream(1, 0)}, []

        @contextlib.contextmanager
        def device(d):
            old, self.at = self.at, torch.device(d).index if not isinstance(d, int) else d
            yield
            self.at = old

        @contextlib.contextmanager
        def stream(s):
            old, self.at = self.at, s.device.index
            before, self.streams[self.at] = self.streams[self.at], s
            yield
            self.streams[self.at], self.at = before, old

        def external(handle, device=None):
            return Stream(torch.device(device).index, handle)

        self.cuda = types.SimpleNamespace(
            Stream=Stream, ExternalStream=external, device=device, stream=stream, current_device=lambda: self.at,
            current_stream=lambda d=None: self.streams[self.at if d is None else d if isinstance(d, int) else torch.device(d).index])

    def __getattr__(self, name):
        return getattr(torch, name)

    def made(self, tensor, device):
        out = OnGpu(tensor, torch.device(device).index if torch.device(device).index is not None else self.at, self.log)
        self.log.append(("new", out.data_ptr(), self.at, self.streams[out._index].cuda_stream))
        return out

    def empty(self, *shape, dtype, device):
        return self.made(torch.empty(*shape, dtype=dtype), device)

    def zeros(self, *shape, dtype, device):
        return self.made(torch.zeros(*shape, dtype=dtype), device)

    # ---- the library
    def tent_strerror(self, status):
        return b"refused"

    def tent_kv_packed_page(self, page_tokens, heads, dim):
        return -(-page_tokens * heads * (dim // 2 + dim // 32) // 16) * 16

    def tent_kv_attend_workspace(self, cache, batch, args, need):
        need._obj.value = 4096
        return 0

    def call(self, name, stream):
        self.log.append((name, self.at, stream.value or 0))
        return 0

    def tent_kv_append(self, cache, batch, args, stream):
        return self.call("append", stream)

    def tent_kv_pack(self, src, dst, src_pages, dst_pages, n, errors, stream):
        return self.call("pack", stream)

    def tent_kv_read(self, cache, batch, k, v, stride, stream):
        return self.call("read", stream)

    def tent_kv_attend(self, cache, batch, args, stream):
        return self.call("attend", stream)


class Step:
    """A cache of two pages, a packed one beside it, and a step of two sequences, all on GPU `index`."""

    def __init__(self, gpus, index=0):
        def on(t):
            return OnGpu(t, index, gpus.log)

        def rows(heads):
            return on(torch.zeros(3, heads, 64, dtype=torch.bfloat16))

        self.on = on
        self.cache = kv.Cache(*(on(torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)) for _ in "kv"))
        self.packed = kv.Cache(*(on(torch.zeros(2, 16 * 2 * 34, dtype=torch.uint8)) for _ in "kv"), dtype=torch.bfloat16, page_tokens=16,
                               kv_heads=2, head_dim=64)
        self.batch = kv.Batch(on(torch.zeros(2, 4, dtype=torch.int32)), on(torch.ones(2, dtype=torch.int32)),
                              on(torch.tensor([0, 1, 3], dtype=torch.int32)), 3, 2, 20)
        self.q, self.k, self.v = rows(4), rows(2), rows(2)
        self.weight, self.rope = on(torch.ones(64, dtype=torch.bfloat16)), on(torch.zeros(20, 64))
        self.pages, self.errors = on(torch.zeros(2, dtype=torch.int32)), on(torch.zeros(1, dtype=torch.int32))

    def append(self, **change):
        a = dict(k=self.k, v=self.v, q=self.q, q_weight=self.weight, k_weight=self.weight, rope=self.rope, positions=None)
        a.update(change)
        return kv.append(self.cache, self.batch, a.pop("k"), a.pop("v"), **a)

    def pack(self, **change):
        a = dict(src_pages=self.pages, dst_pages=self.pages, errors=self.errors)
        a.update(change)
        return kv.pack(self.cache, self.packed, **a)

    def read(self, **change):
        return kv.read(self.cache, self.batch, **change)

    def attend(self, **change):
        return kv.attend(self.cache, self.batch, change.pop("q", self.q), want_lse=True, **change)

    def calls(self):
        return {"append": self.append, "pack": self.pack, "read": self.read, "attend": self.attend}


@pytest.fixture
def gpus(monkeypatch):
    g = Gpus()
    monkeypatch.setattr(kv, "torch", g)
    monkeypatch.setattr(kv, "_raw_stream", lambda index: g.streams[index].cuda_stream)
    monkeypatch.setattr(kv, "_current_device", lambda: g.at, raising=False)
    monkeypatch.setattr(T, "lib", lambda: g)
    return g


def test_calls_are_handed_on(gpus):
    for name, call in Step(gpus).calls().items():
        call()
        assert gpus.log[-1] == (name, 0, 0)


def test_a_workspace_that_is_not_whole_or_elsewhere_is_refused(gpus):
    s = Step(gpus)
    room = torch.zeros(1 << 14, dtype=torch.uint8)
    s.attend(workspace=s.on(room))
    # every second byte; the same byte 2^14 times, with nothing behind it; another GPU
    for bad in (s.on(room[::2]), s.on(room[:1].expand(1 << 14)), OnGpu(room, 1, gpus.log), room):
        n = len(gpus.log)
        with pytest.raises(ValueError, match="workspace"):
            s.attend(workspace=bad)
        assert not any(e[0] == "attend" for e in gpus.log[n:])


def test_errors_of_pack_on_another_gpu_are_refused(gpus):
    s = Step(gpus)
    with pytest.raises(ValueError, match="errors"):
        s.pack(errors=OnGpu(torch.zeros(1, dtype=torch.int32), 1, gpus.log))
    assert not any(e[0] == "pack" for e in gpus.log)


def test_what_a_call_allocates_belongs_to_the_stream_it_is_given(gpus):
    s = Step(gpus)
    extra = {"append": (s.k, s.v, s.q, s.weight, s.rope), "pack": (s.pages, s.errors), "read": (), "attend": (s.q,)}
    made_by = {"append": 1, "pack": 0, "read": 2, "attend": 3}           # attend: the output, the logsumexps and the workspace
    for given in (Stream(0, 0x55), 0x55):
        for name, call in s.calls().items():
            gpus.log.clear()
            result = call(stream=given)
            assert (name, 0, 0x55) in gpus.log and gpus.streams[0].cuda_stream == 0
            made = [e for e in gpus.log if e[0] == "new"]
            assert len(made) == made_by[name] and all(e[3] == 0x55 for e in made)
            # the allocator is told of both streams, for what was passed in before the work is enqueued
            at = gpus.log.index((name, 0, 0x55))
            before, behind = ({e[1:] for e in part if e[0] == "record"} for part in (gpus.log[:at], gpus.log[at:]))
            outs = [] if result is None else [result] if isinstance(result, torch.Tensor) else list(result)
            tensors = (*s.cache.tensors, *(s.packed.tensors if name == "pack" else s.batch.tensors), *extra[name])
            assert before == {(t.data_ptr(), 0x55) for t in tensors} and behind == {(t.data_ptr(), 0) for t in outs}


def test_tensors_that_are_passed_in_are_not_made_anew(gpus):
    s = Step(gpus)
    out = s.on(torch.zeros(3, 4, 64, dtype=torch.bfloat16))
    room = s.on(torch.zeros(4096, dtype=torch.uint8))
    gpus.log.clear()
    assert s.append(q_out=out, stream=0x55) is out and s.attend(out=out, workspace=room, stream=0x55)[0] is out
    k, v = (s.on(torch.zeros(3, 2, 64, dtype=torch.bfloat16)) for _ in "kv")
    assert s.read(k_out=k, v_out=v, stream=0x55) == (k, v)
    assert len([e for e in gpus.log if e[0] == "new"]) == 1              # the logsumexps
    for t in (out, room, k, v):
        assert ("record", t.data_ptr(), 0x55) in gpus.log and ("record", t.data_ptr(), 0) not in gpus.log


def test_the_current_stream_may_be_given(gpus):
    s = Step(gpus)
    gpus.log.clear()
    with gpus.cuda.stream(Stream(0, 0x77)):
        for call in s.calls().values():
            call()
            call(stream=Stream(0, 0x77))
    assert not [e for e in gpus.log if e[0] == "record"]
    assert all(e[-1] == 0x77 for e in gpus.log)


def test_a_stream_of_another_gpu_is_refused(gpus):
    for name, call in Step(gpus).calls().items():
        with pytest.raises(ValueError, match="stream"):
            call(stream=Stream(1, 0x55))
        assert not any(e[0] == name for e in gpus.log)


@pytest.mark.parametrize("index", [0, 1])
def test_calls_go_to_the_device_of_their_tensors(gpus, index):
    s = Step(gpus, index)
    gpus.streams = {0: Stream(0, 0x10), 1: Stream(1, 0x20)}
    for at in (0, 1):
        gpus.at = at
        for name, call in s.calls().items():
            for given, handle in ((None, (0x10, 0x20)[index]), (Stream(index, 0x55), 0x55), (gpus.streams[index], (0x10, 0x20)[index]), (0x66, 0x66)):
                gpus.log.clear()
                call(stream=given)
                assert (name, index, handle) in gpus.log
                assert gpus.at == at and [gpus.streams[i].cuda_stream for i in (0, 1)] == [0x10, 0x20]


def test_gradients_are_not_dropped_without_a_word(gpus):
    s = Step(gpus)

    def learns(t):
        return s.on(t.as_subclass(torch.Tensor).detach().clone().requires_grad_())

    cases = [(s.append, name, dict([(name, learns(getattr(s, of)))])) for name, of in
             (("k", "k"), ("v", "v"), ("q", "q"), ("q_weight", "weight"), ("k_weight", "weight"), ("rope", "rope"))]
    cases += [(s.append, "q_out", dict(q_out=learns(s.q))), (s.attend, "q", dict(q=learns(s.q))), (s.attend, "out", dict(out=learns(s.q))),
              (s.read, "k_out", dict(k_out=learns(s.k), v_out=s.v))]
    for call, name, change in cases:
        gpus.log.clear()
        with pytest.raises(ValueError, match=f"{name} requires gradients"):
            call(**change)
        assert not [e for e in gpus.log if e[0] in ("append", "attend", "read")]
        with torch.no_grad():                                            # a serving program's weights are parameters, too
            call(**change)
        assert gpus.log[-1][0] in ("append", "attend", "read")
    pool = learns(s.cache.k)
    with pytest.raises(ValueError, match="k requires gradients"):
        kv.Cache(pool, pool)
    with torch.no_grad():
        kv.Cache(pool, pool)


def test_pools_of_nothing_are_refused(gpus):
    s = Step(gpus)
    for shape in ((0, 16, 2, 64), (2, 0, 2, 64), (2, 16, 0, 64), (2, 16, 2, 0)):
        pool = s.on(torch.zeros(*shape, dtype=torch.bfloat16))
        with pytest.raises(ValueError, match="page"):
            kv.Cache(pool, pool)
    pool = s.on(torch.zeros(0, 16 * 2 * 34, dtype=torch.uint8))
    with pytest.raises(ValueError, match="page"):
        kv.Cache(pool, pool, dtype=torch.bfloat16, page_tokens=16, kv_heads=2, head_dim=64)
