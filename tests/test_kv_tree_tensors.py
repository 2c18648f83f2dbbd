"""What the tensor side (kv.py) of trees, verification and eviction refuses and hands on, without a device, and the masks of trees."""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv_tree_reference as R  # noqa: E402
import test_kv_tensors as Base  # noqa: E402
from paper_2604_00368_amd import binding as T, kv  # noqa: E402
from test_kv_tensors import OnGpu, Stream  # noqa: E402

NAMES = ("attend_tree", "verify", "weigh", "choose", "keep")


class Gpus(Base.Gpus):
    def tent_kv_attend_tree_workspace(self, cache, batch, args, need):
        return self.tent_kv_attend_workspace(cache, batch, args, need)

    def tent_kv_attend_tree(self, cache, batch, args, tree, stream):
        self.words = tree._obj.mask_stride
        return self.call("attend_tree", stream)

    def tent_kv_verify_workspace(self, batch, args, need):
        need._obj.value = 4096
        return 0

    def tent_kv_verify(self, batch, args, stream):
        self.args = T.tent_kv_verify_args.from_buffer_copy(args._obj)
        return self.call("verify", stream)

    def tent_kv_weigh_workspace(self, cache, batch, args, need):
        need._obj.value = 4096
        return 0

    def tent_kv_weigh(self, cache, batch, args, stream):
        self.args = T.tent_kv_weigh_args.from_buffer_copy(args._obj)
        return self.call("weigh", stream)

    def tent_kv_choose_workspace(self, batch, args, need):
        need._obj.value = 2048
        return 0

    def tent_kv_choose(self, batch, args, stream):
        self.args = T.tent_kv_choose_args.from_buffer_copy(args._obj)
        return self.call("choose", stream)

    def tent_kv_keep(self, cache, batch, args, stream):
        self.args = T.tent_kv_keep_args.from_buffer_copy(args._obj)
        return self.call("keep", stream)


class Step(Base.Step):
    """Two sequences of one and two rows, 20 tokens at most, two heads of the cache."""

    def __init__(self, gpus, index=0):
        super().__init__(gpus, index)
        on = self.on
        i32 = torch.int32
        self.tree, self.tokens, self.parents = on(torch.zeros(3, 1, dtype=torch.int64)), on(torch.zeros(3, dtype=i32)), on(torch.zeros(3, dtype=i32))
        self.target, self.draft, self.accept, self.next = on(torch.zeros(3, 50)), on(torch.zeros(3, 50)), on(torch.zeros(3)), on(torch.zeros(2))
        self.lse, self.weights = on(torch.zeros(3, 4)), on(torch.zeros(2, 2, 20))
        self.lists, self.counts, self.to_table = on(torch.zeros(2, 2, 7, dtype=i32)), on(torch.zeros(2, dtype=i32)), on(torch.zeros(2, 3, dtype=i32))

    def attend_tree(self, **change):
        return kv.attend(self.cache, self.batch, change.pop("q", self.q), want_lse=True, **{"tree": self.tree, **change})

    def verify(self, **change):
        a = dict(target=self.target, tokens=self.tokens, accept=self.accept, next=self.next, parents=self.parents, draft=self.draft)
        return kv.verify(self.batch, **{**a, **change})

    def weigh(self, **change):
        return kv.weigh(self.cache, self.batch, **{**dict(q=self.q, lse=self.lse, weights=self.weights), **change})

    def choose(self, **change):
        return kv.choose(self.batch, **{**dict(weights=self.weights, budget=7, first=1, recent=2), **change})

    def keep(self, **change):
        return kv.keep(self.cache, self.batch, **{**dict(lists=self.lists, counts=self.counts, weights=self.weights), **change})

    def calls(self):
        return {n: getattr(self, n) for n in NAMES}


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


def test_what_a_call_allocates_belongs_to_the_stream_it_is_given(gpus):
    s = Step(gpus)
    extra = {"attend_tree": (s.q, s.tree), "verify": (s.target, s.tokens, s.accept, s.next, s.parents, s.draft), "weigh": (s.q, s.lse, s.weights),
             "choose": (s.weights,), "keep": (s.lists, s.counts, s.weights)}
    made_by = {"attend_tree": 3, "verify": 4, "weigh": 1, "choose": 2, "keep": 1}
    for given in (Stream(0, 0x55), 0x55):
        for name, call in s.calls().items():
            gpus.log.clear()
            result = call(stream=given)
            assert (name, 0, 0x55) in gpus.log and gpus.streams[0].cuda_stream == 0
            made = [e for e in gpus.log if e[0] == "new"]
            assert len(made) == made_by[name] and all(e[3] == 0x55 for e in made)
            at = gpus.log.index((name, 0, 0x55))
            before, behind = ({e[1:] for e in part if e[0] == "record"} for part in (gpus.log[:at], gpus.log[at:]))
            outs = [result] if isinstance(result, torch.Tensor) else [x for x in result if x is not s.weights]
            cache = () if name in ("verify", "choose") else s.cache.tensors
            assert before == {(t.data_ptr(), 0x55) for t in (*cache, *s.batch.tensors, *extra[name])} and behind == {(t.data_ptr(), 0) for t in outs}


def test_tensors_that_are_passed_in_are_not_made_anew(gpus):
    s = Step(gpus)
    path, room, out, length = s.on(torch.zeros(2, 2, dtype=torch.int32)), s.on(torch.zeros(4096, dtype=torch.uint8)), s.on(torch.zeros(2, 2, 20)), s.on(torch.zeros(2, dtype=torch.int32))
    assert s.verify(path=path, workspace=room, stream=0x55)[0] is path
    assert s.weigh(out=out, stream=0x55) is out and s.weigh(out=s.weights, stream=0x55) is s.weights
    got = s.keep(weights_out=out, kv_len_out=length, stream=0x55)
    assert got[0] is length and got[1] is out
    assert s.keep(kv_len_out=length, stream=0x55)[1] is s.weights        # in place
    assert s.keep(weights=None, kv_len_out=length) is length
    for t in (path, room, out, length, s.weights):
        assert ("record", t.data_ptr(), 0x55) in gpus.log and ("record", t.data_ptr(), 0) not in gpus.log


def test_choose_from_long_lists_takes_a_workspace(gpus):
    s = Step(gpus)
    i32 = dict(dtype=torch.int32)
    batch = kv.Batch(s.on(torch.zeros(2, 20000, **i32)), s.on(torch.zeros(2, **i32)), s.on(torch.zeros(3, **i32)), 3, 2, 20000)
    weights, room = s.on(torch.zeros(2, 2, 20000)), s.on(torch.zeros(2100, dtype=torch.uint8))
    gpus.log.clear()
    kv.choose(batch, weights, 9, stream=0x55)
    assert gpus.args.workspace_bytes == 2048 and len([e for e in gpus.log if e[0] == "new"]) == 3
    kv.choose(batch, weights, 9, workspace=room, stream=0x55)
    assert (gpus.args.workspace, gpus.args.workspace_bytes) == (room.data_ptr(), 2100) and ("record", room.data_ptr(), 0x55) in gpus.log
    for wrong in (s.on(torch.zeros(2100, **i32)), s.on(torch.zeros(2, 4096, dtype=torch.uint8)[:, :2100]), torch.zeros(2100, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            kv.choose(batch, weights, 9, workspace=wrong)


@pytest.mark.parametrize("index", [0, 1])
def test_calls_go_to_the_device_of_their_tensors(gpus, index):
    s = Step(gpus, index)
    gpus.streams = {0: Stream(0, 0x10), 1: Stream(1, 0x20)}
    for at in (0, 1):
        gpus.at = at
        for name, call in s.calls().items():
            for given, handle in ((None, (0x10, 0x20)[index]), (Stream(index, 0x55), 0x55), (0x66, 0x66)):
                gpus.log.clear()
                call(stream=given)
                assert (name, index, handle) in gpus.log
                assert gpus.at == at and [gpus.streams[i].cuda_stream for i in (0, 1)] == [0x10, 0x20]
            with pytest.raises(ValueError, match="stream"):
                call(stream=Stream(1 - index, 0x55))


def test_gradients_are_not_dropped_without_a_word(gpus):
    s = Step(gpus)

    def learns(t):
        return s.on(t.as_subclass(torch.Tensor).detach().clone().requires_grad_())

    for call, name in ((s.attend_tree, "q"), (s.verify, "target"), (s.verify, "draft"), (s.verify, "accept"), (s.weigh, "q"), (s.weigh, "lse"), (s.weigh, "weights"),
                       (s.choose, "weights"), (s.keep, "weights")):
        gpus.log.clear()
        change = {name: learns(getattr(s, name))}
        with pytest.raises(ValueError, match=f"{name} requires gradients"):
            call(**change)
        assert not [e for e in gpus.log if e[0] in NAMES]
        with torch.no_grad():
            call(**change)
        assert [e for e in gpus.log if e[0] in NAMES]


def test_tensors_that_are_refused(gpus):
    s = Step(gpus)
    on, i32 = s.on, torch.int32
    away = lambda t: OnGpu(t, 1, gpus.log)  # noqa: E731
    bad = [
        (s.attend_tree, "tree", [on(torch.zeros(3, 1, dtype=i32)), on(torch.zeros(2, 1, dtype=torch.int64)), on(torch.zeros(3, dtype=torch.int64)),
                                 on(torch.zeros(3, 2, dtype=torch.int64)[:, :1]), away(torch.zeros(3, 1, dtype=torch.int64)), torch.zeros(3, 1, dtype=torch.int64)]),
        (s.verify, "target", [on(torch.zeros(3, 50, dtype=torch.float64)), on(torch.zeros(2, 50)), on(torch.zeros(50)), on(torch.zeros(3, 100)[:, ::2]), away(torch.zeros(3, 50)),
                              on(torch.zeros(1, 50).expand(3, 50)), None]),
        (s.verify, "draft", [on(torch.zeros(3, 50, dtype=torch.bfloat16)), on(torch.zeros(3, 51)), away(torch.zeros(3, 50))]),
        (s.verify, "tokens", [on(torch.zeros(3, dtype=torch.int64)), on(torch.zeros(2, dtype=i32)), on(torch.zeros(6, dtype=i32)[::2]), away(torch.zeros(3, dtype=i32))]),
        (s.verify, "parents", [on(torch.zeros(4, dtype=i32))]), (s.verify, "accept", [on(torch.zeros(3, dtype=torch.float64)), on(torch.zeros(2))]),
        (s.verify, "next", [on(torch.zeros(3))]), (s.verify, "path", [on(torch.zeros(2, 3, dtype=i32))]),
        (s.verify, "workspace", [on(torch.zeros(8192, dtype=torch.uint8)[::2]), away(torch.zeros(4096, dtype=torch.uint8))]),
        (s.weigh, "lse", [on(torch.zeros(3, 5)), on(torch.zeros(3, 8)[:, ::2]), away(torch.zeros(3, 4)), on(torch.zeros(3, 4, dtype=torch.bfloat16))]),
        (s.weigh, "weights", [on(torch.zeros(2, 2, 19)), on(torch.zeros(2, 20)), on(torch.zeros(2, 2, 40)[..., ::2]), on(torch.zeros(3, 2, 20)), away(torch.zeros(2, 2, 20))]),
        (lambda **change: s.weigh(weights=None, per_head=False, **change), "workspace", [on(torch.zeros(8192, dtype=torch.uint8)[::2]), away(torch.zeros(4096, dtype=torch.uint8))]),
        (s.weigh, "out", [on(torch.zeros(2, 2, 21)), on(torch.zeros(2, 1, 20))]),
        (s.choose, "weights", [on(torch.zeros(2, 2, 19)), on(torch.zeros(2, 2, 20, dtype=torch.float16)), on(torch.zeros(1, 2, 20).expand(2, 2, 20)), away(torch.zeros(2, 2, 20))]),
        (s.keep, "lists", [on(torch.zeros(2, 3, 7, dtype=i32)), on(torch.zeros(1, 2, 7, dtype=i32)), on(torch.zeros(2, 2, 7)), on(torch.zeros(2, 2, 14, dtype=i32)[..., ::2])]),
        (s.keep, "counts", [on(torch.zeros(3, dtype=i32)), on(torch.zeros(2))]), (s.keep, "kv_len_out", [on(torch.zeros(3, dtype=i32))]),
        (s.keep, "to_table", [on(torch.zeros(1, 3, dtype=i32)), on(torch.zeros(2, 3)), on(torch.zeros(1, 3, dtype=i32).expand(2, 3)), on(torch.zeros(2, 6, dtype=i32)[:, ::2])]),
        (s.keep, "weights", [on(torch.zeros(2, 1, 20)), on(torch.zeros(2, 2, 19))]), (s.keep, "weights_out", [on(torch.zeros(2, 2, 24))]),
    ]
    for call, name, tensors in bad:
        for t in tensors:
            n = len(gpus.log)
            with pytest.raises(ValueError):
                call(**{name: t})
            assert not any(e[0] in NAMES for e in gpus.log[n:]), (name, t.shape)
    for change in (dict(budget=0), dict(budget=2, first=1, recent=2), dict(first=-1), dict(recent=-1)):
        with pytest.raises(ValueError, match="budget"):
            s.choose(**change)
    with pytest.raises(ValueError, match="causal"):
        s.attend_tree(causal=False)
    with pytest.raises(ValueError, match="weights"):
        s.keep(weights=None, weights_out=s.weights)


def test_strides_are_handed_on(gpus):
    s = Step(gpus)
    on = s.on
    s.verify(target=on(torch.zeros(3, 64)[:, :50]), draft=None, parents=None)
    assert (gpus.args.target_stride, gpus.args.draft_stride, gpus.args.draft, gpus.args.parents, gpus.args.vocab, gpus.args.path_stride) == (64, 0, None, None, 50, 2)
    wide = on(torch.zeros(2, 2, 32)[..., :20])
    s.weigh(weights=wide, out=wide)
    assert gpus.args.weights_stride == 32 and gpus.args.weights == gpus.args.weights_out
    s.weigh(weights=None, per_head=False)
    assert gpus.args.n_lists == 1 and gpus.args.weights is None and gpus.args.weights_stride == 20 and gpus.args.workspace_bytes == 4096
    s.choose(weights=on(torch.zeros(2, 2, 32)), budget=5)
    assert (gpus.args.weights_stride, gpus.args.list_stride, gpus.args.n_lists) == (32, 5, 2)
    s.choose(weights=on(torch.zeros(2, 24)), budget=5)
    assert (gpus.args.weights_stride, gpus.args.n_lists, gpus.args.workspace) == (24, 1, None)
    s.keep(lists=on(torch.zeros(2, 9, dtype=torch.int32)[:, :4]), to_table=on(torch.zeros(2, 8, dtype=torch.int32)[:, :3]), rows=True)
    assert (gpus.args.list_stride, gpus.args.most, gpus.args.n_lists, gpus.args.to_stride, gpus.args.n_weights, gpus.args.flags) == (9, 4, 1, 8, 2, 1)
    assert gpus.args.weights != gpus.args.weights_out                    # to other pages: not in place


def test_tables_to_move_to_end_with_their_rows(gpus):
    """What lies between the rows of a table is not its own, and a table of no pages is not taken for none."""
    s = Step(gpus)
    on, i32 = s.on, torch.int32
    for table, stride, entries in ((torch.zeros(2, 8, dtype=i32)[:, 5:], 8, 3), (torch.zeros(2, 3, dtype=i32), 3, 3), (torch.zeros(2, 8, dtype=i32)[:, :1], 8, 1)):
        s.keep(to_table=on(table))
        assert (gpus.args.to_stride, gpus.args.to_entries) == (stride, entries) and gpus.args.to_table == table.data_ptr()
    s.keep()
    assert gpus.args.to_table is None and gpus.args.to_entries == 0
    n = len(gpus.log)
    far = torch.zeros(5, dtype=i32)
    for table in (torch.zeros(2, 0, dtype=i32), torch.zeros(2, 8, dtype=i32)[:, 3:3], far.as_strided((2, 3), (2, 1))):
        with pytest.raises(ValueError, match="to_table"):
            s.keep(to_table=on(table))
    assert not any(e[0] in NAMES for e in gpus.log[n:])
    nobody = kv.Batch(on(torch.zeros(0, 3, dtype=i32)), on(torch.zeros(0, dtype=i32)), on(torch.zeros(1, dtype=i32)), 0, 0, 20)
    kv.keep(s.cache, nobody, on(torch.zeros(0, 7, dtype=i32)), on(torch.zeros(0, dtype=i32)), to_table=on(torch.zeros(0, 3, dtype=i32)))
    assert gpus.log[-1][0] == "keep"


def test_outputs_that_share_memory_with_what_is_read_are_refused(gpus):
    s = Step(gpus)
    i32 = torch.int32
    store = torch.zeros(64, dtype=i32)
    part = lambda at, *shape, dtype=i32: s.on(store[at:at + int(np.prod(shape))].view(shape).view(dtype))  # noqa: E731
    rows = lambda at, n, width, apart: s.on(store.as_strided((n, width), (apart, 1), at))  # noqa: E731
    for at in range(12):                                                 # path: four values from 3 on
        for name, n in (("tokens", 3), ("parents", 3), ("accept", 3), ("next", 2)):
            x = part(at, n, dtype=torch.float32 if name in ("accept", "next") else i32)
            refused(gpus, s.verify, {"path": part(3, 2, 2), name: x}, at < 7 and at + n > 3)
    s.batch = kv.Batch(s.batch.page_table, part(40, 2), part(50, 3), 3, 2, 20)
    for at in range(36, 56):
        refused(gpus, s.verify, dict(path=part(at, 2, 2)), any(at <= x < at + 4 for x in (40, 41, 50, 51, 52)))
        if at not in (39, 40, 41, 49, 50, 51, 52):                       # those the library refuses
            refused(gpus, s.keep, dict(kv_len_out=part(at, 2)), False)
    for at in range(0, 30):                                              # lists of two values, nine apart, from 3 on: 3, 4, 12, 13
        refused(gpus, s.keep, dict(kv_len_out=part(at, 2), lists=rows(3, 2, 2, 9), weights=None), any(at <= x < at + 2 for x in (3, 4, 12, 13)))
        refused(gpus, s.keep, dict(kv_len_out=part(at, 2), to_table=rows(3, 2, 2, 9), weights=None), any(at <= x < at + 2 for x in (3, 4, 12, 13)))


def refused(gpus, call, change, is_refused):
    n = len(gpus.log)
    if is_refused:
        with pytest.raises(ValueError, match="share memory"):
            call(**change)
    else:
        call(**change)
    assert any(e[0] in NAMES for e in gpus.log[n:]) != is_refused


@pytest.mark.parametrize("seed", range(6))
def test_masks_of_trees(seed):
    rng = random.Random(seed)
    rows = [rng.choice([0, 1, 2, 17, 63, 64, 65, 130]) for _ in range(rng.randint(1, 7))] + [5]
    trees = [[rng.choice([i - 1, rng.randrange(-2, i + 2), rng.randrange(max(i, 1))]) for i in range(n)] for n in rows]
    starts = torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], dtype=torch.int32)
    masks, deep = kv.tree_masks(torch.tensor([p for t in trees for p in t], dtype=torch.int32), starts, max(rows))
    assert masks.dtype == torch.int64 and masks.is_contiguous() and deep.dtype == torch.int32
    seen = [R.ancestors(t) for t in trees if t]
    want = np.concatenate([R.words(x, masks.shape[1]) for x in seen])
    assert (masks.numpy() == want).all() and (deep.numpy() == np.concatenate([x.sum(1) - 1 for x in seen])).all()


def test_masks_of_no_rows():
    masks, deep = kv.tree_masks(torch.zeros(0, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 0)
    assert masks.shape == (0, 1) and deep.shape == (0,)
