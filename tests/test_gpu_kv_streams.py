"""Paged cache operators on streams of the caller's, with memory that they allocate themselves, on a GPU."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_kv import Setup, kv  # noqa: E402,F401

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("rows", [[1, 2], [70, 3]])
def test_split_calls_on_several_streams_do_not_share_their_workspaces(kv, rows, bits):
    s = Setup(kv, rows, [9001, 4447], BF16, bits, 8, 2, 128, 16, seed=3)
    need = kv.attend_workspace(s.cache, s.batch, 8)
    assert need > 0
    qs = [(2 * torch.randn(s.n_rows, 8, 128, generator=s.g)).to(BF16).cuda() for _ in range(4)]
    want = [kv.attend(s.cache, s.batch, q, want_lse=True) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(3)]
    given = streams + [streams[0].cuda_stream]                           # a handle is as good as a stream
    torch.cuda.synchronize()
    for _ in range(8):
        got = []
        for q, stream in zip(qs, given):
            got.append(kv.attend(s.cache, s.batch, q, want_lse=True, stream=stream))
            torch.full((need,), 0x7F, dtype=torch.uint8, device="cuda")  # allocated, written and given back on the current stream
        torch.cuda.synchronize()
        for (out, lse), (want_out, want_lse) in zip(got, want):
            assert torch.equal(out, want_out) and torch.equal(lse, want_lse)


def test_a_step_on_a_stream_of_the_callers(kv):
    s = Setup(kv, [1, 30], [5000, 90], BF16, 4, 8, 2, 128, 16, seed=4)
    q, k, v = (torch.randn(s.n_rows, h, 128, generator=s.g).to(BF16).cuda() for h in (8, 2, 2))
    rope = kv.rope_table(5000, 128)
    stream = torch.cuda.Stream()

    def step(on):
        turned = kv.append(s.cache, s.batch, k, v, q=q.clone() if on is None else q, rope=rope, stream=on)
        return (turned, *kv.read(s.cache, s.batch, stream=on), kv.attend(s.cache, s.batch, turned, stream=on))

    want = step(None)
    torch.cuda.synchronize()
    for _ in range(4):
        got = step(stream)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert int(s.batch.errors) == 0


def test_the_default_stream_by_its_handle(kv):
    s = Setup(kv, [2, 1], [5000, 7], BF16, 16, 4, 2, 64, 16, seed=5)
    q = s.q.cuda()
    want = kv.attend(s.cache, s.batch, q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for given in (0, torch.cuda.default_stream()):
            out = kv.attend(s.cache, s.batch, q, stream=given)
            torch.cuda.default_stream().synchronize()
            assert torch.equal(out, want)
        assert torch.cuda.current_stream() == side
