"""The example that runs the paged cache operators around a migration (examples/migrate_and_answer.py), end to end."""
import importlib.util
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("migrate_and_answer", os.path.join(ROOT, "examples", "migrate_and_answer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def pages_of(cache, table, n):
    """K and V of a sequence's first n tokens in 64 bits."""
    at = torch.from_numpy(table[:-(-n // cache.page_tokens)]).long().cuda()
    return [R.page_values(p[at], cache.bits, cache.page_tokens, cache.kv_heads, cache.head_dim).reshape(-1, cache.kv_heads, cache.head_dim)[:n]
            for p in (cache.k, cache.v)]


def test_what_arrives_is_what_was_packed_and_the_answers_are_attention_over_it(example):
    prompts, steps = [70, 1, 133], 3
    r = example.run(prompts, steps, seed=4)
    assert r["moved"] * 3.7 < r["moved16"] < r["moved"] * 3.8
    assert r["answers"].shape == (sum(prompts), example.Q_HEADS, example.DIM) and bool(r["answers"].isfinite().all())
    assert len(r["outs"]) == steps
    for i, n in enumerate(prompts):
        arrived = pages_of(r["cache4"], r["table4"][i], n + steps)
        for got, source in zip(arrived, pages_of(r["cache16"], r["table16"][i], n)):
            assert np.array_equal(got[:n], R.decode4(*R.encode4(source, example.DTYPE)))
        want, _, mass, size = R.attend(r["last_q"][i:i + 1].cpu().double().numpy(), *arrived, 1 / math.sqrt(example.DIM), 0, True)
        bound, _ = R.attend_bounds(want, mass, size, n + steps, example.DIM, example.DTYPE)
        assert (np.abs(r["outs"][-1][i:i + 1].cpu().double().numpy() - want) <= bound).all()


def test_the_command(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["migrate_and_answer.py", "--prompts", "20", "33", "--steps", "2"])
    example.main()
    assert "2 prompts of 53 tokens answered" in capsys.readouterr().out
