"""The example's books of pages, which need no GPU: a refusal leaves them as they were."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def cache():
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module.Cache(4, 1, 64, 16, 40, "cpu")


def books(cache):
    return [list(p) for p in cache.of], list(cache.lengths), sorted(cache.free)


def test_a_sequence_that_does_not_fit(cache):
    s, t = cache.new(), cache.new()
    cache.grow(s, 17)
    cache.grow(t, 1)
    before = books(cache)
    with pytest.raises(ValueError, match="longer than 40"):
        cache.grow(s, 24)
    assert books(cache) == before
    cache.free.clear()
    before = books(cache)
    with pytest.raises(MemoryError):
        cache.grow(t, 16)
    assert books(cache) == before
    assert cache.grow(t, 15)[0] == list(range(1, 16))


def test_all_sequences_of_a_step_or_none(cache):
    s, t = cache.new(), cache.new()
    cache.grow(s, 16)
    cache.grow(t, 32)
    before = books(cache)
    for seqs, tokens, refusal in [([s, t], 1, MemoryError), ([s, t], 9, ValueError), ([s, s], 1, ValueError)]:
        with pytest.raises(refusal):
            cache.grow_all(seqs, tokens)
        assert books(cache) == before
    positions, slots = cache.grow_all([s], 1)
    assert positions == [16] and slots == [cache.of[s][1] * 16]
    table, lengths = cache.table([t, s])
    assert lengths.tolist() == [32, 17] and table.tolist() == [cache.of[t] + [-1], cache.of[s] + [-1]]


def test_rooms_of_several_sequences_lie_one_behind_the_other(cache):
    s, t = cache.new(), cache.new()
    cache.grow(s, 15)
    positions, slots = cache.grow_all([t, s], 2)
    assert positions == [0, 1, 15, 16]
    assert slots == [cache.of[t][0] * 16, cache.of[t][0] * 16 + 1, cache.of[s][0] * 16 + 15, cache.of[s][1] * 16]
