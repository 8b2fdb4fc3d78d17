"""The order of PagedCache's calls, without a GPU: a chunk's rows belong to the last `begin`, until pages or slots go to something else."""
import types

import pytest
import torch

from paper_2512_14069_b200 import binding as rb
from paper_2512_14069_b200.cache import PagedCache


@pytest.fixture
def calls(monkeypatch):
    """What reaches the library."""
    seen = []
    for name in ("radar_cache_extend", "radar_paged_store", "radar_chunk_attention"):
        monkeypatch.setattr(rb, name, lambda ctx, name=name, **kw: seen.append((name, kw)))
    monkeypatch.setattr(rb, "radar_chunk_attn_workspace_bytes", lambda *a: 4096)
    return seen


def _cache():
    return PagedCache(None, n_layers=2, B=2, Hq=4, Hkv=2, d=64, page_size=16, n_pages=8, max_len=64, max_new=40, device="cpu")


K = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
Q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
NEW = torch.tensor([3, 2], dtype=torch.int32)
STEP = types.SimpleNamespace(accept_len=torch.zeros(2, dtype=torch.int32), path_nodes=torch.zeros(2, 4, dtype=torch.int32))
TREE = torch.zeros(2, 2, 12, 2, 64, dtype=torch.bfloat16)


def _both(c):
    c.store(1, K, K)
    c.attention(1, Q, Q)


def _refused(c, calls):
    n = len(calls)
    with pytest.raises(ValueError, match="begin"):
        c.store(1, K, K)
    with pytest.raises(ValueError, match="begin"):
        c.attention(1, Q, Q)
    with pytest.raises(ValueError, match="begin"):
        c.attention(1, Q, Q, max_new=3)
    assert len(calls) == n


def test_a_chunk_is_there_from_begin_to_append_or_release(calls):
    c = _cache()
    _refused(c, calls)
    for end in (lambda: c.release(torch.tensor([0, 1])), lambda: c.append(STEP, TREE, TREE)):
        c.begin(NEW, 5)
        _both(c)
        _both(c)
        assert [name for name, _ in calls[-4:]] == ["radar_paged_store", "radar_chunk_attention"] * 2 and calls[-1][1]["max_new"] == 5 and calls[-2][1]["slots"].numel() == 5
        end()
        _refused(c, calls)
    c.begin(NEW, 5)
    c.begin(NEW, 4)                                      # the last one counts
    _both(c)
    assert calls[-1][1]["max_new"] == 4 and calls[-2][1]["slots"].numel() == 4


def test_a_call_that_is_refused_leaves_the_chunk(calls):
    c = _cache()
    c.begin(NEW, 5)
    with pytest.raises(ValueError, match="made for 40"):
        c.begin(NEW, 41)
    with pytest.raises(ValueError, match="made for 40"):
        c.append(types.SimpleNamespace(accept_len=STEP.accept_len, path_nodes=torch.zeros(2, 30, dtype=torch.int32)), TREE, TREE)
    _both(c)


def test_a_chunk_of_nothing_is_one(calls):
    c = _cache()
    c.begin(torch.zeros(2, dtype=torch.int32), 0)
    c.store(0, K[:0], K[:0])
    c.attention(0, Q[:0], Q[:0])


def test_positions_without_a_rotation_are_refused(calls):
    """pos, pair_axis and neighbours say how inv_freq turns rows; without it they would be left out of account."""
    c = _cache()
    c.begin(NEW, 5)
    n = len(calls)
    pos, axis, freq = torch.zeros(5, dtype=torch.int32), torch.zeros(32, dtype=torch.uint8), torch.ones(32)
    for turn in (dict(pos=pos), dict(pair_axis=axis), dict(neighbours=True), dict(pos=pos, pair_axis=axis, neighbours=True, inv_freq=None)):
        with pytest.raises(ValueError, match="inv_freq"):
            c.store(0, K, K, **turn)
    assert len(calls) == n
    c.store(0, K, K, neighbours=False, pair_axis=None, inv_freq=None)
    assert calls[-1][1].get("pos") is None
    c.store(0, K, K, inv_freq=freq, pair_axis=axis, neighbours=True)
    assert calls[-1][1]["pos"].data_ptr() == c.pos.data_ptr() and calls[-1][1]["pos"].numel() == 5
    c.store(0, K, K, inv_freq=freq, pos=pos)
    assert calls[-1][1]["pos"] is pos


def test_an_append_is_of_the_steps_size(calls):
    """... and not of the room for a chunk: a step accepts path_nodes.numel() tokens at most, whatever the cache was made for."""
    c = _cache()
    c.append(STEP, TREE, TREE)
    (_, extend), (_, store) = calls[-2:]
    assert extend["slots"].numel() == extend["src_row"].numel() == store["slots"].numel() == store["src_row"].numel() == STEP.path_nodes.numel() < c.slots.numel()
    assert extend["slots"].data_ptr() == store["slots"].data_ptr() and extend["src_row"].data_ptr() == store["src_row"].data_ptr()
