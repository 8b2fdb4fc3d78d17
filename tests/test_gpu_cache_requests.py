"""Requests that a 4-bit cache has no room for, beside others that it holds; rows that are not in use; bounds of the lengths."""
import numpy as np
import pytest

from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


def _rows(seed, L, n, Hkv, d):
    import torch
    g = torch.Generator().manual_seed(seed)
    return tuple(torch.randn(L, n, Hkv, d, generator=g).cuda() for _ in range(2))


def _held(x):
    x = x.double().cpu().numpy()
    return C.values(*C.quantise(x)) if x.size else x


def _load(cache, lens):
    """The first lens[b] tokens of each request, as they come back: (K, V) a request."""
    import torch
    i32 = torch.int32
    start = torch.tensor([0] + list(np.cumsum(lens)), dtype=i32, device="cuda")
    n = int(sum(lens))
    K = torch.zeros(cache.n_layers, n, cache.Hkv, cache.d, device="cuda")
    V = torch.zeros_like(K)
    cache.load(torch.zeros(len(lens), dtype=i32, device="cuda"), start, K, V)
    cut = [slice(int(a), int(b)) for a, b in zip(start[:-1], start[1:])]
    return [(K[:, c].double().cpu().numpy(), V[:, c].double().cpu().numpy()) for c in cut]


def _i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(ctx, **kw):
    from paper_2512_14069_b200.cache import FourBitCache
    return FourBitCache(ctx, **dict(dict(n_layers=2, B=4, Hq=4, Hkv=2, d=64, page_size=16, n_pages=40, max_len=64, max_new=300), **kw))


# ---- admission ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("where", [0, 1, 2])
def test_a_prompt_that_is_too_long_takes_nobodys_rows(ctx, where):
    """The others get their own rows, and a request admitted before keeps its own."""
    c = _cache(ctx)
    before = _rows(1, 2, 40, 2, 64)
    c.admit(_i32([0, 0, 0, 40]), *before)
    new = [20, 5]
    new.insert(where, 100)
    rows = _rows(2, 2, 125, 2, 64)
    c.admit(_i32(new + [0]), *rows)
    assert ctx.read_device_status() == -1
    kept = [n if n < 100 else 0 for n in new] + [40]
    assert c.cache_len.tolist() == kept and c.granted.tolist() == [int(n < 100) for n in new] + [1]
    got = _load(c, kept)
    ctx.check_device_status()
    at = 0
    for b, n in enumerate(new):
        for x, have in zip(rows, got[b]):
            assert np.array_equal(have, _held(x[:, at:at + kept[b]])), b
        at += n
    for x, have in zip(before, got[3]):
        assert np.array_equal(have, _held(x))


def test_refused_requests_count_their_tokens(ctx):
    """... in the running sum, with no slots: lengths that do not fit, lengths that are none."""
    import torch
    from paper_2512_14069_b200 import binding as rb
    lens, new = [3, 0, -7, 60, 16], [10, 9, 4, 5, 8]
    t = dict(cache_len=_i32(lens), new_len=_i32(new), block_table=_i32(np.arange(20).reshape(5, 4).tolist()), free_pages=_i32(list(range(20, 40))), free_count=_i32([20]),
             slots=torch.full((50,), 77, dtype=torch.int64, device="cuda"), start=_i32([0] * 6), granted=torch.zeros(5, dtype=torch.uint8, device="cuda"))
    rb.radar_cache_extend(ctx, page_size=16, **t)
    assert ctx.read_device_status() == -1
    assert t["start"].tolist() == [0, 10, 19, 23, 28, 36] and t["granted"].tolist() == [1, 1, 0, 0, 1]
    assert t["cache_len"].tolist() == [13, 9, -7, 60, 24]
    s = t["slots"].tolist()
    assert s[:10] == list(range(3, 13)) and s[10:19] == [39 * 16 + i for i in range(9)] and s[19:28] == [-1] * 9 and s[28:36] == [38 * 16 + i for i in range(8)]
def test_rows_beyond_the_new_tokens_are_nobodys(ctx):
    """K and V of a fixed size, as a captured admission has them, hold more rows than are added."""
    c = _cache(ctx)
    a, b = _rows(3, 2, 200, 2, 64), _rows(4, 2, 200, 2, 64)
    c.admit(_i32([60, 30, 0, 0]), *a)
    c.admit(_i32([0, 0, 7, 21]), *b)
    ctx.check_device_status()
    got = _load(c, [60, 30, 7, 21])
    ctx.check_device_status()
    for i, (x, at, n) in enumerate(((a, 0, 60), (a, 60, 30), (b, 0, 7), (b, 7, 21))):
        for v in range(2):
            assert np.array_equal(got[i][v], _held(x[v][:, at:at + n])), i


@pytest.mark.parametrize("capacity", [0, 1, 40, 5000, 40000])
@pytest.mark.parametrize("in_place", [False, True])
def test_slots_behind_the_last_token_hold_none(ctx, capacity, in_place):
    import torch
    from paper_2512_14069_b200 import binding as rb
    n = min(capacity, 33)
    t = dict(cache_len=_i32([5, 0]), new_len=_i32([n, 0]), block_table=_i32([[0, 1, 2], [3, 4, 5]]), free_pages=_i32(list(range(10))), free_count=_i32([10]),
             slots=torch.full((capacity,), 9, dtype=torch.int64, device="cuda"), start=_i32([0] * 3), granted=torch.zeros(2, dtype=torch.uint8, device="cuda"))
    if not in_place:
        t.update(cache_len_out=_i32([0, 0]), free_count_out=_i32([0]))
    rb.radar_cache_extend(ctx, page_size=16, **t)
    ctx.check_device_status()
    s = t["slots"].cpu()
    assert bool((s[:n] >= 0).all()) and bool((s[n:] == -1).all())
