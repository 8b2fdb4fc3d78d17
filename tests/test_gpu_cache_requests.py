"""Requests that a 4-bit cache has no room for, beside others that it holds; rows that are not in use; bounds of the lengths."""
import types

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


# ---- room for slots -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,most,capacity", [(2, 8, 6), (5, 9, 11), (300, 40, 4000), (300, 40, 4500), (300, 60, 0), (700, 33, 8000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_tokens_without_a_slot_are_not_granted(ctx, B, most, capacity, in_place):
    """A length counts only tokens that have a slot to be stored in: from the first request whose tokens pass the slots' capacity on,
    requests that add tokens are not granted, take no pages and keep their lengths."""
    import torch
    from paper_2512_14069_b200 import binding as rb
    rng = np.random.default_rng(B + capacity)
    page, columns = 16, 8
    lens = rng.integers(0, 40, B)
    new = np.where(rng.random(B) < 0.2, -rng.integers(0, lens + 1), rng.integers(0, most, B))
    new[0] = min(4, most)
    table, n_pages = np.arange(B * columns).reshape(B, columns), B * columns
    stack = np.arange(n_pages, 2 * n_pages)
    t = dict(cache_len=_i32(lens.tolist()), new_len=_i32(new.tolist()), block_table=_i32(table.tolist()), free_pages=_i32(stack.tolist()), free_count=_i32([n_pages - 3 * B]),
             slots=torch.full((capacity,), 9, dtype=torch.int64, device="cuda"), start=_i32([0] * (B + 1)), granted=torch.zeros(B, dtype=torch.uint8, device="cuda"))
    if not in_place:
        t.update(cache_len_out=_i32([0] * B), free_count_out=_i32([0]))
    rb.radar_cache_extend(ctx, page_size=page, **t)
    add = np.maximum(new, 0)
    end = np.cumsum(add)
    assert end[-1] > capacity and ctx.read_device_status() == -1
    out = (new > 0) & (end > capacity)
    want = C.extend(page, lens, np.where(out, 0, new), table, stack, n_pages - 3 * B)
    got = lambda name: (t[name] if in_place or name + "_out" not in t else t[name + "_out"]).cpu().numpy()
    assert np.array_equal(t["granted"].cpu().numpy().astype(bool), want[5] & ~out)
    assert np.array_equal(got("cache_len"), want[3]) and got("free_count")[0] == want[2]
    assert np.array_equal(t["block_table"].cpu().numpy(), want[0]) and np.array_equal(t["free_pages"].cpu().numpy()[:want[2]], want[1][:want[2]])
    assert np.array_equal(t["start"].cpu().numpy(), np.concatenate([[0], end]))
    slots = np.concatenate([[-1] * add[b] if out[b] else want[4][b] for b in range(B)])[:capacity]
    assert np.array_equal(t["slots"].cpu().numpy(), slots)


def test_counts_that_no_int_holds(ctx):
    """The running sum ends at the largest int: what lies behind has no slots and is not granted."""
    import torch
    from paper_2512_14069_b200 import binding as rb
    t = dict(cache_len=_i32([0, 0]), new_len=_i32([2 ** 31 - 1, 4]), block_table=_i32([[0], [1]]), free_pages=_i32(list(range(20))), free_count=_i32([20]),
             slots=torch.full((50,), 77, dtype=torch.int64, device="cuda"), start=_i32([0] * 3), granted=torch.zeros(2, dtype=torch.uint8, device="cuda"))
    rb.radar_cache_extend(ctx, page_size=16, extra=5, **t)
    assert ctx.read_device_status() == -1
    assert t["cache_len"].tolist() == [0, 0] and t["granted"].tolist() == [0, 0] and t["start"].tolist() == [0, 2 ** 31 - 1, 2 ** 31 - 1]
    assert t["slots"].tolist() == [-1] * 50 and t["free_count"].tolist() == [20]


def _step(accept, columns=4):
    n = len(accept)
    return types.SimpleNamespace(accept_len=_i32(accept), path_nodes=_i32([list(range(columns))] * n))


def test_append_wants_room_for_what_a_step_may_accept(ctx):
    c = _cache(ctx, max_new=15)
    K, V = _rows(5, 2, 4 * 64, 2, 64)
    c.admit(_i32([2, 3, 1, 1]), K[:, :7], V[:, :7])
    with pytest.raises(ValueError, match="made for 15"):
        c.append(_step([0, 0, 0, 0]), K.view(2, 4, 64, 2, 64), V.view(2, 4, 64, 2, 64))
    assert c.cache_len.tolist() == [2, 3, 1, 1]


# ---- rows that hold no request ----------------------------------------------------------------------------------------------
def test_append_leaves_out_rows_that_hold_no_request(ctx):
    """Never admitted, refused, released: none of them grows or takes a page, and one that is admitted again does."""
    import torch
    c = _cache(ctx, n_pages=6)
    K, V = _rows(6, 2, 4 * 64, 2, 64)
    tree = K.view(2, 4, 64, 2, 64), V.view(2, 4, 64, 2, 64)
    c.admit(_i32([20, 16, 60, 0]), K[:, :96], V[:, :96])             # two pages, one, four (refused), never
    assert c.granted.tolist() == [1, 1, 0, 1] and int(c.free_count) == 3
    c.append(_step([3, 1, 3, 3]), *tree)
    ctx.check_device_status()
    assert c.cache_len.tolist() == [24, 18, 0, 0] and int(c.free_count) == 2
    c.release(torch.tensor([1, 0, 0, 0], dtype=torch.uint8, device="cuda"))
    free = int(c.free_count)
    for _ in range(3):
        c.append(_step([3, 0, 3, 3]), *tree)
    ctx.check_device_status()
    assert c.cache_len.tolist() == [0, 21, 0, 0] and int(c.free_count) == free == 4
    c.admit(_i32([0, 0, 5, 0]), K[:, :5], V[:, :5])
    c.append(_step([1, 1, 1, 1]), *tree)
    ctx.check_device_status()
    assert c.cache_len.tolist() == [0, 23, 7, 0]
    got = _load(c, [0, 23, 7, 0])
    want = np.concatenate([_held(K[:, :5]), _held(K[:, 2 * 64:2 * 64 + 2])], 1)
    assert np.array_equal(got[2][0], want)


def test_a_request_without_cached_tokens_may_be_admitted(ctx):
    """A prompt of one token, the first step's root: nothing is cached yet, and its steps count."""
    import torch
    c = _cache(ctx)
    K, V = _rows(7, 2, 4 * 64, 2, 64)
    c.admit(_i32([0, 0, 0, 0]), K[:, :0], V[:, :0], requests=torch.tensor([0, 1, 0, 0], dtype=torch.uint8, device="cuda"))
    c.append(_step([2, 2, 2, 2]), K.view(2, 4, 64, 2, 64), V.view(2, 4, 64, 2, 64))
    ctx.check_device_status()
    assert c.cache_len.tolist() == [0, 3, 0, 0]


def test_an_idle_row_takes_no_page_from_a_live_one(ctx):
    import torch
    c = _cache(ctx, n_pages=3)
    K, V = _rows(8, 2, 4 * 64, 2, 64)
    tree = K.view(2, 4, 64, 2, 64), V.view(2, 4, 64, 2, 64)
    c.admit(_i32([15, 31, 0, 0]), K[:, :46], V[:, :46])
    c.release(torch.tensor([1, 0, 0, 0], dtype=torch.uint8, device="cuda"))
    c.append(_step([0, 0, 0, 0]), *tree)
    c.append(_step([0, 1, 0, 0]), *tree)
    ctx.check_device_status()
    assert c.granted.tolist() == [1, 1, 1, 1] and c.cache_len.tolist() == [0, 34, 0, 0]


def test_a_step_that_finds_no_page_is_taken_again():
    """The example's decoder: a request whose tokens were not granted emits none and keeps its root, until there are pages."""
    import os
    import sys
    import torch
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import decode_with_cache as D
    from paper_2512_14069_b200 import binding as rb
    ctx = rb.Context(0)
    model = D.Model(layers=2, Hq=4, Hkv=2, d=64, V=100, max_len=128, seed=4)
    texts = []
    for n_pages in (20, 4):
        dec = D.Decoder(ctx, model, B=2, n_pages=n_pages, max_len=128)
        assert dec.admit(0, list(range(17))) and dec.admit(1, list(range(30, 63)))       # one page, two
        text = []
        for step in range(40):
            if step == 12:
                dec.cache.release(torch.tensor([1, 0], dtype=torch.uint8, device="cuda"))
            before, root = dec.cache.cache_len.tolist(), dec.root.tolist()
            new = dec.decode_step()
            ctx.check_device_status()
            assert [a - b for a, b in zip(dec.cache.cache_len.tolist(), before)] == [len(e) for e in new]
            if not new[1]:
                assert dec.root[1] == root[1]
            text += new[1]
            if step >= 12:
                assert new[0] == []
        texts.append(text)
        assert dec.cache.granted.tolist()[1] == (n_pages == 20 or len(text) + 32 <= 64)
    assert len(texts[1]) < len(texts[0])
    assert texts[1] == texts[0][:len(texts[1])]
    ctx.close()


def test_the_example_with_few_pages_answers_every_request():
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import decode_with_cache as D
    text, dec = D.main(n_pages=8)
    assert len(text) == 6 and all(len(t) >= 24 for t in text.values())
    assert int(dec.cache.free_count) == 8 and dec.cache.cache_len.tolist() == [0] * dec.B
    with pytest.raises(RuntimeError, match="pages"):
        D.main(n_pages=1)


# ---- bounds of the lengths --------------------------------------------------------------------------------------------------
def _attend(c, ctx, rows, **kw):
    import torch
    g = torch.Generator().manual_seed(9)
    Q, Kt, Vt = (torch.randn(c.B, rows, h, c.d, generator=g).bfloat16().cuda() for h in (c.Hq, c.Hkv, c.Hkv))
    O = torch.full_like(Q, 7.0)
    lse = torch.full((c.B, c.Hq, rows), 7.0, device="cuda")
    ctx.reset_launch_counts()
    c.attention(1, Q, Kt, Vt, O, lse, **kw)
    n = {k: v[0] for k, v in ctx.kernel_stats().items()}
    return O, lse, (Q, Kt, Vt), n["cache_attention"], n["cache_attention_combine"]


@pytest.mark.parametrize("rows", [1, 9, 64])
def test_a_bound_of_the_lengths_may_be_given(ctx, rows):
    """Which form takes a call goes by it: a short request in a cache made for long ones runs as one among short ones."""
    c = _cache(ctx, B=1, max_len=32768, Hq=8, d=128)
    c.admit(_i32([300]), *_rows(10, 2, 300, 2, 128))
    O, lse, _, one, joined = _attend(c, ctx, rows)
    O2, lse2, _, one2, joined2 = _attend(c, ctx, rows, max_cache_len=300)
    ctx.check_device_status()
    assert (one, joined) == (1, 1) and (one2, joined2) == (1, 0)
    # each is off by up to 1.1 2^-7 sum p |v| <= 1.1 2^-7 max |v|; normal rows lie within 6
    assert float((O.float() - O2.float()).abs().max()) <= 2.2 * 2.0 ** -7 * 6 and float((lse - lse2).abs().max()) <= 1e-4
    _attend(c, ctx, rows, max_cache_len=299)
    assert ctx.read_device_status() == -1


@pytest.mark.parametrize("rows", [1, 33])
def test_a_request_may_fill_its_last_page(ctx, rows):
    """Capacities that are no multiple of the page size: what is granted can be attended to."""
    c = _cache(ctx, B=1, page_size=64, max_len=100, Hq=4, n_pages=3)
    rows_in = _rows(11, 2, 120, 2, 64)
    c.admit(_i32([120]), *rows_in)
    ctx.check_device_status()
    if c.granted.tolist() == [0]:
        return
    O, lse, (Q, Kt, Vt), _, _ = _attend(c, ctx, rows)
    ctx.check_device_status()
    q, kt, vt = (x[0].double().cpu().numpy() for x in (Q, Kt, Vt))
    k, v = (np.concatenate([_held(x)[1], t]) for x, t in zip(rows_in, (kt, vt)))
    see = np.concatenate([np.ones((rows, 120), bool), np.tril(np.ones((rows, rows), bool))], 1)
    o, _ = C.attention(q, k, v, see, 64 ** -0.5)
    size, _ = C.attention(q, k, np.abs(v), see, 64 ** -0.5)
    assert np.all(np.abs(O[0].double().cpu().numpy() - o) <= 1.2 * 2.0 ** -7 * size)
