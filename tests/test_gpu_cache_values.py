"""Values and shapes at the edge of what the 4-bit cache's attention takes: empty pools, scales from end to end, infinities and NaN in
Q, K and V, many sequences, layouts whose strides differ where they count for nothing."""
import functools

import numpy as np
import pytest

from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu
FAR = 40000          # a bound of the lengths that leaves nothing to clusters


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


# ---- nothing cached -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,Hq,Hkv,d,rows", [(2, 8, 2, 64, 1), (2, 8, 2, 128, 64), (70, 8, 8, 64, 4), (16, 32, 8, 128, 64), (40, 40, 40, 64, 64)])
def test_attention_over_an_empty_pool(ctx, B, Hq, Hkv, d, rows):
    """No pages at all: a null address, a bound of 0.  Few units, and more than clusters take; few rows and many."""
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    g = torch.Generator().manual_seed(B)
    Q, Kt, Vt = (torch.randn(B, rows, h, d, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    O, lse = torch.zeros_like(Q), torch.zeros(B, Hq, rows, device="cuda")
    pages = torch.empty(0, rb.radar_cache_page_bytes(Hkv, d, 16), dtype=torch.uint8, device="cuda")
    rb.radar_cache_attention(ctx, Q=Q, Kt=Kt, Vt=Vt, pages=pages, page_size=16, block_table=T.dev(np.full((B, 1), -1), torch.int32),
                             cache_len=T.dev(np.zeros(B), torch.int32), max_cache_len=0, O=O, lse=lse,
                             workspace=T.workspace(rb.radar_cache_attn_workspace_bytes(ctx, B, Hq, Hkv, d, rows, 0)))
    ctx.check_device_status()
    see = np.tril(np.ones((rows, rows), bool))
    for b in range(B):
        q, k, v = (x[b].double().cpu().numpy() for x in (Q, Kt, Vt))
        o, l = C.attention(q, k, v, see, d ** -0.5)
        size, _ = C.attention(q, k, np.abs(v), see, d ** -0.5)
        move = 2.0 ** -23 * d ** 0.5 * np.abs(q).max() * np.abs(k).max()
        assert np.all(np.abs(O[b].double().cpu().numpy() - o) <= (1.1 * 2.0 ** -7 + 2 * move) * size)
        assert np.all(np.abs(lse[b].double().cpu().numpy() - l) <= 2.0 ** -20 + move + 2.0 ** -23 * np.abs(l))


# ---- scales -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", [1, 7, 64])
@pytest.mark.parametrize("max_len", [None, FAR])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_from_the_smallest_to_the_largest(ctx, monkeypatch, rows, max_len, d):
    """Scale bytes 0 to 255 (values from 2^-20 to 30720) side by side, and pools of one end alone."""
    import cache_harness as T
    whole = T.random_pool
    for i, (lo, hi, gain) in enumerate(((0, 256, 2.0 ** -8), (0, 1, 1.0), (255, 256, 2.0 ** -12))):
        monkeypatch.setattr(T, "random_pool", functools.partial(whole, lo=lo, hi=hi))
        T.check_attention(ctx, np.random.default_rng(31 + i), [700, 33], 8, 2, d, 32, rows, max_len=max_len, gain=gain)


# ---- many sequences -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,Hq,Hkv,d,rows", [(97, 8, 2, 64, 1), (133, 4, 1, 128, 8), (130, 8, 2, 64, 20), (161, 8, 8, 128, 50)])
@pytest.mark.parametrize("max_len", [None, FAR])
def test_attention_of_more_sequences_than_a_warp_has_lanes(ctx, B, Hq, Hkv, d, rows, max_len):
    import cache_harness as T
    rng = np.random.default_rng(B)
    lens, n = rng.integers(0, 90, B), rng.integers(0, rows + 1, B)
    lens[::5], n[::6], lens[-1] = 0, 0, 600
    n[-1] = rows
    T.check_attention(ctx, rng, list(lens), Hq, Hkv, d, 16, rows, n_nodes=n, max_len=max_len)


# ---- infinities and NaN ---------------------------------------------------------------------------------------------------------
FORMS = [([300, 20], 1, None), ([300, 20], 12, None), ([300, 20], 64, None), ([9000, 100], 1, FAR), ([9000, 100], 7, FAR), ([9000, 100], 64, FAR), ([100, 30], 64, FAR)]


def _run(ctx, kw, **changed):
    from paper_2512_14069_b200 import binding as rb
    kw["O"].fill_(7.0), kw["lse"].fill_(7.0)
    rb.radar_cache_attention(ctx, **dict(kw, **changed))
    ctx.check_device_status()
    return kw["O"].double().cpu().numpy(), kw["lse"].double().cpu().numpy()


@pytest.mark.parametrize("lens,rows,max_len", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_a_row_of_nan_is_nan_and_the_others_are_not(ctx, lens, rows, max_len, d):
    """However its keys are shared out: O and lse of that row and head, and no others."""
    import cache_harness as T
    kw = T.check_attention(ctx, np.random.default_rng(41), lens, 8, 2, d, 16, rows, max_len=max_len)
    lse0 = kw["lse"].double().cpu().numpy()
    Q = kw["Q"].clone()
    Q[0, rows - 1, 5, 3] = float("nan")
    O, lse = _run(ctx, kw, Q=Q)
    assert np.isnan(O[0, rows - 1, 5]).all() and np.isnan(lse[0, 5, rows - 1])
    hit = np.zeros(O.shape[:3], bool)
    hit[0, rows - 1, 5] = True
    for b in range(2):
        o, bound = T.held_to[b]
        assert np.all((np.abs(O[b] - o) <= bound)[~hit[b]])
    at = ~hit.transpose(0, 2, 1)
    assert np.all(np.abs(lse - lse0)[at] <= 2e-4)            # twice 2^-20 + 2^-23 d max|q| max|k| / sqrt(d) + 2^-23 |lse|, with |q| < 6, |k| < 8, |lse| < 100


@pytest.mark.parametrize("lens,rows,max_len", [f for f in FORMS if f[1] > 1])
@pytest.mark.parametrize("value", ["nan", "inf", "-inf"])
def test_a_key_that_no_row_sees_is_not_there(ctx, lens, rows, max_len, value):
    """Whatever it is: the same bits as with zeros in its place."""
    import torch
    import cache_harness as T
    kw = T.check_attention(ctx, np.random.default_rng(42), lens, 8, 2, 128, 16, rows, max_len=max_len)
    t = rows - 3
    mask = kw["mask"] & ~(1 << t)
    Kt = kw["Kt"].clone()
    Kt[:, t] = 0.0
    want = _run(ctx, kw, mask=mask, Kt=Kt)
    Kt[:, t] = float(value)
    got = _run(ctx, kw, mask=mask, Kt=Kt)
    assert np.isfinite(want[0]).all()
    assert np.array_equal(want[0], got[0]) and np.array_equal(want[1], got[1])


@pytest.mark.parametrize("lens,rows,max_len", FORMS)
def test_keys_that_are_infinite(ctx, lens, rows, max_len):
    """A score of +inf leaves a row without a value, one of -inf takes the key from it, as in the definition."""
    import torch
    import cache_harness as T
    kw = T.check_attention(ctx, np.random.default_rng(43), lens, 8, 2, 128, 16, rows, max_len=max_len)
    Kt = kw["Kt"].clone()
    Kt[0, 0, 1, 9] = float("inf")                            # of the root, which all rows see
    O, lse = _run(ctx, kw, Kt=Kt)
    q = kw["Q"][0].double().cpu().numpy()
    see = np.ones(rows, bool)
    plus = see[:, None] & (q[:, :, 9] > 0) & (np.arange(8) >= 4)[None]
    assert plus.any() and np.array_equal(np.isnan(O[0]).all(-1), plus) and np.array_equal(np.isnan(O[0]).any(-1), plus)
    assert not np.isfinite(lse[0].T[plus]).any() and np.isfinite(lse[0].T[~plus]).all()
    # the others: as if the key were hidden from them
    hidden = kw["mask"].clone()
    hidden[0] &= ~1
    O2, lse2 = _run(ctx, kw, mask=hidden)
    minus = see[:, None] & (q[:, :, 9] < 0) & (np.arange(8) >= 4)[None]
    most = 2 * 1.1 * 2.0 ** -7 * 8                           # of two results, |v| < 8
    assert np.all(np.abs(O[0] - O2[0])[minus] <= most)
    o, bound = T.held_to[0]
    assert np.all((np.abs(O[0] - o) <= bound)[~plus & ~minus])


@pytest.mark.parametrize("lens,rows,max_len", FORMS)
def test_a_value_of_nan_reaches_its_head_and_no_other(ctx, lens, rows, max_len):
    """A probability of zero does not hide it: V of a live node has to be finite.  Other KV heads and sequences do not see it."""
    import cache_harness as T
    kw = T.check_attention(ctx, np.random.default_rng(44), lens, 8, 2, 64, 16, rows, max_len=max_len)
    Vt = kw["Vt"].clone()
    Vt[0, rows - 1, 1, 7] = float("nan")
    O, lse = _run(ctx, kw, Vt=Vt)
    o, bound = T.held_to[0]
    assert np.isnan(O[0, rows - 1, 4:, 7]).all()
    hit = np.zeros(O.shape[1:], bool)
    hit[:, 4:, 7] = True
    assert np.all((np.abs(O[0] - o) <= bound)[~hit])
    o, bound = T.held_to[1]
    assert np.all(np.abs(O[1] - o) <= bound)
    assert np.isfinite(lse).all()


# ---- layouts ----------------------------------------------------------------------------------------------------------------------
def test_strides_of_dimensions_of_one_element_do_not_matter(ctx):
    """Keys as [B, heads, rows, d] with one row, values as [B, rows, heads, d]: alike in memory."""
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    kw = T.check_attention(ctx, np.random.default_rng(51), [100, 7, 40], 8, 2, 64, 16, 1)
    first = kw["O"].clone()
    Kt = torch.empty_strided(kw["Kt"].shape, (2 * 64, 64, 64, 1), dtype=torch.bfloat16, device="cuda").copy_(kw["Kt"])
    assert Kt.stride() != kw["Vt"].stride()
    kw["O"].zero_()
    rb.radar_cache_attention(ctx, **dict(kw, Kt=Kt))
    ctx.check_device_status()
    assert torch.equal(kw["O"], first)
    K = torch.randn(1, 5, 3, 64, device="cuda")
    V = torch.empty_strided(K.shape, (7, 192, 64, 1), device="cuda").copy_(torch.randn_like(K))      # one layer
    pool = torch.zeros(1, 1, 3 * 18 * 64, dtype=torch.uint8, device="cuda")
    rb.radar_cache_store(ctx, K=K, V=V, slots=torch.arange(5, device="cuda"), pages=pool, page_size=16)
    K2, V2 = torch.zeros_like(K), torch.zeros(1, 5, 3, 64, device="cuda")
    rb.radar_cache_load(ctx, pages=pool, page_size=16, block_table=T.dev([[0]], torch.int32), first=T.dev([0], torch.int32), start=T.dev([0, 5], torch.int32), K=K2, V=V2)
    ctx.check_device_status()
    for x, y in ((K, K2), (V, V2)):
        assert np.array_equal(y.double().cpu().numpy(), C.values(*C.quantise(x.double().cpu().numpy())))
