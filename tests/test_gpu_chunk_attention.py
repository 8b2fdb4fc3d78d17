"""radar_chunk_attention: chunks of new tokens over the paged cache, against float64."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


def _rng(*key):
    return np.random.default_rng([list(map(ord, str(k)))[0] if isinstance(k, str) else k for k in key])


# (rows of each request, cached tokens of each)
SHAPES = {
    "one token": ([1], [1]),
    "token, end of a tile": ([1, 1, 1], [127, 128, 129]),
    "tokens": ([1] * 9, [5, 300, 64, 1000, 33, 2, 777, 128, 256]),
    "whole prompts": ([1, 17, 128, 200], [1, 17, 128, 200]),
    "chunk of a long one": ([65], [3000]),
    "two units and a row": ([513], [700]),
    "mixed": ([1, 130, 0, 64, 7, 1], [900, 130, 50, 1111, 7, 1]),
    "no keys for the first rows": ([9, 200], [4, 30]),
    "nothing cached": ([3, 5], [0, 8]),
    "rows without tokens": ([0, 4, 0], [10, 4, 0]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(8, 2, 128, 64), (3, 3, 64, 16), (7, 1, 128, 32)])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_against_float64(ctx, shape, Hq, Hkv, d, page, dtype):
    import paged_harness as T
    news, lens = SHAPES[shape]
    T.check_chunk(ctx, _rng(len(shape), Hq, page), news, lens, Hq, Hkv, d, page, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 5), (6, 2), (16, 1), (24, 8), (28, 4), (64, 1), (65, 1), (128, 1), (96, 1), (256, 2)])
def test_head_ratios(ctx, Hq, Hkv, dtype):
    import paged_harness as T
    T.check_chunk(ctx, _rng(Hq, Hkv), [3, 1, 40], [200, 77, 40], Hq, Hkv, 64, 16, dtype)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 384])
@pytest.mark.parametrize("d", [64, 128])
def test_page_sizes(ctx, page, d):
    import paged_harness as T
    for dtype in ("bf16", "f32"):
        T.check_chunk(ctx, _rng(page, d), [30, 1, 200], [500, 385, 200], 4, 2, d, page, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_fused_projection_and_rows_of_nobody(ctx, dtype):
    import paged_harness as T
    T.check_chunk(ctx, _rng(3), [5, 130], [60, 400], 8, 2, 128, 64, dtype, fused=True, lead=3, tail=6, rows_behind=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_bounds_and_no_lse(ctx, dtype):
    """Bounds far above what the requests have."""
    import paged_harness as T
    T.check_chunk(ctx, _rng(4), [5, 1], [60, 400], 8, 2, 128, 16, dtype, max_new=5000, max_len=100000, want_lse=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gain,scale", [(4.0, 0.0), (1.0, 0.5), (0.01, 0.0)])
def test_scores_small_and_large(ctx, gain, scale, dtype):
    import paged_harness as T
    T.check_chunk(ctx, _rng(5), [70, 1, 9], [500, 300, 9], 4, 2, 64, 16, dtype, gain=gain, scale=scale)


@pytest.mark.parametrize("news,lens,Hq,Hkv", [([1], [40000], 8, 2), ([1] * 64, list(range(1, 4100, 64)), 4, 1), ([300], [20000], 4, 1), ([1, 1000, 1, 500], [5000, 1000, 20, 4000], 8, 8)])
def test_units_over_many_blocks(ctx, news, lens, Hq, Hkv):
    import paged_harness as T
    T.check_chunk(ctx, _rng(len(news), Hq), news, lens[:len(news)], Hq, Hkv, 128, 64)


def test_many_requests_f32(ctx):
    import paged_harness as T
    T.check_chunk(ctx, _rng(6), [1] * 40 + [90], list(range(1, 41)) + [2500], 6, 2, 64, 16, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_repeats_are_bit_equal(ctx, dtype):
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    kw = T.check_chunk(ctx, _rng(7), [130, 1, 40], [2000, 1500, 40], 8, 2, 128, 64, dtype)
    first = kw["O"].clone(), kw["lse"].clone()
    for _ in range(3):
        kw["O"].fill_(3.0)
        rb.radar_chunk_attention(ctx, **kw)
        torch.cuda.synchronize()
        assert torch.equal(kw["O"], first[0]) and torch.equal(kw["lse"], first[1])


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (4, 2), (9, 1), (16, 1), (32, 2), (17, 1), (6, 6)])
@pytest.mark.parametrize("d", [64, 128])
def test_few_rows(ctx, Hq, Hkv, d):
    """Single tokens and two of them, at lengths around a chunk, a block's keys, a cluster's, and behind the bound of the form."""
    import paged_harness as T
    lens = [1, 15, 16, 17, 127, 128, 129, 250]
    T.check_chunk(ctx, _rng(Hq, d), [1] * 8, lens, Hq, Hkv, d, 16)
    T.check_chunk(ctx, _rng(Hq, d, 1), [2, 1, 0, 2], [2, 1, 5, 640], Hq, Hkv, d, 32)
    for n in (300, 2047, 2048, 2049, 5000, 17000):
        T.check_chunk(ctx, _rng(Hq, n), [1], [n], Hq, Hkv, d, 64)
    T.check_chunk(ctx, _rng(Hq, d, 2), [2, 1], [0, 0], Hq, Hkv, d, 16, max_len=400)


def test_few_rows_of_many_requests(ctx):
    import paged_harness as T
    T.check_chunk(ctx, _rng(1), [1] * 150, [3 * i % 700 for i in range(150)], 4, 2, 128, 16)
    T.check_chunk(ctx, _rng(2), [2] * 40, [11 * i % 500 + 2 for i in range(40)], 8, 1, 64, 128)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,lens,d", [([1, 1], [40, 300], 128), ([30, 1, 200], [200, 900, 200], 64), ([300], [3000], 128)])
def test_keys_and_values_that_are_no_numbers(ctx, news, lens, d, dtype):
    """A NaN key makes exactly the rows that see it NaN; keys behind a row's last, and infinite ones there, reach nothing."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    rng = _rng(len(news), d)
    Hq, Hkv, page = 4, 2, 16
    kw = T.check_chunk(ctx, rng, news, lens, Hq, Hkv, d, page, dtype)
    want = kw["O"].clone()
    for value in (float("nan"), float("inf")):
        b = len(news) - 1
        n, L = news[b], lens[b]
        j = L - max(1, n // 2)                                    # hidden from the rows before token j
        table = kw["block_table"][b].tolist()
        slot = table[j // page] * page + j % page
        keep = kw["Kc"][slot, 0].clone()
        kw["Kc"][slot, 0] = value
        kw["O"].fill_(5.0)
        rb.radar_chunk_attention(ctx, **kw)
        torch.cuda.synchronize()
        ctx.check_device_status()
        kw["Kc"][slot, 0] = keep
        first = int(kw["q_start"][b]) + n - (L - j)               # the first row that sees the key
        G = Hq // Hkv
        assert torch.equal(kw["O"][:first], want[:first]) and torch.equal(kw["O"][:, G:], want[:, G:])
        if value != value:
            last = int(kw["q_start"][b + 1])
            assert torch.isnan(kw["O"][first:last, :G]).all() and torch.isnan(kw["lse"][first:last, :G]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_pages_and_requests(ctx, dtype):
    """A page that is not in the cache is told and read as page 0; a request out of bounds is told and skipped, the others are as ever."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    for news, lens in (([20, 1, 70], [200, 300, 90]), ([1, 1, 1], [50, 300, 90])):
        kw = T.check_chunk(ctx, _rng(9), news, lens, 4, 2, 64, 16, dtype)
        start = kw["q_start"].tolist()
        for name, at, value in (("cache_len", 1, -1), ("cache_len", 1, max(lens) + 1), ("cache_len", 1, 2 ** 31 - 1), ("block_table", (1, 2), 10 ** 6), ("block_table", (1, 2), -3)):
            x = kw[name]
            keep = x[at].clone()
            x[at] = value
            kw["O"].fill_(5.0)
            rb.radar_chunk_attention(ctx, **kw)
            assert ctx.read_device_status() == -1, (name, value)
            x[at] = keep
            T.hold_again(kw, [0, 2])
            if name == "cache_len":
                assert torch.all(kw["O"][start[1]:start[2]] == 5.0)
        bad = kw["q_start"].clone()
        bad[1], bad[2] = start[2] + 1, start[1]                     # request 1 runs backwards, 0 and 2 have too many rows or others'
        rb.radar_chunk_attention(ctx, **dict(kw, q_start=bad))
        assert ctx.read_device_status() == -1
        bad = torch.tensor([start[0], start[1], start[2], kw["Q"].shape[0] + 1], dtype=torch.int32, device="cuda")
        kw["O"].fill_(5.0)
        rb.radar_chunk_attention(ctx, **dict(kw, q_start=bad))
        assert ctx.read_device_status() == -1
        T.hold_again(kw, [0, 1])
        assert torch.all(kw["O"][start[2]:] == 5.0)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (4, 2), (9, 1), (16, 1), (17, 1), (6, 6)])
@pytest.mark.parametrize("d", [64, 128])
def test_few_rows_f32(ctx, Hq, Hkv, d):
    import paged_harness as T
    T.check_chunk(ctx, _rng(Hq, d), [1] * 8, [1, 7, 8, 9, 63, 64, 65, 250], Hq, Hkv, d, 16, "f32")
    T.check_chunk(ctx, _rng(Hq, d, 1), [2, 1, 0, 2], [2, 1, 5, 640], Hq, Hkv, d, 32, "f32")
    for n in (300, 1023, 1024, 1025, 5000, 17000):
        T.check_chunk(ctx, _rng(Hq, n), [1], [n], Hq, Hkv, d, 64, "f32")
    T.check_chunk(ctx, _rng(Hq, d, 2), [2, 1], [0, 0], Hq, Hkv, d, 16, "f32", max_len=400)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 384])
def test_few_rows_in_pages_of_all_sizes_from_a_fused_projection(ctx, page, dtype):
    import paged_harness as T
    T.check_chunk(ctx, _rng(page), [1, 2, 0, 1], [500, 385, 7, 900], 8, 2, 128, page, dtype, fused=True, lead=2, tail=3, rows_behind=2)


def test_more_requests_than_a_warp_has_lanes(ctx):
    """Ranges over 70 requests of 5 and more rows, some of them empty, in one launch of the tensor cores' form."""
    import paged_harness as T
    news = [0 if i % 9 == 4 else 5 + i % 7 for i in range(70)]
    T.check_chunk(ctx, _rng(3), news, [n + (37 * i) % 600 for i, n in enumerate(news)], 4, 1, 128, 32)
    T.check_chunk(ctx, _rng(4), [0] * 33 + [140] + [0] * 40, [50] * 33 + [1400] + [3] * 40, 4, 2, 64, 16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1], [40, 7]])
def test_the_first_call_of_a_context_may_be_captured(dtype, news):
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    kw = T.check_chunk(c, _rng(5), news, [300, 100], 4, 2, 64, 16, dtype)
    c.close()
    want, c = kw["O"].clone(), rb.Context(0)
    kw["O"].fill_(5.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rb.radar_chunk_attention(c, **kw)
    assert torch.all(kw["O"] == 5.0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kw["O"], want) and c.read_device_status() == 0
    del graph
    c.close()


def test_two_calls_at_once(ctx):
    """On two streams, with a workspace each: what either gives alone."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    calls = [T.check_chunk(ctx, _rng(i), news, lens, 8, 2, 128, 64) for i, (news, lens) in enumerate([([300, 40], [4000, 900]), ([130, 1, 60], [2000, 3000, 60])])]
    want = [(k["O"].clone(), k["lse"].clone()) for k in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for k, s in zip(calls, streams):
            rb.radar_chunk_attention(ctx, stream=s, **k)
    torch.cuda.synchronize()
    for k, w in zip(calls, want):
        assert torch.equal(k["O"], w[0]) and torch.equal(k["lse"], w[1])
    assert ctx.read_device_status() == 0


@pytest.mark.parametrize("news,dtype", [([1, 1], "bf16"), ([40, 7], "bf16"), ([1, 1], "f32"), ([40, 7], "f32")])
def test_a_cache_beyond_32_bits(ctx, news, dtype):
    """Pages at the end of a pool of more than 2^31 elements give what the same pages give at the start of a small one."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    Hkv, d, page = 16, 128, 64
    kw = T.check_chunk(ctx, _rng(8), news, [300, 1000], 32, Hkv, d, page, dtype)
    want, lse = kw["O"].clone(), kw["lse"].clone()
    small = kw["Kc"].shape[0]
    rows = 2 ** 31 // (Hkv * d) + small
    rows -= rows % page
    for name in ("Kc", "Vc"):
        big = torch.empty(rows, Hkv, d, dtype=T.DT[dtype], device="cuda")
        big[rows - small:] = kw[name]
        kw[name] = big
    table = kw["block_table"]
    kw["block_table"] = torch.where(table >= 0, table + (rows - small) // page, table)
    kw["O"].fill_(7.0)
    rb.radar_chunk_attention(ctx, **kw)
    torch.cuda.synchronize()
    ctx.check_device_status()
    assert torch.equal(kw["O"], want) and torch.equal(kw["lse"], lse)


def test_pools_at_addresses_of_16_bytes(ctx):
    """Single tokens over pools that 32-byte reads cannot take."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    for dtype in ("bf16", "f32"):
        kw = T.check_chunk(ctx, _rng(9), [1, 1, 0], [300, 70, 5], 8, 2, 64, 16, dtype)
        for name in ("Kc", "Vc"):
            room = torch.empty(kw[name].numel() + 16, dtype=T.DT[dtype], device="cuda")
            at = 16 // room.element_size()
            moved = room[at:at + kw[name].numel()].view_as(kw[name])
            assert moved.data_ptr() % 32 == 16
            moved.copy_(kw[name])
            kw[name] = moved
        kw["O"].fill_(7.0)
        rb.radar_chunk_attention(ctx, **kw)
        torch.cuda.synchronize()
        ctx.check_device_status()
        T.hold_again(kw, range(3))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (32, 8), (16, 1), (17, 1)])
def test_few_rows_in_tiles(ctx, Hq, Hkv, d):
    """Units of up to 16 rows, and of 17, in the tiles that long caches take; pieces of them in several blocks."""
    import paged_harness as T
    G = Hq // Hkv
    for news, lens in (([1, 16 // G if G <= 16 else 1, 0, 1], [5000, 700, 40, 128]), ([16 // G + 1, 1], [257, 9000])):
        T.check_chunk(ctx, _rng(G), news, lens, Hq, Hkv, d, 32, max_len=60000)


@pytest.mark.parametrize("rows", [17, 32, 33, 63, 64, 65, 100])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (32, 8, 64), (17, 1, 128), (40, 1, 64)])
def test_small_units_in_tiles(ctx, Hq, Hkv, d, rows):
    """Units at the bounds of the products' sizes, whole and in pieces, beside smaller ones."""
    import paged_harness as T
    n = max(1, rows // (Hq // Hkv))
    T.check_chunk(ctx, _rng(rows), [n, 1, max(1, n // 2)], [n + 700, 9000, 300], Hq, Hkv, d, 32, max_len=60000)
