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
