"""radar_chunk_attention under the loosest bounds: max_new is any int, and says no more than that requests have no more rows."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (6, 6), (65, 1)])
def test_the_largest_bound_of_rows(ctx, Hq, Hkv, dtype):
    """With many units the launch fills the machine whatever the bound, and how the work is cut follows from the requests alone: the same bits."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    kw = T.check_chunk(ctx, np.random.default_rng(Hq), [40, 130, 7, 300], [5000, 3000, 900, 4000], Hq, Hkv, 128, 64, dtype)
    want, lse = kw["O"].clone(), kw["lse"].clone()
    for bound in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 30):
        kw["O"].fill_(7.0)
        kw["lse"].fill_(7.0)
        rb.radar_chunk_attention(ctx, **dict(kw, max_new=bound))
        torch.cuda.synchronize()
        ctx.check_device_status()
        assert torch.equal(kw["O"], want) and torch.equal(kw["lse"], lse), bound


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_bounds_of_rows_and_tokens(ctx, dtype):
    """... and tokens: a table with room for max_cache_len is what bounds it, so pages are large ones; few rows and many heads."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    kw = T.check_chunk(ctx, np.random.default_rng(1), [3, 1, 40], [200, 77, 40], 16, 8, 64, 128, dtype)
    most = 2 ** 31 - 2 ** 14 - 1
    table = torch.full((3, -(-most // 128)), -7, dtype=torch.int32, device="cuda")
    table[:, :kw["block_table"].shape[1]] = kw["block_table"]
    kw.update(block_table=table, max_cache_len=most, max_new=2 ** 31 - 1)
    kw["O"].fill_(7.0)
    rb.radar_chunk_attention(ctx, **kw)
    torch.cuda.synchronize()
    ctx.check_device_status()
    T.hold_again(kw, range(3))
