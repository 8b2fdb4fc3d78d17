"""The 4-bit cache's attention, launched again and again behind itself: the same bits every time.

Keys and values pass from copies to decoders to products through rings in shared memory.  A tile that was handed on before all
lanes had written it, or a stage that was filled again while a lane still read it, would show as a result that differs between
launches."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("lens,Hq,Hkv,d,page,rows", [([5000, 3001, 64], 64, 8, 128, 16, 64), ([4000, 2222], 32, 8, 128, 128, 20), ([3000, 777], 32, 8, 64, 32, 64)])
def test_launches_behind_one_another_agree(ctx, lens, Hq, Hkv, d, page, rows):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    kw = T.check_attention(ctx, np.random.default_rng(21), lens, Hq, Hkv, d, page, rows, max_len=40000)
    outs = [(torch.zeros_like(kw["O"]), torch.zeros_like(kw["lse"])) for _ in range(30)]
    for O, lse in outs:
        rb.radar_cache_attention(ctx, **dict(kw, O=O, lse=lse))
    ctx.check_device_status()
    for O, lse in outs:
        assert torch.equal(O, kw["O"]) and torch.equal(lse, kw["lse"])
