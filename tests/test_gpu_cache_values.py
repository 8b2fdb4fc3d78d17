"""Values and shapes at the edge of what the 4-bit cache's attention takes: empty pools, scales from end to end, infinities and NaN in
Q, K and V, many sequences, layouts whose strides differ where they count for nothing."""
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
