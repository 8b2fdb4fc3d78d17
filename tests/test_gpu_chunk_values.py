"""radar_chunk_attention deep in long caches: outputs that every page's values go into (paged_values; test_chunk_values.py shows that one wrong page is
seen)."""
import numpy as np
import pytest

import paged_values as V

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(V.CASES))
def test_every_page_of_values(ctx, name, dtype):
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    news, lens, Hq, Hkv, d, page, bounds = V.CASES[name]
    requests, start = V.make(name, dtype)
    Kc, Vc, table = V.pool(np.random.default_rng(7), requests, Hkv, d, page, dtype)
    max_len = bounds.get("max_len", max(lens))
    table = np.pad(table, ((0, 0), (0, max(0, -(-max_len // page) - table.shape[1]))), constant_values=-7)
    Q = T.dev(np.concatenate([q for q, _, _ in requests]), T.DT[dtype])
    O, lse = torch.full_like(Q, 7.0), torch.full(Q.shape[:2], 7.0, device="cuda")
    ws = T.workspace(rb.radar_chunk_attn_workspace_bytes(ctx, len(news), Hq, Hkv, d, T.CODE[dtype], max(news), max_len))
    ws.random_(0, 256)                                       # (what stands in a workspace is nobody's)
    rb.radar_chunk_attention(ctx, Q=Q, q_start=T.dev(start, torch.int32), Kc=Kc.cuda(), Vc=Vc.cuda(), page_size=page, block_table=T.dev(table, torch.int32),
                             cache_len=T.dev(lens, torch.int32), max_new=max(news), max_cache_len=max_len, O=O, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    ctx.check_device_status()
    assert V.hold(O.double().cpu().numpy(), lse.double().cpu().numpy(), requests, start, dtype) < 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_page_of_a_decoding_loop(ctx, dtype):
    """PagedCache: prompts stored in chunks, then single tokens and a chunk over all of it."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200.cache import PagedCache
    B, Hq, Hkv, d, page = 3, 8, 2, 64, 32
    rng = np.random.default_rng(5)
    lens, news = [3000, 900, 4100], [1, 40, 1]
    requests = [V.request(rng, n, L, Hq, Hkv, d, page, dtype) for n, L in zip(news, lens)]
    c = PagedCache(ctx, n_layers=1, B=B, Hq=Hq, Hkv=Hkv, d=d, page_size=page, n_pages=260, max_len=4200, max_new=700, dtype=T.DT[dtype])
    done = np.zeros(B, int)
    while np.any(done < lens):
        n = [min(233, L - new - have) for L, new, have in zip(lens, news, done)]
        n = n if any(n) else news                             # the rows that attend, at last
        c.begin(torch.tensor(n, dtype=torch.int32, device="cuda"), sum(n))
        c.store(0, *(T.dev(np.concatenate([r[i][have:have + m] for r, have, m in zip(requests, done, n)]), T.DT[dtype]) for i in (1, 2)))
        done += n
    Q = T.dev(np.concatenate([q for q, _, _ in requests]), T.DT[dtype])
    O, lse = torch.full_like(Q, 7.0), torch.full(Q.shape[:2], 7.0, device="cuda")
    c.attention(0, Q, O, lse, max_new=max(news))
    torch.cuda.synchronize()
    ctx.check_device_status()
    start = np.concatenate([[0], np.cumsum(news)])
    assert V.hold(O.double().cpu().numpy(), lse.double().cpu().numpy(), requests, start, dtype) < 1.0
