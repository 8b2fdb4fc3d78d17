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


@pytest.mark.parametrize("rows,max_len", [(1, 600), (1, 40000), (24, 600), (24, 40000)])
def test_attention_right_behind_new_pages(ctx, rows, max_len):
    """Pages are granted and attended to by calls behind one another, with nothing between them: the lookups see the table as the call
    before has left it.  Each step again on its own, over the table of that time, gives the same bits."""
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    i32, B, Hq, Hkv, d, page, steps = torch.int32, 3, 32, 8, 64, 16, 24
    rng = np.random.default_rng(rows)
    n_pages = 130
    pool = torch.from_numpy(T.random_pool(rng, n_pages, Hkv, d, page).reshape(n_pages, -1)).cuda()
    table, lens = torch.full((B, -(-max_len // page)), -1, dtype=i32, device="cuda"), torch.zeros(B, dtype=i32, device="cuda")
    stack, count = T.dev(rng.permutation(n_pages), i32), T.dev([n_pages], i32)
    new = T.dev([16, 15, 3], i32)
    slots, start, granted = torch.zeros(34, dtype=torch.int64, device="cuda"), T.dev([0] * 4, i32), torch.zeros(B, dtype=torch.uint8, device="cuda")
    g = torch.Generator().manual_seed(rows)
    Q, Kt, Vt = (torch.randn(B, rows, h, d, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    ws = T.workspace(rb.radar_cache_attn_workspace_bytes(ctx, B, Hq, Hkv, d, rows, max_len))
    outs = [torch.zeros_like(Q) for _ in range(steps)]

    def attend(O, table, lens):
        rb.radar_cache_attention(ctx, Q=Q, Kt=Kt, Vt=Vt, pages=pool, page_size=page, block_table=table, cache_len=lens, max_cache_len=max_len, O=O, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    attend(outs[0], table, lens)                             # (nothing that is set up once is left to the capture)
    rb.radar_cache_extend(ctx, page_size=page, cache_len=lens, new_len=torch.zeros_like(new), block_table=table, free_pages=stack, free_count=count, slots=slots, start=start,
                          granted=granted)
    with torch.cuda.graph(graph):
        for O in outs:
            rb.radar_cache_extend(ctx, page_size=page, cache_len=lens, new_len=new, block_table=table, free_pages=stack, free_count=count, slots=slots, start=start, granted=granted)
            attend(O, table, lens)
    graph.replay()
    torch.cuda.synchronize()
    ctx.check_device_status()
    assert lens.tolist() == [16 * steps, 15 * steps, 3 * steps]
    for i, O in enumerate(outs):
        alone, at = torch.zeros_like(O), T.dev([16 * (i + 1), 15 * (i + 1), 3 * (i + 1)], i32)
        torch.cuda.synchronize()
        attend(alone, table, at)
        torch.cuda.synchronize()
        assert torch.equal(alone, O), i
