"""The paged bf16 / fp32 cache's operators together, as a decoding loop uses them: prompts in chunks, trees, accepted rows, single tokens, release."""
import os
import sys
import types

import numpy as np
import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    return rb.Context(0)


def test_the_example_runs_and_gives_its_pages_back(capsys):
    import decode_with_cache as D
    text, dec = D.main(paged=True)
    assert len(text) == 6 and all(len(t) >= 24 for t in text.values())
    assert int(dec.cache.free_count) == dec.cache.free_pages.numel()
    assert dec.cache.cache_len.tolist() == [0] * dec.B
    again, _ = D.main(paged=True)
    assert again == text
    # few pages: requests wait and start over, their text is that of the prompt and what was emitted before
    scarce, dec = D.main(paged=True, n_pages=9)
    assert all(len(t) >= 24 for t in scarce.values()) and int(dec.cache.free_count) == 9
    assert "pages free" in capsys.readouterr().out


def _cache(ctx, dtype="bf16", **kw):
    import paged_harness as T
    from paper_2512_14069_b200.cache import PagedCache
    args = dict(n_layers=2, B=3, Hq=6, Hkv=2, d=64, page_size=16, n_pages=60, max_len=300, max_new=200, dtype=T.DT[dtype])
    return PagedCache(ctx, **dict(args, **kw))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunks_and_tokens_are_a_prompt(ctx, dtype):
    """Prompts that come in chunks of all sizes, single tokens and nothing among them, request by request at different times: every row's
    output is the attention over the rotated rows up to it, and the cache holds the rotated rows."""
    import paged_harness as T
    import torch
    c = _cache(ctx, dtype)
    rng = np.random.default_rng(3)
    L, B, Hq, Hkv, d = 2, 3, 6, 2, 64
    freq = (10000.0 ** (-np.arange(0, d, 2) / d)).astype(np.float32)
    inv = T.dev(freq, torch.float32)
    kept = [[([], []) for _ in range(L)] for _ in range(B)]
    lens = np.zeros(B, int)
    for news in ([40, 0, 7], [1, 1, 1], [0, 130, 3], [17, 0, 0], [2, 1, 1], [1, 1, 1]):
        n = sum(news)
        start = np.concatenate([[0], np.cumsum(news)])
        c.begin(T.dev(news, torch.int32), n)
        pos = np.concatenate([lens[b] + np.arange(news[b]) for b in range(B)])
        assert c.pos[:n].tolist() == pos.tolist()
        lens = lens + news
        assert c.cache_len.tolist() == lens.tolist() and c.granted.tolist() == [1] * B
        for layer in range(L):
            qkv = torch.from_numpy(rng.standard_normal((n, Hq + 2 * Hkv, d))).to(T.DT[dtype])
            g = qkv.cuda()
            Q, K, V = g[:, :Hq], g[:, Hq:Hq + Hkv], g[:, Hq + Hkv:]
            O, lse = torch.zeros(n, Hq, d, dtype=T.DT[dtype], device="cuda"), torch.zeros(n, Hq, device="cuda")
            c.store(layer, K, V, Q=Q, Q_out=Q, inv_freq=inv)
            c.attention(layer, Q, O, lse, max_new=max(news))
            torch.cuda.synchronize()
            ctx.check_device_status()
            x = qkv.double().numpy()
            want, size = T.turned(x[:, :Hq + Hkv], pos[None], freq, np.zeros(d // 2, int), False)
            T.hold_turned(g[:, :Hq].double().cpu().numpy(), want[:, :Hq], size[:, :Hq], dtype, d)
            rows = []
            for b in range(B):
                at = slice(start[b], start[b + 1])
                table = c.block_table[b].tolist()
                slots = [table[j // 16] * 16 + j % 16 for j in range(lens[b])]
                k, v = (p[layer][slots].double().cpu().numpy() for p in (c.Kc, c.Vc))
                T.hold_turned(k[lens[b] - news[b]:], want[at, Hq:], size[at, Hq:], dtype, d)
                ks, vs = kept[b][layer]
                ks.append(k[lens[b] - news[b]:]), vs.append(x[at, Hq + Hkv:])
                assert np.array_equal(np.concatenate(ks), k) and np.array_equal(np.concatenate(vs), v)       # what was there stays
                rows.append((k, v))
            T.hold_chunk(O, lse, g[:, :Hq].double().cpu().numpy(), rows, start, lens, d, dtype)


def test_a_chunk_attends_as_the_tree_attention_does(ctx):
    """A tree that is a chain, verified over the paged cache, and the same tokens stored and attended to as a chunk: both round probabilities and O
    to bf16, each is off by up to 2^-7 sum p |v| (a tenth more for the fp32 sums), which is at most the largest |v|."""
    import torch
    from paper_2512_14069_b200 import binding as rb
    from paper_2512_14069_b200.pipeline import SpecStep
    B, Hq, Hkv, d, R = 3, 8, 2, 64, rb.RADAR_MAX_NODES
    c = _cache(ctx, Hq=Hq, Hkv=Hkv, n_layers=1, max_new=300)
    g = torch.Generator().manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    c.begin(i32([90, 16, 129]), 235)
    c.store(0, rand(235, Hkv, d), rand(235, Hkv, d))
    step = SpecStep(ctx, B=B, V=64, k=4, t_max=4, N=16, Hq=Hq, Hkv=Hkv, d=d, kv_dtype=torch.bfloat16, max_prefix_len=300)
    Q, Kt, Vt = rand(B, R, Hq, d), rand(B, R, Hkv, d), rand(B, R, Hkv, d)
    news = [20, 1, 33]
    step.n_nodes.copy_(i32(news))
    step.tree_mask.copy_(torch.tensor([-1 if i == 63 else (1 << (i + 1)) - 1 for i in range(R)], dtype=torch.int64).expand(B, R))
    step.attention_paged(c, 0, Q, Kt, Vt)
    pick = lambda x: torch.cat([x[b, :n] for b, n in enumerate(news)])
    c.begin(i32(news), sum(news))
    c.store(0, pick(Kt), pick(Vt))
    O, lse = torch.zeros(sum(news), Hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(sum(news), Hq, device="cuda")
    c.attention(0, pick(Q), O, lse, max_new=33)
    torch.cuda.synchronize()
    ctx.check_device_status()
    most = float(c.Vc.float().abs().max())
    assert float((O.float() - pick(step.O).float()).abs().max()) <= 2.2 * 2.0 ** -7 * most
    assert float((lse - pick(step.lse.transpose(1, 2))).abs().max()) <= 1e-4


def test_accepted_rows_and_release(ctx):
    """append takes the accepted rows of the trees as they are; rows without a request take nothing; released pages come back."""
    import torch
    c = _cache(ctx, B=4, max_new=64)
    g = torch.Generator().manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    c.begin(i32([15, 0, 30, 0]), 45, requests=i32([1, 0, 1, 1]))
    for layer in range(2):
        c.store(layer, rand(45, 2, 64), rand(45, 2, 64))
    before = c.Kc.clone()
    step = types.SimpleNamespace(accept_len=i32([2, 3, 0, 1]), path_nodes=i32([[0, 4, 9, -1], [0, 1, 2, 3], [0, -1, -1, -1], [0, 5, -1, -1]]))
    K, V = rand(2, 4, 12, 2, 64), rand(2, 4, 12, 2, 64)
    c.append(step, K, V)
    ctx.check_device_status()
    assert c.cache_len.tolist() == [18, 0, 31, 2] and c.live.tolist() == [True, False, True, True]
    touched = []
    for b, first, nodes in ((0, 15, [0, 4, 9]), (2, 30, [0]), (3, 0, [0, 5])):
        table = c.block_table[b].tolist()
        slots = [table[j // 16] * 16 + j % 16 for j in range(first, first + len(nodes))]
        assert torch.equal(c.Kc[:, slots], K[:, b, nodes]) and torch.equal(c.Vc[:, slots], V[:, b, nodes])
        touched += slots
    others = [i for i in range(c.Kc.shape[1]) if i not in touched]
    assert torch.equal(c.Kc[:, others], before[:, others])
    c.release(i32([1, 0, 1, 1]))
    assert c.cache_len.tolist() == [0] * 4 and int(c.free_count) == 60 and not c.live.any()
    with pytest.raises(ValueError, match="made for 64"):
        c.begin(i32([70, 0, 0, 0]), 70)


def test_a_full_pool_grants_no_pages(ctx):
    import torch
    c = _cache(ctx, n_pages=3, B=2, n_layers=1)
    K = torch.randn(60, 2, 64).bfloat16().cuda()
    c.begin(torch.tensor([30, 30], dtype=torch.int32, device="cuda"), 60)
    assert c.granted.tolist() == [1, 0] and c.cache_len.tolist() == [30, 0] and c.live.tolist() == [True, False]
    c.store(0, K, K)
    O = torch.full((60, 6, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    c.attention(0, torch.randn(60, 6, 64).bfloat16().cuda(), O)
    ctx.check_device_status()
    table = c.block_table[0].tolist()
    assert torch.equal(c.Kc[0, [table[j // 16] * 16 + j % 16 for j in range(30)]], K[:30])
    assert torch.isfinite(O).all()


def test_a_captured_round_is_the_round(ctx):
    """A chunk, a token, a step's accepted rows and a release as one CUDA graph, replayed: the same outputs, pages, lengths and tables as the
    calls issued one by one.  Two captures share one workspace."""
    import torch
    from paper_2512_14069_b200 import binding as rb
    g = torch.Generator().manual_seed(6)
    rand = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    inv = torch.tensor([100.0 ** (-i / 16) for i in range(16)], device="cuda")
    chunk, token, zero = i32([50, 3, 0]), i32([1, 1, 1]), i32([0, 0, 1])
    q, k, v, tk, tv = rand(53, 6, 64), rand(53, 2, 64), rand(53, 2, 64), rand(2, 3, 12, 2, 64), rand(2, 3, 12, 2, 64)
    step = types.SimpleNamespace(accept_len=i32([2, 0, 1]), path_nodes=i32([[0, 4, 9], [0, -1, -1], [0, 7, -1]]))
    caches = [_cache(ctx) for _ in range(2)]
    caches[1].workspace = caches[0].workspace
    outs = [(torch.zeros(2, 53, 6, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 3, 6, 64, dtype=torch.bfloat16, device="cuda")) for _ in caches]

    def run(c, o):
        turned = torch.empty_like(q)
        c.begin(chunk, 53)
        for layer in range(2):
            c.store(layer, k, v, Q=q, Q_out=turned, inv_freq=inv)
            c.attention(layer, turned, o[0][layer])
        c.begin(token, 3)
        for layer in range(2):
            c.store(layer, k[:3], v[:3])
            c.attention(layer, q[:3], o[1][layer], max_new=1)
        c.append(step, tk, tv)
        c.release(zero)
    run(caches[0], outs[0])                       # (also what is asked once of the device)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(caches[1], outs[1])
    assert caches[1].cache_len.tolist() == [0, 0, 0]
    graph.replay()
    torch.cuda.synchronize()
    ctx.check_device_status()
    assert caches[1].cache_len.tolist() == [54, 5, 0]
    for name in ("Kc", "Vc", "cache_len", "block_table", "free_pages", "free_count", "granted", "live"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), name
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_refusals(ctx):
    import torch
    from paper_2512_14069_b200 import binding as rb
    from paper_2512_14069_b200.pipeline import SpecStep
    c = _cache(ctx)
    s = SpecStep(ctx, B=3, V=64, k=4, t_max=4, N=16, Hq=6, Hkv=2, d=64, kv_dtype=torch.bfloat16, max_prefix_len=400)
    with pytest.raises(ValueError, match="has room for"):
        s.attention_paged(c, 0, None, None, None)
    bf = lambda *x: torch.zeros(*x, dtype=torch.bfloat16, device="cuda")
    i32 = lambda *x: torch.zeros(*x, dtype=torch.int32, device="cuda")
    f32 = lambda *x: torch.zeros(*x, device="cuda")
    rotate = dict(Q=bf(4, 2, 64), Q_out=bf(4, 2, 64), pos=i32(4), inv_freq=f32(32))
    rb.radar_rotate(ctx, **rotate)
    for change in (dict(Q=None), dict(Q_out=None), dict(Q_out=bf(4, 3, 64)), dict(Q_out=f32(4, 2, 64)), dict(K=bf(5, 2, 64), K_out=bf(5, 2, 64)), dict(pos=None), dict(pos=i32(3)),
                   dict(pos=torch.zeros(4, dtype=torch.int64, device="cuda")), dict(pos=i32(2, 2, 4)), dict(inv_freq=bf(32)), dict(pair_axis=torch.zeros(31, dtype=torch.uint8, device="cuda")),
                   dict(Q=bf(4, 2, 64).cpu()), dict(Q=bf(4, 64, 2).transpose(1, 2)), dict(Q=bf(8, 64)), dict(Q=bf(4, 2, 64).half(), Q_out=bf(4, 2, 64).half())):
        with pytest.raises((ValueError, TypeError)):
            rb.radar_rotate(ctx, **dict(rotate, **change))
    with pytest.raises(rb.RadarError):
        rb.radar_rotate(ctx, **dict(rotate, inv_freq=f32(33)))
    store = dict(K=bf(4, 2, 64), V=bf(4, 2, 64), slots=torch.arange(4, device="cuda"), Kc=bf(16, 2, 64), Vc=bf(16, 2, 64))
    rb.radar_paged_store(ctx, **store)
    rb.radar_paged_store(ctx, **dict(store, Kc=bf(1, 16, 2, 64), Vc=bf(1, 16, 2, 64)))          # (pages of 16 rows)
    for change in (dict(V=bf(3, 2, 64)), dict(V=f32(4, 2, 64)), dict(V=bf(4, 4, 64)[:, :2]), dict(slots=i32(4)), dict(slots=torch.arange(5, device="cuda")), dict(src_row=i32(3)), dict(Kc=f32(16, 2, 64)),
                   dict(Kc=bf(16, 3, 64), Vc=bf(16, 3, 64)), dict(Vc=bf(17, 2, 64)), dict(Q=bf(4, 6, 64)), dict(Q_out=bf(4, 6, 64)), dict(Q=bf(5, 6, 64), Q_out=bf(5, 6, 64)),
                   dict(Q=bf(4, 6, 64), Q_out=bf(3, 6, 64)), dict(Q=f32(4, 6, 64), Q_out=f32(4, 6, 64)), dict(K=bf(4, 2, 64).cpu(), V=bf(4, 2, 64).cpu()), dict(pos=i32(3), inv_freq=f32(8))):
        with pytest.raises((ValueError, TypeError)):
            rb.radar_paged_store(ctx, **dict(store, **change))
    attend = dict(Q=bf(5, 6, 64), q_start=i32(3), Kc=bf(64, 2, 64), Vc=bf(64, 2, 64), page_size=16, block_table=i32(2, 4), cache_len=i32(2), max_new=5, max_cache_len=64, O=bf(5, 6, 64),
                  workspace=c.workspace)
    rb.radar_chunk_attention(ctx, **attend)
    for change in (dict(Q=f32(5, 6, 64)), dict(O=bf(4, 6, 64)), dict(O=bf(5, 12, 64)[:, ::2]), dict(q_start=i32(2)), dict(block_table=i32(3, 4)), dict(block_table=i32(8)), dict(Vc=bf(63, 2, 64)),
                   dict(Kc=bf(64, 2, 128), Vc=bf(64, 2, 128)), dict(lse=f32(6, 5)), dict(lse=bf(5, 6)), dict(cache_len=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(workspace=f32(1 << 20)),
                   dict(page_size=None), dict(max_new=1 << 40)):
        with pytest.raises((ValueError, TypeError, OverflowError)):
            rb.radar_chunk_attention(ctx, **dict(attend, **change))
    for change in (dict(page_size=24), dict(max_cache_len=65), dict(workspace=c.workspace[:1024]), dict(workspace=c.workspace[16:]), dict(Kc=bf(64, 4, 64), Vc=bf(64, 4, 64))):
        with pytest.raises(rb.RadarError):
            rb.radar_chunk_attention(ctx, **dict(attend, **change))
    assert ctx.read_device_status() == 0


def test_a_chunk_of_nothing(ctx):
    import torch
    c = _cache(ctx, B=2, n_layers=1)
    c.begin(torch.tensor([0, 0], dtype=torch.int32, device="cuda"), 0, requests=torch.tensor([0, 1], device="cuda"))
    z = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(0, 6, 64, dtype=torch.bfloat16, device="cuda")
    c.store(0, z, z, Q=q, Q_out=q, inv_freq=torch.ones(32, device="cuda"))
    c.attention(0, q, q)
    ctx.check_device_status()
    assert c.cache_len.tolist() == [0, 0] and c.live.tolist() == [False, True]
