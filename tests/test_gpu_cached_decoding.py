"""The 4-bit cache's operators as a decoding loop uses them: admission, steps, release, over `FourBitCache` and `SpecStep`."""
import os
import sys

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
    text, dec = D.main()
    assert len(text) == 6 and all(len(t) >= 24 for t in text.values())
    assert int(dec.cache.free_count) == dec.cache.free_pages.numel()
    assert sorted(dec.cache.free_pages.tolist()) == list(range(dec.cache.free_pages.numel()))
    assert dec.cache.cache_len.tolist() == [0] * dec.B
    again, _ = D.main()
    assert again == text
    assert "pages free" in capsys.readouterr().out


def test_a_step_is_what_the_tree_attention_makes_of_the_loaded_rows(ctx):
    """radar_tree_attention over the rows that the cache gives back (exact in bf16), on each layer's own inputs.  Both kernels'
    probabilities enter their product as bf16 and O is rounded to bf16: each is off by up to 2^-7 sum p |v|, the two by twice that
    (a tenth more for the fp32 sums); sum p |v| is at most the largest |v|."""
    import torch
    import decode_with_cache as D
    from paper_2512_14069_b200 import binding as rb
    model = D.Model(layers=2, Hq=8, Hkv=2, d=64, V=300, max_len=200, seed=3)
    dec = D.Decoder(ctx, model, B=3, n_pages=40, max_len=200)
    rng = np.random.default_rng(5)
    for b, n in enumerate((2, 40, 61)):
        dec.admit(b, rng.integers(0, model.V, n).tolist())
    s, c, seen = dec.step, dec.cache, []

    def check(layer, Q, Kt, Vt):
        lens = c.cache_len.cpu()
        start = torch.zeros(4, dtype=torch.int32)
        start[1:] = lens.cumsum(0)
        n = int(start[3])
        K = torch.zeros(model.layers, n, model.Hkv, model.d, dtype=torch.bfloat16, device="cuda")
        V = torch.zeros_like(K)
        c.load(torch.zeros(3, dtype=torch.int32, device="cuda"), start.cuda(), K, V)
        O, lse = s.O.clone(), s.lse.clone()
        s.attention(Q.contiguous(), K[layer], V[layer], start[:3].long().cuda(), c.cache_len, Kt.contiguous(), Vt.contiguous())
        for b in range(3):
            m = int(s.n_nodes[b])
            most = max(float(V[layer, start[b]:start[b + 1]].abs().max()), float(Vt[b, :m].abs().max()))
            assert float((O[b, :m].float() - s.O[b, :m].float()).abs().max()) <= 2.2 * 2.0 ** -7 * most
            assert float((lse[b, :, :m] - s.lse[b, :, :m]).abs().max()) <= 1e-4
        s.O.copy_(O), s.lse.copy_(lse)
        seen.append(n)

    before = c.cache_len.tolist()
    for _ in range(6):
        emitted = dec.decode_step(check)
        ctx.check_device_status()
        after = c.cache_len.tolist()
        assert [a - x for a, x in zip(after, before)] == [len(e) for e in emitted] and c.granted.tolist() == [1, 1, 1]
        before = after
    assert len(seen) == 12 and seen == sorted(seen)


def test_appended_rows_are_the_accepted_ones(ctx):
    """The rows that a step adds, loaded back, are the quantised rows of the accepted nodes in their order."""
    import torch
    import decode_with_cache as D
    from oracle import cache_oracle as C
    model = D.Model(layers=2, Hq=4, Hkv=4, d=128, V=100, max_len=128, seed=4)
    dec = D.Decoder(ctx, model, B=2, page_size=32, n_pages=20, max_len=128)
    for b, n in enumerate((9, 33)):
        dec.admit(b, list(range(n)))
    first = dec.cache.cache_len.clone()
    emitted = dec.decode_step()
    n = sum(map(len, emitted))
    K = torch.zeros(2, n, 4, 128, device="cuda")
    V = torch.zeros_like(K)
    dec.cache.load(first, dec.cache.start, K, V)
    ctx.check_device_status()
    at = 0
    for b, e in enumerate(emitted):
        nodes = dec.step.path_nodes[b, :len(e)].tolist()
        assert nodes[0] == 0
        for got, rows in ((K, dec.K), (V, dec.V)):
            want = rows[:, b, nodes].double().cpu().numpy()
            codes, numbers = C.quantise(want)
            assert np.array_equal(got[:, at:at + len(e)].double().cpu().numpy(), C.values(codes, numbers))
        at += len(e)


def test_a_full_pool_grants_no_pages(ctx):
    import torch
    from paper_2512_14069_b200.cache import FourBitCache
    c = FourBitCache(ctx, n_layers=1, B=2, Hq=2, Hkv=2, d=64, page_size=16, n_pages=3, max_len=64, max_new=64)
    rows = torch.randn(1, 60, 2, 64, device="cuda")
    c.admit(torch.tensor([30, 30], dtype=torch.int32, device="cuda"), rows, rows)
    ctx.check_device_status()
    assert c.granted.tolist() == [1, 0] and c.cache_len.tolist() == [30, 0] and int(c.free_count) == 1
    with pytest.raises(ValueError, match="made for 64"):
        c.admit(torch.tensor([40, 40], dtype=torch.int32, device="cuda"), torch.randn(1, 80, 2, 64, device="cuda"), torch.randn(1, 80, 2, 64, device="cuda"))
    c.release(torch.tensor([1, 0], dtype=torch.uint8, device="cuda"))
    assert int(c.free_count) == 3 and c.cache_len.tolist() == [0, 0]


def test_a_captured_step_is_the_step(ctx):
    """Attention and append as a CUDA graph, replayed: the same output, pages, lengths and tables as the calls issued one by one."""
    import types
    import torch
    from paper_2512_14069_b200 import binding as rb
    from paper_2512_14069_b200.cache import FourBitCache
    B, L, Hq, Hkv, d, R = 3, 2, 8, 2, 64, rb.RADAR_MAX_NODES
    g = torch.Generator().manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    prompt, rows, Q = (rand(L, 90, Hkv, d), rand(L, 90, Hkv, d)), (rand(L, B, R, Hkv, d), rand(L, B, R, Hkv, d)), rand(B, R, Hq, d)
    n_nodes = torch.tensor([20, 33, 1], dtype=torch.int32, device="cuda")
    step = types.SimpleNamespace(accept_len=torch.tensor([2, 0, 0], dtype=torch.int32, device="cuda"),
                                 path_nodes=torch.tensor([[0, 3, 7, -1], [0, -1, -1, -1], [0, -1, -1, -1]], dtype=torch.int32, device="cuda"))
    caches = [FourBitCache(ctx, n_layers=L, B=B, Hq=Hq, Hkv=Hkv, d=d, page_size=16, n_pages=30, max_len=160, max_new=90) for _ in range(2)]
    O = [torch.zeros(L, B, R, Hq, d, dtype=torch.bfloat16, device="cuda") for _ in caches]
    for c in caches:
        c.admit(torch.tensor([40, 33, 17], dtype=torch.int32, device="cuda"), *prompt)

    def run(c, out):
        for _ in range(2):
            for layer in range(L):
                c.attention(layer, Q, rows[0][layer], rows[1][layer], out[layer], n_nodes=n_nodes)
            c.append(step, *rows)
    run(caches[0], O[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(caches[1], O[1])
    assert caches[1].cache_len.tolist() == [40, 33, 17]
    graph.replay()
    torch.cuda.synchronize()
    ctx.check_device_status()
    assert caches[1].cache_len.tolist() == [46, 35, 19]
    for name in ("pages", "cache_len", "block_table", "free_pages", "free_count", "granted"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), name
    assert torch.equal(O[0], O[1])
