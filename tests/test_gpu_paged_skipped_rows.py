"""Tokens that are skipped (a slot below 0) in radar_paged_store and PagedCache.append: what stands in src_row for them is nobody's."""
import types

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


def _i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_trees_of_fewer_rows_after_larger_ones(ctx, dtype):
    """Accepted rows of trees of 64 rows, then of 12: the source rows that the first ones left behind the second ones' are not there any more."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200.cache import PagedCache
    B, L, Hkv, d, page = 2, 3, 2, 64, 16
    c = PagedCache(ctx, n_layers=L, B=B, Hq=4, Hkv=Hkv, d=d, page_size=page, n_pages=12, max_len=80, max_new=40, dtype=T.DT[dtype])
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g).to(T.DT[dtype]).cuda()
    c.begin(_i32([5, 17]), 22)
    kept = [rand(L, n, Hkv, d) for n in (5, 17)]
    for layer in range(L):
        rows = torch.cat([k[layer] for k in kept])
        c.store(layer, rows, rows)
    for R, accept, nodes in ((64, [3, 3], [[0, 60, 61, 63], [0, 50, 62, 63]]), (12, [0, 1], [[0, -1, -1, -1], [0, 11, -1, -1]]), (1, [0, 0], [[0, -1, -1, -1]] * 2)):
        K = rand(L, B, R, Hkv, d)
        c.append(types.SimpleNamespace(accept_len=_i32(accept), path_nodes=_i32(nodes)), K, K)
        ctx.check_device_status()
        for b in range(B):
            kept[b] = torch.cat([kept[b], K[:, b, nodes[b][:accept[b] + 1]]], 1)
    for b in range(B):
        table, n = c.block_table[b].tolist(), kept[b].shape[1]
        slots = [table[j // page] * page + j % page for j in range(n)]
        assert int(c.cache_len[b]) == n and torch.equal(c.Kc[:, slots], kept[b]) and torch.equal(c.Vc[:, slots], kept[b])


@pytest.mark.parametrize("tokens", [6, 2600])
def test_rows_that_are_not_there_behind_skipped_slots(ctx, tokens):
    """No error without queries; a token's query is turned whatever its slot, so that with queries its row has to be there."""
    import torch
    from paper_2512_14069_b200 import binding as rb
    K = torch.randn(tokens, 2, 64, device="cuda")
    slots, src = torch.arange(tokens, device="cuda"), torch.arange(tokens, dtype=torch.int32, device="cuda")
    slots[::5], src[::5] = -1, _i32([tokens, -1, 2 ** 31 - 1, -2 ** 31, tokens + 7]).repeat(-(-tokens // 25))[:-(-tokens // 5)]
    stored = slots >= 0
    Kc, Vc = torch.full((tokens, 2, 64), 3.0, device="cuda"), torch.full((tokens, 2, 64), 3.0, device="cuda")
    rb.radar_paged_store(ctx, K=K, V=K, slots=slots, src_row=src, Kc=Kc, Vc=Vc)
    assert ctx.read_device_status() == 0
    for c in (Kc, Vc):
        assert torch.equal(c[stored], K[stored]) and torch.all(c[~stored] == 3.0)
    Q, out = torch.randn(tokens, 3, 64, device="cuda"), torch.full((tokens, 3, 64), 3.0, device="cuda")
    rb.radar_paged_store(ctx, K=K, V=K, slots=slots, src_row=src, Kc=Kc, Vc=Vc, Q=Q, Q_out=out)
    assert ctx.read_device_status() == -1
    assert torch.equal(out[stored], Q[stored]) and torch.all(out[~stored] == 3.0) and torch.equal(Kc[stored], K[stored])
