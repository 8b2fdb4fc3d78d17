"""The 4-bit paged cache on the GPU: pages and slots, rows in and out, attention; against the oracle, request by request and in
float64.  Codes, scales, slots and tables have to be equal; the attention's tolerances are derived in cache_harness.py."""
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


# ---- pages and slots --------------------------------------------------------------------------------------------------
def _extend(ctx, page, lens, new, table, stack, n_free, *, extra=0, in_place=False, capacity=None, path=None, rows=0):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    i32, B = torch.int32, len(lens)
    total = int(np.maximum(new, 0).sum()) if capacity is None else capacity
    t = dict(cache_len=T.dev(lens, i32), new_len=T.dev(np.asarray(new) - extra, i32), block_table=T.dev(table, i32), free_pages=T.dev(stack, i32),
             free_count=T.dev([n_free], i32), slots=torch.full((total,), -5, dtype=torch.int64, device="cuda"), start=torch.zeros(B + 1, dtype=i32, device="cuda"),
             granted=torch.full((B,), 9, dtype=torch.uint8, device="cuda"))
    if not in_place:
        t.update(cache_len_out=torch.full((B,), -1, dtype=i32, device="cuda"), free_count_out=torch.full((1,), -1, dtype=i32, device="cuda"))
    if path is not None:
        t.update(path_nodes=T.dev(path, i32), rows=rows, src_row=torch.full((max(total, 1),), -7, dtype=i32, device="cuda"))
    rb.radar_cache_extend(ctx, page_size=page, extra=extra, **t)
    out = {k: v.cpu().numpy() for k, v in t.items() if hasattr(v, "cpu")}
    if in_place:
        out["cache_len_out"], out["free_count_out"] = out["cache_len"], out["free_count"]
    return out


@pytest.mark.parametrize("B,page,columns,long", [(1, 16, 8, 60), (3, 64, 9, 200), (31, 16, 40, 300), (33, 32, 17, 500), (1025, 16, 20, 100), (300, 128, 64, 3000), (64, 384, 30, 9000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_pages_and_slots(ctx, B, page, columns, long, in_place):
    """Rounds of requests that grow, shrink and end; the stack runs short in some.  One block and several."""
    rng = np.random.default_rng(B + page)
    n_pages = max(2, int(B * columns * 0.45))
    table, stack, n_free, lens = np.full((B, columns), -3), np.arange(n_pages)[::-1].copy(), n_pages, np.zeros(B, int)
    short = 0
    for it in range(8):
        new = np.minimum(rng.integers(0, long, B), columns * page - lens)
        new = np.where(rng.random(B) < 0.25, -rng.integers(0, lens + 1), new)
        new = np.where(rng.random(B) < 0.1, -lens, new)
        want = C.extend(page, lens, new, table, stack, n_free)
        got = _extend(ctx, page, lens, new, table, stack, n_free, extra=it % 3, in_place=in_place)
        ctx.check_device_status()
        table, stack, n_free, lens, slots, granted = want
        short += int((~granted).sum())
        assert np.array_equal(got["block_table"], table)
        assert got["free_count_out"][0] == n_free and np.array_equal(got["free_pages"][:n_free], stack[:n_free])
        assert np.array_equal(got["cache_len_out"], lens) and np.array_equal(got["granted"], granted.astype(np.uint8))
        assert np.array_equal(got["start"], np.concatenate([[0], np.cumsum([len(s) for s in slots])]))
        assert got["slots"].tolist() == [x for s in slots for x in s]
    assert short > 0 or B in (1, 1025)              # (those stacks are never short)


def test_source_rows_of_accepted_paths(ctx):
    rng = np.random.default_rng(1)
    B, rows = 5, 64
    n = np.array([1, 4, 9, 2, 6])
    path = np.full((B, 9), -1)
    for b in range(B):
        path[b, :n[b]] = np.sort(rng.choice(rows, n[b], replace=False))
    got = _extend(ctx, 16, np.array([3, 14, 30, 0, 16]), n, np.tile(np.arange(4), (B, 1)), np.arange(50), 40, extra=1, path=path, rows=rows)
    ctx.check_device_status()
    assert got["src_row"].tolist() == [b * rows + x for b in range(B) for x in path[b, :n[b]]]


def test_extend_reports_what_does_not_fit(ctx):
    from paper_2512_14069_b200 import binding as rb
    table, stack = np.zeros((2, 3), int), np.arange(10)
    for lens, new, n_free, kw in (([0, -1], [4, 4], 5, {}), ([0, 40], [4, 9], 5, {}), ([0, 5], [4, -6], 5, {}), ([0, 0], [4, 4], 11, {}), ([0, 0], [4, 4], -2, {}),
                                  ([0, 0], [4, 4], 5, dict(capacity=6)), ([0, 40], [4, -40], 9, {}), ([0, 0], [4, 4], 5, dict(path=np.array([[0, 1, 2, -1]] * 2), rows=3))):
        got = _extend(ctx, 16, np.array(lens), np.array(new), table, stack, n_free, **kw)
        assert ctx.read_device_status() == -1, (lens, new, n_free)
        assert got["cache_len_out"][0] == 4 or n_free < 0                   # the other request is served
        assert np.all(got["slots"][:4] >= 0) or n_free < 0
    _extend(ctx, 16, np.array([0]), np.array([0]), table[:1], stack, 5)          # nothing to add, no slots at all
    ctx.check_device_status()
    with pytest.raises(rb.RadarError):
        _extend(ctx, 24, np.array([0]), np.array([4]), table[:1], stack, 5)
    with pytest.raises(ValueError, match="disagree"):
        _extend(ctx, 16, np.array([0, 0]), np.array([4]), table, stack, 5)


# ---- rows in and out ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hkv,page,L,long,fused", [(1, 1, 16, 1, 1, False), (3, 3, 32, 2, 40, True), (2, 8, 64, 1, 150, True), (5, 2, 256, 3, 300, False), (1, 5, 128, 1, 129, False)])
def test_rows_come_back_as_the_format_holds_them(ctx, d, dtype, B, Hkv, page, L, long, fused):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    rng = np.random.default_rng(d + B * 7 + Hkv)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    old, new = rng.integers(0, 40, B), np.maximum(rng.integers(0, long + 1, B), np.arange(B) == 0)
    start = np.concatenate([[0], np.cumsum(new)])
    n = int(start[-1])
    pages = -(-(old + new) // page)
    n_pages = int(pages.sum()) + 1
    table = np.full((B, int(pages.max()) + 1), -4)
    order = rng.permutation(n_pages)
    for b in range(B):
        table[b, :pages[b]] = order[pages[:b].sum():pages[:b + 1].sum()]
    slots = np.array([table[b, p // page] * page + p % page for b in range(B) for p in range(old[b], old[b] + new[b])], np.int64)
    n_src = n + 3
    x = rng.standard_normal((L, n_src, 3 * Hkv, d)) * np.exp(rng.uniform(-9, 7, (L, n_src, 3 * Hkv, 1)))
    x[0, 0] = 0.0
    x[0, 1, :, :16] = np.arange(16) - 7.5                       # ties: 7.5 / 7 is a scale's tie too
    x[0, 2, :, 3] = np.inf
    x[0, 2, :, 20] = -1e30
    x[0, -1] = 1e-38
    rows = torch.from_numpy(x).to(dt)
    g = rows.cuda()
    K, V = g[:, :, Hkv:2 * Hkv], g[:, :, 2 * Hkv:]
    if not fused:
        K, V = K.contiguous(), V.contiguous()
    src = rng.permutation(n_src)[:n]
    pool = torch.from_numpy(rng.integers(0, 256, (L, n_pages, Hkv * page // 16 * 18 * d), dtype=np.uint8)).cuda()
    before = pool.clone()
    if L == 1:
        K, V = K[0], V[0]
    rb.radar_cache_store(ctx, K=K, V=V, slots=T.dev(slots, torch.int64), src_row=T.dev(src, torch.int32), pages=pool if L > 1 else pool[0], page_size=page)
    ctx.check_device_status()
    want = C.values(*C.quantise(rows.double().numpy()[:, src]))
    # the bytes: every stored token's, and nobody else's
    blocks = pool.cpu().numpy().reshape(L, n_pages, Hkv, page // 16, 18 * d)
    left = before.cpu().numpy().reshape(L, n_pages, Hkv, page // 16, 18 * d)
    kq, kn, vq, vn = (u.reshape(L, n_pages, Hkv, page, -1) for u in C.unpack_blocks(blocks.reshape(-1, 18 * d)))
    old_parts = [u.reshape(L, n_pages, Hkv, page, -1) for u in C.unpack_blocks(left.reshape(-1, 18 * d))]
    touched = np.zeros((n_pages, page), bool)
    touched[slots // page, slots % page] = True
    for now, then in zip((kq, kn, vq, vn), old_parts):
        assert np.array_equal(np.moveaxis(now, 3, 2)[:, ~touched], np.moveaxis(then, 3, 2)[:, ~touched])
    K_held = np.moveaxis(C.values(kq, kn), 3, 2)[:, slots // page, slots % page]
    V_held = np.moveaxis(C.values(vq, vn), 3, 2)[:, slots // page, slots % page]
    assert np.array_equal(K_held, want[:, :, Hkv:2 * Hkv]) and np.array_equal(V_held, want[:, :, 2 * Hkv:])
    # and read back
    for out_dt in (torch.bfloat16, torch.float32):
        K2, V2 = (torch.full((L, n + 2, Hkv, d), 3.0, dtype=out_dt, device="cuda") for _ in range(2))
        rb.radar_cache_load(ctx, pages=pool, page_size=page, block_table=T.dev(table, torch.int32), first=T.dev(old, torch.int32), start=T.dev(start, torch.int32), K=K2, V=V2)
        ctx.check_device_status()
        assert np.array_equal(K2[:, :n].double().cpu().numpy(), K_held) and np.array_equal(V2[:, :n].double().cpu().numpy(), V_held)
        assert bool((K2[:, n:] == 3).all()) and bool((V2[:, n:] == 3).all())


def test_prompt_stores_with_rows_in_order(ctx):
    """Whole prompts: consecutive slots, rows in order, blocks that are full, begun and ended in the middle; some not granted."""
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    for d, dt, Hkv, page in ((128, torch.bfloat16, 8, 64), (128, torch.float32, 3, 16), (64, torch.bfloat16, 4, 128), (64, torch.float32, 1, 32)):
        rng = np.random.default_rng(Hkv)
        old, new = np.array([0, 5, 16, 31, 0, 48]), np.array([100, 60, 16, 1, 257, 15])
        start = np.concatenate([[0], np.cumsum(new)])
        columns = 20
        table = rng.permutation(6 * columns).reshape(6, columns)
        slots = np.concatenate([[table[b, p // page] * page + p % page for p in range(old[b], old[b] + new[b])] if b != 1 else [-1] * new[b] for b in range(6)])
        x = torch.from_numpy(rng.standard_normal((2, int(start[-1]), Hkv, d))).to(dt)
        pool = torch.zeros(6 * columns, Hkv * page // 16 * 18 * d, dtype=torch.uint8, device="cuda")
        rb.radar_cache_store(ctx, K=x[0].cuda(), V=x[1].cuda(), slots=T.dev(slots, torch.int64), pages=pool, page_size=page)
        K, V = (torch.zeros(int(start[-1]), Hkv, d, dtype=dt, device="cuda") for _ in range(2))
        rb.radar_cache_load(ctx, pages=pool, page_size=page, block_table=T.dev(table, torch.int32), first=T.dev(old, torch.int32), start=T.dev(start, torch.int32), K=K, V=V)
        ctx.check_device_status()
        want = C.values(*C.quantise(x.double().numpy()))
        on = np.concatenate([[b != 1] * new[b] for b in range(6)])
        assert np.array_equal(K.double().cpu().numpy()[on], want[0][on]) and np.array_equal(V.double().cpu().numpy()[on], want[1][on])


def test_nan_is_stored_as_zero_and_reported(ctx):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    for d, n in ((64, 1), (128, 40)):
        x = torch.randn(n, 2, d, device="cuda")
        x[0, 1, 5] = float("nan")
        pool = torch.zeros(3, 2 * 18 * d, dtype=torch.uint8, device="cuda")
        slots = torch.arange(n, device="cuda")
        rb.radar_cache_store(ctx, K=x, V=torch.zeros_like(x), slots=slots, pages=pool, page_size=16)
        assert ctx.read_device_status() == -6
        K, V = torch.zeros_like(x), torch.ones_like(x)
        rb.radar_cache_load(ctx, pages=pool, page_size=16, block_table=T.dev([[0, 1, 2]], torch.int32), first=T.dev([0], torch.int32), start=T.dev([0, n], torch.int32),
                            K=K, V=V)
        ctx.check_device_status()
        want = C.values(*C.quantise(torch.nan_to_num(x, nan=0.0).double().cpu().numpy()))
        assert np.array_equal(K.double().cpu().numpy(), want) and float(V.abs().max()) == 0.0


def test_store_and_load_report_what_is_out_of_range(ctx):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    i32, d = torch.int32, 64
    K, V = torch.randn(8, 1, d, device="cuda"), torch.randn(8, 1, d, device="cuda")
    pool = torch.zeros(2, 18 * d, dtype=torch.uint8, device="cuda")
    store = lambda slots, **kw: rb.radar_cache_store(ctx, K=K, V=V, slots=T.dev(slots, torch.int64), pages=pool, page_size=16, **kw)
    store([0, -1, -8, 31])
    ctx.check_device_status()
    for slots, kw in (([0, 32], {}), ([1 << 40, 3], {}), ([3, 4], dict(src_row=T.dev([0, 8], i32))), ([3, 4], dict(src_row=T.dev([-1, 0], i32)))):
        store(slots, **kw)
        assert ctx.read_device_status() == -1
    out = torch.zeros(4, 1, d, device="cuda")
    load = lambda table, first, start: rb.radar_cache_load(ctx, pages=pool, page_size=16, block_table=T.dev(table, i32), first=T.dev(first, i32), start=T.dev(start, i32),
                                                           K=out, V=torch.zeros_like(out))
    load([[1, -1]], [0], [0, 4])
    ctx.check_device_status()
    for args in (([[1, 2]], [15], [0, 4]), ([[1, -1]], [15], [0, 4]), ([[1, 0]], [30], [0, 4]), ([[1, 0]], [-1], [0, 4]), ([[1, 0]], [0], [0, 5])):
        load(*args)
        assert ctx.read_device_status() == -1, args
    empty = torch.zeros(0, dtype=torch.int64, device="cuda")
    rb.radar_cache_store(ctx, K=K, V=V, slots=empty, pages=pool, page_size=16)
    ctx.check_device_status()
    with pytest.raises(ValueError, match="pages: expected"):
        rb.radar_cache_store(ctx, K=K, V=V, slots=empty, pages=pool, page_size=32)
    with pytest.raises(ValueError, match="fewer rows"):
        store(list(range(9)))
    with pytest.raises(ValueError, match="last two are contiguous"):
        wide = torch.randn(8, 1, 2 * d, device="cuda")
        rb.radar_cache_store(ctx, K=wide[..., ::2], V=wide[..., 1::2], slots=empty, pages=pool, page_size=16)
    with pytest.raises(ValueError):
        rb.radar_cache_store(ctx, K=K.half(), V=V.half(), slots=T.dev([0], torch.int64), pages=pool, page_size=16)
    with pytest.raises(rb.RadarError):                           # rows that do not start on 16 bytes
        wide = torch.randn(8 * (d + 1) + 4, device="cuda")
        odd = wide[:8 * (d + 1)].view(8, 1, d + 1)[..., :d]
        rb.radar_cache_store(ctx, K=odd, V=odd, slots=T.dev([0], torch.int64), pages=pool, page_size=16)


# ---- attention ----------------------------------------------------------------------------------------------------------
SHAPES = [  # lens, Hq, Hkv, d, page, rows
    ([0], 1, 1, 64, 16, 1), ([1], 4, 4, 64, 16, 1), ([15, 16, 17], 8, 2, 128, 16, 1), ([127, 128, 129, 0], 32, 8, 128, 64, 1), ([2048], 32, 8, 128, 64, 1),
    ([31, 33, 1000, 5], 40, 40, 128, 32, 1), ([4097], 16, 1, 128, 256, 1), ([700, 0, 3], 24, 8, 64, 128, 4), ([300], 28, 4, 128, 16, 5), ([1, 0, 97], 6, 2, 64, 16, 16),
    ([500, 20], 8, 8, 128, 128, 33), ([129, 1500], 32, 8, 128, 64, 64), ([640], 64, 8, 128, 16, 61), ([256, 0], 28, 4, 64, 32, 64), ([90], 128, 1, 64, 16, 3),
    ([333, 40], 40, 40, 128, 16, 60), ([7], 64, 2, 128, 384, 17), ([3000, 2999], 16, 1, 64, 64, 64), ([6000], 4, 4, 64, 16, 64), ([5, 1111], 48, 16, 128, 128, 50)]


@pytest.mark.parametrize("lens,Hq,Hkv,d,page,rows", SHAPES)
@pytest.mark.parametrize("mask", ["tree", None])
def test_attention(ctx, lens, Hq, Hkv, d, page, rows, mask):
    import cache_harness as T
    rng = np.random.default_rng(sum(lens) + rows)
    T.check_attention(ctx, rng, lens, Hq, Hkv, d, page, rows, mask=mask, fused=mask is None)


@pytest.mark.parametrize("lens,Hq,Hkv,d,page,rows", [s for s in SHAPES if s[5] > 3])
def test_attention_with_ragged_trees_and_empty_rows(ctx, lens, Hq, Hkv, d, page, rows):
    import cache_harness as T
    rng = np.random.default_rng(sum(lens) + rows + 1)
    n = rng.integers(0, rows + 1, len(lens))
    n[0] = rows - 1
    T.check_attention(ctx, rng, lens, Hq, Hkv, d, page, rows, n_nodes=n, mask="holes", max_len=max(lens) + 300)


@pytest.mark.parametrize("rows", [1, 7, 64])
def test_attention_with_scores_that_jump(ctx, rows):
    """Scores of some hundreds: the maximum moves again and again, probabilities are far apart."""
    import cache_harness as T
    T.check_attention(ctx, np.random.default_rng(3), [1500, 70], 8, 2, 128, 32, rows, gain=30.0)
    T.check_attention(ctx, np.random.default_rng(4), [900], 8, 2, 64, 16, rows, gain=8.0, scale=0.7, want_lse=False)


@pytest.mark.parametrize("rows", [1, 64])
def test_attention_on_another_stream(ctx, rows):
    import torch
    import cache_harness as T
    T.check_attention(ctx, np.random.default_rng(6), [600, 64], 8, 2, 128, 16, rows, stream=torch.cuda.Stream())


@pytest.mark.parametrize("rows", [1, 60])
def test_pages_beyond_four_gigabytes(ctx, rows):
    import cache_harness as T
    page_bytes = 8 * 8 * 18 * 128
    T.check_attention(ctx, np.random.default_rng(7), [300, 130], 8, 8, 128, 128, rows, first_page=(1 << 32) // page_bytes + 5)


def test_results_do_not_change_from_run_to_run(ctx):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    for rows in (1, 64):
        kw = T.check_attention(ctx, np.random.default_rng(8), [3000, 1200, 50], 32, 8, 128, 64, rows)
        first = kw["O"].clone(), kw["lse"].clone()
        for _ in range(5):
            kw["O"].zero_(), kw["lse"].zero_()
            rb.radar_cache_attention(ctx, **kw)
            assert torch.equal(kw["O"], first[0]) and torch.equal(kw["lse"], first[1])


def test_a_workspace_serves_smaller_calls(ctx):
    from paper_2512_14069_b200 import binding as rb
    for Hq, Hkv, d, rows in ((32, 8, 128, 1), (32, 8, 128, 64), (64, 8, 128, 64), (40, 40, 128, 64), (6, 2, 64, 7), (16, 1, 128, 33), (8, 1, 64, 64)):
        most = rb.radar_cache_attn_workspace_bytes(ctx, 16, Hq, Hkv, d, rows, 20000)
        for B in (1, 2, 3, 5, 8, 11, 16):
            for n in list(range(0, 3000, 117)) + [4096, 8192, 9999, 20000]:
                assert rb.radar_cache_attn_workspace_bytes(ctx, B, Hq, Hkv, d, rows, n) <= most


def test_attention_reports_what_is_out_of_range(ctx):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    for rows in (1, 64):
        kw = T.check_attention(ctx, np.random.default_rng(9), [300, 40], 8, 2, 64, 16, rows, n_nodes=[rows, rows])
        o, bound = T.held_to[1]
        good = lambda: bool(np.all(np.abs(kw["O"][1].double().cpu().numpy() - o) <= bound))       # (not bit for bit: without the first sequence the keys are shared out differently)
        for name, value in (("cache_len", [301, 40]), ("cache_len", [-1, 40]), ("n_nodes", [rows + 1, rows]), ("n_nodes", [-1, rows])):
            kw["O"].zero_()
            rb.radar_cache_attention(ctx, **dict(kw, **{name: T.dev(value, torch.int32)}))
            assert ctx.read_device_status() == -1, name
            assert float(kw["O"][0].float().abs().max()) == 0.0 and good()
        for page in (-1, kw["pages"].shape[0]):
            table = kw["block_table"].clone()
            table[0, 3] = page
            rb.radar_cache_attention(ctx, **dict(kw, block_table=table))
            assert ctx.read_device_status() == -1
            assert good()
        with pytest.raises(rb.RadarError) as e:
            rb.radar_cache_attention(ctx, **dict(kw, max_cache_len=20000))
        assert e.value.status == -1                              # the table is too narrow
        with pytest.raises(rb.RadarError) as e:
            rb.radar_cache_attention(ctx, **dict(kw, workspace=kw["workspace"][8:]))
        assert e.value.status == -3
        if kw["workspace"].numel() > 256:
            with pytest.raises(rb.RadarError) as e:
                rb.radar_cache_attention(ctx, **dict(kw, workspace=kw["workspace"][:256]))
            assert e.value.status == -3
        with pytest.raises(ValueError, match="bfloat16"):
            rb.radar_cache_attention(ctx, **dict(kw, Q=kw["Q"].float()))
        with pytest.raises(ValueError, match="disagree"):
            rb.radar_cache_attention(ctx, **dict(kw, cache_len=kw["cache_len"][:1]))
        with pytest.raises(ValueError, match="pages: expected"):
            rb.radar_cache_attention(ctx, **dict(kw, page_size=64))
        if rows > 1:
            with pytest.raises(ValueError, match="must follow"):
                rb.radar_cache_attention(ctx, **dict(kw, Q=torch.zeros(2, 2 * rows, 8, 64, dtype=torch.bfloat16, device="cuda")[:, :rows]))


# ---- attention by each of its forms --------------------------------------------------------------------------------------
# Which form takes a call goes by max_cache_len, not by the lengths, which only the GPU knows: with a bound this far off, clusters take nothing
# (a warp would have more stages than they take), up to 32 rows go in ranges, and more to the tensor cores.
FAR = 40000


@pytest.mark.parametrize("lens,Hq,Hkv,d,page,rows", SHAPES)
@pytest.mark.parametrize("mask", ["tree", None])
def test_attention_under_a_far_bound(ctx, lens, Hq, Hkv, d, page, rows, mask):
    import cache_harness as T
    T.check_attention(ctx, np.random.default_rng(sum(lens) + rows + 5), lens, Hq, Hkv, d, page, rows, mask=mask, fused=mask is None, max_len=FAR)


@pytest.mark.parametrize("lens,Hq,Hkv,d,page,rows", [s for s in SHAPES if s[5] > 3])
def test_ragged_trees_under_a_far_bound(ctx, lens, Hq, Hkv, d, page, rows):
    import cache_harness as T
    rng = np.random.default_rng(sum(lens) + rows + 6)
    n = rng.integers(0, rows + 1, len(lens))
    n[-1] = rows
    T.check_attention(ctx, rng, lens, Hq, Hkv, d, page, rows, n_nodes=n, mask="holes", max_len=FAR)


@pytest.mark.parametrize("Hq,Hkv,rows", [(8, 8, 33), (8, 8, 32), (32, 8, 8), (32, 8, 9), (56, 8, 5), (40, 8, 64)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_many_short_sequences(ctx, Hq, Hkv, rows, d):
    """More units than fit clusters; units of one and of two row blocks, and of none, in turn."""
    import cache_harness as T
    rng = np.random.default_rng(rows + d)
    lens, n = rng.integers(0, 150, 60), rng.integers(0, rows + 1, 60)
    lens[::7], n[::5] = 0, rows
    T.check_attention(ctx, rng, list(lens), Hq, Hkv, d, 16, rows, n_nodes=n)


@pytest.mark.parametrize("lens,Hq,Hkv,d,rows", [([8000], 32, 8, 128, 1), ([7777, 20, 6400], 6, 2, 64, 2), ([9000, 0], 4, 4, 128, 8), ([6200], 32, 2, 64, 16), ([7000], 16, 1, 128, 4)])
def test_attention_of_long_sequences_by_large_clusters(ctx, lens, Hq, Hkv, d, rows):
    import cache_harness as T
    T.check_attention(ctx, np.random.default_rng(lens[0]), lens, Hq, Hkv, d, 64, rows)


@pytest.mark.parametrize("rows", [7, 64])
def test_scores_that_jump_under_a_far_bound(ctx, rows):
    import cache_harness as T
    T.check_attention(ctx, np.random.default_rng(13), [1500, 70], 8, 2, 128, 32, rows, gain=30.0, max_len=FAR)
    T.check_attention(ctx, np.random.default_rng(14), [900], 8, 2, 64, 16, rows, gain=8.0, scale=0.7, want_lse=False, max_len=FAR)


@pytest.mark.parametrize("rows", [1, 60])
def test_pages_beyond_four_gigabytes_under_a_far_bound(ctx, rows):
    import torch
    import cache_harness as T
    T.check_attention(ctx, np.random.default_rng(17), [300, 130], 8, 8, 128, 128, rows, first_page=(1 << 32) // (8 * 8 * 18 * 128) + 5, max_len=FAR, stream=torch.cuda.Stream())


@pytest.mark.parametrize("rows", [1, 64])
def test_a_far_bound_reports_what_is_out_of_range(ctx, rows):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    kw = T.check_attention(ctx, np.random.default_rng(19), [300, 40], 8, 2, 64, 16, rows, n_nodes=[rows, rows], max_len=FAR)
    first = kw["O"].clone(), kw["lse"].clone()
    o, bound = T.held_to[1]
    good = lambda: bool(np.all(np.abs(kw["O"][1].double().cpu().numpy() - o) <= bound))
    rb.radar_cache_attention(ctx, **kw)
    assert (kw["O"] == first[0]).all() and (kw["lse"] == first[1]).all()
    for name, value in (("cache_len", [FAR + 1, 40]), ("cache_len", [-1, 40]), ("n_nodes", [rows + 1, rows]), ("n_nodes", [-1, rows])):
        kw["O"].zero_()
        rb.radar_cache_attention(ctx, **dict(kw, **{name: T.dev(value, torch.int32)}))
        assert ctx.read_device_status() == -1, name
        assert float(kw["O"][0].float().abs().max()) == 0.0 and good()
    for page in (-1, kw["pages"].shape[0]):
        table = kw["block_table"].clone()
        table[0, 3] = page
        rb.radar_cache_attention(ctx, **dict(kw, block_table=table))
        assert ctx.read_device_status() == -1
        assert good()
