"""radar_rotate and radar_paged_store against 64-bit references (angles in 80)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


def _freq(rng, P):
    return np.concatenate([[1.0], np.exp(-rng.uniform(0, 13, P - 1))]).astype(np.float32)


def _case(rng, rows, heads, d, P, axes, dtype, far=50000):
    import paged_harness as T
    import torch
    x = torch.from_numpy(rng.standard_normal((rows, heads, d))).to(T.DT[dtype])
    return x, rng.integers(-far, far, (axes, rows)), _freq(rng, P), rng.integers(0, axes, P)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("d,P,axes", [(128, 64, 1), (64, 16, 3), (80, 40, 2), (72, 36, 2), (96, 24, 1), (7, 3, 2), (2, 1, 1), (1024, 512, 4), (130, 8, 1), (72, 8, 1)])
@pytest.mark.parametrize("rows", [1, 3, 2501])
def test_rotation(ctx, rows, d, P, axes, neighbours, dtype):
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    Hq, Hkv = (5, 2) if d < 1000 else (2, 1)
    rng = np.random.default_rng([rows, d, P, neighbours])
    q, pos, freq, axis = _case(rng, rows, Hq, d, P, axes, dtype)
    k = torch.from_numpy(rng.standard_normal((rows, Hkv, d))).to(T.DT[dtype])
    Q, K = q.cuda(), k.cuda()
    Qo, Ko = torch.full_like(Q, 9.0), torch.full_like(K, 9.0)
    for inverse in (False, True):
        rb.radar_rotate(ctx, Q=Q, Q_out=Qo, K=K, K_out=Ko, pos=T.dev(pos, torch.int32), inv_freq=T.dev(freq, torch.float32), pair_axis=T.dev(axis, torch.uint8), neighbours=neighbours,
                        inverse=inverse)
        torch.cuda.synchronize()
        ctx.check_device_status()
        for x, out in ((q, Qo), (k, Ko)):
            want, size = T.turned(x.double().numpy(), pos, freq, axis, neighbours, inverse)
            T.hold_turned(out.double().cpu().numpy(), want, size, dtype, 2 * P)
        assert torch.equal(Q.cpu(), q) and torch.equal(K.cpu(), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions(ctx, dtype):
    """Every 32-bit position, the ends among them, and frequencies that are no powers of anything."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    rng = np.random.default_rng(5)
    rows, P = 400, 32
    q, _, freq, _ = _case(rng, rows, 2, 64, P, 1, dtype)
    pos = rng.integers(-2 ** 31, 2 ** 31, (1, rows))
    pos[0, :4] = [2 ** 31 - 1, -2 ** 31, 0, 2 ** 24 + 1]
    freq[1] = np.float32(3.14159274)
    Q = q.cuda()
    rb.radar_rotate(ctx, Q=Q, Q_out=Q, pos=T.dev(pos[0], torch.int32), inv_freq=T.dev(freq, torch.float32))
    torch.cuda.synchronize()
    want, size = T.turned(q.double().numpy(), pos, freq, np.zeros(P, int), False)
    T.hold_turned(Q.double().cpu().numpy(), want, size, dtype, 64)


@pytest.mark.parametrize("rows", [2, 900])
@pytest.mark.parametrize("offset", [0, 1])
def test_parts_of_a_fused_projection_in_place(ctx, rows, offset):
    """Q and K as slices of one buffer, at addresses of 16 bytes and at odd ones; the rest of the buffer stays."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    rng = np.random.default_rng([rows, offset])
    Hq, Hkv, d, P = 6, 2, 64, 32
    flat = torch.from_numpy(rng.standard_normal(rows * (Hq + 2 * Hkv) * d + offset)).bfloat16()
    g = flat.cuda()
    qkv, orig = (x[offset:].view(rows, Hq + 2 * Hkv, d) for x in (g, flat))
    pos, freq = rng.integers(0, 9000, (1, rows)), _freq(rng, P)
    Q, K = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
    rb.radar_rotate(ctx, Q=Q, Q_out=Q, K=K, K_out=K, pos=T.dev(pos, torch.int32), inv_freq=T.dev(freq, torch.float32))
    torch.cuda.synchronize()
    want, size = T.turned(orig[:, :Hq + Hkv].double().numpy(), pos, freq, np.zeros(P, int), False)
    T.hold_turned(qkv[:, :Hq + Hkv].double().cpu().numpy(), want, size, "bf16", d)
    assert torch.equal(qkv[:, Hq + Hkv:].cpu(), orig[:, Hq + Hkv:]) and torch.equal(g[:offset].cpu(), flat[:offset])


@pytest.mark.parametrize("neighbours", [False, True])
def test_inverse_is_the_gradient(ctx, neighbours):
    """<R x, g> = <x, R^T g> for the transpose, and differences of <R x, g> along every channel of a row: R is linear, so a difference of any
    step is the gradient; held to the roundings of the values and of the difference."""
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    rng = np.random.default_rng(8)
    d, P = 24, 8
    _, pos, freq, axis = _case(rng, 1, 1, d, P, 2, "f32")
    kw = dict(inv_freq=T.dev(freq, torch.float32), pair_axis=T.dev(axis, torch.uint8), neighbours=neighbours)
    x, g = rng.standard_normal((1, 1, d)).astype(np.float32), rng.standard_normal((1, 1, d)).astype(np.float32)
    grad = torch.zeros(1, 1, d, device="cuda")
    rb.radar_rotate(ctx, Q=T.dev(g, torch.float32), Q_out=grad, pos=T.dev(pos, torch.int32), inverse=True, **kw)
    step = np.repeat(x, 2 * d, 0)
    for c in range(d):
        step[2 * c, 0, c] += 1.0
        step[2 * c + 1, 0, c] -= 1.0
    S = T.dev(step, torch.float32)
    rb.radar_rotate(ctx, Q=S, Q_out=S, pos=T.dev(np.repeat(pos, 2 * d, 1), torch.int32), **kw)
    y = (S.double().cpu().numpy()[:, 0] * g[0, 0]).sum(-1)
    diff = (y[0::2] - y[1::2]) / (step[0::2].astype(np.float64) - step[1::2])[:, 0].max(-1)
    bound = 2 * d * (2.0 ** -21 + 2.0 ** -24) * 2 * (np.abs(x).max() + 1) * np.abs(g).max()
    assert np.all(np.abs(diff - grad.double().cpu().numpy()[0, 0]) <= bound)


def test_no_rows_and_bad_axes(ctx):
    import paged_harness as T
    import torch
    from paper_2512_14069_b200 import binding as rb
    z = torch.zeros(0, 2, 64, device="cuda")
    rb.radar_rotate(ctx, Q=z, Q_out=z, pos=torch.zeros(0, dtype=torch.int32, device="cuda"), inv_freq=torch.ones(32, device="cuda"))
    rng = np.random.default_rng(9)
    q, pos, freq, axis = _case(rng, 6, 2, 64, 32, 2, "f32")
    Q = q.cuda()
    axis[5] = 7                                                  # no such axis: counts as axis 0, and is told
    rb.radar_rotate(ctx, Q=Q, Q_out=Q, pos=T.dev(pos, torch.int32), inv_freq=T.dev(freq, torch.float32), pair_axis=T.dev(axis, torch.uint8))
    assert ctx.read_device_status() == -1
    axis[5] = 0
    want, size = T.turned(q.double().numpy(), pos, freq, axis, False)
    T.hold_turned(Q.double().cpu().numpy(), want, size, "f32", 64)


# ---- stores ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,T,n_rows,Hq,Hkv,d,P,fused,picked", [
    (1, 1, 1, 8, 2, 128, 64, True, False), (1, 700, 700, 8, 2, 128, 64, True, False), (3, 37, 200, 0, 4, 64, 0, False, True), (2, 9, 9, 4, 4, 64, 16, False, False),
    (1, 2600, 2600, 3, 1, 72, 36, False, False), (5, 11, 64, 2, 1, 128, 64, False, True), (1, 50, 60, 2, 2, 9, 4, True, False), (40, 130, 130, 0, 2, 128, 64, False, False)])
def test_store(ctx, L, T, n_rows, Hq, Hkv, d, P, fused, picked, dtype):
    import paged_harness as H
    import torch
    from paper_2512_14069_b200 import binding as rb
    rng = np.random.default_rng([L, T, Hkv, d])
    lead = (L, n_rows) if L > 1 else (n_rows,)
    x = torch.from_numpy(rng.standard_normal((*lead, max(Hq, 1) + 2 * Hkv, d))).to(H.DT[dtype])
    g = x.cuda()
    hq = max(Hq, 1)
    q, k, v = x[..., :hq, :], x[..., hq:hq + Hkv, :], x[..., hq + Hkv:, :]
    Q, K, V = g[..., :hq, :], g[..., hq:hq + Hkv, :], g[..., hq + Hkv:, :]
    if not fused:
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
    cache_rows = T + 21
    slots = rng.permutation(cache_rows)[:T]
    slots[::5] = -1 if T > 1 else slots[0]
    src = rng.integers(0, n_rows, T) if picked else None
    Kc, Vc = (torch.full((L, cache_rows, Hkv, d) if L > 1 else (cache_rows, Hkv, d), 5.0, dtype=H.DT[dtype], device="cuda") for _ in range(2))
    Qo = torch.full((*((L, T) if L > 1 else (T,)), Hq, d), 5.0, dtype=H.DT[dtype], device="cuda") if Hq else None
    pos, freq, axis = rng.integers(0, 5000, (2, T)), _freq(rng, P) if P else None, rng.integers(0, 2, P) if P else None
    turn = dict(pos=H.dev(pos, torch.int32), inv_freq=H.dev(freq, torch.float32), pair_axis=H.dev(axis, torch.uint8)) if P else {}
    rb.radar_paged_store(ctx, K=K, V=V, slots=H.dev(slots, torch.int64), Kc=Kc, Vc=Vc, src_row=None if src is None else H.dev(src, torch.int32), Q=Q if Hq else None, Q_out=Qo, **turn)
    torch.cuda.synchronize()
    ctx.check_device_status()
    row = np.arange(T) if src is None else src
    kept = slots >= 0
    others = np.setdiff1d(np.arange(cache_rows), slots)
    for l in range(L):
        at = (lambda t: t[l]) if L > 1 else (lambda t: t)
        for name, xs, out, to in (("K", k, Kc, slots[kept]), ("Q", q, Qo, np.arange(T))):
            if out is None:
                continue
            keep = kept if name == "K" else np.ones(T, bool)
            rows = at(xs).double().numpy()[row][keep]
            got = at(out).double().cpu().numpy()
            if P:
                want, size = H.turned(rows, pos[:, keep], freq, axis, False)
                H.hold_turned(got[to], want, size, dtype, 2 * P)
            else:
                assert np.array_equal(got[to], rows)
        assert np.array_equal(at(Vc).double().cpu().numpy()[slots[kept]], at(v).double().numpy()[row][kept])
        for c in (Kc, Vc):
            assert np.all(at(c).double().cpu().numpy()[others] == 5.0)
    assert torch.equal(g.cpu(), x)


def test_store_bad_slots_and_rows(ctx):
    """Slots at or beyond the cache's end and rows that are not there are left out and told; the rest is stored."""
    import paged_harness as H
    import torch
    from paper_2512_14069_b200 import binding as rb
    K = torch.randn(6, 2, 64, device="cuda")
    for slots, src in (([0, 1, 16, 3], None), ([0, 1, 2 ** 40, 3], None), ([0, 1, 2, 3], [0, 1, 6, 3]), ([0, 1, 2, 3], [0, 1, -1, 3])):
        Kc, Vc = torch.zeros(16, 2, 64, device="cuda"), torch.zeros(16, 2, 64, device="cuda")
        rb.radar_paged_store(ctx, K=K, V=K, slots=H.dev(slots, torch.int64), Kc=Kc, Vc=Vc, src_row=None if src is None else H.dev(src, torch.int32))
        assert ctx.read_device_status() == -1
        for c in (Kc, Vc):
            assert torch.equal(c[[0, 1, 3]], K[[0, 1, 3]]) and torch.all(c[2] == 0) and torch.all(c[4:] == 0)
    assert ctx.read_device_status() == 0


def test_store_queries_in_place(ctx):
    import paged_harness as H
    import torch
    from paper_2512_14069_b200 import binding as rb
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((700, 8, 64))).bfloat16()
    g = x.cuda()
    Kc, Vc = (torch.zeros(700, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos, freq = rng.integers(0, 100, (1, 700)), _freq(rng, 32)
    rb.radar_paged_store(ctx, K=g[:, 4:6], V=g[:, 6:], slots=torch.arange(700, device="cuda"), Kc=Kc, Vc=Vc, Q=g[:, :4], Q_out=g[:, :4], pos=H.dev(pos, torch.int32),
                         inv_freq=H.dev(freq, torch.float32))
    torch.cuda.synchronize()
    want, size = H.turned(x[:, :6].double().numpy(), pos, freq, np.zeros(32, int), False)
    H.hold_turned(g[:, :4].double().cpu().numpy(), want[:, :4], size[:, :4], "bf16", 64)
    H.hold_turned(Kc.double().cpu().numpy(), want[:, 4:], size[:, 4:], "bf16", 64)
    assert torch.equal(Vc.cpu(), x[:, 6:]) and torch.equal(g[:, 4:].cpu(), x[:, 4:])


def test_slots_beyond_32_bits(ctx):
    """Rows of two layers at the end of pools of more than 2^31 elements."""
    import torch
    from paper_2512_14069_b200 import binding as rb
    Hkv, d = 8, 128
    rows = 2 ** 31 // (Hkv * d) + 64
    pools = [torch.empty(2, rows, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    K, V = (torch.randn(2, 5, Hkv, d, device="cuda").bfloat16() for _ in range(2))
    slots = torch.tensor([rows - 1, rows - 40, 3, -1, rows - 64], device="cuda")
    for p in pools:
        p[:, slots[slots >= 0]] = 7.0
        p[:, rows - 2] = 7.0
    rb.radar_paged_store(ctx, K=K, V=V, slots=slots, Kc=pools[0], Vc=pools[1])
    torch.cuda.synchronize()
    ctx.check_device_status()
    for p, x in zip(pools, (K, V)):
        assert torch.equal(p[:, slots[slots >= 0]], x[:, slots >= 0]) and torch.all(p[:, rows - 2] == 7.0)
