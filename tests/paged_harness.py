"""Inputs, references in 64 bits and bounds of the paged cache's GPU tests."""
import numpy as np
import torch

from paper_2512_14069_b200 import binding as rb

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}          # a rounding moves a number by at most this share of it
CODE = {"f32": rb.RADAR_F32, "bf16": rb.RADAR_BF16}


def dev(x, dt):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dt).cuda()


def workspace(n):
    w = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
    return w[(-w.data_ptr()) % 256:][:n]


# ---- rotation --------------------------------------------------------------------------------------------------------------
def turned(x, pos, freq, axis, neighbours, inverse=False):
    """x float64 [rows, heads, d] turned; the angles in 80-bit numbers, which hold a 32-bit position times a float32 frequency exactly."""
    P = len(freq)
    two_pi = np.longdouble("6.28318530717958647692528676655900577")
    angle = pos[axis].T.astype(np.longdouble) * np.asarray(freq, np.float32).astype(np.longdouble)
    angle = angle - np.rint(angle / two_pi) * two_pi
    c, s = (f(angle).astype(np.float64)[:, None] for f in (np.cos, np.sin))
    s = -s if inverse else s
    first, second = (np.arange(0, 2 * P, 2), np.arange(1, 2 * P, 2)) if neighbours else (np.arange(P), np.arange(P, 2 * P))
    y, size = x.copy(), np.abs(x)
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    size[..., first] = size[..., second] = np.abs(x[..., first]) + np.abs(x[..., second])
    return y, size


def hold_turned(got, want, size, dtype, turned_channels):
    """cos and sin: the angle in half turns (at most 1) is rounded to fp32 (pi 2^-25 of an angle) and the functions are good to two of their
    last places (2^-23); a product and a sum are rounded (2^-24 each): together below 2^-21 of |x| + |y|.  Then the result's rounding.
    Channels behind the pairs are copied."""
    bound = 2.0 ** -21 * size + EPS[dtype] * (np.abs(want) + 2.0 ** -21 * size)
    bound[..., turned_channels:] = 0
    assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / (bound + 1e-300))


# ---- attention -------------------------------------------------------------------------------------------------------------
def make_cache(rng, lens, page, Hkv, d, dtype, spare=2, poison=True, gain=1.0):
    """A cache of requests with these lengths: rows in random pages; what belongs to no request is NaN.  (Kc, Vc, table, K and V of
    each request in float64)."""
    lens = np.asarray(lens)
    have = -(-lens // page)
    n_pages = int(have.sum()) + spare
    order = rng.permutation(n_pages)
    table = np.full((len(lens), max(1, int(have.max()) + 1)), -7)
    Kc, Vc = (torch.full((n_pages * page, Hkv, d), float("nan") if poison else 0.0, dtype=DT[dtype]) for _ in range(2))
    rows, at = [], 0
    for b, n in enumerate(lens):
        table[b, :have[b]] = order[at:at + have[b]]
        at += have[b]
        k, v = (torch.from_numpy(rng.standard_normal((n, Hkv, d)) * gain).to(DT[dtype]) for _ in range(2))
        if n:
            j = np.arange(n)
            slots = torch.from_numpy(table[b, j // page] * page + j % page)
            Kc[slots], Vc[slots] = k, v
        rows.append((k.double().numpy(), v.double().numpy()))
    return Kc, Vc, table, rows


def attention(q, k, v, seen, scale):
    """float64 (O, lse, sum p |v|) of rows q [n, Hq, d], row i over the first seen[i] of k, v [L, Hkv, d]."""
    n, Hq, d = q.shape
    G = Hq // k.shape[1]
    O, size, lse = np.zeros((n, Hq, d)), np.zeros((n, Hq, d)), np.full((n, Hq), -np.inf)
    hidden = np.arange(len(k)) >= seen[:, None]
    live = seen > 0
    for h in range(Hq):
        z = np.where(hidden, -np.inf, (q[:, h] @ k[:, h // G].T) * scale)[live]
        if not z.size:
            continue
        top = z.max(-1, keepdims=True)
        p = np.exp(z - top)
        total = p.sum(-1, keepdims=True)
        O[live, h], size[live, h] = p / total @ v[:, h // G], p / total @ np.abs(v[:, h // G])
        lse[live, h] = (np.log(total) + top)[:, 0]
    return O, lse, size


held = {}            # of the last check_chunk: what its outputs were compared with


def hold_again(kw, requests):
    """The outputs of another call with check_chunk's arguments, for some of its requests (the sums' order follows from all requests' sizes, so
    that they are not the same to the bit where others change)."""
    for b in requests:
        hold_chunk(kw["O"], kw["lse"], held["q64"], [held["rows"][b]], held["start"][b:b + 2], held["lens"][b:b + 1], held["d"], held["dtype"], held["scale"])


def check_chunk(ctx, rng, news, lens, Hq, Hkv, d, page, dtype="bf16", fused=False, lead=0, tail=0, scale=0.0, gain=1.0, max_new=None, max_len=None, want_lse=True, stream=None,
                rows_behind=0):
    """Runs radar_chunk_attention and holds it to float64.

    Bounds.  A score is d products summed in fp32: each sum is off by 2^-24 of what it holds (2^-23 on the tensor cores, which truncate),
    at most |q| |k|, so d 2^-23 |q| |k| scale; its product with the scale and the maximum's subtraction add 2^-22 of it.  An
    exponential is good to 2^-22.  So a probability is off by a share r of itself, and the sums of n of them or of n products by n 2^-23
    more.  bf16: a probability is rounded for its product (2^-8); O is rounded once (2^-8, fp32 2^-24).  lse: the scores' and the sum's
    errors, and its own rounding."""
    news, lens = np.asarray(news), np.asarray(lens)
    B, T = len(news), int(news.sum())
    Kc, Vc, table, rows = make_cache(rng, lens, page, Hkv, d, dtype, gain=gain)
    start = lead + np.concatenate([[0], np.cumsum(news)])
    n_rows = lead + T + tail
    qkv = torch.from_numpy(rng.standard_normal((max(1, n_rows + rows_behind), Hq + 2, d)) * gain).to(DT[dtype])
    q64 = qkv[:, :Hq].double().numpy()
    Q = qkv.cuda()[:n_rows, :Hq] if fused else qkv[:n_rows, :Hq].contiguous().cuda()
    O, lse = torch.full((n_rows, Hq, d), 7.0, dtype=DT[dtype], device="cuda"), torch.full((n_rows, Hq), 7.0, device="cuda")
    max_new = int(news.max()) if max_new is None else max_new
    max_len = int(lens.max()) if max_len is None else max_len
    table = np.pad(table, ((0, 0), (0, max(0, -(-max_len // page) - table.shape[1]))), constant_values=-7)
    ws = workspace(rb.radar_chunk_attn_workspace_bytes(ctx, B, Hq, Hkv, d, CODE[dtype], max_new, max_len))
    kw = dict(Q=Q, q_start=dev(start, torch.int32), Kc=Kc.cuda(), Vc=Vc.cuda(), page_size=page, block_table=dev(table, torch.int32), cache_len=dev(lens, torch.int32), max_new=max_new,
              max_cache_len=max_len, O=O, lse=lse if want_lse else None, workspace=ws, scale=scale)
    torch.cuda.synchronize()
    rb.radar_chunk_attention(ctx, stream=stream, **kw)
    torch.cuda.synchronize()
    ctx.check_device_status()
    held.update(q64=q64, rows=rows, start=start, lens=lens, d=d, dtype=dtype, scale=scale)
    hold_chunk(O, lse if want_lse else None, q64, rows, start, lens, d, dtype, scale)
    assert torch.all(O[:start[0]] == 7.0) and torch.all(O[start[-1]:] == 7.0)
    if want_lse:
        assert torch.all(lse[:start[0]] == 7.0) and torch.all(lse[start[-1]:] == 7.0)
    return kw


def hold_chunk(O, lse, q64, rows, start, lens, d, dtype, scale=0.0):
    """The comparison of check_chunk: rows [(K, V)] of each request in float64."""
    o_gpu, lse_gpu = O.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    sc = scale if scale > 0 else d ** -0.5
    for b, (k, v) in enumerate(rows):
        at = slice(int(start[b]), int(start[b + 1]))
        n, L = at.stop - at.start, int(lens[b])
        if n == 0:
            continue
        seen = np.maximum(L - n + 1 + np.arange(n), 0)
        o, l, size = attention(q64[at], k, v, seen, sc)
        norm = lambda x: np.sqrt((x ** 2).sum(-1)).max(initial=0)
        top = norm(q64[at]) * norm(k) * sc
        move = top * (d * 2.0 ** -23 + 2.0 ** -22)
        r = np.expm1(move) + 2.0 ** -22 + L * 2.0 ** -23
        p = 2.0 ** -8 if dtype == "bf16" else 0.0
        # (fp32 has no probability below 2^-126 of the largest, 2^-118 where the reference lags: L of them at most)
        bound = (2.1 * r + p + EPS[dtype] + 0.1 * p) * size + L * 2.0 ** -118 * np.abs(v).max(initial=0)
        err = np.abs(o_gpu[at] - o)
        assert np.all(err <= bound), (b, n, L, float(np.max(err / (bound + 1e-300))), np.argwhere(~(err <= bound))[:4].tolist())
        if lse is not None:
            got, empty = lse_gpu[at], np.isneginf(l)
            assert np.array_equal(empty, np.isneginf(got)), (b, n, L)
            assert np.all(np.abs(got[~empty] - l[~empty]) <= move + 2.0 ** -21 + L * 2.0 ** -23 + 2.0 ** -22 * np.abs(l[~empty])), (b, n, L)
