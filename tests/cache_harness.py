"""Inputs and references of the 4-bit cache's GPU tests."""
import numpy as np
import torch

from oracle import cache_oracle as C
from paper_2512_14069_b200 import binding as rb


def dev(x, dt):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dt).cuda()


def random_pool(rng, n_pages, Hkv, d, page, lo=130, hi=160):
    """Pages of random codes and of scales around one (numbers lo .. hi - 1 of 256)."""
    pool = rng.integers(0, 256, (n_pages, Hkv, page // 16, 18 * d), dtype=np.uint8)
    for at in (8 * d, 17 * d):
        pool[..., at:at + d] = rng.integers(lo, hi, pool[..., at:at + d].shape, dtype=np.uint8)
    return pool


def rows_of(pool, table, n, page, Hkv, d):
    """float64 K and V [n, Hkv, d] of a request's first n tokens."""
    if n == 0:
        return np.zeros((0, Hkv, d)), np.zeros((0, Hkv, d))
    blocks = pool[table[:-(-n // page)]].transpose(0, 2, 1, 3).reshape(-1, Hkv, 18 * d)
    kq, kn, vq, vn = C.unpack_blocks(blocks.reshape(-1, 18 * d))
    k, v = C.values(kq, kn), C.values(vq, vn)
    return tuple(x.reshape(-1, Hkv, 16, d).transpose(0, 2, 1, 3).reshape(-1, Hkv, d)[:n] for x in (k, v))


def tree_masks(rng, B, rows):
    mask = np.zeros((B, rows), np.uint64)
    for b in range(B):
        for i in range(rows):
            up = mask[b, rng.integers(0, i)] if i else np.uint64(0)
            mask[b, i] = up | np.uint64(1 << i)
    return mask


held_to = []         # of each sequence of the last check_attention: (O in float64, what O may be off)


def workspace(n):
    w = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
    return w[(-w.data_ptr()) % 256:][:n]


def check_attention(ctx, rng, lens, Hq, Hkv, d, page, rows, n_nodes=None, mask="tree", fused=False, max_len=None, want_lse=True, scale=0.0, gain=1.0, first_page=0,
                    stream=None):
    """Runs radar_cache_attention and holds it to float64.

    Tolerances.  bf16 has eight significant bits, so rounding to it moves a number by up to 2^-8 of itself.  O: a probability
    enters its product as bf16 (2^-8 of it) and O is rounded to bf16 (2^-8): 2^-7 sum p |v|, and a tenth more for the fp32 sums
    and exponentials; a probability below 2^-126 of the largest (2^-118: the reference may lag by 2^8) is none in fp32.  Scores: at most d products of bf16 numbers summed in fp32, each sum off by
    2^-24 of what has been added up (doubled for the tensor cores' truncation), which moves a probability and lse by as much:
    2^-23 d max|q| max|k| scale.  lse adds the fp32 exponentials and sums, 2^-20, and its own rounding."""
    B = len(lens)
    lens = np.asarray(lens)
    pages = -(-lens // page)
    n_pages = int(pages.sum()) + 2
    pool = random_pool(rng, n_pages, Hkv, d, page)
    order = rng.permutation(n_pages)
    table = np.full((B, int(pages.max()) + 1), -9)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = order[at:at + pages[b]]
        at += pages[b]
    M = np.full(B, rows) if n_nodes is None else np.asarray(n_nodes)
    qkv = torch.from_numpy(rng.standard_normal((B, rows, Hq + 2 * Hkv, d))).float().mul_(gain).bfloat16()
    for b in range(B):
        qkv[b, M[b]:, Hq:] = float("nan")                     # rows that belong to no node reach nothing
    masks = tree_masks(rng, B, rows)
    if mask == "holes":                                        # rows that see nothing of the tree, others with foreign bits
        masks[:, ::3] = 0
        masks[:, 1::3] |= np.uint64(1) << np.uint64(63)
    g = qkv.cuda()
    Q, Kt, Vt = g[:, :, :Hq], g[:, :, Hq:Hq + Hkv], g[:, :, Hq + Hkv:]
    if not fused:
        Q, Kt, Vt = Q.contiguous(), Kt.contiguous(), Vt.contiguous()
    O, lse = torch.full((B, rows, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, Hq, rows), 7.0, device="cuda")
    max_len = int(lens.max()) if max_len is None else max_len
    table = np.pad(table, ((0, 0), (0, max(0, -(-max_len // page) - table.shape[1]))), constant_values=-9)
    dpool = torch.empty(first_page + n_pages, Hkv * page // 16 * 18 * d, dtype=torch.uint8, device="cuda")
    dpool[first_page:] = torch.from_numpy(pool.reshape(n_pages, -1))
    ws = workspace(rb.radar_cache_attn_workspace_bytes(ctx, B, Hq, Hkv, d, rows, max_len))
    kw = dict(Q=Q, Kt=Kt, Vt=Vt, pages=dpool, page_size=page, block_table=dev(np.where(table < 0, table, table + first_page), torch.int32), cache_len=dev(lens, torch.int32),
              max_cache_len=max_len, O=O, lse=lse if want_lse else None, workspace=ws, mask=None if mask is None else dev(masks.view(np.int64), torch.int64),
              n_nodes=None if n_nodes is None else dev(M, torch.int32), scale=scale)
    torch.cuda.synchronize()
    rb.radar_cache_attention(ctx, stream=stream, **kw)
    torch.cuda.synchronize()
    ctx.check_device_status()
    o_gpu, lse_gpu = O.double().cpu().numpy(), lse.double().cpu().numpy()
    q64 = qkv.double().numpy()
    sc = scale if scale > 0 else d ** -0.5
    held_to.clear()
    for b in range(B):
        m, n = int(M[b]), int(lens[b])
        K, V = rows_of(pool, table[b], n, page, Hkv, d)
        k, v = np.concatenate([K, q64[b, :m, Hq:Hq + Hkv]]), np.concatenate([V, q64[b, :m, Hq + Hkv:]])
        see = np.ones((m, n + m), bool)
        for i in range(m):
            for t in range(m):
                see[i, n + t] = t <= i if mask is None else bool(int(masks[b, i]) >> t & 1)
        q = q64[b, :m, :Hq]
        o, l = C.attention(q, k, v, see, sc)
        size, _ = C.attention(q, k, np.abs(v), see, sc)
        move = 2.0 ** -23 * d * sc * (np.abs(q).max() if q.size else 0) * (np.abs(k).max() if k.size else 0)
        bound = (1.1 * 2.0 ** -7 + 2 * move) * size + len(v) * 2.0 ** -118 * np.abs(v).max(initial=0)
        held_to.append((o, bound))
        assert np.all(np.abs(o_gpu[b, :m] - o) <= bound), (b, np.max(np.abs(o_gpu[b, :m] - o) / (size + 1e-30)))
        assert np.all(o_gpu[b, m:] == 7.0)
        if want_lse:
            got, empty = lse_gpu[b, :, :m], np.isneginf(l)
            assert np.array_equal(empty, np.isneginf(got))
            assert np.all(np.abs(got - l)[~empty] <= 2.0 ** -20 + move + 2.0 ** -23 * np.abs(l[~empty]))
            assert np.all(lse_gpu[b, :, m:] == 7.0)
    return kw
