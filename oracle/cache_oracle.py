"""The 4-bit paged cache from its definition: the format, the page and slot arithmetic, and attention over it in float64.

Shares no code with the CUDA path.  Codes and scales are kept as arrays; `pack_block` is the one place that knows where they lie in
a block's bytes.
"""
from __future__ import annotations

import numpy as np

GROUP = 16


def quantise(x):
    """Codes (int, -8 .. 7) and scale numbers (0 .. 255) of rows [..., d]; a NaN counts as 0."""
    v = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, GROUP)
    v = np.where(np.isnan(v), 0.0, v)
    top = np.abs(v).max(-1)
    with np.errstate(all="ignore"):
        half, e = np.frexp(np.where(np.isinf(top), np.float64(2.0 ** 60), top) / 7.0)
        number = (e - 1 + 20) * 8 + np.rint(half * 16).astype(int) - 8
        number = np.where(half == 0, 0, np.clip(number, 0, 255))
        q = np.clip(np.rint(v / scale(number)[..., None]), -8, 7).astype(int)
    return q.reshape(x.shape), number


def scale(number):
    number = np.asarray(number)
    return np.ldexp(1.0 + (number % 8) / 8.0, number // 8 - 20)


def values(q, number):
    return (q.reshape(*q.shape[:-1], -1, GROUP) * scale(number)[..., None]).reshape(q.shape)


def place(r):
    """Where row r of a block stands among the V codes."""
    return r % 2 * 4 + r % 8 // 2 + r // 8 * 8


def pack_block(kq, kn, vq, vn):
    """The bytes of a block: codes [16, d] and scale numbers [16, d / 16] of K and V."""
    d = kq.shape[1]
    w = d // 64
    out = np.zeros(18 * d, np.uint8)

    def put(at, q, swapped):
        for c in range(d):
            byte = c // 8 * 4 + (c % 8 // 2 + c % 2 * 4) // 2
            out[at + (byte ^ (32 if swapped else 0))] |= np.uint8(int(q[c]) + 8 << (c % 8 // 2 + c % 2 * 4) % 2 * 4)
    for r in range(16):
        put(r * d // 2, kq[r], False)
        put(9 * d + place(r) * d // 2, vq[r], d == 128 and place(r) % 4 >= 2)
        for g in range(d // 16):
            out[8 * d + r % 8 * (d // 8) + g // w * 2 * w + r // 8 * w + g % w] = kn[r, g]
            out[17 * d + g * 16 + place(r) % 4 * 4 + place(r) // 4] = vn[r, g]
    return out


def unpack_blocks(blocks):
    """Codes [N, 16, d] and scale numbers [N, 16, d / 16] of K, then of V, of blocks [N, 18 d]."""
    blocks = np.asarray(blocks).astype(int)
    d = blocks.shape[1] // 18
    w, r, c, g = d // 64, np.arange(16)[:, None], np.arange(d), np.arange(d // 16)
    nibble = c % 8 // 2 + c % 2 * 4
    byte, shift = c // 8 * 4 + nibble // 2, nibble % 2 * 4
    swap = np.where((d == 128) & (place(r) % 4 >= 2), 32, 0)
    kq = (blocks[:, r * d // 2 + byte] >> shift) % 16 - 8
    vq = (blocks[:, 9 * d + place(r) * d // 2 + (byte ^ swap)] >> shift) % 16 - 8
    return (kq, blocks[:, 8 * d + r % 8 * (d // 8) + g // w * 2 * w + r // 8 * w + g % w], vq,
            blocks[:, 17 * d + g * 16 + place(r) % 4 * 4 + place(r) // 4])


def extend(page, cache_len, new, table, stack, n_free):
    """Request by request: (table, stack, free count, lengths, slots per request, granted)."""
    table, stack, lens = table.copy(), list(stack), list(cache_len)
    pages = lambda n: -(-n // page)
    for b, n in enumerate(new):                                 # what is given up first
        if n < 0:
            for i in range(pages(lens[b] + n), pages(lens[b])):
                stack[n_free] = table[b, i]
                n_free += 1
    slots, granted, asked, top = [], [], 0, n_free
    for b, n in enumerate(new):
        have, want = pages(lens[b]), pages(lens[b] + n)
        lack = max(want - have, 0)
        asked += lack
        ok = lack == 0 or asked <= top
        granted.append(ok)
        if ok:
            for i in range(lack):
                table[b, have + i] = stack[top - 1 - (asked - lack) - i]
            n_free -= lack
            slots.append([table[b, p // page] * page + p % page for p in range(lens[b], lens[b] + max(n, 0))])
            lens[b] += n
        else:
            slots.append([-1] * max(n, 0))
    return table, np.array(stack), n_free, np.array(lens), slots, np.array(granted)


def attention(q, k, v, see, scale_):
    """O [M, Hq, d] and lse [Hq, M] in float64 of q [M, Hq, d] over k, v [n, Hkv, d]; see [M, n]: which keys a row attends to."""
    M, Hq, d = q.shape
    k, v = (np.repeat(x, Hq // k.shape[1], axis=1) for x in (k, v))
    z = np.einsum("mhd,nhd->hmn", q, k) * scale_
    z = np.where(see[None], z, -np.inf)
    if z.shape[-1] == 0:
        return np.zeros((M, Hq, d)), np.full((Hq, M), -np.inf)
    top = z.max(-1, keepdims=True)
    p = np.exp(z - np.where(np.isinf(top), 0.0, top))
    total = p.sum(-1)
    with np.errstate(all="ignore"):
        o = np.einsum("hmn,nhd->mhd", p, v) / np.where(total == 0, 1.0, total).T[:, :, None]
        return o, np.log(total) + np.where(np.isinf(top), 0.0, top)[..., 0]
