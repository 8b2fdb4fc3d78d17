"""Requests whose attention depends on every page of a long cache, and a bound that shows it where one page's values are wrong.

Rows of randn keys and values average a long cache out: |O| shrinks as the root of what a row attends to, and a bound that counts roundings at
their worst does not.  Here a key of every page (of every 128 tokens where pages are larger) points along one of a few directions, and a query
points along one of them: its row's mass lies on those keys, in parts of about one size, and what stands in any of their pages moves O."""
import numpy as np
import torch

import paged_harness as T

TILE = 128
LOUD = 2.5           # length of a planted key, in lengths of a query
SURE = 9.0           # deviations that a sum of independent roundings does not reach: 2 exp(-SURE^2 / 2) = 5e-18 for each output

# (rows of each request, cached tokens of each, query heads, KV heads, head size, page, types, bounds: greater ones select the forms of long caches)
CASES = {
    "a token over 40000": ([1], [40000], 8, 2, 128, 64, {}),
    "a token over 40000, one KV head": ([1], [40000], 8, 1, 64, 64, {}),
    "a token of one head": ([1], [17000], 1, 1, 128, 64, {}),
    "a token of two groups": ([1], [17000], 4, 2, 64, 64, {}),
    "16 rows of one KV head": ([1], [17000], 16, 1, 128, 64, {}),
    "17 rows of one KV head": ([1], [17000], 17, 1, 64, 32, {}),
    "a token, pages of 16": ([1], [9000], 8, 2, 128, 16, {}),
    "two tokens, pages of 32": ([2, 1, 0, 2], [5000, 900, 7, 300], 4, 4, 64, 32, {}),
    "tokens of many requests": ([1] * 40, list(range(3, 6000, 150)), 4, 1, 128, 64, {}),
    "few rows in tiles": ([1, 4, 0, 1], [5000, 700, 40, 128], 32, 8, 128, 32, dict(max_len=60000)),
    "few rows in tiles, one head": ([1, 16, 1], [9000, 700, 257], 4, 4, 64, 32, dict(max_len=60000)),
    "33 rows in tiles": ([33, 1, 16], [733, 9000, 300], 4, 4, 128, 32, dict(max_len=60000)),
    "64 rows in tiles": ([16, 1, 8], [6000, 9000, 300], 32, 8, 64, 32, dict(max_len=60000)),
    "100 rows in tiles": ([100, 1, 50], [9000, 3000, 300], 4, 4, 64, 32, dict(max_len=60000)),
    "300 rows over 20000": ([300], [20000], 4, 1, 128, 64, {}),
    "a chunk, pages of 16": ([150], [9000], 6, 2, 128, 16, {}),
    "a chunk, pages of 128": ([70], [17000], 6, 2, 64, 128, {}),
    "a chunk, pages of 384": ([70, 1], [17000, 9000], 4, 2, 128, 384, {}),
    "chunks and tokens": ([1, 500, 1, 260], [5000, 1500, 20, 4000], 8, 8, 128, 64, {}),
}


def grain(page):
    """Tokens that share a planted key."""
    return min(page, TILE)


def request(rng, n, L, Hq, Hkv, d, page, dtype):
    """(q [n, Hq, d], k, v [L, Hkv, d]) in float64, rounded to the type.  Pieces and rows of a KV head take the directions in turn."""
    G = Hq // Hkv
    C = max(1, min(8, G * n))
    along = rng.standard_normal((Hkv, C, d))
    along *= np.sqrt(d) / np.linalg.norm(along, axis=-1, keepdims=True)
    k, v = rng.standard_normal((2, L, Hkv, d))
    for piece, first in enumerate(range(0, L, grain(page))):
        j = first + int(rng.integers(0, min(grain(page), L - first)))
        k[j] = LOUD * along[:, piece % C] + 0.2 * rng.standard_normal((Hkv, d))      # (their masses differ by some 20 %, and so do the roundings)
    row = (np.arange(n)[:, None] * G + np.arange(Hq) % G) % C
    q = along[np.arange(Hq) // G, row] + 0.1 * rng.standard_normal((n, Hq, d))
    return tuple(torch.from_numpy(x).to(T.DT[dtype]).double().numpy() for x in (q, k, v))


def attention(q, k, v, seen):
    """float64 (O, lse, sum p |v|, root of sum (p v)^2, p [Hq, n, L])."""
    n, Hq, d = q.shape
    G = Hq // k.shape[1]
    O, size, root, lse, ps = np.zeros((n, Hq, d)), np.zeros((n, Hq, d)), np.zeros((n, Hq, d)), np.full((n, Hq), -np.inf), np.zeros((Hq, n, len(k)))
    hidden, live = np.arange(len(k)) >= seen[:, None], seen > 0
    for h in range(Hq):
        if not live.any():
            continue
        z = np.where(hidden, -np.inf, q[:, h] @ k[:, h // G].T * d ** -0.5)[live]
        top = z.max(-1, keepdims=True)
        p = np.exp(z - top)
        total = p.sum(-1, keepdims=True)
        p /= total
        ps[h, live], x = p, v[:, h // G]
        O[live, h], size[live, h], root[live, h] = p @ x, p @ np.abs(x), np.sqrt(p ** 2 @ x ** 2)
        lse[live, h] = (np.log(total) + top)[:, 0]
    return O, lse, size, root, ps


def bound(q, k, v, O, size, root, p, dtype):
    """What O may be off by.

    Scores and exponentials as in paged_harness.check_chunk: a probability is off by a share r of itself, at its worst in one direction.  A sum in
    fp32 is rounded with each addend (2^-24 of what it holds, 2^-23 on the tensor cores, which take 16 at a time and truncate), and what it holds is
    a part of the whole, chosen without a look at the values: |O| and SURE times the root of the squares.  An addend that is below 2^-23 of that
    moves the sum by itself at most, and so the many that are next to nothing are counted by their mass, and by one rounding for 16 of them.  256:
    what joins and moves of the maximum add.  bf16: each probability is rounded for its product by up to 2^-8 of itself, the one's rounding
    independent of the other's but for a share common to all: SURE roots, and 2^-8 |O|.  O is rounded once."""
    d, L = q.shape[-1], len(k)
    most = np.abs(v).max(initial=0)
    small = p <= 2.0 ** -23 * root.min(-1, initial=np.inf).T[..., None] / max(most, 1e-300)
    roundings = ((~small).sum(-1) + L / 16 + 256).T[..., None]
    nothing = (p * small).sum(-1).T[..., None] * most
    norm = lambda x: np.sqrt((x ** 2).sum(-1)).max(initial=0)
    move = norm(q) * norm(k) * d ** -0.5 * (d * 2.0 ** -23 + 2.0 ** -22)
    r = np.expm1(move) + 2.0 ** -22
    out = 2.1 * r * size + roundings * 2.0 ** -23 * (2 * np.abs(O) + SURE * root) + nothing + T.EPS[dtype] * np.abs(O)
    if dtype == "bf16":
        out = out + 2.0 ** -8 * (np.abs(O) + SURE * root)
    return out, move


def hold(O, lse, requests, start, dtype):
    """O and lse as they came, float64 [rows, Hq, d] and [rows, Hq]: the largest share of the bound that an output is off by, below 1 where all are
    right."""
    worst = 0.0
    for b, (q, k, v) in enumerate(requests):
        at, n, L = slice(int(start[b]), int(start[b + 1])), len(q), len(k)
        if n == 0:
            continue
        want, l, size, root, p = attention(q, k, v, np.maximum(L - n + 1 + np.arange(n), 0))
        most, move = bound(q, k, v, want, size, root, p, dtype)
        err = np.abs(O[at] - want)
        assert np.all(np.isfinite(err)), (b, n, L)
        worst = max(worst, float(np.max(err / (most + 1e-300))))
        empty = np.isneginf(l)
        assert np.array_equal(empty, np.isneginf(lse[at])), (b, n, L)
        assert np.all(np.abs(lse[at][~empty] - l[~empty]) <= move + 2.0 ** -21 + L * 2.0 ** -23 + 2.0 ** -22 * np.abs(l[~empty])), (b, n, L)
    return worst


def pool(rng, requests, Hkv, d, page, dtype):
    """(Kc, Vc, table): the requests' rows in random pages, NaN where no token is."""
    have = [-(-len(k) // page) for _, k, _ in requests]
    order, at = rng.permutation(sum(have) + 2), 0
    table = np.full((len(requests), max(1, max(have))), -7)
    Kc, Vc = (torch.full((len(order) * page, Hkv, d), float("nan"), dtype=T.DT[dtype]) for _ in range(2))
    for b, (_, k, v) in enumerate(requests):
        table[b, :have[b]] = order[at:at + have[b]]
        at += have[b]
        if len(k):
            j = np.arange(len(k))
            slots = torch.from_numpy(table[b, j // page] * page + j % page)
            Kc[slots], Vc[slots] = torch.from_numpy(k).to(T.DT[dtype]), torch.from_numpy(v).to(T.DT[dtype])
    return Kc, Vc, table


def make(name, dtype):
    """(requests, start) of a case, the same each time."""
    news, lens, Hq, Hkv, d, page, _ = CASES[name]
    rng = np.random.default_rng([list(CASES).index(name), dtype == "bf16"])
    return [request(rng, n, L, Hq, Hkv, d, page, dtype) for n, L in zip(news, lens)], np.concatenate([[0], np.cumsum(news)])
