"""The timed cases of the 4-bit paged KV cache: its block tables, its writes, its reads and the attention over it.

blocks   `radar_cache_extend`: pages and slots for the tokens that requests add, pages back from those that give some up.
store    `radar_cache_store`: rows of K and V of all layers into their slots in 4 bits; read back through `radar_cache_load`.
load     `radar_cache_load`: cached tokens as dense rows.
attend   `radar_cache_attention`: one layer's attention of single tokens or draft trees over the cache.
step     the three of a decoding step, one behind the other: accepted tokens get their slots, are stored, and the next tree attends.

The cache.  A group of 16 channels of a token is eight bits of scale, s = 2^(E - 20) (1 + m / 8) as E << 3 | m, and 16 codes
q = -8 .. 7, held as q + 8; the value is q s.  16 tokens of a KV head are a block of 18 d bytes: K codes, K scales, V codes, V
scales; a page is [KV head][page / 16] blocks.
  K codes  row r: d / 8 words of 32 bits; nibble n < 4 of a word is its channel 2 n, nibble 4 + n its channel 2 n + 1.
  K scales group g of row r at (r % 8) * d / 8 + g / w * 2 w + r / 8 * w + g % w, w = d / 64.
  V codes  row r is at place p = r % 2 * 4 + r % 8 / 2 + r / 8 * 8; words as in K; with d = 128 the places 2, 3 mod 4 have their
           two halves of 32 bytes exchanged.
  V scales group g of place p at g * 16 + p % 4 * 4 + p / 4.
"""
import math

import numpy as np
import torch

own = False

_KV_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SCALE_BIAS = 107 * 8          # exponent field and three mantissa bits of 2^-20 as a float32


def listed():
    return [
        # one request decoding: the smallest call, all latency
        dict(kind="blocks", name="blocks_b1", B=1, page=64, len_lo=2048, len_hi=2048, new_lo=5, new_hi=5, gone=0),
        # a server's admission: prompts of many requests at once, one in eight finished and giving its pages back
        dict(kind="blocks", name="blocks_admit_b512", B=512, page=16, len_lo=0, len_hi=0, new_lo=17, new_hi=4096, gone=8),
        # accepted paths of 32 requests, all 32 layers of an 8B model, rows picked from the trees
        dict(kind="store", name="store_accepted_8b_b32", L=32, Hkv=8, d=128, page=64, dtype="bf16", B=32, len_lo=100, len_hi=1000,
             new_lo=1, new_hi=9, tree=True, fused=False),
        # a prompt chunk of 2048 tokens, all layers of the same model, K and V as parts of the fused projection
        dict(kind="store", name="store_prompt_8b", L=32, Hkv=8, d=128, page=64, dtype="bf16", B=1, len_lo=0, len_hi=0, new_lo=2048,
             new_hi=2048, tree=False, fused=True),
        # prompts of a small fp32 model, ragged
        dict(kind="store", name="store_prompts_f32_d64", L=4, Hkv=3, d=64, page=16, dtype="f32", B=7, len_lo=1, len_hi=33, new_lo=1, new_hi=301,
             tree=False, fused=False),
        # shared prefixes read back for the dense attention of the next prompt chunk
        dict(kind="load", name="load_prefix_b4", L=1, Hkv=8, d=128, page=128, dtype="bf16", B=4, len_lo=3000, len_hi=16384),
        dict(kind="load", name="load_prefix_f32_d64", L=2, Hkv=4, d=64, page=16, dtype="f32", B=3, len_lo=5, len_hi=777),
        # single tokens: one interactive request
        dict(kind="attend", name="token_8b_b1", B=1, Hq=32, Hkv=8, d=128, page=64, P_lo=2048, P_hi=2048, rows=1, n_lo=1, fused=False),
        # ... and a server under load with long contexts
        dict(kind="attend", name="token_8b_b32", B=32, Hq=32, Hkv=8, d=128, page=64, P_lo=4096, P_hi=32768, rows=1, n_lo=1, fused=True),
        # whole draft trees: a 70B model's layer
        dict(kind="attend", name="tree_70b_b8", B=8, Hq=64, Hkv=8, d=128, page=128, P_lo=8192, P_hi=8192, rows=64, n_lo=61, fused=False),
        # ... ragged trees over long contexts, the largest case
        dict(kind="attend", name="tree_8b_b32", B=32, Hq=32, Hkv=8, d=128, page=64, P_lo=4096, P_hi=32768, rows=64, n_lo=9, fused=False),
        # a decoding step's calls for one layer: multi-head attention, small trees, odd lengths
        dict(kind="step", name="step_13b_b4", B=4, Hq=40, Hkv=40, d=128, page=16, P_lo=1001, P_hi=4096, rows=64, n_lo=20, new_hi=7, fused=False),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choices(["blocks", "store", "load", "attend", "step"], [0.15, 0.2, 0.1, 0.4, 0.15])[0]
    page = rng.choice([16, 16, 32, 64, 128, 256])
    d = rng.choice([64, 128, 128])
    if kind == "blocks":
        B = log_int(1, 2048)
        prompts = rng.random() < 0.5
        new_hi = log_int(1, max(1, min(8192, 1000000 // B))) if prompts else rng.randint(1, 9)
        len_hi = 0 if prompts else log_int(1, 32768)
        return dict(kind=kind, B=B, page=page, len_lo=len_hi // 4, len_hi=len_hi, new_lo=rng.randint(1, new_hi), new_hi=new_hi, gone=rng.choice([0, 4, 16]))
    Hkv = rng.choice([1, 2, 3, 4, 8, 8, 16, 40])
    if kind in ("store", "load"):
        L = log_int(1, 32)
        B = log_int(1, 32)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if kind == "load":
            len_hi = log_int(1, max(1, min(16384, int(4.0e7 / (L * B * Hkv * d)) + 1)))
            return dict(kind=kind, L=L, Hkv=Hkv, d=d, page=page, dtype=dtype, B=B, len_lo=rng.randint(1, len_hi), len_hi=len_hi)
        tree = rng.random() < 0.5
        new_hi = rng.randint(1, 9) if tree else log_int(1, max(1, min(4096, int(4.0e7 / (L * B * Hkv * d)) + 1)))
        len_hi = log_int(1, 2000)
        return dict(kind=kind, L=L, Hkv=Hkv, d=d, page=page, dtype=dtype, B=B, len_lo=rng.randint(0, len_hi), len_hi=len_hi, new_lo=rng.randint(1, new_hi),
                    new_hi=new_hi, tree=tree, fused=not tree and rng.random() < 0.5)
    Hq, Hkv = rng.choice([(4, 4), (16, 16), (40, 40), (32, 8), (32, 8), (64, 8), (24, 8), (28, 4), (16, 1), (6, 2)])
    B = log_int(1, 64)
    rows = rng.choice([1, 1, 1, 4, 8, 16, 33, 64, 64])
    most = max(16, min(32768, int(6.0e8 / (B * Hkv * d)), int(8.0e8 / (B * Hq * rows))))
    P_hi = log_int(16, most)
    case = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, P_lo=rng.randint(1, P_hi), P_hi=P_hi, rows=rows, n_lo=rng.randint(max(1, rows // 3), rows),
                fused=rng.random() < 0.3)
    if kind == "step":
        case["new_hi"] = rng.randint(1, 9)
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n lengths spread evenly over lo .. hi, the same for every seed."""
    return np.linspace(hi, lo, n).round().astype(np.int64) if n > 1 else np.array([hi], np.int64)


def _dev(x, dt):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dt).cuda()


def _tables(rng, lens, page, spare):
    """A pool of pages dealt out to requests of these lengths: (block table, free pages, free count, pages in the pool)."""
    have = -(-lens // page)
    n_pages = int(have.sum() + spare)
    order = rng.permutation(n_pages)
    table = np.zeros((len(lens), int(have.max()) + spare), np.int64)
    at = 0
    for b, n in enumerate(have):
        table[b, :n] = order[at:at + n]
        at += n
    free = np.zeros(n_pages, np.int64)
    free[:n_pages - at] = order[at:]
    return table, free, n_pages - at, n_pages


def _rows(g, *shape):
    """K-like or V-like rows: some channels of a head are several times as large as the others, as rotated keys have them."""
    x = torch.randn(shape, device="cuda", generator=g)
    loud = torch.rand(shape[-2:], device="cuda", generator=g) < 0.05
    return x.mul_(torch.where(loud, 5.0, 1.0))


def _pool(g, n_pages, Hkv, d, page, L=1):
    """A cache that has been written: [L, n_pages, bytes of a page]."""
    out = []
    for _ in range(L):
        parts = []
        for _ in range(2):
            x = _rows(g, n_pages * page // 16, 16, Hkv, d).transpose(1, 2)
            parts.append(_quantise(x))
        out.append(_pack(*parts[0], *parts[1]).view(n_pages, page // 16, Hkv, 18 * d).transpose(1, 2).reshape(n_pages, -1))
        del parts, x
    return torch.stack(out)


def _pack(kq, ks, vq, vs):
    """Codes [N, Hkv, 16, d] and scale bytes [N, Hkv, 16, d / 16] as blocks [N, Hkv, 18 d]."""
    N, H, _, d = kq.shape
    place = torch.tensor([((p & 3) << 1) | ((p >> 2) & 1) | (p & 8) for p in range(16)], device=kq.device)

    def words(q):
        u = (q + 8).to(torch.uint8).view(N, H, 16, d // 8, 8)[..., [0, 2, 4, 6, 1, 3, 5, 7]]
        return (u[..., 0::2] | (u[..., 1::2] << 4)).view(N, H, 16, d // 2)
    w = d // 64
    k_codes, v_codes = words(kq), words(vq)[:, :, place]
    if d == 128:
        halves = v_codes.view(N, H, 4, 2, 2, 2, 32)
        v_codes = torch.stack([halves[:, :, :, 0], halves[:, :, :, 1].flip(-2)], 3)
    k_scales = ks.view(N, H, 2, 8, 4, w).permute(0, 1, 3, 4, 2, 5)
    v_scales = vs[:, :, place].view(N, H, 4, 4, d // 16).permute(0, 1, 4, 3, 2)
    return torch.cat([x.reshape(N, H, -1) for x in (k_codes, k_scales, v_codes, v_scales)], -1)


def _trees(rng, B, rows, n_lo):
    """Ancestor masks of random draft trees with n_lo .. rows nodes, and of each a path from the root."""
    n = _spread(B, n_lo, rows)
    mask = np.zeros((B, rows), np.uint64)
    mask[:, 0] = 1
    for b in range(B):
        parent = np.maximum(np.arange(rows) - 1 - rng.integers(0, 12, rows), 0)
        for i in range(1, int(n[b])):
            mask[b, i] = mask[b, parent[i]] | np.uint64(1 << i)
    return n, mask.view(np.int64)


def _attention_inputs(s, case, rng, g):
    B, Hq, Hkv, d, rows = (case[k] for k in ("B", "Hq", "Hkv", "d", "rows"))
    n, mask = _trees(rng, B, rows, case["n_lo"])
    if case["fused"]:
        qkv = torch.randn(B, rows, Hq + 2 * Hkv, d, device="cuda", generator=g).bfloat16()
        s["Q"], s["Kt"], s["Vt"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    else:
        s["Q"], s["Kt"], s["Vt"] = (torch.randn(B, rows, h, d, device="cuda", generator=g).bfloat16() for h in (Hq, Hkv, Hkv))
    s["mask"], s["n_nodes"] = _dev(mask, torch.int64), _dev(n, torch.int32)
    s["O"] = torch.zeros(B, rows, Hq, d, dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros(B, Hq, rows, device="cuda")


def prepare(case, seed):
    rng = np.random.default_rng([seed, 77])
    g = torch.Generator(device="cuda").manual_seed(seed)
    i32, kind, B, page = torch.int32, case["kind"], case["B"], case["page"]
    s = dict(case)
    if kind == "load":
        lens = rng.permutation(_spread(B, case["len_lo"], case["len_hi"]))
        table, _, _, n_pages = _tables(rng, lens, page, 2)
        T = int(lens.sum())
        s.update(block_table=_dev(table, i32), first=torch.zeros(B, dtype=i32, device="cuda"), start=_dev(np.concatenate([[0], np.cumsum(lens)]), i32), T=T,
                 pages=_pool(g, n_pages, case["Hkv"], case["d"], page, case["L"]))
        s["K_out"], s["V_out"] = (torch.zeros(case["L"], T, case["Hkv"], case["d"], dtype=_KV_DT[case["dtype"]], device="cuda") for _ in range(2))
        return s
    if kind == "attend":
        lens = rng.permutation(_spread(B, case["P_lo"], case["P_hi"]))
        table, _, _, n_pages = _tables(rng, lens, page, 2)
        s.update(block_table=_dev(table, i32), cache_len=_dev(lens, i32), max_len=case["P_hi"], pages=_pool(g, n_pages, case["Hkv"], case["d"], page)[0])
        _attention_inputs(s, case, rng, g)
        return s
    # the others give requests new tokens
    if kind == "step":
        lens, new = rng.permutation(_spread(B, case["P_lo"], case["P_hi"])), rng.permutation(_spread(B, 1, case["new_hi"]))
    else:
        lens, new = rng.permutation(_spread(B, case["len_lo"], case["len_hi"])), _spread(B, case["new_lo"], case["new_hi"])
        if case.get("gone"):
            new[::case["gone"]] = 0
            lens = lens + 40
        new = rng.permutation(new)
        new = np.where(new == 0, -lens, new)
    add = np.maximum(new, 0)
    spare = int((-(-add // page)).sum()) + B
    table, free, n_free, n_pages = _tables(rng, lens, page, int(-(-add.max() // page)) + 1 if kind != "blocks" else 0)
    need = int((-(-(lens + add) // page)).max())
    table = np.pad(table, ((0, 0), (0, max(0, need - table.shape[1]))))
    free = np.concatenate([free[:n_free], rng.permutation(np.arange(n_pages, n_pages + spare)), np.zeros(n_pages, np.int64)])
    n_free, n_pages, T = n_free + spare, n_pages + spare, int(add.sum())
    tree = kind == "step" or bool(case.get("tree"))
    s.update(block_table=_dev(table, i32), free_pages=_dev(free, i32), free_count=_dev([n_free], i32), free_count_out=_dev([0], i32), cache_len=_dev(lens, i32),
             cache_len_out=_dev(lens, i32), slots=torch.zeros(T, dtype=torch.int64, device="cuda"), start=torch.zeros(B + 1, dtype=i32, device="cuda"),
             granted=torch.zeros(B, dtype=torch.uint8, device="cuda"), T=T, path_nodes=None, src_row=None)
    if tree:           # accept_len + 1 rows of each tree are kept: its root and a path
        path = np.full((B, 9), -1, np.int64)
        for b in range(B):
            path[b, :new[b]] = np.concatenate([[0], np.sort(rng.choice(np.arange(1, 20), new[b] - 1, replace=False))])
        s.update(new_len=_dev(new - 1, i32), extra=1, path_nodes=_dev(path, i32), src_row=torch.zeros(T, dtype=i32, device="cuda"))
    else:
        s.update(new_len=_dev(new, i32), extra=0)
    if kind == "blocks":
        return s
    L, Hkv, d = case.get("L", 1), case["Hkv"], case["d"]
    dt = _KV_DT[case.get("dtype", "bf16")]
    n_src = B * 64 if tree else T
    if kind == "store" and case["fused"]:
        qkv = _rows(g, L, n_src, 6 * Hkv, d).to(dt)
        s["K"], s["V"] = qkv[:, :, 4 * Hkv:5 * Hkv], qkv[:, :, 5 * Hkv:]
    else:
        s["K"], s["V"] = _rows(g, L, n_src, Hkv, d).to(dt), _rows(g, L, n_src, Hkv, d).to(dt)
    if kind == "store":
        s["pages"] = torch.zeros(L, n_pages, Hkv * page // 16 * 18 * d, dtype=torch.uint8, device="cuda")
        s["K_out"], s["V_out"] = (torch.zeros(L, T, Hkv, d, dtype=dt, device="cuda") for _ in range(2))
    else:
        s["pages"], s["max_len"] = _pool(g, n_pages, Hkv, d, page), int(case["P_hi"] + case["new_hi"])
        _attention_inputs(s, case, rng, g)
    return s


# ---- the operators in elementary operations, in 32 bits ----------------------------------------------------------------
def _quantise(x):
    """Codes and scale bytes of float32 rows [..., d], in groups of 16 channels."""
    x = x.reshape(*x.shape[:-1], -1, 16)
    bits = (x.abs().amax(-1) / torch.full((), 7.0, device=x.device)).view(torch.int32)     # (a Python number would be multiplied by its reciprocal)
    byte = (((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - _SCALE_BIAS).clamp(0, 255)
    q = torch.round(x / _scale(byte)[..., None]).clamp(-8, 7)
    return q.flatten(-2).to(torch.int8), byte.to(torch.uint8)


def _scale(byte):
    return ((byte.to(torch.int32) + _SCALE_BIAS) << 20).view(torch.float32)


def _values(q, byte):
    return (q.float().unflatten(-1, (-1, 16)) * _scale(byte)[..., None]).flatten(-2)


def _unpack(blocks, d):
    """float32 K and V, [..., 16, d] each, of blocks [..., 18 d]."""
    lead, w = blocks.shape[:-1], d // 64
    k_codes, k_scales, v_codes, v_scales = blocks.split([8 * d, d, 8 * d, d], -1)
    place = torch.tensor([r % 2 * 4 + r % 8 // 2 + r // 8 * 8 for r in range(16)], device=blocks.device)

    def codes(c):
        c = c.view(*c.shape[:-1], d // 8, 4)
        u = torch.stack([c & 15, c >> 4], -1).flatten(-2)                # nibbles 0 .. 7
        return (u[..., [0, 4, 1, 5, 2, 6, 3, 7]].to(torch.int8) - 8).flatten(-2)
    v_codes = v_codes.reshape(*lead, 16, d // 2)
    if d == 128:
        v = v_codes.view(*lead, 4, 2, 2, 2, 32)
        v_codes = torch.stack([v[..., 0, :, :, :], v[..., 1, :, :, :].flip(-2)], -4).reshape(*lead, 16, d // 2)
    k_s = k_scales.reshape(*lead, 8, 4, 2, w).movedim(-2, -4).reshape(*lead, 16, d // 16)
    v_s = v_scales.reshape(*lead, d // 16, 4, 4).movedim(-1, -3).movedim(-1, -2).reshape(*lead, 16, d // 16)
    return (_values(codes(k_codes.reshape(*lead, 16, d // 2)), k_s),
            _values(codes(v_codes[..., place, :]), v_s[..., place, :]))


def _plain_extend(s):
    page, B, T = s["page"], s["B"], s["T"]
    lens, new, n_free = s["cache_len"].long(), s["new_len"].long() + s["extra"], s["free_count"].long()
    total = lens + new
    have, want = (lens + page - 1) // page, (total + page - 1) // page
    grow, back = (want - have).clamp(min=0), (have - want).clamp(min=0)
    table, stack = s["block_table"].long(), s["free_pages"].long()
    column = torch.arange(table.shape[1], device=table.device)
    # what is given up goes onto the stack, in order
    end = back.cumsum(0)
    given = (column >= want[:, None]) & (column < have[:, None])
    where = torch.where(given, n_free + (end - back)[:, None] + column - want[:, None], stack.numel())
    stack = torch.cat([stack, stack[:1]]).scatter(0, where.flatten(), table.flatten())[:-1]
    n_free = n_free + end[-1:]
    # what is needed comes from its top, in order
    end = grow.cumsum(0)
    granted = (grow == 0) | (end <= n_free)
    taken = (column >= have[:, None]) & (column < want[:, None]) & granted[:, None]
    where = (n_free - 1 - (end - grow)[:, None] - (column - have[:, None])).clamp(0, stack.numel() - 1)
    table = torch.where(taken, stack[where], table)
    start = torch.cat([end.new_zeros(1), new.clamp(min=0).cumsum(0)])
    b = torch.repeat_interleave(torch.arange(B, device=table.device), new.clamp(min=0), output_size=T)
    j = torch.arange(T, device=table.device) - start[b]
    at = lens[b] + j
    slots = torch.where(granted[b], table[b, at // page] * page + at % page, -1)
    out = {"block_table": table.int(), "free_pages": stack.int(), "free_count": (n_free - (grow * granted).sum()).int(),
           "cache_len": torch.where(granted, total, lens).int(), "slots": slots, "start": start.int(), "granted": granted.to(torch.uint8)}
    if s["src_row"] is not None:
        out["src_row"] = (b * 64 + s["path_nodes"].long()[b, j]).int()
    return out, b, at


def _plain_store(s, e):
    def kept(x):
        x = x if s["src_row"] is None else x[:, e["src_row"].long()]
        return _values(*_quantise(x.float()))
    return kept(s["K"]), kept(s["V"])


def _gathered(pages, table, n_blocks, page, Hkv, d):
    """float32 K and V [B, n_blocks * 16, Hkv, d] of the first n_blocks blocks of 16 tokens that the table's rows name."""
    blocks = pages.view(-1, Hkv, page // 16, 18 * d).transpose(1, 2).reshape(-1, Hkv, 18 * d)
    i = torch.arange(n_blocks, device=pages.device)
    got = blocks[table.long()[:, i // (page // 16)] * (page // 16) + i % (page // 16)]
    return tuple(x.transpose(2, 3).flatten(1, 2) for x in _unpack(got, d))


def _plain_load(s):
    n_blocks = -(-s["len_hi"] // 16)
    lens = (s["start"][1:] - s["start"][:-1]).long()
    b = torch.repeat_interleave(torch.arange(s["B"], device="cuda"), lens, output_size=s["T"])
    j = torch.arange(s["T"], device="cuda") - s["start"].long()[b]
    kv = [_gathered(p, s["block_table"], n_blocks, s["page"], s["Hkv"], s["d"]) for p in s["pages"].unbind(0)]
    return tuple(torch.stack([x[i][b, j] for x in kv]).to(_KV_DT[s["dtype"]]) for i in (0, 1))


def _plain_attend(s, K, V, cache_len):
    B, Hq, Hkv, d, rows = (s[k] for k in ("B", "Hq", "Hkv", "d", "rows"))
    K, V = torch.cat([K, s["Kt"].float()], 1), torch.cat([V, s["Vt"].float()], 1)
    n = K.shape[1] - rows
    q = s["Q"].float().view(B, rows, Hkv, Hq // Hkv, d) * (1.0 / math.sqrt(d))
    z = torch.einsum("bmhgd,bphd->bhgmp", q, K)
    node = torch.arange(rows, device="cuda")
    live = node < s["n_nodes"][:, None]
    prefix = (torch.arange(n, device="cuda") < cache_len[:, None])[:, None].expand(B, rows, n)
    tree = (((s["mask"][:, :, None] >> node) & 1) == 1) & live[:, None]
    z.masked_fill_(~torch.cat([prefix, tree], 2)[:, None, None], float("-inf"))
    top = z.amax(-1, keepdim=True)
    z = z.sub_(top).exp_()
    total = z.sum(-1)
    o = torch.einsum("bhgmp,bphd->bmhgd", z, V) / total.permute(0, 3, 1, 2)[..., None]
    o = (o * live[:, :, None, None, None]).reshape(B, rows, Hq, d)
    lse = (total.log() + top[..., 0]).reshape(B, Hq, rows) * live[:, None]
    return {"O": o.bfloat16(), "lse": lse}


def _plain(s):
    kind = s["kind"]
    if kind == "blocks":
        return _plain_extend(s)[0]
    if kind == "store":
        e, _, _ = _plain_extend(s)
        k, v = _plain_store(s, e)
        return {"K": k.to(s["K"].dtype), "V": v.to(s["V"].dtype), "slots": e["slots"], "cache_len": e["cache_len"]}
    if kind == "load":
        k, v = _plain_load(s)
        return {"K": k, "V": v}
    n_blocks = -(-s["max_len"] // 16)
    if kind == "attend":
        K, V = _gathered(s["pages"], s["block_table"], n_blocks, s["page"], s["Hkv"], s["d"])
        return _plain_attend(s, K, V, s["cache_len"])
    e, b, at = _plain_extend(s)
    k, v = _plain_store(s, e)
    K, V = _gathered(s["pages"][0], e["block_table"], n_blocks, s["page"], s["Hkv"], s["d"])
    K[b, at], V[b, at] = k[0], v[0]
    return dict(_plain_attend(s, K, V, e["cache_len"]), slots=e["slots"], cache_len=e["cache_len"])


# ---- the framework's calls ------------------------------------------------------------------------------------------
_kept = {}


def _context():
    from paper_2512_14069_b200 import binding as rb
    if "ctx" not in _kept:
        _kept["ctx"] = rb.Context(torch.cuda.current_device())
    return rb, _kept["ctx"]


def _workspace(n):
    """One workspace for all calls on the stream, as large as the largest call so far needs."""
    w = _kept.get("workspace")
    if w is None or w.numel() < n:
        w = _kept["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return w


def _extend(rb, ctx, s):
    rb.radar_cache_extend(ctx, page_size=s["page"], cache_len=s["cache_len"], new_len=s["new_len"], extra=s["extra"], block_table=s["block_table"],
                          free_pages=s["free_pages"], free_count=s["free_count"], free_count_out=s["free_count_out"], cache_len_out=s["cache_len_out"],
                          slots=s["slots"], start=s["start"], granted=s["granted"], path_nodes=s["path_nodes"], rows=64, src_row=s["src_row"])


def _attend(rb, ctx, s, pages, cache_len):
    n = rb.radar_cache_attn_workspace_bytes(ctx, s["B"], s["Hq"], s["Hkv"], s["d"], s["rows"], s["max_len"])
    rb.radar_cache_attention(ctx, Q=s["Q"], Kt=s["Kt"], Vt=s["Vt"], pages=pages, page_size=s["page"], block_table=s["block_table"], cache_len=cache_len,
                             max_cache_len=s["max_len"], mask=s["mask"], n_nodes=s["n_nodes"], O=s["O"], lse=s["lse"], workspace=_workspace(n))


def _run_own(s):
    rb, ctx = _context()
    kind = s["kind"]
    if kind == "attend":
        _attend(rb, ctx, s, s["pages"], s["cache_len"])
        return {"O": s["O"], "lse": s["lse"]}
    if kind == "load":
        rb.radar_cache_load(ctx, pages=s["pages"], page_size=s["page"], block_table=s["block_table"], first=s["first"], start=s["start"], K=s["K_out"],
                            V=s["V_out"])
        return {"K": s["K_out"], "V": s["V_out"]}
    _extend(rb, ctx, s)
    if kind == "blocks":
        return {"block_table": s["block_table"], "free_pages": s["free_pages"], "free_count": s["free_count_out"], "cache_len": s["cache_len_out"],
                "slots": s["slots"], "start": s["start"], "granted": s["granted"]}
    rb.radar_cache_store(ctx, K=s["K"], V=s["V"], slots=s["slots"], src_row=s["src_row"], pages=s["pages"], page_size=s["page"])
    if kind == "store":
        rb.radar_cache_load(ctx, pages=s["pages"], page_size=s["page"], block_table=s["block_table"], first=s["cache_len"], start=s["start"], K=s["K_out"],
                            V=s["V_out"])
        return {"K": s["K_out"], "V": s["V_out"], "slots": s["slots"], "cache_len": s["cache_len_out"]}
    _attend(rb, ctx, s, s["pages"][0], s["cache_len_out"])
    return {"O": s["O"], "lse": s["lse"], "slots": s["slots"], "cache_len": s["cache_len_out"]}


def run(state):
    return _run_own(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def work(case):
    kind, B, page = case["kind"], case["B"], case["page"]
    if kind == "blocks":
        lens, new = _spread(B, case["len_lo"], case["len_hi"]), _spread(B, case["new_lo"], case["new_hi"])
        pages = int((-(-(lens + new) // page) + -lens // page).sum())
        return {"bytes": 20 * B + 8 * pages + 8 * int(new.sum()), "flops": 0}
    Hkv, d, L = case["Hkv"], case["d"], case.get("L", 1)
    row = Hkv * (d + d // 8)                      # K and V of a cached token
    if kind in ("store", "load"):
        size = 2 if case["dtype"] == "bf16" else 4
        T = int(_spread(B, case["len_lo"], case["len_hi"]).sum() if kind == "load" else _spread(B, case["new_lo"], case["new_hi"]).sum())
        wide = 2 * Hkv * d * size
        return {"bytes": L * T * (wide + row if kind == "load" else 2 * (wide + row)), "flops": 0}
    Hq, P, n = case["Hq"], _spread(B, case["P_lo"], case["P_hi"]), _spread(B, case["n_lo"], case["rows"])
    new = int(_spread(B, 1, case["new_hi"]).sum()) if kind == "step" else 0
    tree = int(n.sum()) * ((2 * Hq + 2 * Hkv) * d * 2 + 8 + 4 * Hq)
    return {"bytes": (int(P.sum()) + 2 * new) * row + new * Hkv * d * 4 + tree + 4 * int((-(-P // page)).sum()),
            "flops": 4 * Hq * d * int((n * P.mean() + n * n / 2).sum())}


# ---- from the definition, in 64 bits ----------------------------------------------------------------------------------
def _exact_kept(x):
    """What the cache holds of rows x [..., d], float64."""
    x = x.double()
    v = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    half, e = torch.frexp(v.abs().amax(-1) / 7)                              # half in [1/2, 1)
    number = ((e - 1 + 20) * 8 + torch.round(half * 16).int() - 8).clamp(0, 255)
    number = torch.where(half == 0, torch.zeros_like(number), number)
    s = torch.ldexp(1 + (number % 8).double() / 8, number // 8 - 20)[..., None]
    return (torch.round(v / s).clamp(-8, 7) * s).reshape(x.shape)


def _exact_tokens(pages, page, Hkv, d, slots):
    """Cached K and V [n, Hkv, d] at `slots`, looked up byte by byte."""
    c, h, r = torch.arange(d, device="cuda"), torch.arange(Hkv, device="cuda")[:, None], slots % 16
    r = r[:, None, None]
    block = ((slots // page)[:, None, None] * Hkv + h) * (page // 16) + (slots % page // 16)[:, None, None]
    flat, w = pages.reshape(-1), d // 64

    def value(codes_at, row, swap, scale_at):
        nibble = c % 8 // 2 + 4 * (c % 2)
        at = codes_at + row * (d // 2) + ((c // 8 * 4) ^ swap) + nibble // 2
        q = (flat[block * 18 * d + at].long() >> (nibble % 2 * 4)) % 16 - 8
        e = flat[block * 18 * d + scale_at].long()
        return q.double() * torch.ldexp(1 + (e % 8).double() / 8, e // 8 - 20)
    grp = c // 16
    place = r % 2 * 4 + r % 8 // 2 + r // 8 * 8
    K = value(0, r, 0, 8 * d + r % 8 * (d // 8) + grp // w * 2 * w + r // 8 * w + grp % w)
    V = value(9 * d, place, (place % 4 // 2) * 32 if d == 128 else 0, 17 * d + grp * 16 + place % 4 * 4 + place // 4)
    return K, V


def _slots_of(table, b, at, page):
    return table[b].long()[at // page] * page + at % page


def exact(case, seed):
    kind, page = case["kind"], case["page"]
    if kind == "blocks":
        return None
    s = prepare(case, seed)
    B, Hkv, d, none = s["B"], s["Hkv"], s["d"], {"slots": None, "cache_len": None}
    if kind == "load":
        start = s["start"].tolist()
        K, V = (torch.empty(s["L"], s["T"], Hkv, d, dtype=torch.float64, device="cuda") for _ in range(2))
        for b in range(B):
            at = torch.arange(start[b + 1] - start[b], device="cuda")
            for l in range(s["L"]):
                K[l, start[b]:start[b + 1]], V[l, start[b]:start[b + 1]] = _exact_tokens(s["pages"][l], page, Hkv, d, _slots_of(s["block_table"], b, at, page))
        return {"K": K, "V": V}
    kept = {}
    if kind in ("store", "step"):
        new, rows = (s["new_len"] + s["extra"]).tolist(), []
        for b, n in enumerate(new):
            rows += (b * 64 + s["path_nodes"][b, :n]).tolist() if s["path_nodes"] is not None else range(len(rows), len(rows) + n)
        if kind == "store":
            return dict({k: torch.stack([_exact_kept(x[rows]) for x in s[k]]) for k in ("K", "V")}, **none)
        ends = np.cumsum([0] + new)
        for b in range(B):
            kept[b] = tuple(_exact_kept(s[k][0][rows[ends[b]:ends[b + 1]]]) for k in ("K", "V"))
    Hq, R = s["Hq"], s["rows"]
    O, lse = torch.zeros(B, R, Hq, d, dtype=torch.float64, device="cuda"), torch.zeros(B, Hq, R, dtype=torch.float64, device="cuda")
    pages, lens, nodes = s["pages"].reshape(-1), s["cache_len"].tolist(), s["n_nodes"].tolist()
    masks = s["mask"].cpu().numpy().view(np.uint64)
    for b in range(B):
        P, M = lens[b], nodes[b]
        K, V = _exact_tokens(pages, page, Hkv, d, _slots_of(s["block_table"], b, torch.arange(P, device="cuda"), page))
        more = [kept[b]] if b in kept else []
        K, V = (torch.cat([x, *(m[i] for m in more), s[t][b, :M].double()]) for i, (x, t) in enumerate(((K, "Kt"), (V, "Vt"))))
        see = torch.ones(M, len(K), dtype=torch.bool)
        for i in range(M):
            for t in range(M):
                see[i, len(K) - M + t] = bool(int(masks[b, i]) >> t & 1)
        see = see.cuda()
        for h in range(Hq):
            z = (s["Q"][b, :M, h].double() @ K[:, h // (Hq // Hkv)].T / math.sqrt(d)).masked_fill(~see, -math.inf)
            lse[b, h, :M] = torch.logsumexp(z, -1)
            O[b, :M, h] = torch.softmax(z, -1) @ V[:, h // (Hq // Hkv)]
    return dict({"O": O, "lse": lse}, **(none if kind == "step" else {}))
