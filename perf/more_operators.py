"""The timed cases of the bf16 / float32 paged KV cache: rotary positions, its writes, and the attention of new tokens over it.

rotate   `radar_rotate`: rows of queries and keys turned by their positions, on one axis or several; inverse: its backward pass.
store    `radar_paged_store`: keys (turned on the way) and values into their slots, the queries turned beside them.
attend   `radar_chunk_attention`: ragged chunks of new tokens, single tokens among them, over the paged cache.
admit    the two of a prompt chunk, one behind the other: a chunk's rows are turned and stored, and attend to all that is stored.

Row i of a request with n new rows and L cached tokens (the new ones among them) attends to the tokens 0 .. L - n + i.  Pair p of a
head's first 2 P channels (P frequencies) is channels (p, p + P), or (2 p, 2 p + 1); its angle is position * inv_freq[p], the position
on the pair's axis.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one request's draft tree before its verification: the smallest call, all latency
        dict(kind="rotate", name="rotate_tree_8b_b1", rows=61, Hq=32, Hkv=8, d=128, rot=128, axes=1, neighbours=False, inverse=False, fused=False, dtype="bf16", far=2048),
        # a prompt with images, three axes (time, height, width), queries and keys as parts of the fused projection
        dict(kind="rotate", name="rotate_images_7b", rows=8192, Hq=28, Hkv=4, d=128, rot=128, axes=3, neighbours=False, inverse=False, fused=True, dtype="bf16", far=131072),
        # the gradient of an image encoder's two axes, patches of an odd picture, neighbouring channels
        dict(kind="rotate", name="rotate_grad_f32_d80", rows=5329, Hq=16, Hkv=16, d=80, rot=80, axes=2, neighbours=True, inverse=True, fused=False, dtype="f32", far=73),
        # one request's next token
        dict(kind="store", name="store_token_8b_b1", L=1, Hq=32, Hkv=8, d=128, rot=128, axes=1, neighbours=False, dtype="bf16", tokens=1, page=64, tree=False, fused=True, far=8192),
        # a prompt chunk of one layer, rows of the fused projection, far positions
        dict(kind="store", name="store_prompt_8b", L=1, Hq=32, Hkv=8, d=128, rot=128, axes=1, neighbours=False, dtype="bf16", tokens=8192, page=64, tree=False, fused=True,
             far=131072),
        # what 32 requests accepted, in all layers, picked from the trees' rows (turned before their verification)
        dict(kind="store", name="store_accepted_13b_b32", L=40, Hq=0, Hkv=40, d=128, rot=0, axes=0, neighbours=False, dtype="bf16", tokens=157, page=16, tree=True, fused=False,
             far=4096),
        # single tokens: one interactive request
        dict(kind="attend", name="token_8b_b1", B=1, Hq=32, Hkv=8, d=128, page=64, dtype="bf16", P_lo=2048, P_hi=2048, n_lo=1, n_hi=1, fused=False),
        # ... and a server under load
        dict(kind="attend", name="tokens_8b_b64", B=64, Hq=32, Hkv=8, d=128, page=64, dtype="bf16", P_lo=1000, P_hi=16384, n_lo=1, n_hi=1, fused=True),
        # a chunk of a long prompt, the largest case
        dict(kind="attend", name="chunk_8b_32k", B=1, Hq=32, Hkv=8, d=128, page=64, dtype="bf16", P_lo=32768, P_hi=32768, n_lo=2048, n_hi=2048, fused=False),
        # chunks of many requests beside single tokens, a 70B model's layer, ragged
        dict(kind="attend", name="mixed_70b_b8", B=8, Hq=64, Hkv=8, d=128, page=128, dtype="bf16", P_lo=1500, P_hi=8191, n_lo=1, n_hi=511, fused=False),
        # prompts of a small float32 model
        dict(kind="attend", name="prompts_f32_d64", B=5, Hq=12, Hkv=12, d=64, page=16, dtype="f32", P_lo=37, P_hi=1000, n_lo=37, n_hi=500, fused=False),
        # whole prompts admitted: multi-head attention from the first token on, odd lengths
        dict(kind="admit", name="admit_13b_b4", B=4, Hq=40, Hkv=40, d=128, rot=128, axes=1, neighbours=False, page=16, dtype="bf16", P_lo=1001, P_hi=1777, n_lo=1001, n_hi=1777,
             fused=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choices(["rotate", "store", "attend", "admit"], [0.2, 0.25, 0.35, 0.2])[0]
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    Hq, Hkv = rng.choice([(4, 4), (12, 12), (16, 16), (40, 40), (32, 8), (32, 8), (64, 8), (24, 8), (28, 4), (16, 1), (6, 2)])
    neighbours, axes, far = rng.random() < 0.3, rng.choice([1, 1, 2, 3]), log_int(16, 1000000)
    if kind == "rotate":
        d = rng.choice([64, 72, 80, 128, 128, 256])
        most = int(3.0e7 / ((Hq + Hkv) * d))
        return dict(kind=kind, rows=log_int(1, most), Hq=Hq, Hkv=rng.choice([Hkv, Hkv, 0]), d=d, rot=rng.choice([d, d, d // 8 * 4]), axes=axes, neighbours=neighbours,
                    inverse=rng.random() < 0.5, fused=rng.random() < 0.4, dtype=dtype, far=far)
    d, page = rng.choice([64, 128, 128]), rng.choice([16, 16, 32, 64, 128, 256])
    if kind == "store":
        tree = rng.random() < 0.4
        L = log_int(1, 40)
        rot = 0 if tree else rng.choice([d, d, d // 2])
        Hq = 0 if tree else rng.choice([0, Hq, Hq])
        tokens = log_int(1, max(1, min(8192, int(4.0e7 / (L * (Hq + 2 * Hkv) * d)))))
        return dict(kind=kind, L=L, Hq=Hq, Hkv=Hkv, d=d, rot=rot, axes=axes if rot else 0, neighbours=neighbours, dtype=dtype, tokens=tokens, page=page, tree=tree,
                    fused=not tree and Hq > 0 and rng.random() < 0.5, far=far)
    f32 = dtype == "f32"
    B = log_int(1, 16 if f32 else 64)
    n_hi = rng.choice([1, log_int(1, 64), log_int(16, 2048), log_int(128, 4096)])
    score = 1.0e8 if f32 else 8.0e8                          # rows times keys of all heads
    n_hi = max(1, min(n_hi, int(math.sqrt(score / (B * Hq)))))
    most = max(n_hi, min(32768, int(score / (B * Hq * n_hi)), int(4.0e8 / (B * Hkv * d))))
    P_hi = n_hi if kind == "admit" else log_int(n_hi, most)
    n_lo = rng.randint(1, n_hi)
    case = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, dtype=dtype, P_lo=rng.randint(n_hi, P_hi), P_hi=P_hi, n_lo=n_lo, n_hi=n_hi, fused=rng.random() < 0.4)
    if kind == "admit":
        case.update(P_lo=n_lo, rot=rng.choice([d, d, d // 2]), axes=axes, neighbours=neighbours)
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n lengths spread evenly over lo .. hi, the same for every seed."""
    return np.linspace(hi, lo, n).round().astype(np.int64) if n > 1 else np.array([hi], np.int64)


def _dev(x, dt):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dt).cuda()


def _rows(g, *shape):
    """K-like rows: some channels of a head are several times as large as the others."""
    x = torch.randn(shape, device="cuda", generator=g)
    loud = torch.rand(shape[-2:], device="cuda", generator=g) < 0.05
    return x.mul_(torch.where(loud, 3.0, 1.0))


def _frequencies(rot, axes):
    """1 / 500000^(2 i / rot), and the axis of each pair: runs of about equal length, the first axis' a little shorter."""
    P = rot // 2
    freq = 500000.0 ** (-np.arange(P) / P)
    cut = [P * (a + 1) // axes - (P // 16 if axes > 1 and a < axes - 1 else 0) for a in range(axes)]
    return _dev(freq, torch.float32), _dev(np.searchsorted(cut, np.arange(P), side="right"), torch.uint8) if axes > 1 else None


def _qkv(g, lead, Hq, Hkv, d, dt, fused):
    if fused:
        x = _rows(g, *lead, Hq + 2 * Hkv, d).to(dt)
        return x[..., :Hq, :], x[..., Hq:Hq + Hkv, :], x[..., Hq + Hkv:, :]
    return tuple(_rows(g, *lead, h, d).to(dt) if h else None for h in (Hq, Hkv, Hkv))


def prepare(case, seed):
    rng = np.random.default_rng([seed, 99])
    g = torch.Generator(device="cuda").manual_seed(seed)
    s, kind, dt = dict(case), case["kind"], _DT[case["dtype"]]
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    if case.get("rot"):
        s["inv_freq"], s["pair_axis"] = _frequencies(case["rot"], case["axes"])
    if kind == "rotate":
        rows = case["rows"]
        s["Q"], s["K"], _ = _qkv(g, (rows,), Hq, Hkv, d, dt, case["fused"])
        s["K"] = s["K"] if Hkv else None
        s["pos"] = _dev(rng.integers(0, case["far"], (case["axes"], rows)), torch.int32)
        s["Q_out"], s["K_out"] = torch.zeros(rows, Hq, d, dtype=dt, device="cuda"), torch.zeros(rows, Hkv, d, dtype=dt, device="cuda") if Hkv else None
        return s
    page = case["page"]
    if kind == "store":
        L, T = case["L"], case["tokens"]
        n_rows = 12 * T if case["tree"] else T
        s["Q"], s["K"], s["V"] = _qkv(g, (L, n_rows), Hq, Hkv, d, dt, case["fused"])
        s["src_row"] = _dev(np.sort(rng.choice(n_rows, T, replace=False)), torch.int32) if case["tree"] else None
        n_pages = -(-T // page) + 3
        slots = (rng.permutation(n_pages)[:, None] * page + np.arange(page)).reshape(-1)[rng.integers(0, page):][:T]
        if T > 8:
            slots[::37] = -1                                     # tokens that were not granted a slot
        s["slots"] = _dev(slots, torch.int64)
        s["pos"] = _dev(np.stack([rng.integers(0, case["far"]) + np.arange(T) // (1 + a) for a in range(case["axes"])]), torch.int32) if case["rot"] else None
        s["Kc"], s["Vc"] = (torch.zeros(L, n_pages * page, Hkv, d, dtype=dt, device="cuda") for _ in range(2))
        s["Q_out"] = torch.zeros(L, T, Hq, d, dtype=dt, device="cuda") if Hq else None
        return s
    # requests over a paged cache
    B = case["B"]
    n = _spread(B, case["n_lo"], case["n_hi"])
    lens = n if kind == "admit" else np.maximum(_spread(B, case["P_lo"], case["P_hi"])[::-1], n)
    order = rng.permutation(B)
    n, lens = n[order], lens[order]
    T, have = int(n.sum()), -(-lens // page)
    n_pages = int(have.sum()) + 2
    table, at, pages = np.zeros((B, int(have.max()) + 1), np.int64), 0, rng.permutation(n_pages)
    for b in range(B):
        table[b, :have[b]] = pages[at:at + have[b]]
        at += have[b]
    request, start = np.repeat(np.arange(B), n), np.concatenate([[0], np.cumsum(n)])
    position = np.concatenate([np.arange(lens[b] - n[b], lens[b]) for b in range(B)])
    s.update(T=T, max_len=int(lens.max()), block_table=_dev(table, torch.int32), cache_len=_dev(lens, torch.int32), q_start=_dev(start, torch.int32),
             request=_dev(request, torch.int64), place=_dev(np.arange(T) - start[request], torch.int64))
    s["Q"], s["K"], s["V"] = _qkv(g, (T,), Hq, Hkv, d, dt, case["fused"])
    if kind == "attend":
        s["Kc"], s["Vc"] = (_rows(g, n_pages * page, Hkv, d).to(dt) for _ in range(2))
    else:
        s["Kc"], s["Vc"] = (torch.zeros(n_pages * page, Hkv, d, dtype=dt, device="cuda") for _ in range(2))
        s["slots"] = _dev(table[request, position // page] * page + position % page, torch.int64)
        s["pos"] = _dev(np.stack([position // (1 + a) for a in range(case["axes"])]), torch.int32)
        s["Q_out"] = torch.zeros(T, Hq, d, dtype=dt, device="cuda")
    s["O"], s["lse"] = torch.zeros(T, Hq, d, dtype=dt, device="cuda"), torch.zeros(T, Hq, device="cuda")
    return s


# ---- the operators in elementary operations, in 32 bits (angles in 64) -------------------------------------------------
def _turned(s, x):
    """float32 rows [..., rows, heads, d] turned by s["pos"] (back, where s["inverse"])."""
    x = x.float()
    P = s["rot"] // 2
    axis = s["pair_axis"].long() if s["pair_axis"] is not None else torch.zeros(P, dtype=torch.int64, device="cuda")
    angle = s["pos"].double()[axis].T * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    sin = -sin if s.get("inverse") else sin
    a, b = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if s["neighbours"] else (x[..., :P], x[..., P:2 * P])
    pair = (a * cos - b * sin, b * cos + a * sin)
    return torch.cat([torch.stack(pair, -1).flatten(-2) if s["neighbours"] else torch.cat(pair, -1), x[..., 2 * P:]], -1)


def _plain_store(s):
    dt = _DT[s["dtype"]]
    K, V = (x if s.get("src_row") is None else x[..., s["src_row"].long(), :, :] for x in (s["K"], s["V"]))
    if s["rot"]:
        K = _turned(s, K).to(dt)
    slots, last = s["slots"], s["slots"].argmax()          # a row without a slot writes what the last slot's row does, where it does
    row = torch.where(slots >= 0, torch.arange(len(slots), device="cuda"), last)
    for pool, rows in ((s["Kc"], K), (s["Vc"], V)):
        pool.index_copy_(-3, slots[row], rows.index_select(-3, row))
    if s["Q"] is not None:
        s["Q_out"].copy_(_turned(s, s["Q"]) if s["rot"] else s["Q"])


def _plain_attend(s, Q):
    B, Hq, Hkv, d, n, P = s["B"], s["Hq"], s["Hkv"], s["d"], s["n_hi"], s["max_len"]
    G, page = Hq // Hkv, s["page"]
    token = torch.arange(P, device="cuda")
    slots = s["block_table"].long()[:, token // page] * page + token % page
    K, V = s["Kc"][slots].float(), s["Vc"][slots].float()
    q = torch.zeros(B, n, Hq, d, device="cuda")
    q[s["request"], s["place"]] = Q.float() * (1.0 / math.sqrt(d))
    z = torch.einsum("bnhgd,bphd->bhngp", q.view(B, n, Hkv, G, d), K)
    count = (s["q_start"][1:] - s["q_start"][:-1]).long()
    sees = (s["cache_len"].long() - count)[:, None] + torch.arange(n, device="cuda")            # the last token that a row sees
    z.masked_fill_((token > sees[..., None])[:, None, :, None], float("-inf"))
    top = z.amax(-1, keepdim=True)
    z = z.sub_(top).exp_()
    total = z.sum(-1)
    o = torch.einsum("bhngp,bphd->bnhgd", z, V) / total.permute(0, 2, 1, 3)[..., None]
    lse = (total.log() + top[..., 0]).permute(0, 2, 1, 3)
    return {"O": o.reshape(B, n, Hq, d)[s["request"], s["place"]].to(_DT[s["dtype"]]), "lse": lse.reshape(B, n, Hq)[s["request"], s["place"]]}


def _plain(s):
    kind, dt = s["kind"], _DT[s["dtype"]]
    if kind == "rotate":
        return {k: _turned(s, s[k]).to(dt) for k in ("Q", "K") if s[k] is not None}
    if kind == "store":
        _plain_store(s)
        return {k: s[n] for k, n in (("Q", "Q_out"), ("K", "Kc"), ("V", "Vc")) if s[n] is not None}
    if kind == "attend":
        return _plain_attend(s, s["Q"])
    _plain_store(s)
    return dict(_plain_attend(s, s["Q_out"]), K=s["Kc"], V=s["Vc"])


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


def _store(rb, ctx, s):
    rotation = dict(pos=s["pos"], inv_freq=s["inv_freq"], pair_axis=s["pair_axis"], neighbours=s["neighbours"]) if s["rot"] else {}
    rb.radar_paged_store(ctx, K=s["K"], V=s["V"], slots=s["slots"], src_row=s.get("src_row"), Kc=s["Kc"], Vc=s["Vc"], Q=s["Q"], Q_out=s["Q_out"], **rotation)


def _attend(rb, ctx, s, Q):
    n = rb.radar_chunk_attn_workspace_bytes(ctx, s["B"], s["Hq"], s["Hkv"], s["d"], rb.dtype_code(s["O"]), s["n_hi"], s["max_len"])
    rb.radar_chunk_attention(ctx, Q=Q, q_start=s["q_start"], Kc=s["Kc"], Vc=s["Vc"], page_size=s["page"], block_table=s["block_table"], cache_len=s["cache_len"],
                             max_new=s["n_hi"], max_cache_len=s["max_len"], O=s["O"], lse=s["lse"], workspace=_workspace(n))
    return {"O": s["O"], "lse": s["lse"]}


def _run_own(s):
    rb, ctx = _context()
    kind = s["kind"]
    if kind == "rotate":
        rb.radar_rotate(ctx, Q=s["Q"], Q_out=s["Q_out"], K=s["K"], K_out=s["K_out"], pos=s["pos"], inv_freq=s["inv_freq"], pair_axis=s["pair_axis"],
                        neighbours=s["neighbours"], inverse=s["inverse"])
        return {k: s[n] for k, n in (("Q", "Q_out"), ("K", "K_out")) if s[n] is not None}
    if kind == "attend":
        return _attend(rb, ctx, s, s["Q"])
    _store(rb, ctx, s)
    if kind == "store":
        return {k: s[n] for k, n in (("Q", "Q_out"), ("K", "Kc"), ("V", "Vc")) if s[n] is not None}
    return dict(_attend(rb, ctx, s, s["Q_out"]), K=s["Kc"], V=s["Vc"])


def run(state):
    return _run_own(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def work(case):
    kind, size, Hq, Hkv, d = case["kind"], 2 if case["dtype"] == "bf16" else 4, case["Hq"], case["Hkv"], case["d"]
    if kind == "rotate":
        return {"bytes": case["rows"] * (2 * (Hq + Hkv) * d * size + 4 * case["axes"]), "flops": 3 * case["rows"] * (Hq + Hkv) * case["rot"]}
    if kind == "store":
        T = case["tokens"]
        return {"bytes": case["L"] * T * 2 * (Hq + 2 * Hkv) * d * size + T * (8 + 4 * case["axes"] + 4 * case["tree"]), "flops": 3 * case["L"] * T * (Hq + Hkv) * case["rot"]}
    n = _spread(case["B"], case["n_lo"], case["n_hi"])
    lens = n if kind == "admit" else np.maximum(_spread(case["B"], case["P_lo"], case["P_hi"])[::-1], n)
    T, seen = int(n.sum()), int((n * (lens - n) + n * (n + 1) // 2).sum())
    out = {"bytes": T * (2 * Hq * d * size + 4 * Hq) + int(lens.sum()) * 2 * Hkv * d * size + 4 * int((-(-lens // case["page"])).sum()), "flops": 4 * Hq * d * seen}
    if kind == "admit":                                    # the rows as they come, the cache written and the attention's own bytes but Q
        out["bytes"] += T * (2 * Hkv * d * size + 8 + 4 * case["axes"])
        out["flops"] += 3 * T * (Hq + Hkv) * case["rot"]
    return out


# ---- from the definition, in 64 bits ----------------------------------------------------------------------------------
def _exact_turned(s, x):
    """Each pair as a complex number times e^(i angle), float64."""
    P = s["rot"] // 2
    y = x.double().clone()
    if not P:
        return y
    first, step = (range(0, 2 * P, 2), 1) if s["neighbours"] else (range(P), P)
    first = torch.tensor(list(first), device="cuda")
    axis = s["pair_axis"].tolist() if s["pair_axis"] is not None else [0] * P
    angle = torch.stack([s["pos"][axis[p]].double() * float(s["inv_freq"][p]) for p in range(P)], -1)
    turn = torch.polar(torch.ones_like(angle), -angle if s.get("inverse") else angle)[:, None]
    z = torch.complex(y[..., first], y[..., first + step]) * turn
    y[..., first], y[..., first + step] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind, dt = case["kind"], _DT[case["dtype"]]
    if kind == "rotate":
        return {k: _exact_turned(s, s[k]) for k in ("Q", "K") if s[k] is not None}
    out = {}
    Q = s["Q"]
    if kind in ("store", "admit"):
        K, V = (x if s.get("src_row") is None else x[..., s["src_row"].long(), :, :] for x in (s["K"], s["V"]))
        K, V = _exact_turned(s, K), V.double()
        Q = _exact_turned(s, Q) if Q is not None else None
        for name, rows in (("K", K), ("V", V)):
            pool = torch.zeros(s["Kc"].shape, dtype=torch.float64, device="cuda")
            kept = s["slots"] >= 0
            pool[..., s["slots"][kept], :, :] = rows[..., kept, :, :]
            out[name] = pool
        if kind == "store":
            return dict({"Q": Q} if Q is not None else {}, **out)
    Kc, Vc = (out["K"].to(dt), out["V"].to(dt)) if kind == "admit" else (s["Kc"], s["Vc"])       # what the attention reads is rounded
    Q = Q.to(dt)
    B, Hq, Hkv, d, page = s["B"], s["Hq"], s["Hkv"], s["d"], s["page"]
    O, lse = torch.zeros(s["T"], Hq, d, dtype=torch.float64, device="cuda"), torch.zeros(s["T"], Hq, dtype=torch.float64, device="cuda")
    start, lens, table = s["q_start"].tolist(), s["cache_len"].tolist(), s["block_table"].tolist()
    for b in range(B):
        rows, n, P = slice(start[b], start[b + 1]), start[b + 1] - start[b], lens[b]
        slots = torch.tensor([table[b][j // page] * page + j % page for j in range(P)], device="cuda")
        hidden = torch.arange(P, device="cuda") > torch.arange(P - n, P, device="cuda")[:, None]
        for h in range(Hq):
            k, v = (x[slots, h // (Hq // Hkv)].double() for x in (Kc, Vc))
            z = (Q[rows, h].double() @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[rows, h] = torch.logsumexp(z, -1)
            O[rows, h] = torch.softmax(z, -1) @ v
    return dict({"O": O, "lse": lse}, **out)
