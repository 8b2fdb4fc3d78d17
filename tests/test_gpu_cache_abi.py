"""The 4-bit cache's four calls through the C ABI itself, with argument structs filled field by field: what the Python calls give, and
the refusals that those never reach."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_14069_b200 import binding as rb
    c = rb.Context(0)
    yield c
    c.close()


def _fill(struct, **kw):
    a = struct()
    for k, v in kw.items():
        assert any(k == f for f, _ in struct._fields_), k
        setattr(a, k, v.data_ptr() if hasattr(v, "data_ptr") else v)
    return a


def _call(ctx, name, a):
    import torch
    from paper_2512_14069_b200 import binding as rb
    return getattr(rb.lib(), "radar_cache_" + name)(ctx.handle, ctypes.byref(a), torch.cuda.current_stream().cuda_stream)


def _inputs(seed, L=2, B=3, Hq=8, Hkv=2, d=64, page=16, rows=9):
    import torch
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    i32, n_pages = torch.int32, 30
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    s = dict(L=L, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, rows=rows, n_pages=n_pages, T=70)
    s.update(cache_len=T.dev([0] * B, i32), new_len=T.dev([40, 13, 17], i32), table=torch.full((B, 6), -1, dtype=i32, device="cuda"), stack=T.dev(np.arange(n_pages), i32),
             count=T.dev([n_pages], i32), granted=torch.zeros(B, dtype=torch.uint8, device="cuda"), start=T.dev([0] * (B + 1), i32),
             slots=torch.zeros(70, dtype=torch.int64, device="cuda"), pages=torch.zeros(L, n_pages, rb.radar_cache_page_bytes(Hkv, d, page), dtype=torch.uint8, device="cuda"),
             K=rand(L, 70, Hkv, d), V=rand(L, 70, Hkv, d), K_out=torch.zeros(L, 70, Hkv, d, device="cuda"), V_out=torch.zeros(L, 70, Hkv, d, device="cuda"),
             first=T.dev([0] * B, i32), Q=rand(B, rows, Hq, d), Kt=rand(B, rows, Hkv, d), Vt=rand(B, rows, Hkv, d), O=torch.zeros(B, rows, Hq, d, dtype=torch.bfloat16, device="cuda"),
             lse=torch.zeros(B, Hq, rows, device="cuda"))
    return s


def _structs(ctx, s):
    """The four calls' structs over the inputs."""
    import cache_harness as T
    from paper_2512_14069_b200 import binding as rb
    row = s["Hkv"] * s["d"]
    layer_bytes = s["pages"][0].numel()
    s["ws"] = T.workspace(rb.radar_cache_attn_workspace_bytes(ctx, s["B"], s["Hq"], s["Hkv"], s["d"], s["rows"], 96))
    return dict(
        extend=_fill(rb.CacheExtendArgs, B=s["B"], page_size=s["page"], max_pages=6, cache_len=s["cache_len"], new_len=s["new_len"], block_table=s["table"], free_pages=s["stack"],
                     free_count=s["count"], free_capacity=s["n_pages"], cache_len_out=s["cache_len"], free_count_out=s["count"], granted=s["granted"], start=s["start"], slots=s["slots"],
                     slot_capacity=s["T"]),
        store=_fill(rb.CacheStoreArgs, n_layers=s["L"], Hkv=s["Hkv"], d=s["d"], page_size=s["page"], dtype=rb.RADAR_BF16, n_tokens=s["T"], n_rows=s["T"], n_pages=s["n_pages"], K=s["K"],
                    V=s["V"], row_stride=row, row_layer_stride=s["T"] * row, slots=s["slots"], pages=s["pages"], page_layer_stride=layer_bytes),
        load=_fill(rb.CacheLoadArgs, n_layers=s["L"], B=s["B"], Hkv=s["Hkv"], d=s["d"], page_size=s["page"], max_pages=6, dtype=rb.RADAR_F32, n_rows=s["T"], n_pages=s["n_pages"],
                   pages=s["pages"], page_layer_stride=layer_bytes, block_table=s["table"], first=s["first"], start=s["start"], K=s["K_out"], V=s["V_out"], row_layer_stride=s["T"] * row),
        attention=_fill(rb.CacheAttnArgs, B=s["B"], Hq=s["Hq"], Hkv=s["Hkv"], d=s["d"], rows=s["rows"], dtype=rb.RADAR_BF16, Q=s["Q"], Kt=s["Kt"], Vt=s["Vt"],
                        q_row_stride=s["Hq"] * s["d"], kv_row_stride=row, pages=s["pages"], n_pages=s["n_pages"], page_size=s["page"], max_pages=6, block_table=s["table"],
                        cache_len=s["cache_len"], max_cache_len=96, O=s["O"], lse=s["lse"], workspace=s["ws"], workspace_bytes=s["ws"].numel()))


def test_structs_and_python_calls_agree(ctx):
    import torch
    from paper_2512_14069_b200 import binding as rb
    a, b = _inputs(1), _inputs(1)
    args = _structs(ctx, a)
    _structs(ctx, b)
    for name in ("extend", "store", "load", "attention"):
        assert _call(ctx, name, args[name]) == rb.RADAR_OK, name
    rb.radar_cache_extend(ctx, page_size=b["page"], cache_len=b["cache_len"], new_len=b["new_len"], block_table=b["table"], free_pages=b["stack"], free_count=b["count"],
                          slots=b["slots"], start=b["start"], granted=b["granted"])
    rb.radar_cache_store(ctx, K=b["K"], V=b["V"], slots=b["slots"], pages=b["pages"], page_size=b["page"])
    rb.radar_cache_load(ctx, pages=b["pages"], page_size=b["page"], block_table=b["table"], first=b["first"], start=b["start"], K=b["K_out"], V=b["V_out"])
    rb.radar_cache_attention(ctx, Q=b["Q"], Kt=b["Kt"], Vt=b["Vt"], pages=b["pages"][0], page_size=b["page"], block_table=b["table"], cache_len=b["cache_len"], max_cache_len=96,
                             O=b["O"], lse=b["lse"], workspace=b["ws"])
    ctx.check_device_status()
    assert a["cache_len"].tolist() == [40, 13, 17] and int(a["count"]) == 24
    for k in ("cache_len", "table", "count", "granted", "start", "slots", "pages", "K_out", "V_out", "O", "lse"):
        assert torch.equal(a[k], b[k]), k
    assert float(a["O"].float().abs().max()) > 0 and float(a["K_out"].abs().max()) > 0


def test_refusals_of_the_library(ctx):
    """Nothing is launched: null pointers, sizes that are none or not supported, rows and workspaces that are not aligned."""
    from paper_2512_14069_b200 import binding as rb
    s = _inputs(2)
    args = _structs(ctx, s)
    invalid, unsupported, workspace = -1, -2, -3
    bad = dict(
        extend=[(f, 0, invalid) for f in ("B", "max_pages", "free_capacity", "cache_len", "new_len", "block_table", "free_pages", "free_count", "cache_len_out", "free_count_out",
                                          "granted", "start", "slots")] +
               [("page_size", 24, invalid), ("slot_capacity", -1, invalid), ("path_nodes", s["start"].data_ptr(), invalid), ("B", 8193, unsupported)],
        store=[(f, 0, invalid) for f in ("n_layers", "Hkv", "K", "V", "slots", "pages", "row_stride", "row_layer_stride", "page_layer_stride")] +
              [("page_size", 48, invalid), ("n_tokens", -1, invalid), ("n_rows", -1, invalid), ("d", 96, unsupported), ("dtype", 7, unsupported), ("n_layers", 65536, unsupported),
               ("K", s["K"].data_ptr() + 2, invalid), ("pages", s["pages"].data_ptr() + 8, invalid), ("row_stride", s["Hkv"] * s["d"] + 4, invalid)],
        load=[(f, 0, invalid) for f in ("n_layers", "B", "Hkv", "max_pages", "K", "V", "pages", "block_table", "first", "start", "row_layer_stride", "page_layer_stride")] +
             [("page_size", 0, invalid), ("d", 32, unsupported), ("dtype", 9, unsupported), ("V", s["V_out"].data_ptr() + 4, invalid)],
        attention=[(f, 0, invalid) for f in ("B", "Hq", "Hkv", "rows", "Q", "Kt", "Vt", "O", "pages", "n_pages", "block_table", "cache_len", "workspace", "max_pages")] +
                  [("rows", 65, invalid), ("Hkv", 3, invalid), ("d", 80, unsupported), ("dtype", rb.RADAR_F32, unsupported), ("max_cache_len", -1, invalid), ("max_cache_len", 97, invalid),
                   ("page_size", 20, invalid), ("q_row_stride", 8 * 64 - 8, invalid), ("kv_row_stride", 2 * 64 + 4, invalid), ("Q", s["Q"].data_ptr() + 2, invalid),
                   ("workspace", s["ws"].data_ptr() + 128, workspace), ("workspace_bytes", 1024, workspace)])
    for name, changes in bad.items():
        for field, value, status in changes:
            a = type(args[name]).from_buffer_copy(args[name])
            setattr(a, field, value)
            assert _call(ctx, name, a) == status, (name, field, value)
    for name in args:
        assert getattr(rb.lib(), "radar_cache_" + name)(ctx.handle, None, None) == invalid
        assert getattr(rb.lib(), "radar_cache_" + name)(None, ctypes.byref(args[name]), None) == invalid
    ctx.check_device_status()
    assert float(s["O"].float().abs().max()) == 0.0 and s["cache_len"].tolist() == [0, 0, 0]


def test_lengths_that_an_int_cannot_look_ahead_of_are_refused(ctx):
    """A bound near 2^31 (a table of many pages that share one): lookups run ahead of the keys, beyond what an int counts."""
    from paper_2512_14069_b200 import binding as rb
    a = _structs(ctx, _inputs(3))["attention"]
    a.max_pages = 2 ** 31 // 16
    for bound in (2 ** 31 - 1, 2 ** 31 - 2 ** 14):
        a.max_cache_len = bound
        assert _call(ctx, "attention", a) == -1
    ctx.check_device_status()
