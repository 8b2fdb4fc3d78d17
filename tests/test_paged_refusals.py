"""The refusals of radar_rotate, radar_paged_store and radar_chunk_attention, without a GPU: they come before anything of the context or of the
arguments' memory is touched, so that a context of zeros and addresses that lead nowhere will do."""
import ctypes
import os
import subprocess

import pytest

from paper_2512_14069_b200 import binding as rb

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
AT = 1 << 20                                             # an aligned address


@pytest.fixture(scope="module")
def ctx():
    return ctypes.create_string_buffer(1 << 16)          # (sm_count 0, no status word)


def _call(ctx, name, a):
    return getattr(rb.lib(), name)(ctypes.cast(ctx, ctypes.c_void_p), ctypes.byref(a), None)


def _set(a, changes):
    for k, v in changes.items():
        o, f = (a.rotation, k[2:]) if k.startswith("r.") else (a, k)
        assert any(f == x for x, _ in o._fields_), k
        setattr(o, f, v)
    return a


def _rotate():
    return _set(rb.RotateArgs(), dict(Hq=4, Hkv=2, d=64, dtype=rb.RADAR_BF16, n_rows=10, Q=AT, K=2 * AT, q_row_stride=256, k_row_stride=128, Q_out=3 * AT, K_out=4 * AT,
                                      q_out_row_stride=256, k_out_row_stride=128, **{"r.pos": AT, "r.pos_stride": 10, "r.n_axes": 2, "r.n_pairs": 32, "r.inv_freq": AT}))


@pytest.mark.parametrize("changes,status", [
    (dict(n_rows=0), OK), (dict(n_rows=-1), INVALID), (dict(n_rows=1 << 31), UNSUPPORTED), (dict(Hq=-1), INVALID), (dict(Hq=0, Hkv=0), INVALID), (dict(d=0), INVALID),
    (dict(d=1026, q_row_stride=1 << 14, k_row_stride=1 << 14, q_out_row_stride=1 << 14, k_out_row_stride=1 << 14), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(Q=None), INVALID), (dict(K_out=None), INVALID), (dict(q_row_stride=255), INVALID), (dict(k_out_row_stride=127), INVALID), (dict(Q=AT + 1), INVALID),
    (dict(Q_out=AT, q_out_row_stride=512), INVALID), ({"r.pos": None}, INVALID), ({"r.inv_freq": None}, INVALID), ({"r.n_axes": 0}, INVALID), ({"r.n_pairs": 0}, INVALID),
    ({"r.n_pairs": 33}, INVALID), ({"r.pos_stride": 9}, INVALID)])
def test_rotate(ctx, changes, status):
    assert _call(ctx, "radar_rotate", _set(_rotate(), changes)) == status
    assert rb.lib().radar_rotate(None, ctypes.byref(_rotate()), None) == INVALID and rb.lib().radar_rotate(ctypes.cast(ctx, ctypes.c_void_p), None, None) == INVALID


def _store():
    return _set(rb.PagedStoreArgs(), dict(n_layers=2, Hq=4, Hkv=2, d=64, dtype=rb.RADAR_F32, n_tokens=8, n_rows=10, cache_rows=64, Q=AT, K=2 * AT, V=3 * AT, q_row_stride=256,
                                          kv_row_stride=128, q_layer_stride=2560, kv_layer_stride=1280, slots=AT, Q_out=4 * AT, q_out_row_stride=256, q_out_layer_stride=2048,
                                          Kc=5 * AT, Vc=6 * AT, cache_layer_stride=64 * 128))


@pytest.mark.parametrize("changes,status", [
    (dict(n_tokens=0), OK), (dict(n_tokens=-1), INVALID), (dict(n_tokens=11), INVALID), (dict(n_tokens=1 << 31, src_row=AT), UNSUPPORTED), (dict(n_layers=0), INVALID),
    (dict(n_layers=65536), UNSUPPORTED), (dict(Hkv=0), INVALID), (dict(Hq=-1), INVALID), (dict(d=0), INVALID), (dict(d=2000), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
    (dict(cache_rows=-1), INVALID), (dict(K=None), INVALID), (dict(V=None), INVALID), (dict(Kc=None), INVALID), (dict(Vc=None), INVALID), (dict(slots=None), INVALID),
    (dict(kv_row_stride=127), INVALID), (dict(kv_layer_stride=0), INVALID), (dict(cache_layer_stride=64 * 128 - 1), INVALID), (dict(K=AT + 2), INVALID), (dict(Vc=AT + 2), INVALID),
    (dict(Q=None), INVALID), (dict(Q_out=None), INVALID), (dict(q_row_stride=255), INVALID), (dict(q_out_row_stride=255), INVALID), (dict(q_layer_stride=0), INVALID),
    (dict(q_out_layer_stride=0), INVALID), (dict(Q_out=AT, src_row=AT), INVALID), (dict(Q_out=AT, q_out_row_stride=512), INVALID), (dict(Q_out=AT), INVALID),
    ({"r.pos": AT}, INVALID), ({"r.pos": AT, "r.inv_freq": AT, "r.n_axes": 1, "r.n_pairs": 33}, INVALID), ({"r.pos": AT, "r.inv_freq": AT, "r.n_axes": 3, "r.n_pairs": 8, "r.pos_stride": 7}, INVALID)])
def test_store(ctx, changes, status):
    assert _call(ctx, "radar_paged_store", _set(_store(), changes)) == status
    assert rb.lib().radar_paged_store(None, ctypes.byref(_store()), None) == INVALID


def _attend():
    return _set(rb.ChunkAttnArgs(), dict(B=3, Hq=8, Hkv=2, d=64, dtype=rb.RADAR_BF16, n_rows=20, Q=AT, q_row_stride=512, q_start=AT, Kc=AT, Vc=AT, cache_rows=640, page_size=16,
                                         max_pages=10, block_table=AT, cache_len=AT, max_new=20, max_cache_len=160, O=AT, workspace=AT, workspace_bytes=1 << 30))


@pytest.mark.parametrize("changes,status", [
    (dict(n_rows=0), OK), (dict(max_new=0), OK), (dict(B=0), INVALID), (dict(B=65536), UNSUPPORTED), (dict(Hq=7), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID),
    (dict(Hq=258, q_row_stride=1 << 15), UNSUPPORTED), (dict(d=32), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(n_rows=-1), INVALID),
    (dict(n_rows=1 << 31), UNSUPPORTED), (dict(cache_rows=1 << 31), UNSUPPORTED), (dict(cache_rows=0), INVALID), (dict(max_new=-1), INVALID), (dict(max_cache_len=-1), INVALID),
    (dict(max_cache_len=161), INVALID), (dict(max_cache_len=(1 << 31) - (1 << 14), page_size=1 << 30), UNSUPPORTED), (dict(page_size=8), INVALID), (dict(page_size=48), INVALID),
    (dict(page_size=0), INVALID), (dict(page_size=-16), INVALID), (dict(max_pages=-1), INVALID), (dict(Q=None), INVALID), (dict(q_start=None), INVALID), (dict(Kc=None), INVALID),
    (dict(Vc=None), INVALID), (dict(block_table=None), INVALID), (dict(cache_len=None), INVALID), (dict(O=None), INVALID), (dict(q_row_stride=511), INVALID), (dict(q_row_stride=516), INVALID),
    (dict(Q=AT + 8), INVALID), (dict(Kc=AT + 8), INVALID), (dict(O=AT + 4), INVALID), (dict(workspace=None), WORKSPACE), (dict(workspace=AT + 16), WORKSPACE),
    (dict(dtype=rb.RADAR_F32, q_row_stride=514), INVALID)])
def test_attention(ctx, changes, status):
    assert _call(ctx, "radar_chunk_attention", _set(_attend(), changes)) == status
    assert rb.lib().radar_chunk_attention(None, ctypes.byref(_attend()), None) == INVALID


def test_workspace_sizes(ctx):
    size = lambda *a: rb.lib().radar_chunk_attn_workspace_bytes(ctypes.cast(ctx, ctypes.c_void_p), *a)
    for bad in ((0, 8, 2, 64, 1, 1, 1), (1, 7, 2, 64, 1, 1, 1), (1, 8, 2, 96, 1, 1, 1), (1, 8, 2, 64, 2, 1, 1), (1, 8, 2, 64, 1, -1, 1), (1, 8, 2, 64, 1, 1, -1)):
        assert size(*bad) == 0
    assert rb.lib().radar_chunk_attn_workspace_bytes(None, 1, 8, 2, 64, 1, 1, 1) == 0


def test_structs_have_the_headers_layout(tmp_path):
    structs = {"radar_rotation": rb.Rotation, "radar_rotate_args": rb.RotateArgs, "radar_paged_store_args": rb.PagedStoreArgs, "radar_chunk_attn_args": rb.ChunkAttnArgs}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "radar.h"', "int main(void){"]
    for c, st in structs.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (c, c))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (c, f, c, f) for f, _ in st._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0;}"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")])
    out = dict(l.split() for l in subprocess.check_output([str(tmp_path / "layout")], text=True).splitlines())
    for c, st in structs.items():
        assert int(out[c]) == ctypes.sizeof(st), c
        for f, _ in st._fields_:
            assert int(out["%s.%s" % (c, f)]) == getattr(st, f).offset, (c, f)
