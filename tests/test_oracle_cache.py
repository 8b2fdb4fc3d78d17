"""Pins of the 4-bit cache's oracle: the format's numbers by hand and by brute force, the page arithmetic by its invariants,
attention against torch; the binding's refusals, which need no GPU."""
import ctypes

import numpy as np
import pytest

from oracle import cache_oracle as C


def test_scales_and_codes_by_hand():
    x = np.zeros((3, 16))
    x[0, :4] = [7.0, -8.0, 1.5, 2.5]            # 8 / 7 rounds to 1.125 (nine eighths: 9.14 of 8)
    x[1, 0] = 1e-9                               # below the smallest scale's half step
    x[2, :2] = [3.0e4, -1.0e6]                   # beyond the largest: saturates
    q, n = C.quantise(x)
    assert C.scale(n[0, 0]) == 1.125 and q[0, :4].tolist() == [6, -7, 1, 2]
    assert n[1, 0] == 0 and not q[1].any()
    assert n[2, 0] == 255 and C.values(q, n)[2, :2].tolist() == [7 * 3840.0, -8 * 3840.0]
    assert C.scale(0) == 2.0 ** -20 and C.scale(255) == 3840.0


def test_every_number_is_its_nearest_code():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 32)) * np.exp(rng.uniform(-8, 8, (200, 1)))
    q, n = C.quantise(x)
    s = np.repeat(C.scale(n), 16, axis=1)
    every = np.arange(-8, 8)
    best = np.abs(x[..., None] - every * s[..., None]).min(-1)
    assert np.all(np.abs(x - q * s) <= best * (1 + 1e-12))
    top = np.abs(x).reshape(200, 2, 16).max(-1)
    assert np.all(np.abs(C.scale(n) - top / 7) <= top / 7 / 16 * (1 + 1e-12))       # half a unit of four significant bits


@pytest.mark.parametrize("d", [64, 128])
def test_blocks_are_a_permutation_of_their_parts(d):
    rng = np.random.default_rng(d)
    parts = [rng.integers(-8, 8, (16, d)), rng.integers(0, 256, (16, d // 16)), rng.integers(-8, 8, (16, d)), rng.integers(0, 256, (16, d // 16))]
    block = C.pack_block(*parts)
    for a, b in zip(parts, C.unpack_blocks(np.stack([block, block[::-1]]))):
        assert np.array_equal(a, b[0])


def test_pages_change_hands_and_none_is_lost():
    rng = np.random.default_rng(5)
    B, page, columns, n_pages = 9, 16, 12, 60
    table, stack, n_free = np.full((B, columns), -1), np.arange(n_pages), n_pages
    lens, short = np.zeros(B, int), 0
    for _ in range(300):
        new = np.where(rng.random(B) < 0.2, -rng.integers(0, lens + 1), np.minimum(rng.integers(0, 70, B), columns * page - lens))
        before = lens.copy()
        table, stack, n_free, lens, slots, granted = C.extend(page, lens, new, table, stack, n_free)
        short += int((~granted).sum())
        held = [table[b, i] for b in range(B) for i in range(-(-lens[b] // page))]
        assert sorted(held + list(stack[:n_free])) == list(range(n_pages))
        for b in range(B):
            assert lens[b] == before[b] + (new[b] if granted[b] else 0)
            assert slots[b] == ([table[b, p // page] * page + p % page for p in range(before[b], lens[b])] if granted[b] else [-1] * max(new[b], 0))
    assert short > 20


def test_attention_is_softmax_attention():
    import torch
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((11, 2, 8)), rng.standard_normal((11, 2, 8))
    see = rng.random((5, 11)) < 0.6
    see[3] = False
    o, lse = C.attention(q, k, v, see, 0.3)
    t = torch.nn.functional.scaled_dot_product_attention(
        *(torch.from_numpy(np.repeat(x, r, 1)).transpose(0, 1) for x, r in ((q, 1), (k, 2), (v, 2))), attn_mask=torch.from_numpy(see), scale=0.3).transpose(0, 1).numpy()
    rows = [0, 1, 2, 4]
    assert np.abs(o[rows] - t[rows]).max() < 1e-12
    assert np.all(o[3] == 0) and np.all(np.isneginf(lse[:, 3]))


def test_struct_layouts_match_the_header(tmp_path):
    import os
    import subprocess
    from paper_2512_14069_b200 import binding as rb
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"radar_cache_extend_args": rb.CacheExtendArgs, "radar_cache_store_args": rb.CacheStoreArgs, "radar_cache_load_args": rb.CacheLoadArgs,
               "radar_cache_attn_args": rb.CacheAttnArgs}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "radar.h"', "int main(void){"]
    for c, st in structs.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (c, c))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (c, f, c, f) for f, _ in st._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0;}"]))
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")])
    out = dict(l.split() for l in subprocess.check_output([str(tmp_path / "layout")], text=True).splitlines())
    for c, st in structs.items():
        assert int(out[c]) == ctypes.sizeof(st)
        for f, _ in st._fields_:
            assert int(out["%s.%s" % (c, f)]) == getattr(st, f).offset, (c, f)
