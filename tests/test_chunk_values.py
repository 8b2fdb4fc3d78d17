"""That the GPU tests of values in long caches can fail: what O would be with one page's values from elsewhere is beyond their bound."""
import numpy as np
import pytest

import paged_values as V


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(V.CASES))
def test_a_wrong_page_of_values_is_beyond_the_bound(name, dtype):
    """In the first request and in the longest one: every page's values exchanged for another page's, zeros in their place, and a key and value taken
    twice or left out."""
    requests, _ = V.make(name, dtype)
    _, _, Hq, Hkv, d, page, _ = V.CASES[name]
    G, unit = Hq // Hkv, V.grain(page)
    rng = np.random.default_rng(1)
    for q, k, v in {id(r): r for r in (requests[0], max(requests, key=lambda r: len(r[1]) * (len(r[0]) > 0)))}.values():
        n, L = len(q), len(k)
        seen = np.maximum(L - n + 1 + np.arange(n), 0)
        O, _, size, root, p = V.attention(q, k, v, seen)
        most, _ = V.bound(q, k, v, O, size, root, p, dtype)
        first = np.arange(0, max(1, (L - n) // unit * unit), unit)      # pages that all rows see
        for f in first if len(first) < 60 else rng.choice(first, 60, replace=False):
            rows = np.arange(f, min(f + unit, L - n))
            if not len(rows):
                continue
            other = rng.choice([x for x in first if x != f] or [f])
            from_there = (other + rows - f) % L
            part = p[:, :, rows]
            change = lambda values: np.stack([part[h] @ values[:, h // G] for h in range(Hq)], 1)
            wrongs = {"zeros": -v[rows], "twice": v[rows], "not zeroed": 3.0 - v[rows]}
            if other != f:
                wrongs["another page"] = v[from_there] - v[rows]
            for what, values in wrongs.items():
                assert np.any(np.abs(change(values)) > 1.5 * most), (what, f, other, float(np.max(np.abs(change(values)) / most)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(V.CASES))
def test_the_outputs_rounded_are_within_the_bound(name, dtype):
    """The operator in fp32 with its probabilities rounded as the kernels round them, and one request's O from a pool whose pages are exchanged."""
    import torch
    import paged_harness as T
    requests, start = V.make(name, dtype)
    _, _, Hq, Hkv, d, page, _ = V.CASES[name]
    G, dt = Hq // Hkv, T.DT[dtype]
    O, lse = np.zeros((start[-1], Hq, d)), np.full((start[-1], Hq), -np.inf)
    for b, (q, k, v) in enumerate(requests):
        n, L = len(q), len(k)
        hidden = torch.arange(L) > torch.arange(L - n, L)[:, None]
        for h in range(Hq if n else 0):
            z = (torch.from_numpy(q[:, h]).float() @ torch.from_numpy(k[:, h // G]).float().T * d ** -0.5).masked_fill(hidden, -float("inf"))
            top = z.amax(-1, keepdim=True)
            p = (z - top).exp()
            total = p.sum(-1, keepdim=True)
            O[start[b]:start[b + 1], h] = (p.to(dt).float() @ torch.from_numpy(v[:, h // G]).float() / total).to(dt).double().numpy()
            lse[start[b]:start[b + 1], h] = (total.log() + top)[:, 0].double().numpy()
    assert V.hold(O, lse, requests, start, dtype) < 1.0
    # the same outputs against a request whose pages of values are one place off
    b = int(np.argmax([len(k) * (len(q) > 0) for q, k, _ in requests]))
    q, k, v = requests[b]
    if len(k) >= 4 * V.grain(page):
        assert V.hold(O, lse, [(q, k, np.roll(v, V.grain(page), 0)) if i == b else r for i, r in enumerate(requests)], start, dtype) > 1.0
