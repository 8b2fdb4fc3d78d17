"""Speculative decoding of a small model over a paged cache, from admission to release.

A random-weight transformer decodes for a batch of requests: a bigram table is the draft model, a step's tree is verified in one
pass whose attention reads the cache, and what was accepted is appended to it.  Requests that reach their length give their
pages back, and prompts that wait take their places.  Between steps the host reads only the tokens.

    python examples/decode_with_cache.py            # the 4-bit cache; learned positions, a prompt attends by itself
    python examples/decode_with_cache.py --paged    # the bf16 cache; rotary positions, a prompt comes in chunks and attends over the cache
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_14069_b200 import binding as rb  # noqa: E402
from paper_2512_14069_b200 import workloads as W  # noqa: E402
from paper_2512_14069_b200.cache import FourBitCache, PagedCache  # noqa: E402
from paper_2512_14069_b200.pipeline import SpecStep  # noqa: E402

ROWS = rb.RADAR_MAX_NODES


class Model:
    """Decoder layers of fused projection, attention and output projection; positions are learned, or (inv_freq) turn queries and keys."""

    def __init__(self, *, layers, Hq, Hkv, d, V, max_len, seed=0, rotary=False):
        g = torch.Generator().manual_seed(seed)
        w = lambda *shape: (torch.randn(*shape, generator=g) * shape[-1] ** -0.5).bfloat16().cuda()
        self.layers, self.Hq, self.Hkv, self.d, self.V, D = layers, Hq, Hkv, d, V, Hq * d
        self.E, self.pos, self.draft = w(V, D) * D ** 0.5, w(max_len, D) * D ** 0.5, w(V, V) * V ** 0.5
        self.inv_freq = 10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d) if rotary else None
        self.qkv, self.out = [w((Hq + 2 * Hkv) * d, D) for _ in range(layers)], [w(D, D) for _ in range(layers)]

    def split(self, qkv):
        a, b = self.Hq, self.Hq + self.Hkv
        return qkv[..., :a, :], qkv[..., a:b, :], qkv[..., b:, :]

    def forward(self, tokens, positions, attend):
        """Logits of tokens [B, rows]; attend(layer, Q, K, V) gives that layer's attention output [B, rows, Hq, d]."""
        x = (self.E[tokens] if self.inv_freq is not None else self.E[tokens] + self.pos[positions]).float()
        for i in range(self.layers):
            h = torch.nn.functional.normalize(x, dim=-1).mul(x.shape[-1] ** 0.5).bfloat16()
            o = attend(i, *self.split((h @ self.qkv[i].T).unflatten(-1, (-1, self.d))))
            x = x + (o.flatten(-2) @ self.out[i].T).float()
        return torch.nn.functional.normalize(x, dim=-1).bfloat16().float() @ self.E.T.float()


class Decoder:
    def __init__(self, ctx, model, *, B, k=4, t_max=4, N=16, page_size=16, n_pages=64, max_len=256, max_prompt=64, chunk=24):
        self.ctx, self.model, self.B, self.k, self.t_max = ctx, model, B, k, t_max
        m = model
        self.step = SpecStep(ctx, B=B, V=m.V, k=k, t_max=t_max, N=N, Hq=m.Hq, Hkv=m.Hkv, d=m.d, kv_dtype=torch.bfloat16, max_prefix_len=max_len)
        self.paged, self.chunk = model.inv_freq is not None, chunk
        self.cache = (PagedCache if self.paged else FourBitCache)(ctx, n_layers=m.layers, B=B, Hq=m.Hq, Hkv=m.Hkv, d=m.d, page_size=page_size, n_pages=n_pages, max_len=max_len,
                                  max_new=max(B * (t_max + 1), max_prompt))
        self.gate = {n: torch.from_numpy(v).cuda() for n, v in W.gate_weights(W.shrink(W.CONFIGS[1], k=k)).items()}
        self.draft_logits = torch.zeros(B, self.step.R, m.V, device="cuda")
        self.K = torch.zeros(m.layers, B, ROWS, m.Hkv, m.d, dtype=torch.bfloat16, device="cuda")
        self.V = torch.zeros_like(self.K)
        self.root = torch.zeros(B, dtype=torch.int32, device="cuda")

    def admit(self, b, prompt):
        """A prompt for request b, which must be empty.  Its last token becomes the root of the first step.  False: there are no pages
        for it."""
        if self.paged:
            return self.admit_chunks(b, prompt)
        m, n = self.model, len(prompt) - 1
        tokens = torch.tensor(prompt, device="cuda")
        K = torch.empty(m.layers, n, m.Hkv, m.d, dtype=torch.bfloat16, device="cuda")
        V = torch.empty_like(K)

        def attend(layer, Q, Kt, Vt):                    # the prompt by itself: rows attend to those before them
            K[layer], V[layer] = Kt[0], Vt[0]
            heads = lambda x: x[0].repeat_interleave(m.Hq // x.shape[2], 1).transpose(0, 1).float()
            s = heads(Q) @ heads(Kt).transpose(1, 2) * m.d ** -0.5
            s = s.masked_fill(torch.ones(n, n, device="cuda", dtype=torch.bool).triu(1), float("-inf"))
            return (s.softmax(-1) @ heads(Vt)).transpose(0, 1)[None].bfloat16()
        m.forward(tokens[None, :n], torch.arange(n, device="cuda")[None], attend)
        which = torch.arange(self.B, device="cuda") == b
        self.cache.admit(torch.where(which, n, 0).to(torch.int32), K, V, requests=which)
        self.root[b] = int(prompt[-1])
        return bool(self.cache.granted[b])

    def admit_chunks(self, b, prompt):
        """The prompt in chunks: a layer's rows are stored, their keys turned on the way, and attend to all that is there."""
        m, c = self.model, self.cache
        which = torch.arange(self.B, device="cuda") == b
        tokens = torch.tensor(prompt, device="cuda")
        for first in range(0, max(len(prompt) - 1, 1), self.chunk):
            n = min(self.chunk, len(prompt) - 1 - first)
            c.begin(torch.where(which, n, 0).to(torch.int32), n, requests=which)
            if not c.granted[b]:                         # what is there goes back
                c.release(which)
                return False
            if n == 0:
                break

            def attend(layer, Q, K, V):
                turned, O = Q[0].contiguous(), torch.empty_like(Q[0])
                c.store(layer, K[0], V[0], Q=turned, Q_out=turned, inv_freq=m.inv_freq)
                c.attention(layer, turned, O)
                return O[None]
            m.forward(tokens[None, first:first + n], c.pos[None, :n].long(), attend)
        self.root[b] = int(prompt[-1])
        return True

    def draft(self):
        """The draft calls of a step: rows of the bigram table for the root, then for each call's frontier."""
        s, k = self.step, self.k
        self.draft_logits[:, 0] = self.model.draft[self.root.long()].float()
        for t in range(1, self.t_max + 1):
            if t > 1:
                self.draft_logits[:, 1 + (t - 2) * k:1 + (t - 1) * k] = self.model.draft[s.frontier_tok[t - 2].long()].float()
            s.expand(t, self.draft_logits, self.gate)

    def verify(self, check=None):
        """The target's pass over the tree.  check(layer, Q, Kt, Vt) sees each layer's inputs behind its attention."""
        s, c = self.step, self.cache

        def attend(layer, Q, Kt, Vt):
            if self.paged:
                Q, Kt, Vt = Q.contiguous(), Kt.contiguous(), Vt.contiguous()
                rb.radar_rotate(self.ctx, Q=Q.flatten(0, 1), Q_out=Q.flatten(0, 1), K=Kt.flatten(0, 1), K_out=Kt.flatten(0, 1), pos=s.tree_pos.flatten(),
                                inv_freq=self.model.inv_freq)
                s.attention_paged(c, layer, Q, Kt, Vt)
            else:
                s.attention_cached(c, layer, Q, Kt, Vt)
            self.K[layer], self.V[layer] = Kt, Vt
            if check is not None:
                check(layer, Q, Kt, Vt)
            return torch.where(live[:, :, None, None], s.O, 0)       # (rows that hold no node are left as they were)
        live = torch.arange(ROWS, device="cuda") < s.n_nodes[:, None]
        tokens, positions = (torch.where(live, x, 0).long() for x in (s.tree_tok, s.tree_pos))
        return self.model.forward(tokens, positions, attend)

    def decode_step(self, check=None):
        """One step of all requests; the tokens that it emitted, by request.  A request that the pool has no page for emits none and keeps
        its root: the same step again when there are pages."""
        s, c = self.step, self.cache
        self.draft()
        s.build_tree(self.root, c.cache_len)
        s.accept(self.verify(check), self.draft_logits)
        c.append(s, self.K, self.V)
        took = c.live & (c.granted != 0)
        self.root.copy_(torch.where(took, s.next_token, self.root))
        took, lens, path, nxt = took.tolist(), s.accept_len.tolist(), s.path_tokens.tolist(), s.next_token.tolist()
        return [path[b][1:1 + lens[b]] + [nxt[b]] if took[b] else [] for b in range(self.B)]


def main(requests=6, B=3, tokens=24, seed=1, n_pages=64, paged=False):
    torch.manual_seed(seed)
    ctx = rb.Context(0)
    model = Model(layers=2, Hq=8, Hkv=2, d=64, V=512, max_len=256, rotary=paged)
    dec = Decoder(ctx, model, B=B, n_pages=n_pages)
    prompts = [torch.randint(0, model.V, (int(n),)).tolist() for n in torch.randint(5, 60, (requests,))]
    waiting, text = list(range(requests)), [[] for _ in range(requests)]
    slot, admitted, starved, steps = [None] * B, [], False, 0            # requests in the batch's rows; rows in the order of their admission
    while waiting or admitted:
        for b in range(B):
            if slot[b] is None and waiting and not (starved and admitted):     # (pages go to those that run before new ones come in)
                if not dec.admit(b, prompts[waiting[0]] + text[waiting[0]]):
                    break
                slot[b] = waiting.pop(0)
                admitted.append(b)
        if not admitted:
            raise RuntimeError("too few pages for a prompt")
        new, steps = dec.decode_step(), steps + 1
        starved = not all(new[b] for b in admitted)
        done = torch.zeros(B, dtype=torch.uint8)
        for b in list(admitted):
            text[slot[b]] += new[b]
            if len(text[slot[b]]) >= tokens:
                done[b] = 1
        if not any(new[b] for b in admitted):                            # nobody goes on: the last one makes room, and waits
            if len(admitted) == 1:
                raise RuntimeError("too few pages for a request")
            done[admitted[-1]] = 1
            waiting.insert(0, slot[admitted[-1]])
        for b in range(B):
            if done[b]:
                admitted.remove(b)
                slot[b] = None
        dec.cache.release(done.cuda())
        ctx.check_device_status()
    for i in range(requests):
        print(i, *text[i][:tokens])
    print(f"{sum(map(len, text))} tokens in {steps} steps, {int(dec.cache.free_count)} of {dec.cache.free_pages.numel()} pages free")
    return dict(enumerate(text)), dec


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description="speculative decoding over a paged cache")
    parser.add_argument("--paged", action="store_true", help="the bf16 cache, rotary positions, prompts in chunks")
    main(paged=parser.parse_args().paged)
