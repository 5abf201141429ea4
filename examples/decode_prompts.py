"""Decode S prompts with N lattice codes each through a small random transformer, all on the library's calls.

Per step and lane: pages for one more token (as_pages_grow), keys and values into the 4-bit cache (as_cache4_append),
attention over it, the prompt's pages read once for its N lanes (as_cache4_attend), logit edits (as_logits_edit), the
decode step (as_step).  The prompts are stored and attended as chunks; as_pages_fork hands each to its N lanes, and later
drops lanes that have ended; as_pages_compact packs the pool when it has holes.

    python examples/decode_prompts.py [--prompts 4] [--codes 8] [--steps 40]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2210_15458_b200 import binding as B  # noqa: E402

EOS = 0


class TinyLM:
    """Random weights; `layers` of attention with a residual, query heads that share key heads."""

    def __init__(self, V=600, layers=2, q_heads=8, heads=2, D=64, dtype=torch.float32, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.V, self.layers, self.Hq, self.H, self.D, self.dtype = V, layers, q_heads, heads, D, dtype
        w = q_heads * D
        r = lambda *s: (torch.randn(*s, generator=g) / math.sqrt(s[0])).to(device=device, dtype=dtype)
        self.emb = torch.randn(V, w, generator=g).to(device=device, dtype=dtype)
        self.qkv = [r(w, (q_heads + 2 * heads) * D) for _ in range(layers)]
        self.out = [r(w, w) for _ in range(layers)]
        self.head = r(w, V) * 2.0

    def forward(self, tokens, pools, table, length, N=1, shared=None):
        """Logits [lanes, V] of the last of tokens [lanes, T]; stores their keys and values (pages are there already)."""
        lanes, T = tokens.shape
        x = self.emb[tokens.long()]
        for i in range(self.layers):
            qkv = (x @ self.qkv[i]).view(lanes, T, self.Hq + 2 * self.H, self.D)
            q, k, v = qkv[:, :, :self.Hq], qkv[:, :, self.Hq:self.Hq + self.H], qkv[:, :, self.Hq + self.H:]
            B.as_cache4_append(pools[i], k, v, table, length)
            o = B.as_cache4_attend(pools[i], q, table, length, 1 / math.sqrt(self.D), N=N, shared=shared)
            x = x + o.view(lanes, T, -1) @ self.out[i]
        return x[:, -1] @ self.head


def i32(v, device="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=device)


def decode(lm, prompts, N, u, steps, page_size=16, n_pages=2000, temp=1.0, top_p=0.95, repetition=1.2, presence=0.1, frequency=0.1,
           mask=None, keep_logits=False):
    """(sequences as lists, pool state) for `prompts` (lists of tokens), N codes each with shift u.  mask: int32
    [2, ceil(V / 32)]: the tokens allowed after an even and after an odd token (a grammar of two states), or None."""
    S, lanes = len(prompts), len(prompts) * N
    T = max(len(p) for p in prompts)
    M = -(-(T + steps + 1) // page_size) + 1
    pools = B.cache4_pages(n_pages, lm.H, lm.D, page_size, planes=lm.layers)
    table, length = torch.full((S, M), -1, dtype=torch.int32, device="cuda"), i32([0] * S)
    ref = i32([0] * n_pages)
    # the prompts, padded at their front, all but the last token of each
    B.as_pages_grow(i32([len(p) - 1 for p in prompts]), table, length, ref, page_size)
    body = i32([[EOS] * (T - len(p)) + p[:-1] for p in prompts])
    if T > 1:
        lm.forward(body, pools, table, length)
    # hand each to its codes
    table, length, ref = B.as_pages_fork(i32([s for s in range(S) for _ in range(N)]), table, length, ref, page_size, pools)
    shared = i32([(len(p) - 1) // page_size * page_size for p in prompts])
    codes = B.as_lattice_codes(N, u).repeat(S)
    seq = torch.zeros(lanes, T + steps, dtype=torch.int32, device="cuda")       # prompt, then what is decoded
    for s, p in enumerate(prompts):
        seq[s * N:(s + 1) * N, :len(p)] = i32(p)
    plen = i32([len(p) for p in prompts for _ in range(N)])
    n = plen.clone()
    prev = i32([p[-1] for p in prompts for _ in range(N)])
    alive = torch.ones(lanes, dtype=torch.bool, device="cuda")
    rows = torch.arange(lanes, device="cuda")
    kept = []
    for step in range(steps):
        B.as_pages_grow(alive.int(), table, length, ref, page_size)
        logits = lm.forward(prev.view(-1, 1), pools, table, length, N, shared)
        if keep_logits:
            kept.append((logits.clone(), alive.clone()))
        state = None if mask is None else prev % 2
        B.as_logits_edit(logits, seq, n, plen, repetition, presence, frequency, mask=mask, mask_row=state, out=logits)
        tok, codes = B.as_step(logits, codes, temp, 0, top_p)
        seq[rows, n.long()] = torch.where(alive, tok, seq[rows, n.long()])
        n += alive.int()
        prev = torch.where(alive, tok, prev)
        ended = alive & (tok == EOS)
        alive &= tok != EOS
        if bool(ended.any()):
            # lanes that have ended give their pages back; the pool is packed now and then
            keep = torch.where(alive, rows, -1).int()
            table, length, ref = B.as_pages_fork(keep, table, length, ref, page_size, ref_out=ref)
            shared = (length.view(S, N).amin(1) >= shared).int() * shared       # (a group with an ended lane reads lane by lane)
            if step % 8 == 7:
                B.as_pages_compact(table, ref, pools)
        if not bool(alive.any()):
            break
    ends = n.tolist()
    out = [seq[i, :ends[i]].tolist() for i in range(lanes)]
    return out, dict(pools=pools, table=table, length=length, ref=ref, logits=kept)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--prompts", type=int, default=4)
    ap.add_argument("--codes", type=int, default=8)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    g = torch.Generator().manual_seed(1)
    lm = TinyLM(dtype=torch.bfloat16)
    prompts = [torch.randint(1, lm.V, (20 + 13 * s,), generator=g).tolist() for s in range(a.prompts)]
    seqs, state = decode(lm, prompts, a.codes, 0.37, a.steps)
    for s in range(a.prompts):
        print("prompt %d (%d tokens):" % (s, len(prompts[s])))
        for j in range(a.codes):
            print("  code %d: %s" % (j, seqs[s * a.codes + j][len(prompts[s]):]))
    print("pages held: %d" % int((state["ref"] > 0).sum()))


if __name__ == "__main__":
    main()
