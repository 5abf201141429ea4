"""Decode S prompts with N lattice codes each, several drafted tokens a pass, over caches that stay bounded.

A prompt is stored and attended as a chunk, its last tokens weigh what is stored (as_cache4_weigh), and what they look at least is given
up (as_cache4_evict, as_pages_trim) before as_pages_fork hands the prompt to its N codes.  Each pass then drafts K tokens a lane from a bigram
table (as_step with uniform codes), runs the model over all of them at once, attention with a sliding window and sinks
(as_cache4_attend), accepts what the model agrees to (as_step_verify) and gives the refused tokens' pages, and those that the
window has left behind, back (as_pages_trim).

    python examples/decode_long.py [--prompts 4] [--codes 8] [--passes 20] [--drafts 3] [--keep 48] [--window 64]
"""
import argparse
import importlib.util
import math
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.dirname(HERE))
from paper_2210_15458_b200 import binding as B  # noqa: E402

_spec = importlib.util.spec_from_file_location("decode_prompts", os.path.join(HERE, "decode_prompts.py"))
_prompts = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(_prompts)
TinyLM, i32 = _prompts.TinyLM, _prompts.i32


class LongLM(TinyLM):
    def all_logits(self, tokens, pools, table, length, window=None, sinks=0, weight=None, observers=0):
        """Logits [lanes, T, V] of tokens [lanes, T]; stores their keys and values (pages are there already).  weight [layers][lanes,
        heads, positions]: what the last `observers` tokens give to what is stored."""
        lanes, T = tokens.shape
        x = self.emb[tokens.long()]
        for i in range(self.layers):
            qkv = (x @ self.qkv[i]).view(lanes, T, self.Hq + 2 * self.H, self.D)
            q, k, v = qkv[:, :, :self.Hq], qkv[:, :, self.Hq:self.Hq + self.H], qkv[:, :, self.Hq + self.H:]
            B.as_cache4_append(pools[i], k, v, table, length)
            lse = torch.empty(lanes, T, self.Hq, device=x.device)
            o = B.as_cache4_attend(pools[i], q, table, length, 1 / math.sqrt(self.D), lse=lse, window=window, sinks=sinks if window else 0)
            if weight is not None:
                n = min(T, observers)
                B.as_cache4_weigh(pools[i], q[:, T - n:].contiguous(), lse[:, T - n:].contiguous(), table, length, 1 / math.sqrt(self.D), weight[i],
                                  window=window, sinks=sinks if window else 0, add=False)
            x = x + o.view(lanes, T, -1) @ self.out[i]
        return x @ self.head


def decode(lm, bigram, prompts, N, u, passes, K=3, keep=None, recent=8, window=None, sinks=4, page_size=16, n_pages=2000, temp=1.0, top_p=1.0, seed=0, trace=None):
    """(sequences as lists, state).  keep: tokens of a prompt that stay in the cache (None: all); window, sinks: what a token
    looks at (None: everything); bigram [V, V]: logits of the draft.  trace: a list that gets (target logits, draft logits, drafted, u, codes, tokens,
    accepted) of each pass."""
    S, lanes = len(prompts), len(prompts) * N
    T = max(len(p) for p in prompts)
    M = -(-(T + passes * (K + 1) + K + 1) // page_size) + 1
    pools = B.cache4_pages(n_pages, lm.H, lm.D, page_size, planes=lm.layers)
    table, length, ref = torch.full((S, M), -1, dtype=torch.int32, device="cuda"), i32([0] * S), i32([0] * n_pages)
    # the prompts, padded at their front, all but the last token of each
    B.as_pages_grow(i32([len(p) - 1 for p in prompts]), table, length, ref, page_size)
    if T > 1:
        weight = None if keep is None else [torch.zeros(S, lm.H, M * page_size, device="cuda") for _ in range(lm.layers)]
        lm.all_logits(i32([[0] * (T - len(p)) + p[:-1] for p in prompts]), pools, table, length, window, sinks, weight, observers=recent)
        if keep is not None:
            first = i32([sinks] * S)
            for i in range(lm.layers):
                B.as_cache4_evict(pools[i], weight[i], table, length, i32([keep] * S), recent, first=first, ref=ref)
            B.as_pages_trim(i32([keep] * S), table, length, ref, page_size)
    # hand each to its codes
    table, length, ref = B.as_pages_fork(i32([s for s in range(S) for _ in range(N)]), table, length, ref, page_size, pools)
    codes = B.as_lattice_codes(N, u).repeat(S)
    prev = i32([p[-1] for p in prompts for _ in range(N)])
    out = [list(prompts[i // N]) for i in range(lanes)]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for _ in range(passes):
        draft = torch.empty(lanes, K, lm.V, dtype=lm.dtype, device="cuda")
        drafted = torch.empty(lanes, K, dtype=torch.int32, device="cuda")
        at = prev
        for i in range(K):
            draft[:, i] = bigram[at.long()]
            at, _ = B.as_step(bigram[at.long()], torch.rand(lanes, dtype=torch.float64, device="cuda", generator=gen), temp, 0, top_p)
            drafted[:, i] = at
        B.as_pages_grow(i32([K + 1] * lanes), table, length, ref, page_size)
        logits = lm.all_logits(torch.cat([prev.view(-1, 1), drafted], 1), pools, table, length, window, sinks)
        accept = torch.rand(lanes, K, dtype=torch.float64, device="cuda", generator=gen)
        tokens, accepted, after = B.as_step_verify(logits, draft, drafted, accept, codes, temp, 0, top_p)
        if trace is not None:
            trace.append((logits, draft, drafted, accept, codes, tokens, accepted, after))
        codes = after
        prev = tokens.gather(1, accepted.long().view(-1, 1)).squeeze(1)
        kept = length - (K - accepted)
        gone = None
        if window:
            # the next token looks back to kept + 1 - window
            gone = torch.stack([torch.full_like(kept, -(-sinks // page_size) * page_size), kept + 1 - window], 1).clamp(min=0)
        B.as_pages_trim(kept, table, length, ref, page_size, gone=gone)
        for lane, (row, n) in enumerate(zip(tokens.tolist(), accepted.tolist())):
            out[lane] += row[:n + 1]
    return out, dict(pools=pools, table=table, length=length, ref=ref)


def main():
    ap = argparse.ArgumentParser()
    for name, n in (("prompts", 4), ("codes", 8), ("passes", 20), ("drafts", 3), ("keep", 48), ("window", 64)):
        ap.add_argument("--" + name, type=int, default=n)
    a = ap.parse_args()
    g = torch.Generator().manual_seed(1)
    lm = LongLM(dtype=torch.bfloat16)
    bigram = (lm.emb @ lm.head).contiguous()                # the model without its layers
    prompts = [torch.randint(1, lm.V, (60 + 33 * s,), generator=g).tolist() for s in range(a.prompts)]
    seqs, state = decode(lm, bigram, prompts, a.codes, 0.37, a.passes, a.drafts, keep=a.keep, window=a.window)
    for s in range(a.prompts):
        print("prompt %d (%d tokens):" % (s, len(prompts[s])))
        for j in range(a.codes):
            print("  code %d: %s" % (j, seqs[s * a.codes + j][len(prompts[s]):]))
    made = sum(len(q) for q in seqs) - a.codes * sum(len(p) for p in prompts)
    print("%.2f tokens a pass and lane; pages held: %d" % (made / (a.passes * len(seqs)), int((state["ref"] > 0).sum())))


if __name__ == "__main__":
    main()
