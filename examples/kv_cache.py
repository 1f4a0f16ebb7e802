"""A transformer's attention layer that keeps its past in 8 bits, used as a serving program would use it.

Prompts of differing lengths are written into the cache (kv_write) and attended (kv_attend) at once, then every sequence
goes on token by token; the codes are all that is kept.  At the end the keys are read back (kv_read) as the points of
a clustering (points_bf16, kmeans_fit): the centroids say which parts of a long context a query looks at.

    python examples/kv_cache.py [--dtype fp8] [--steps 32]
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2608_14648_amd as km  # noqa: E402


class Layer:
    """Random projections of a hidden state to queries, keys and values and back."""

    def __init__(self, heads, group, d, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        hidden = 256
        self.heads, self.q_heads, self.d, self.hidden = heads, heads * group, d, hidden

        def w(n_in, n_out):
            return (torch.randn(n_in, n_out, generator=g, device="cuda") / math.sqrt(n_in)).bfloat16()

        self.wq, self.wk, self.wv = (w(hidden, n * d) for n in (self.q_heads, heads, heads))
        self.wo = w(self.q_heads * d, hidden)

    def qkv(self, x):
        return ((x @ self.wq).view(-1, self.q_heads, self.d), (x @ self.wk).view(-1, self.heads, self.d),
                (x @ self.wv).view(-1, self.heads, self.d))


def plain(q, k, v):
    """Attention of one sequence's last queries over keys and values as they were before the cache, in 64 bits."""
    n, L = q.shape[0], k.shape[0]
    group = q.shape[1] // k.shape[1]
    k, v = (t.double().repeat_interleave(group, 1).transpose(0, 1).contiguous() for t in (k, v))
    z = torch.matmul(q.double().transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) / math.sqrt(q.shape[2])
    hide = torch.arange(L, device=q.device) > torch.arange(L - n, L, device=q.device)[:, None]
    return torch.matmul(torch.softmax(z.masked_fill(hide, -math.inf), 2), v).transpose(0, 1)


def main(prompts=(700, 123, 1), steps=16, heads=4, group=4, d=128, page=64, dtype=torch.int8, clusters=8, seed=0,
         say=print):
    layer = Layer(heads, group, d, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    n = len(prompts)
    # pages of every sequence, room for its steps included
    per = [-(-(p + steps) // page) for p in prompts]
    order = torch.randperm(sum(per), generator=g, device="cuda").int()
    table = torch.full((n, max(per)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, p in enumerate(per):
        table[b, :p] = order[at:at + p]
        at += p
    cache = km.kv_cache(sum(per), heads, d, page, dtype)

    # the prompts, all sequences at once
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    starts = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]), dtype=torch.int32, device="cuda")
    x = torch.randn(sum(prompts), layer.hidden, generator=g, device="cuda").bfloat16()
    q, k, v = layer.qkv(x)
    seqs = km.KvSeqs(table, lens, starts, rows=sum(prompts), max_rows=max(prompts), max_len=max(prompts))
    km.kv_write(cache, seqs, k, v)
    out, _ = km.kv_attend(cache, seqs, q)
    past = [[k[a:b], v[a:b]] for a, b in zip(starts.tolist(), starts.tolist()[1:])]  # for the comparison alone
    first = torch.cat([plain(q[a:b], *past[i]) for i, (a, b) in enumerate(zip(starts.tolist(), starts.tolist()[1:]))])
    err = ((out.double() - first).norm() / first.norm()).item()
    say(f"prompts of {list(prompts)} tokens: {err:.4f} from attention on unquantised keys and values")

    # one token of every sequence at a time; table and lens are read on the device, so one KvSeqs serves every step
    one = km.KvSeqs(table, lens, max_len=max(prompts) + steps)
    last = [b - 1 for b in starts.tolist()[1:]]
    h = x[last] + out[last].reshape(n, -1) @ layer.wo
    for _ in range(steps):
        lens += 1
        q, k, v = layer.qkv(h)
        km.kv_write(cache, one, k, v)
        out, lse = km.kv_attend(cache, one, q, lse=True)
        for b in range(n):
            past[b] = [torch.cat([t, new[b:b + 1]]) for t, new in zip(past[b], (k, v))]
        h = h + out.reshape(n, -1) @ layer.wo
        h = (h.float() / h.float().square().mean(1, keepdim=True).sqrt()).bfloat16()
    want = torch.cat([plain(q[b:b + 1], *past[b]) for b in range(n)])
    err1 = ((out.double() - want).norm() / want.norm()).item()
    say(f"after {steps} single tokens: {err1:.4f}; log-sum-exp of the first head {[round(e, 3) for e in lse[:, 0].tolist()]}")

    # the longest sequence's keys, clustered per head
    b = int(np.argmax(prompts))
    total = prompts[b] + steps
    whole = km.KvSeqs(table[b:b + 1].contiguous(), lens[b:b + 1], rows=total, max_len=total)
    keys, _ = km.kv_read(cache, whole, torch.bfloat16)
    back = ((keys.double() - past[b][0].double()).norm() / past[b][0].double().norm()).item()
    say(f"keys read back: {back:.4f} from what was written")
    idx = torch.randperm(total, generator=g, device="cuda")[:clusters].sort().values.cpu().numpy()
    cost = []
    for hd in range(heads):
        pts = km.points_bf16(keys[:, hd])  # rows of one head, where they lie
        C, assign, J = km.kmeans_fit(pts, min(clusters, total), 5, idx)
        cost.append((J[0].item(), J[-1].item()))
    say("clusters of the keys, objective per head: " + ", ".join(f"{a:.0f} -> {z:.0f}" for a, z in cost))
    return dict(prompt=err, token=err1, read=back, cost=cost)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--dtype", choices=["int8", "fp8"], default="int8")
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    main(steps=a.steps, dtype=torch.int8 if a.dtype == "int8" else torch.float8_e4m3fn)
