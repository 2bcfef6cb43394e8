"""Generation and update of pruned rollouts on one paged pool, as an engine around the library would run them.

A toy transformer (attention layers with a residual, random weights) goes through one step of the method:

  prompts    arrol_attention over the packed prompts, their keys and values into pages that all rollouts of a prompt share
  decode     arrol_decode_attention, one token a rollout, the prompt read once for its group; weights gathered over layers and tokens
  prune      arrol_score on the hidden states, arrol_select, arrol_compact_inplace on rollouts and prompts together
  evict      arrol_evict: the survivors' own caches cut to a budget by the gathered weights
  decode     the survivors go on, on what is left of their caches
  update     arrol_attention on the survivors' packed rows, arrol_logprob, and arrol_attention_grad

  python examples/rollout_attention.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2603_24840_amd as A
from paper_2603_24840_amd import workloads as W


class Toy:
    """`n_layers` times x += attention(x Wqkv) Wo, with the configuration's heads."""

    def __init__(self, cfg, n_heads, dev, seed=11):
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        self.H, self.KV, self.hd = n_heads, cfg.n_kv_heads, cfg.head_dim
        rand = lambda *s: W.randn_bf16(s, g, dev, std=s[-2] ** -0.5)
        self.qkv = [rand(cfg.d, (n_heads + 2 * cfg.n_kv_heads) * cfg.head_dim) for _ in range(cfg.n_layers)]
        self.out = [rand(n_heads * cfg.head_dim, cfg.d) for _ in range(cfg.n_layers)]
        self.embed = W.randn_bf16((cfg.vocab, cfg.d), g, dev)

    def project(self, layer, x):
        """Queries, keys and values as slices of one projection."""
        y = (x @ self.qkv[layer]).view(x.shape[0], -1, self.hd)
        return y[:, :self.H], y[:, self.H:self.H + self.KV], y[:, self.H + self.KV:]

    def add(self, layer, x, attended):
        return x + attended.reshape(x.shape[0], -1) @ self.out[layer]


def offsets(lengths, dev):
    return torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), torch.cumsum(lengths.to(torch.int64), 0)])


def run(cfg=None, n_heads=4, steps=20, budget=12, dev="cuda:0", seed=3):
    cfg = cfg or W.CONFIGS["tiny"]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    toy, page, N, B = Toy(cfg, n_heads, dev), cfg.page_tokens, cfg.n_rollouts, cfg.n_prompts
    own_pages, prompt_pages = -(-2 * steps // page), -(-cfg.ckpt_len // page)
    pages = torch.randperm(N * own_pages + B * prompt_pages, generator=g, device=dev).to(torch.int32)
    # rows of one table: the rollouts' own pages, then the prompts'; as wide as the wider of the two
    width = max(own_pages, prompt_pages)
    table = torch.full((N + B, width), -1, dtype=torch.int32, device=dev)
    table[:N, :own_pages] = pages[:N * own_pages].view(N, own_pages)
    table[N:, :prompt_pages] = pages[N * own_pages:].view(B, prompt_pages)
    kv = torch.zeros(cfg.n_layers, 2, pages.numel(), page, toy.KV, toy.hd, dtype=torch.bfloat16, device=dev)

    def put(layer, rows, at, k, v):
        """Keys and values of token at[i] of table row rows[i]."""
        ids, slot = table[rows, at // page].long(), at % page
        kv[layer, 0, ids, slot], kv[layer, 1, ids, slot] = k, v

    # prompts, packed
    prompt_len = torch.randint(1, cfg.ckpt_len + 1, (B,), generator=g, device=dev, dtype=torch.int32)
    cu = offsets(prompt_len, dev)
    T = int(cu[-1])
    seq = torch.searchsorted(cu, torch.arange(T, device=dev), right=True) - 1
    tokens = torch.randint(0, cfg.vocab, (T,), generator=g, device=dev)
    x = toy.embed[tokens]
    for layer in range(cfg.n_layers):
        q, k, v = toy.project(layer, x)
        put(layer, N + seq, torch.arange(T, device=dev) - cu[seq], k, v)
        x = toy.add(layer, x, A.arrol_attention(q, k, v, cu)[0])

    seq_len = torch.zeros(N, dtype=torch.int32, device=dev)
    group = torch.arange(B + 1, device=dev, dtype=torch.int64) * cfg.G
    weight = torch.zeros(N, width * page, device=dev)
    history = []                                 # every step's tokens

    def decode():
        """One token for every rollout of the table's first rows."""
        nonlocal weight
        n = seq_len.numel()
        new = torch.randint(0, cfg.vocab, (n,), generator=g, device=dev)
        history.append(new)
        rows, at, x = torch.arange(n, device=dev), seq_len.long(), toy.embed[new]
        seq_len.add_(1)
        for layer in range(cfg.n_layers):
            q, k, v = toy.project(layer, x)
            put(layer, rows, at, k, v)
            got = A.arrol_decode_attention(q.contiguous(), kv, layer, table[:n], seq_len, table[n:], prompt_len, group, want_weight=True, weight=weight, out_weight=weight)
            x = toy.add(layer, x, got["out"])
        return x, dict(q=q, k=k, v=v, layer=layer, **got)

    for _ in range(steps):
        hidden, last = decode()
    checkpoint = dict(last=last, tokens=tokens, history=torch.stack(history, 1), cu=cu, kv=kv.clone(), table=table.clone(), seq_len=seq_len.clone(), prompt_len=prompt_len,
                      weight=weight.clone())

    # prune: the survivors' pages and the prompts' move to the front of the pool
    w_head = torch.randn(cfg.d, generator=g, device=dev) * cfg.d ** -0.5
    _, prob = A.arrol_score(hidden, w_head)
    _, kept = A.arrol_select(prob, B, cfg.G, cfg.K, cfg.rho)
    rows = torch.cat([kept, torch.arange(N, N + B, dtype=torch.int32, device=dev)])
    moved = A.arrol_compact_inplace(kv, table, torch.cat([seq_len, prompt_len]), rows)
    n = kept.numel()
    table, seq_len, weight = moved["block_table_dst"], moved["seq_len_dst"][:n].contiguous(), weight[kept.long()].contiguous()
    group = torch.arange(B + 1, device=dev, dtype=torch.int64) * cfg.K
    history = [h[kept.long()] for h in history]

    # evict: the first token and the last four stay, of the others those that have gathered most
    cut = A.arrol_evict(kv, table[:n].contiguous(), seq_len, weight, budget, n_first=1, n_recent=4)
    evicted = dict(before=seq_len, **cut)
    seq_len, weight = cut["seq_len"].clone(), cut["weight"].clone()      # the table keeps its pages: the next tokens need them
    for _ in range(steps - budget):
        hidden, last = decode()

    # update: the survivors' tokens, prompt and response, as packed rows
    response = torch.stack(history, 1)
    lengths = prompt_len.repeat_interleave(cfg.K) + response.shape[1]
    cu_s = offsets(lengths, dev)
    packed = torch.cat([torch.cat([tokens[cu[b]:cu[b + 1]], response[r]]) for r, b in ((r, r // cfg.K) for r in range(n))])
    x = toy.embed[packed]
    q, k, v = toy.project(0, x)
    out, lse = A.arrol_attention(q, k, v, cu_s)
    y = toy.add(0, x, out)
    logprob = A.arrol_logprob(y.contiguous(), toy.embed, torch.roll(packed, -1).to(torch.int32))
    # d(sum of log-probs)/d(attention's output) by way of a stand-in for the rest of the backward pass
    grad = A.arrol_attention_grad(q, k, v, out, lse, (y @ toy.out[0].t()).view(out.shape).contiguous(), cu_s)
    torch.cuda.synchronize()
    return dict(checkpoint=checkpoint, kept=kept, moved=moved, evicted=evicted, last=last, hidden=hidden, toy=toy, logprob=logprob, grad=grad, cfg=cfg)


if __name__ == "__main__":
    r = run()
    print("rollouts %d -> %d, own tokens %d -> %d, then %d; %d log-probs, mean %.3f" %
          (r["cfg"].n_rollouts, r["kept"].numel(), int(r["evicted"]["before"].max()), int(r["evicted"]["seq_len"].max()), r["last"]["weight"].gt(0).sum(1).max(),
           r["logprob"].numel(), float(r["logprob"].mean())))
