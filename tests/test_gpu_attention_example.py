"""examples/rollout_attention.py runs the attention calls with the pruning path; what they hand on to each other is looked at here."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rollout_attention.py")


def test_generation_and_update_of_pruned_rollouts():
    print("[case] example: prompts, decode, prune, evict, decode, update", flush=True)
    spec = importlib.util.spec_from_file_location("rollout_attention", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    import paper_2603_24840_amd as A
    r = example.run()
    c, cfg, toy = r["checkpoint"], r["cfg"], r["toy"]
    last = c["last"]
    # the last decode step of the last layer against the packed form over the same keys (bf16 outputs of magnitude about 1: two roundings each)
    page, G = cfg.page_tokens, cfg.G
    keys, values, lengths = [], [], []
    for i in range(cfg.n_rollouts):
        for row, n in ((cfg.n_rollouts + i // G, int(c["prompt_len"][i // G])), (i, int(c["seq_len"][i]))):
            t = torch.arange(n, device="cuda:0")
            ids = c["table"][row, t // page].long()
            keys.append(c["kv"][last["layer"], 0, ids, t % page])
            values.append(c["kv"][last["layer"], 1, ids, t % page])
        lengths.append(int(c["prompt_len"][i // G]) + int(c["seq_len"][i]))
    cu = example.offsets(torch.tensor(lengths, device="cuda:0"), "cuda:0")
    out, lse = A.arrol_attention(last["q"], torch.cat(keys), torch.cat(values), torch.arange(cfg.n_rollouts + 1, device="cuda:0"), cu)
    values_max = float(torch.cat(values).abs().max())
    assert float((out.float() - last["out"].float()).abs().max()) <= 4 * 2.0 ** -8 * values_max
    assert float((lse.t() - last["lse"]).abs().max()) <= 1e-4
    # what a rollout's own tokens have gathered is less than one per head, layer and step, and nothing lies behind its length
    w = c["weight"]
    steps = c["history"].shape[1]
    assert bool((w[:, :steps] > 0).all()) and not w[:, steps:].any() and float(w.sum(1).max()) < toy.H * cfg.n_layers * steps
    # eviction kept the first, the last four and the heaviest between them
    e = r["evicted"]
    weight = w[r["kept"].long()]
    for row in range(weight.shape[0]):
        n = int(e["seq_len"][row])
        where = e["position"][row, :n].long()
        between = torch.arange(1, steps - 4, device="cuda:0")
        kept = torch.zeros(steps, dtype=torch.bool, device="cuda:0")
        kept[where] = True
        assert n == 12 and bool(kept[0]) and bool(kept[steps - 4:].all()) and torch.equal(e["weight"][row, :n], weight[row, where])
        inside = kept[between]
        assert float(weight[row, between][inside].min()) >= float(weight[row, between][~inside].max())
    assert bool(torch.isfinite(r["logprob"][:-1]).all()) and all(bool(torch.isfinite(x.float()).all()) and bool(x.any()) for x in r["grad"].values())
    assert bool(torch.isfinite(r["hidden"].float()).all())
