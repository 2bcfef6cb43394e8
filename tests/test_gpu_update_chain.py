"""Rotary, attention, log-probs and their gradients together, as an update runs them, and append with the attention that reads the pool, as a rollout does."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -8


@pytest.fixture(scope="module")
def A():
    import paper_2603_24840_amd as pkg
    pkg.lib()
    return pkg


def rotate(x, position, inv_freq):
    """x [T, heads, hd] in 64 bits, elements i and i + hd/2 as complex numbers."""
    n = inv_freq.numel()
    turn = torch.polar(torch.ones(position.numel(), n, dtype=torch.float64, device=x.device), torch.outer(position.double(), inv_freq))[:, None]
    z = torch.complex(x[..., :n], x[..., n:2 * n]) * turn
    return torch.cat([z.real, z.imag, x[..., 2 * n:]], -1)


def attend(q, k, v, cu):
    """Causal attention in 64 bits, sequence by sequence."""
    out, per = [], q.shape[1] // k.shape[1]
    for a, b in zip(cu.tolist(), cu.tolist()[1:]):
        z = torch.matmul(q[a:b].transpose(0, 1), k[a:b].repeat_interleave(per, 1).permute(1, 2, 0)) / math.sqrt(q.shape[2])
        z = z + torch.full((b - a, b - a), -math.inf, dtype=torch.float64, device=z.device).triu(1)
        out.append(torch.matmul(torch.softmax(z, -1), v[a:b].repeat_interleave(per, 1).transpose(0, 1)).transpose(0, 1))
    return torch.cat(out)


def test_update_of_the_example_against_differentiation():
    """The gradients that examples/rollout_attention.py ends with, against those of its layer differentiated in 64 bits, with the objective's derivative as given.

    In norm.  Rounded to bf16, each by at most U / sqrt(3) of the values in the root mean square: forward the projection, q and k turned, the weights, their product, its
    projection and the sum with the residual (7; a logit is off by what its row is, and these are of size 1, so a probability is too); back dz, the hidden
    gradient, its projection, p and ds, D, the attention's gradient, the turned one, and the product with x (8).  15 uncorrelated ones are sqrt(15 / 3) U = 2.3 U; the
    LM head's gradient has 7 + 2 behind it, the hidden one's as well.  Half as much again for what one rounding does to two paths: 3.5 U.
    """
    print("[case] chain: gradients of the example", flush=True)
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rollout_attention.py")
    spec = importlib.util.spec_from_file_location("rollout_attention_update", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.run()
    toy, u, grad = r["toy"], r["update"], r["grad"]
    x, g = u["x"].double(), u["grad_logp"].double()
    qkv, head = toy.qkv[0].double().requires_grad_(True), toy.head.double().requires_grad_(True)
    y_q = torch.matmul(x, qkv).view(x.shape[0], -1, toy.hd)
    q, k, v = y_q[:, :toy.H], y_q[:, toy.H:toy.H + toy.KV], y_q[:, toy.H + toy.KV:]
    out = attend(rotate(q, u["position"], toy.inv_freq), rotate(k, u["position"], toy.inv_freq), v, u["cu"])
    hidden = x + torch.matmul(out.flatten(1), toy.out[0].double())
    logp = torch.log_softmax(torch.matmul(hidden, head.t()), 1).gather(1, u["targets"].long()[:, None])[:, 0]
    assert float((logp.detach() - r["logprob"].double()).abs().max()) <= 0.1        # a logit of some 6 at most, off by 4 U of its row's terms
    want = torch.autograd.grad((g * logp).sum(), (qkv, head, hidden))
    used = g != 0
    assert int(used.sum()) > 50 and not grad["grad_hidden"][~used].any()
    for name, ref in (("projection", want[0]), ("grad_lm_head", want[1]), ("grad_hidden", want[2])):
        off = float((grad[name].double() - ref).norm() / ref.norm())
        print("  %s off by %.2g in norm" % (name, off), flush=True)
        assert off <= 3.5 * U, (name, off)
    assert math.isfinite(float(u["objective"]))


@pytest.mark.parametrize("hd,rot,interleaved", [(64, 64, False), (128, 64, False), (80, 40, True)])
def test_rollouts_on_the_pool_attend_as_packed_rows_do(A, hd, rot, interleaved):
    """Prompts and then tokens one by one through append and decode attention, against rotary and attention over the packed whole: the same keys and queries bit for bit, and
    outputs that differ by two roundings each of values and weights."""
    print("[case] chain: append and decode, hd=%d rot=%d" % (hd, rot), flush=True)
    H, KV, page, prompts, steps, G = 4, 2, 16, [5, 33, 16], 18, 2
    g = torch.Generator(device=DEV)
    g.manual_seed(hd)
    f = A.arrol_rotary_frequencies(rot, 1e4, device=DEV)
    n, B = G * len(prompts), len(prompts)
    x = [torch.randn(p, H + 2 * KV, hd, generator=g, device=DEV).to(torch.bfloat16) for p in prompts]
    new = torch.randn(steps, n, H + 2 * KV, hd, generator=g, device=DEV).to(torch.bfloat16)
    table = torch.randperm(n * 2 + B * 3, generator=g, device=DEV).to(torch.int32)
    own, shared = table[:2 * n].view(n, 2), table[2 * n:].view(B, 3)
    kv = torch.full((1, 2, 2 * n + 3 * B, page, KV, hd), float("nan"), dtype=torch.bfloat16, device=DEV)
    prompt_len = torch.tensor(prompts, dtype=torch.int32, device=DEV)
    packed = torch.cat(x)
    cu = torch.tensor([0, 5, 38, 54], device=DEV)
    A.arrol_append(packed[:, H:H + KV], packed[:, H + KV:], kv, 0, shared, torch.zeros(B, dtype=torch.int32, device=DEV), cu, inv_freq=f, interleaved=interleaved)
    seq_len, group = torch.zeros(n, dtype=torch.int32, device=DEV), torch.arange(B + 1, device=DEV) * G
    for t in range(steps):
        q, k, v = new[t, :, :H], new[t, :, H:H + KV], new[t, :, H + KV:]
        q = A.arrol_append(k, v, kv, 0, own, seq_len, q=q, position=prompt_len.repeat_interleave(G) + t, inv_freq=f, interleaved=interleaved)["q"]
        seq_len = seq_len + 1
        got = A.arrol_decode_attention(q, kv, 0, own, seq_len, shared, prompt_len, group)
    whole = torch.cat([torch.cat([x[i // G], new[:, i]]) for i in range(n)])
    lengths = torch.tensor([prompts[i // G] + steps for i in range(n)], device=DEV)
    ends = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lengths.cumsum(0)])
    position = torch.cat([torch.arange(int(m), device=DEV) for m in lengths]).to(torch.int32)
    tq, tk = A.arrol_rotary(whole[:, :H], whole[:, H:H + KV], position, f, interleaved=interleaved)
    out, lse = A.arrol_attention(tq, tk, whole[:, H + KV:], ends)
    last = ends[1:] - 1
    assert torch.equal(tq[last], q)
    for i in range(n):
        slots = torch.arange(steps, device=DEV)
        ids = own[i, slots // page].long()
        assert torch.equal(kv[0, 0, ids, slots % page], tk[ends[i + 1] - steps:ends[i + 1]]) and torch.equal(kv[0, 1, ids, slots % page], new[:, i, H + KV:])
    assert float((out[last].float() - got["out"].float()).abs().max()) <= 4 * U * float(whole[:, H + KV:].float().abs().max())
    assert float((lse[:, last].t() - got["lse"]).abs().max()) <= 1e-4
    assert bool(torch.isfinite(got["out"].float()).all())
