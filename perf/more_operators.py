"""What lies between a model's projections and the calls around it, as cases that can be timed and compared: positions of queries and
keys, new tokens into the paged KV pool, and the gradient of the log-probabilities.

  rotary   queries and keys of packed rows rotated by their positions, or back (the gradient)
  append   keys and values of new tokens into the pool, keys and queries rotated on the way
  grad     the gradient of log pi(y_t) = z_t[y_t] - logsumexp z_t, z = W h, with respect to hidden states and LM head

Tensors are bf16 where the library's are (heads, KV pool, hidden states, LM head, their gradients), fp32 elsewhere and fp64 for frequencies.  Lengths
come from the case alone, values from the seed.
"""
import math

import torch

own = False

DEV = "cuda:0"


def listed():
    return [
        # the tiny configuration's prompts: a call of a few microseconds
        dict(name="rotary_tiny", kind="rotary", n=4, lo=16, hi=64, heads=4, kv=2, hd=64, rot=64, interleaved=False, inverse=False, base=1e4, factor=1.0, context=0,
             magnitude=1.0, far=0),
        # a micro-batch of survivors of an 8B model, frequencies scaled by parts for a longer context
        dict(name="rotary_survivors", kind="rotary", n=4, lo=1024, hi=4096, heads=32, kv=8, hd=128, rot=128, interleaved=False, inverse=False, base=5e5, factor=8.0,
             context=8192, magnitude=1.0, far=0),
        # the gradients of queries and keys of which half the head is rotated in neighbouring pairs, far into a context
        dict(name="rotary_grad_part", kind="rotary", n=64, lo=31, hi=501, heads=16, kv=8, hd=128, rot=64, interleaved=True, inverse=True, base=1e6, factor=4.0,
             context=0, magnitude=1.1386, far=1000000),
        # one prompt's rollouts, a token each: latency
        dict(name="append_one_prompt", kind="append", n=8, lo=1, hi=1, slot_lo=1, slot_hi=60, before=200, heads=32, kv=8, hd=64, rot=64, interleaved=False, page=16,
             want_k=False),
        # a batch of a 1.7B model half way, a token each, behind shared prompts
        dict(name="append_batch", kind="append", n=1024, lo=1, hi=1, slot_lo=1, slot_hi=2000, before=600, heads=16, kv=8, hd=128, rot=128, interleaved=False, page=16,
             want_k=False),
        # the prompts of a 1B-model batch, whose rotated keys the attention over packed rows takes as well
        dict(name="append_prompts", kind="append", n=64, lo=31, hi=512, slot_lo=0, slot_hi=0, before=0, heads=32, kv=8, hd=64, rot=64, interleaved=False, page=16,
             want_k=True),
        # chunks of long prompts behind what is cached of them, part of the head rotated in pairs that no vector of eight fits
        dict(name="append_chunks", kind="append", n=5, lo=300, hi=2047, slot_lo=5, slot_hi=14000, before=0, heads=24, kv=8, hd=80, rot=40, interleaved=False, page=32,
             want_k=False),
        # the tiny configuration's survivors
        dict(name="grad_tiny", kind="grad", n=4, lo=31, hi=128, vocab=4096, d=256, idle=0),
        # few tokens, a whole vocabulary
        dict(name="grad_few", kind="grad", n=1, lo=311, hi=311, vocab=151936, d=2048, idle=0),
        # a micro-batch of survivors of a 1B model
        dict(name="grad_microbatch", kind="grad", n=4, lo=256, hi=2048, vocab=128256, d=2048, idle=0),
        # a batch of a 1.7B model of which three groups in eight have equal rewards, so that their tokens' gradients are zero
        dict(name="grad_equal_rewards", kind="grad", n=16, lo=97, hi=1000, vocab=151936, d=2048, idle=3),
        # a micro-batch of survivors of an 8B model
        dict(name="grad_large", kind="grad", n=2, lo=1000, hi=4096, vocab=151936, d=4096, idle=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "grad"])
    if kind == "grad":
        n, d, vocab = _log_int(rng, 1, 32), 8 * _log_int(rng, 8, 512), _log_int(rng, 300, 152000)
        if rng.random() < 0.7:
            d = 64 * max(1, d // 64)
        hi = _log_int(rng, 1, 4096)
        hi = max(1, min(hi, int(3.5e12 / (n * vocab * d))))
        return dict(kind=kind, n=n, lo=_log_int(rng, 1, hi), hi=hi, vocab=vocab, d=d, idle=rng.choice([0, 0, 1, 4]))
    kv, hd = rng.choice([1, 2, 4, 8]), rng.choice([40, 64, 80, 128])
    heads, rot = kv * rng.choice([1, 2, 3, 4]), 2 * rng.randint(1, hd // 2) if rng.random() < 0.3 else rng.choice([hd, hd // 2])
    if kind == "rotary":
        n, hi = _log_int(rng, 1, 64), _log_int(rng, 1, 4096)
        hi = max(1, min(hi, 16384 * 40 // (n * (heads + kv))))
        return dict(kind=kind, n=n, lo=_log_int(rng, 1, hi), hi=hi, heads=heads, kv=kv, hd=hd, rot=rot, interleaved=rng.random() < 0.4, inverse=rng.random() < 0.5,
                    base=rng.choice([1e4, 5e5, 1e6]), factor=rng.choice([1.0, 4.0, 8.0]), context=rng.choice([0, 8192]), magnitude=rng.choice([1.0, 1.25]),
                    far=rng.choice([0, 30000, 3000000]))
    single = rng.random() < 0.5
    n, hi = (_log_int(rng, 1, 2048), 1) if single else (_log_int(rng, 1, 64), _log_int(rng, 1, 2048))
    hi = max(1, min(hi, 16384 * 40 // (n * (heads + 2 * kv))))
    slot = _log_int(rng, 1, 4096)
    return dict(kind=kind, n=n, lo=_log_int(rng, 1, hi), hi=hi, slot_lo=rng.randint(0, slot), slot_hi=slot, before=rng.choice([0, 100, 20000]), heads=heads, kv=kv, hd=hd,
                rot=rot, interleaved=rng.random() < 0.4, page=rng.choice([8, 16, 32]), want_k=rng.random() < 0.3)


def _lengths(n, lo, hi):
    """n lengths spread over [lo, hi], the longest among them."""
    return [hi - int((hi - lo + 1) * ((0.6180339887498949 * i) % 1.0)) for i in range(n)]


def _offsets(lengths):
    at = [0]
    for x in lengths:
        at.append(at[-1] + x)
    return torch.tensor(at, dtype=torch.int64, device=DEV)


def _places(lengths, first):
    """first[s], first[s] + 1, ... of every packed sequence s."""
    return torch.cat([torch.arange(a, a + n, dtype=torch.int32) for a, n in zip(first, lengths)]).to(DEV)


def _frequencies(rot, base, factor=1.0, context=0):
    """Radians a position: base^(-2i/rot), slower by `factor`; with a context only those that turn less than 4 times in it, in full those that turn less than once."""
    f = torch.tensor(float(base), dtype=torch.float64) ** (torch.arange(rot // 2, dtype=torch.float64) * -2 / rot)
    s = ((context * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
    return (f * (s + (1 - s) / factor)).to(DEV)


def _prepare_rotary(case, g):
    lengths = _lengths(case["n"], case["lo"], case["hi"])
    H, KV, hd = case["heads"], case["kv"], case["hd"]
    x = torch.randn(sum(lengths), H + 2 * KV, hd, generator=g, device=DEV).to(torch.bfloat16)      # slices of one projection's output
    return dict(kind="rotary", q=x[:, :H], k=x[:, H:H + KV], position=_places(lengths, [case["far"] + 17 * i for i in range(case["n"])]),
                inv_freq=_frequencies(case["rot"], case["base"], case["factor"], case["context"]), interleaved=case["interleaved"], inverse=case["inverse"],
                magnitude=case["magnitude"])


def _append_lengths(case):
    return _lengths(case["n"], case["lo"], case["hi"]), _lengths(case["n"], case["slot_lo"], case["slot_hi"])


def _prepare_append(case, g):
    new, start = _append_lengths(case)
    H, KV, hd, per = case["heads"], case["kv"], case["hd"], case["page"]
    need = [-(-(a + b) // per) for a, b in zip(start, new)]
    pages = torch.randperm(sum(need), generator=g, device=DEV).to(torch.int32)
    at = _offsets(need)
    inside = torch.arange(max(need), device=DEV) < (at[1:] - at[:-1])[:, None]
    table = torch.where(inside, pages[(at[:-1, None] + torch.arange(max(need), device=DEV)).clamp(max=sum(need) - 1)], -1)
    kv = torch.zeros(2, 2, sum(need), per, KV, hd, dtype=torch.bfloat16, device=DEV)
    x = torch.randn(sum(new), H + 2 * KV, hd, generator=g, device=DEV).to(torch.bfloat16)
    single = case["hi"] == 1
    return dict(kind="append", q=x[:, :H], k=x[:, H:H + KV], v=x[:, H + KV:], kv=kv, layer=1, table=table, start=torch.tensor(start, dtype=torch.int32, device=DEV),
                cu=None if single else _offsets(new), position=_places(new, [case["before"] + a for a in start]), inv_freq=_frequencies(case["rot"], 5e5),
                interleaved=case["interleaved"], want_k=case["want_k"])


def _active(case):
    """1 for the rows of sequences that are trained on, 0 for those of equal rewards."""
    lengths = _lengths(case["n"], case["lo"], case["hi"])
    return [(int(5 * i % 8 >= case["idle"]), n) for i, n in enumerate(lengths)]


def _prepare_grad(case, g):
    T, V, d = sum(n for _, n in _active(case)), case["vocab"], case["d"]
    lm_head = (torch.randn(V, d, generator=g, device=DEV) * d ** -0.5).to(torch.bfloat16)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    # a sampled token's own logit stands out by 0 to 16: from flat distributions to all but certain ones
    sure = 16 * torch.rand(T, 1, generator=g, device=DEV)
    hidden = (torch.randn(T, d, generator=g, device=DEV) + sure * lm_head[targets.long()].float()).to(torch.bfloat16)
    # derivatives of the clipped objective: advantage over length, a few tokens clipped
    length = torch.cat([torch.full((n,), float(a) / n) for a, n in _active(case)]).to(DEV)
    sequence = torch.cat([torch.full((n,), i) for i, (_, n) in enumerate(_active(case))]).to(DEV)
    advantage = torch.randn(case["n"], generator=g, device=DEV)
    clipped = torch.rand(T, generator=g, device=DEV) < 1 / 32
    grad_logp = torch.where(clipped, torch.zeros_like(length), length * advantage[sequence] * (0.8 + 0.4 * torch.rand(T, generator=g, device=DEV)))
    lse = torch.cat([_logits(hidden[a:a + 2048], lm_head).logsumexp(1) for a in range(0, T, 2048)])
    return dict(kind="grad", hidden=hidden, lm_head=lm_head, targets=targets, lse=lse, grad_logp=grad_logp)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return {"rotary": _prepare_rotary, "append": _prepare_append, "grad": _prepare_grad}[case["kind"]](case, g)


def _rotate(x, position, inv_freq, interleaved, inverse=False, magnitude=1.0):
    rot = 2 * inv_freq.numel()
    angle = position.double()[:, None] * inv_freq
    cos, sin = (f(angle)[:, None].float() * magnitude for f in (torch.cos, torch.sin))
    if inverse:
        sin = -sin
    y = x.float()
    a, b = (y[..., :rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(torch.bfloat16)


def _rotary(s):
    return tuple(_rotate(x, s["position"], s["inv_freq"], s["interleaved"], s["inverse"], s["magnitude"]) for x in (s["q"], s["k"]))


def _append(s):
    q, k = (_rotate(x, s["position"], s["inv_freq"], s["interleaved"]) for x in (s["q"], s["k"]))
    row, slot = torch.arange(q.shape[0], device=DEV), s["start"].long()
    if s["cu"] is not None:
        sequence = torch.searchsorted(s["cu"], row, right=True) - 1
        slot, row = slot[sequence] + row - s["cu"][sequence], sequence
    page = s["kv"].shape[3]
    ids, at = s["table"][row, slot // page].long(), slot % page
    s["kv"][s["layer"], 0, ids, at] = k
    s["kv"][s["layer"], 1, ids, at] = s["v"]
    return (s["kv"], q, k) if s["want_k"] else (s["kv"], q)


def _logits(hidden, lm_head):
    return torch.mm(hidden.float(), lm_head.float().t())


def _grad(s):
    h, w, g = s["hidden"].float(), s["lm_head"].float(), s["grad_logp"][:, None]
    dz = torch.exp(_logits(h, w) - s["lse"][:, None]) * -g
    dz[torch.arange(h.shape[0], device=DEV), s["targets"].long()] += s["grad_logp"]
    return torch.mm(dz, w).to(torch.bfloat16), torch.mm(dz.t(), h).to(torch.bfloat16)


def _run_own(s):
    import paper_2603_24840_amd as A

    if s["kind"] == "rotary":
        return A.arrol_rotary(s["q"], s["k"], s["position"], s["inv_freq"], interleaved=s["interleaved"], inverse=s["inverse"], magnitude=s["magnitude"])
    if s["kind"] == "append":
        got = A.arrol_append(s["k"], s["v"], s["kv"], s["layer"], s["table"], s["start"], s["cu"], q=s["q"], position=s["position"], inv_freq=s["inv_freq"],
                             interleaved=s["interleaved"], want_k=s["want_k"])
        return (s["kv"], got["q"], got["k"]) if s["want_k"] else (s["kv"], got["q"])
    got = A.arrol_logprob_grad(s["hidden"], s["lm_head"], s["targets"], s["lse"], s["grad_logp"])
    return got["grad_hidden"], got["grad_lm_head"]


def run(state):
    if own:
        return _run_own(state)
    return {"rotary": _rotary, "append": _append, "grad": _grad}[state["kind"]](state)


def work(case):
    if case["kind"] == "grad":
        T, V, d = sum(a * n for a, n in _active(case)) * 31 / 32, case["vocab"], case["d"]
        total = sum(n for _, n in _active(case))
        return {"bytes": int(2 * d * (T + total) + 4 * d * V + 12 * total), "flops": int(6 * T * V * d)}
    rot, heads, KV, hd = case["rot"], case["heads"], case["kv"], case["hd"]
    if case["kind"] == "rotary":
        T = sum(_lengths(case["n"], case["lo"], case["hi"]))
        return {"bytes": T * (4 * hd * (heads + KV) + 4), "flops": 3 * T * rot * (heads + KV)}
    T = sum(_append_lengths(case)[0])
    return {"bytes": T * (4 * hd * (heads + 2 * KV) + (2 * hd * KV if case["want_k"] else 0) + 4) + 8 * case["n"], "flops": 3 * T * rot * (heads + KV)}


def _exact_rotate(x, position, inv_freq, interleaved, sign, magnitude):
    """Pairs as complex numbers, turned by e^(i angle)."""
    x, half = x.double(), inv_freq.numel()
    first = torch.arange(half, device=DEV) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    turn = torch.polar(torch.full_like(inv_freq, magnitude).expand(position.numel(), half).contiguous(), sign * torch.outer(position.double(), inv_freq))
    z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_append(s):
    turned = [_exact_rotate(x, s["position"], s["inv_freq"], s["interleaved"], 1.0, 1.0) for x in (s["q"], s["k"])]
    kv, page, start, table = s["kv"].double(), s["kv"].shape[3], s["start"].tolist(), s["table"].tolist()
    ends = s["cu"].tolist() if s["cu"] is not None else list(range(len(start) + 1))
    where = [table[r][(start[r] + j) // page] * page + (start[r] + j) % page for r in range(len(start)) for j in range(ends[r + 1] - ends[r])]
    flat = kv[s["layer"]].flatten(1, 2)
    flat[0, where], flat[1, where] = turned[1], s["v"].double()
    kv[s["layer"]] = flat.view(kv[s["layer"]].shape)
    return (kv, turned[0], turned[1]) if s["want_k"] else (kv, turned[0])


def _exact_grad(s):
    """Token block by token block; what a token's probabilities leave of one, spread over the rows of the LM head."""
    w, V = s["lm_head"].double(), s["lm_head"].shape[0]
    grad_hidden, grad_w = [], torch.zeros_like(w)
    for a in range(0, s["hidden"].shape[0], 1024):
        h, y, lse, g = (s[x][a:a + 1024] for x in ("hidden", "targets", "lse", "grad_logp"))
        h = h.double()
        chosen = (torch.arange(V, device=DEV) == y[:, None]).double()
        left = (chosen - torch.exp(torch.addmm(-lse.double()[:, None], h, w.t()))) * g.double()[:, None]
        grad_hidden.append(torch.mm(left, w))
        grad_w.addmm_(left.t(), h)
    return torch.cat(grad_hidden), grad_w


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        sign = -1.0 if s["inverse"] else 1.0
        return tuple(_exact_rotate(x, s["position"], s["inv_freq"], s["interleaved"], sign, s["magnitude"]) for x in (s["q"], s["k"]))
    return _exact_append(s) if case["kind"] == "append" else _exact_grad(s)
