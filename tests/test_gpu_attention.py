"""Attention over packed sequences and its gradient against a plain implementation in 64 bits.

Tolerances, derived from the roundings (u = 2^-8 for bf16, e = 2^-24 for fp32) before the first run, element by element:
  z      hd products summed in fp32: (hd + 4) e scale sum |q||k|; a weight p is off by that, relatively, and by 2^-21 of exp2 and its argument
  out    weights rounded once (u) and the result once: u |o| + (u + 2 dz + 2^-20) sum p |v|
  lse    dz, its own rounding and up to nk roundings of the sum of positive terms
  ds     p's error and ds' rounding on |ds|, and on p those of dp (as z) and of D = <do, out> (out as above)
  dq, dk, dv   those of their terms, and u of the result
"""
import numpy as np
import pytest
import torch

from helpers import npy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, E = 2.0 ** -8, 2.0 ** -24


@pytest.fixture(scope="module")
def A():
    import paper_2603_24840_amd as pkg
    pkg.lib()
    return pkg


def cu(lengths, start=0):
    return torch.tensor(np.concatenate([[start], start + np.cumsum(lengths)]), dtype=torch.int64, device=DEV)


def f64(t):
    return t.detach().cpu().double().numpy()


def reference(q, k, v, cu_q, cu_k, causal, scale, grad_out=None):
    """fp64 values and tolerances: dict(out, lse[, dq, dk, dv]) and the same of tolerances."""
    q, k, v, cu_q, cu_k = f64(q), f64(k), f64(v), npy(cu_q), npy(cu_k)
    H, KV, hd = q.shape[1], k.shape[1], q.shape[2]
    val = dict(out=np.zeros_like(q), lse=np.full((H, q.shape[0]), -np.inf))
    tol = dict(out=np.zeros_like(q), lse=np.zeros((H, q.shape[0])))
    if grad_out is not None:
        go = f64(grad_out)
        for name, x in (("dq", q), ("dk", k), ("dv", v)):
            val[name], tol[name] = np.zeros_like(x), np.zeros_like(x)
    for a, b, c, d in zip(cu_q, cu_q[1:], cu_k, cu_k[1:]):
        nq, nk = b - a, d - c
        if nq <= 0 or nk <= 0:
            continue
        sees = np.ones((nq, nk), bool)
        if causal:
            sees = np.arange(nk)[None, :] + nq <= np.arange(nq)[:, None] + nk
        for h in range(H):
            g = h * KV // H
            x, y, w = q[a:b, h], k[c:d, g], v[c:d, g]
            z = np.where(sees, scale * (x @ y.T), -np.inf)
            dz = np.where(sees, (hd + 4) * E * scale * (np.abs(x) @ np.abs(y).T), 0)
            top = np.max(z, 1, keepdims=True)
            p = np.exp(z - np.where(np.isfinite(top), top, 0))
            total = p.sum(1, keepdims=True)
            p = p / np.where(total == 0, 1, total)
            o = p @ w
            dp_rel = 2 * dz.max(1, keepdims=True) + 2.0 ** -20 + nk * E + np.abs(np.where(np.isfinite(top), top, 0)) * 4 * E
            out_tol = U * np.abs(o) + (U + dp_rel) * (p @ np.abs(w))
            with np.errstate(divide="ignore"):
                lse = np.where(total > 0, top + np.log(total), -np.inf)
            val["out"][a:b, h], tol["out"][a:b, h] = o, out_tol
            val["lse"][h, a:b] = lse[:, 0]
            tol["lse"][h, a:b] = (dp_rel + 4 * E * np.abs(np.where(np.isfinite(lse), lse, 0)))[:, 0]
            if grad_out is None:
                continue
            do = go[a:b, h]
            rel = 2 * dp_rel                                   # of p from z and from lse
            dp, D = do @ w.T, np.sum(do * o, 1, keepdims=True)
            ds = p * (dp - D)
            ds_tol = (U + rel) * np.abs(ds) + p * (np.sum(np.abs(do) * out_tol, 1, keepdims=True) + 2 * (hd + 4) * E * (np.abs(do) @ np.abs(w).T))
            val["dq"][a:b, h] = scale * ds @ y
            tol["dq"][a:b, h] = scale * (ds_tol + nk * E * np.abs(ds)) @ np.abs(y)
            val["dk"][c:d, g] += scale * ds.T @ x
            tol["dk"][c:d, g] += scale * (ds_tol + nq * H // KV * E * np.abs(ds)).T @ np.abs(x)
            val["dv"][c:d, g] += p.T @ do
            tol["dv"][c:d, g] += (p * (U + rel + nq * H // KV * E)).T @ np.abs(do)
    for name in ("dq", "dk", "dv"):
        if name in val:
            tol[name] += U * np.abs(val[name])
    return val, tol


def agree(name, got, val, tol):
    got = f64(got)
    assert np.array_equal(np.isneginf(got), np.isneginf(val)), name
    fine = np.isfinite(val)
    off, allowed = np.abs(got[fine] - val[fine]), tol[fine] + 1e-30
    assert np.all(off <= allowed), (name, float((off / allowed).max()), float(off.max()))


def make(lengths_q, lengths_k, H, KV, hd, seed, before=0, behind=0, spread=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    Tq = before + sum(lengths_q) + behind
    if lengths_k is None:
        x = torch.randn(Tq, H + 2 * KV, hd, generator=g, device=DEV).to(torch.bfloat16)
        q, k, v = x[:, :H], x[:, H:H + KV], x[:, H + KV:]
    else:
        q = torch.randn(Tq, H, hd, generator=g, device=DEV).to(torch.bfloat16)
        k, v = (torch.randn(before + sum(lengths_k) + behind, KV, hd, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    if spread != 1.0:
        q = (q * spread).to(torch.bfloat16)
    go = torch.randn(Tq, H, hd, generator=g, device=DEV).to(torch.bfloat16)
    cu_q = cu(lengths_q, before)
    return q, k, v, go, cu_q, None if lengths_k is None else cu(lengths_k, before)


def check(A, q, k, v, go, cu_q, cu_k, causal, scale=None):
    out, lse = A.arrol_attention(q, k, v, cu_q, cu_k, causal=causal, scale=scale)
    grad = A.arrol_attention_grad(q, k, v, out, lse, go, cu_q, cu_k, causal=causal, scale=scale)
    torch.cuda.synchronize()
    val, tol = reference(q, k, v, cu_q, cu_q if cu_k is None else cu_k, causal, q.shape[2] ** -0.5 if scale is None else scale, go)
    agree("out", out, val["out"], tol["out"])
    agree("lse", lse, val["lse"], tol["lse"])
    for name, key in (("dv", "grad_v"), ("dk", "grad_k"), ("dq", "grad_q")):
        agree(name, grad[key], val[name], tol[name])
    return out, lse, grad


@pytest.mark.parametrize("lengths", [[1], [2, 1, 1], [31, 32, 33], [0, 63, 0, 64, 65, 0], [127, 128, 129], [300, 7, 511], [1000]])
@pytest.mark.parametrize("H,KV,hd", [(2, 2, 64), (4, 1, 128), (6, 2, 40)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_sequences(A, lengths, H, KV, hd, causal):
    print("[case] attention lengths=%s heads=%d/%d hd=%d causal=%d" % (lengths, H, KV, hd, causal), flush=True)
    check(A, *make(lengths, None, H, KV, hd, sum(lengths) + hd), causal)


@pytest.mark.parametrize("hd", [8, 16, 56, 64, 72, 104, 120, 128])
def test_head_sizes(A, hd):
    print("[case] attention hd=%d" % hd, flush=True)
    check(A, *make([70, 130], None, 3, 3, hd, hd), True)


@pytest.mark.parametrize("H,KV", [(8, 1), (12, 2), (5, 1), (10, 5), (1, 1), (16, 16), (28, 4)])
def test_heads_over_kv_heads(A, H, KV):
    """A workgroup takes four, two or one of the heads that share a kv head."""
    print("[case] attention heads=%d/%d" % (H, KV), flush=True)
    check(A, *make([33, 1, 129, 64], None, H, KV, 64, H), True)
    check(A, *make([40, 3], [70, 300], H, KV, 128, H), True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk", [([1, 1], [500, 1]), ([5, 200, 33], [300, 200, 40]), ([130, 64, 10], [100, 0, 3]), ([40], [1]), ([0, 17], [90, 129])])
def test_keys_of_other_lengths_and_rows_that_see_nothing(A, nq, nk, causal):
    """The queries are the last rows of a longer context; where there are more of them than keys the first ones see nothing: zeros, -inf."""
    print("[case] attention nq=%s nk=%s causal=%d" % (nq, nk, causal), flush=True)
    out, lse, grad = check(A, *make(nq, nk, 4, 2, 64, sum(nk)), causal)
    if causal and nq[0] > nk[0]:
        blind = nq[0] - nk[0]
        assert not out[:blind].any() and not grad["grad_q"][:blind].any() and bool(torch.all(lse[:, :blind] == -float("inf")))


def test_rows_of_no_sequence_get_zeros_and_reach_nothing(A):
    print("[case] attention, rows outside the sequences hold NaN and infinities", flush=True)
    for lengths_k in (None, [50, 140]):
        q, k, v, go, cu_q, cu_k = make([45, 130], lengths_k, 4, 2, 64, 5, before=37, behind=150)
        last = 37 + 45 + 130
        clean = check(A, q, k, v, go, cu_q, cu_k, True)
        assert not clean[0][:37].any() and not clean[0][last:].any() and bool(torch.all(clean[1][:, last:] == -float("inf")))
        for bad in (float("nan"), float("inf")):
            x = [t.clone() for t in (q, k, v, go)]
            for t in x:
                t[:37], t[t.shape[0] - 150:] = bad, bad
            out, lse = A.arrol_attention(x[0], x[1], x[2], cu_q, cu_k)
            safe = out.clone()
            safe[:37], safe[last:] = bad, bad
            grad = A.arrol_attention_grad(x[0], x[1], x[2], safe, lse, x[3], cu_q, cu_k)
            torch.cuda.synchronize()
            assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
            for name in grad:
                assert torch.equal(grad[name], clean[2][name]), name


def test_a_sequence_of_nan_leaves_the_others(A):
    print("[case] attention, one sequence of NaN between two others", flush=True)
    q, k, v, go, cu_q, _ = make([100, 90, 110], None, 4, 2, 128, 6)
    clean = check(A, q, k, v, go, cu_q, None, True)
    x = [t.clone() for t in (q, k, v, go)]
    for t in x:
        t[100:190] = float("nan")
    out, lse = A.arrol_attention(x[0], x[1], x[2], cu_q)
    grad = A.arrol_attention_grad(x[0], x[1], x[2], out, lse, x[3], cu_q)
    torch.cuda.synchronize()
    rest = torch.cat([torch.arange(100), torch.arange(190, 300)]).to(DEV)
    assert torch.equal(out[rest], clean[0][rest]) and torch.equal(lse[:, rest], clean[1][:, rest]) and bool(torch.isnan(out[100:190]).all())
    for name in grad:
        assert torch.equal(grad[name][rest], clean[2][name][rest]), name


@pytest.mark.parametrize("spread", [0.0, 6.0, 40.0])
def test_flat_and_peaked_weights(A, spread):
    """All scores equal, and scores over many powers of e, whose running maximum moves on often."""
    print("[case] attention spread=%g" % spread, flush=True)
    check(A, *make([260, 75], None, 4, 2, 64, 9, spread=spread), True)
    check(A, *make([260, 75], None, 2, 1, 128, 9, spread=spread), False, scale=0.25)


def test_maximum_that_rises_with_every_key(A):
    print("[case] attention, rising scores", flush=True)
    n, hd = 400, 64
    q = torch.zeros(n, 1, hd, device=DEV)
    k = torch.zeros(n, 1, hd, device=DEV)
    q[:, :, 0] = 8.0
    k[:, 0, 0] = torch.arange(n, device=DEV) * 0.5
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    v, go = (torch.randn(n, 1, hd, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    for order in (k, -k):
        check(A, q.to(torch.bfloat16), order.to(torch.bfloat16), v, go, cu([n]), None, True, scale=1.0)


def test_gradient_agrees_with_differences(A):
    """Directional derivatives of <grad_out, out> in 64 bits by central differences (error h^2, h = 1e-4) against the gradient's."""
    print("[case] attention gradient against differences", flush=True)
    q, k, v, go, cu_q, cu_k = make([40, 33], [70, 50], 4, 2, 64, 12)
    out, lse = A.arrol_attention(q, k, v, cu_q, cu_k)
    grad = A.arrol_attention_grad(q, k, v, out, lse, go, cu_q, cu_k)
    _, tol = reference(q, k, v, cu_q, cu_k, True, 0.125, go)
    loss = lambda *x: float(np.sum(f64(go) * reference(*x, cu_q, cu_k, True, 0.125)[0]["out"]))
    rng = np.random.default_rng(4)
    base = [t.double().cpu() for t in (q, k, v)]
    for which, name, short in ((0, "grad_q", "dq"), (1, "grad_k", "dk"), (2, "grad_v", "dv")):
        for _ in range(3):
            step = torch.from_numpy(rng.standard_normal(tuple(base[which].shape)))
            side = []
            for sign in (1, -1):
                x = list(base)
                x[which] = base[which] + sign * 1e-4 * step
                side.append(loss(*x))
            want, got = (side[0] - side[1]) / 2e-4, float((grad[name].double().cpu() * step).sum())
            assert abs(got - want) <= float(np.sum(tol[short] * np.abs(step.numpy()))) + 1e-4 * abs(want) + 1e-3, (name, got, want)


@pytest.mark.parametrize("nq,nk,H,KV,hd", [([1, 200, 33], [5000, 3000, 4097], 4, 2, 64), ([150], [9000], 2, 1, 128), ([64, 0, 7], [2600, 2000, 7], 1, 1, 72), ([2000], None, 2, 2, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_few_queries_over_many_keys_in_ranges(A, nq, nk, H, KV, hd, causal):
    """Given its workspace the call cuts the keys; without it one workgroup walks over all of them.  Both are held to the reference."""
    print("[case] attention in ranges nq=%s nk=%s causal=%d" % (nq, nk, causal), flush=True)
    q, k, v, go, cu_q, cu_k = make(nq, nk, H, KV, hd, 77, before=3, behind=2)
    assert A.lib().arrol_attention_workspace_bytes(q.shape[0], k.shape[0], len(nq), H, hd) > 0
    val, tol = reference(q, k, v, cu_q, cu_q if cu_k is None else cu_k, causal, hd ** -0.5)
    for workspace in ("auto", None):
        out, lse = A.arrol_attention(q, k, v, cu_q, cu_k, causal=causal, workspace=workspace)
        torch.cuda.synchronize()
        agree("out", out, val["out"], tol["out"])
        agree("lse", lse, val["lse"], tol["lse"])


@pytest.mark.parametrize("nq,nk,H,KV,hd", [([1100], None, 4, 1, 64), ([900, 70], None, 2, 2, 128), ([700, 1, 0], [1500, 900, 300], 3, 1, 72), ([60], [2500], 2, 1, 128), ([2500], [64], 4, 2, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_gradient_of_few_heads_in_ranges(A, nq, nk, H, KV, hd, causal):
    """Few workgroups: the walks over keys and queries are cut, and the ranges' sums added."""
    print("[case] attention gradient in ranges nq=%s nk=%s heads=%d/%d hd=%d causal=%d" % (nq, nk, H, KV, hd, causal), flush=True)
    args = make(nq, nk, H, KV, hd, 78, before=5, behind=1)
    T = args[0].shape[0]
    assert A.lib().arrol_attention_grad_workspace_bytes(T, args[1].shape[0], len(nq), H, KV, hd) > 2 * T * H * 4 + 16
    check(A, *args, causal)
    check(A, *args, causal)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("lengths,ranges", [([70, 200, 33], None), ([100], [6000])])
def test_keys_that_a_query_does_not_see_take_no_part(A, lengths, ranges, bad):
    """NaN and infinities in some keys and values: rows that do not see them are what they are without, and the others no numbers."""
    print("[case] attention, %g in hidden keys" % bad, flush=True)
    q, k, v, _, cu_q, cu_k = make(lengths, ranges, 4, 2, 128 if ranges else 64, 5)
    clean = A.arrol_attention(q, k, v, cu_q, cu_k)
    ends, starts = npy(cu_q if cu_k is None else cu_k)[1:], npy(cu_q)[:-1]
    for where in ("k", "v", "both"):
        x, y = k.clone(), v.clone()
        spoiled = [(s, end - back) for s, end in enumerate(ends) for back in (1, 9)]
        for s, at in spoiled:
            if where != "v":
                x[at] = bad
            if where != "k":
                y[at, :, 3::7] = bad
        out, lse = A.arrol_attention(q, x, y, cu_q, cu_k)
        torch.cuda.synchronize()
        for s, n in enumerate(lengths):
            good = torch.arange(starts[s], starts[s] + n - 9, device=DEV)          # the row 9 from the end sees the first spoiled key
            assert torch.equal(lse[:, good], clean[1][:, good]), where
            off = (out[good].float() - clean[0][good].float()).abs()
            assert bool((off <= 2 * U * clean[0][good].float().abs() + U * 4.0).all()) and bool(torch.isfinite(out[good].float()).all()), where
            last = out[starts[s] + n - 1].float()
            assert not bool(torch.isfinite(last if where == "k" and bad != -float("inf") else last[:, 3::7] if where != "k" else torch.full((1,), float("nan"))).any()), where


def test_calls_repeat_bit_for_bit_on_a_side_stream_and_in_a_graph(A):
    print("[case] attention repeated, on a side stream, captured", flush=True)
    q, k, v, go, cu_q, _ = make([200, 90, 333], None, 4, 2, 128, 21)
    out, lse = A.arrol_attention(q, k, v, cu_q)
    grad = A.arrol_attention_grad(q, k, v, out, lse, go, cu_q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out2, lse2 = A.arrol_attention(q, k, v, cu_q, stream=side)
    grad2 = A.arrol_attention_grad(q, k, v, out2, lse2, go, cu_q, stream=side)
    junk = [torch.full((4, 623), float("nan"), device=DEV) for _ in range(8)]
    side.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(grad[n], grad2[n]) for n in grad)
    del junk
    x = [t.clone() for t in (q, k, v, go)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g_out, g_lse = A.arrol_attention(x[0], x[1], x[2], cu_q)
        g_grad = A.arrol_attention_grad(x[0], x[1], x[2], g_out, g_lse, x[3], cu_q)
    for seed in (21, 22, 23):
        fresh = make([200, 90, 333], None, 4, 2, 128, seed)
        want_out, want_lse = A.arrol_attention(*fresh[:3], fresh[4])
        want = A.arrol_attention_grad(*fresh[:3], want_out, want_lse, fresh[3], fresh[4])
        for t, s in zip(x, fresh):
            t.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(g_out, want_out) and torch.equal(g_lse, want_lse) and all(torch.equal(g_grad[n], want[n]) for n in want), seed


def test_offsets_out_of_range_and_out_of_order_stay_inside(A):
    """Offsets are clamped into [0, T]; what comes out is not defined, but nothing outside the buffers is touched."""
    print("[case] attention, bad offsets", flush=True)
    q, k, v, go, _, _ = make([300], None, 4, 2, 64, 2)
    for bad in ([-5, 100, 10 ** 12], [300, 200, 0], [0, -2 ** 62, 2 ** 62, 17], [2 ** 62, -1]):
        offsets = torch.tensor(bad, dtype=torch.int64, device=DEV)
        guard = torch.zeros(300 + 64, 4, 64, dtype=torch.bfloat16, device=DEV)
        out, lse = A.arrol_attention(q, k, v, offsets, out=guard[:300])
        grad = A.arrol_attention_grad(q, k, v, out, lse, go, offsets)
        torch.cuda.synchronize()
        assert not guard[300:].any() and grad["grad_q"].shape == q.shape
    out, lse = A.arrol_attention(q, k, v, torch.tensor([-5, 10 ** 12], dtype=torch.int64, device=DEV))
    want, want_lse = A.arrol_attention(q, k, v, cu([300]))
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_empty_batches(A):
    print("[case] attention, no rows", flush=True)
    q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    out, lse = A.arrol_attention(q, k, k, cu([0]))
    grad = A.arrol_attention_grad(q, k, k, out, lse, out, cu([0]))
    assert out.shape == q.shape and lse.shape == (4, 0) and grad["grad_k"].shape == k.shape
    q = torch.randn(9, 4, 64, device=DEV).to(torch.bfloat16)
    out, lse = A.arrol_attention(q, k, k, cu([9]), cu([0]))           # no keys at all
    grad = A.arrol_attention_grad(q, k, k, out, lse, q, cu([9]), cu([0]))
    torch.cuda.synchronize()
    assert not out.any() and bool(torch.all(lse == -float("inf"))) and not grad["grad_q"].any()
    k = torch.randn(9, 2, 64, device=DEV).to(torch.bfloat16)
    grad = A.arrol_attention_grad(q[:0], k, k, q[:0], lse[:, :0], q[:0], cu([0]), cu([9]))      # keys that nobody reads
    torch.cuda.synchronize()
    assert not grad["grad_k"].any() and not grad["grad_v"].any()
    out, lse = A.arrol_attention(q, k, k, torch.zeros(1, dtype=torch.int64, device=DEV))        # no sequences
    torch.cuda.synchronize()
    assert not out.any() and bool(torch.all(lse == -float("inf")))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk,H,KV,hd,one", [([60], [2500], 2, 1, 128, (512, 832)), ([20, 3], [5000, 2000], 4, 2, 64, (768, 1152))])      # one: keys of one range
def test_nan_is_not_lost_between_ranges(A, nq, nk, H, KV, hd, one, causal):
    """A query, or the keys of a range, whose scores are all NaN: no number comes out, with the keys in ranges as without."""
    print("[case] attention in ranges, NaN, nq=%s nk=%s causal=%d" % (nq, nk, causal), flush=True)
    q, k, v, _, cu_q, cu_k = make(nq, nk, H, KV, hd, 64)
    assert A.lib().arrol_attention_workspace_bytes(q.shape[0], k.shape[0], len(nq), H, hd) > 0
    val, tol = reference(q, k, v, cu_q, cu_k, causal, hd ** -0.5)
    x, y = q.clone(), k.clone()
    x[5], x[7, 1] = float("nan"), float("nan")
    y[one[0]:one[1]] = float("nan")
    for workspace in ("auto", None):
        out, lse = A.arrol_attention(x, k, v, cu_q, cu_k, causal=causal, workspace=workspace)
        torch.cuda.synchronize()
        spoiled = torch.zeros(q.shape[0], H, dtype=torch.bool)
        spoiled[5], spoiled[7, 1] = True, True
        assert torch.equal(torch.isnan(out).all(2).cpu(), spoiled) and torch.equal(torch.isnan(lse).t().cpu(), spoiled), workspace
        good = ~spoiled.numpy()
        agree("out", out[~spoiled.to(DEV)], val["out"][good], tol["out"][good])
        agree("lse", lse.t()[~spoiled.to(DEV)], val["lse"].T[good], tol["lse"].T[good])
        out, lse = A.arrol_attention(q, y, v, cu_q, cu_k, causal=causal, workspace=workspace)
        torch.cuda.synchronize()
        assert bool(torch.isnan(out[:nq[0]]).all()) and bool(torch.isnan(lse[:, :nq[0]]).all()), workspace
        agree("out", out[nq[0]:], val["out"][nq[0]:], tol["out"][nq[0]:])


@pytest.mark.parametrize("bad", [float("inf"), -float("inf")])
@pytest.mark.parametrize("nq,nk,causal", [([1], [70], True), ([40], [70], False), ([1, 9], [129, 33], True), ([33], [2601], False), ([3], [2], False)])
@pytest.mark.parametrize("hd", [64, 72, 128])
def test_an_infinite_value_gives_an_infinite_output(A, nq, nk, causal, hd, bad):
    """Also where it is the last key's, which stands for the missing ones of a tile: their weight is 0, and 0 times infinity would be NaN."""
    print("[case] attention, infinite values, nq=%s nk=%s causal=%d hd=%d" % (nq, nk, causal, hd), flush=True)
    q, k, v, _, cu_q, cu_k = make(nq, nk, 4, 2, hd, 66)
    val, tol = reference(q, k, v, cu_q, cu_k, causal, hd ** -0.5)
    v[nk[0] - 1, 1, 3::5] = bad                                     # the first sequence's last key, second kv head
    expect = np.zeros(val["out"].shape, bool)
    expect[nq[0] - 1 if causal else 0:nq[0], 2:, 3::5] = True
    for workspace in ("auto", None):
        out, lse = A.arrol_attention(q, k, v, cu_q, cu_k, causal=causal, workspace=workspace)
        torch.cuda.synchronize()
        got = f64(out)
        assert np.array_equal(np.isinf(got), expect) and np.all(got[expect] == bad), workspace
        agree("out", out[torch.from_numpy(~expect).to(DEV)], val["out"][~expect], tol["out"][~expect])
        agree("lse", lse, val["lse"], tol["lse"])


@pytest.mark.parametrize("hd", [8, 40, 64, 72, 120, 128])
@pytest.mark.parametrize("nq,nk", [([40, 3], [150, 64]), ([30], [2600])])
def test_a_key_of_minus_infinity_has_no_weight(A, nq, nk, hd):
    """Its score is -inf, and nothing else: what a head is padded with counts 0 in the products."""
    print("[case] attention, keys of -inf, hd=%d nk=%s" % (hd, nk), flush=True)
    q, k, v, go, cu_q, cu_k = make(nq, nk, 4, 2, hd, 65)
    q[:, :, hd - 1] = q[:, :, hd - 1].abs() + 0.5
    hidden = [0, 37, nk[0] - 1]                                     # of the first sequence
    rest = torch.tensor([j for j in range(k.shape[0]) if j not in hidden], device=DEV)
    ends = cu([nk[0] - len(hidden)] + nk[1:])
    val, tol = reference(q, k[rest], v[rest], cu_q, ends, False, hd ** -0.5, go)      # as if they were not there
    k[hidden, :, hd - 1] = -float("inf")
    for workspace in ("auto", None):
        out, lse = A.arrol_attention(q, k, v, cu_q, cu_k, causal=False, workspace=workspace)
        torch.cuda.synchronize()
        agree("out", out, val["out"], tol["out"])
        agree("lse", lse, val["lse"], tol["lse"])
    grad = A.arrol_attention_grad(q, k, v, out, lse, go, cu_q, cu_k, causal=False)
    torch.cuda.synchronize()
    agree("dv", grad["grad_v"][rest], val["dv"], tol["dv"])         # (dq has 0 times infinity in it)
    agree("dk", grad["grad_k"][rest], val["dk"], tol["dk"])
    assert not grad["grad_v"][hidden].any() and not grad["grad_k"][hidden].any()


@pytest.mark.parametrize("more", [0, 1, 31, 32, 40])
@pytest.mark.parametrize("hd", [64, 128])
def test_how_far_nan_reaches_in_the_gradients_of_a_sequence(A, more, hd):
    """Products are made of 32 queries and 32 keys at a time: a NaN may reach rows that do not see it, up to 62 beyond those that do, and no others."""
    print("[case] attention gradient, reach of NaN, nk - nq = %d, hd=%d" % (more, hd), flush=True)
    n = 300
    q, k, v, go, cu_q, cu_k = make([n], [n + more], 2, 1, hd, 69)
    for at in (0, 31, 32, 150, 191, n - 1):
        x, y = go.clone(), k.clone()
        x[at] = float("nan")                                    # query `at` sees the keys up to at + more
        out, lse = A.arrol_attention(q, k, v, cu_q, cu_k)
        grad = A.arrol_attention_grad(q, k, v, out, lse, x, cu_q, cu_k)
        y[at + more] = float("nan")                             # seen by the queries from `at` on
        out, lse = A.arrol_attention(q, y, v, cu_q, cu_k)
        other = A.arrol_attention_grad(q, y, v, out, lse, go, cu_q, cu_k)
        torch.cuda.synchronize()
        odd = lambda t: torch.isnan(t).flatten(1).any(1).cpu().numpy()
        assert np.array_equal(odd(grad["grad_q"]), np.arange(n) == at)
        for name in ("grad_k", "grad_v"):
            got = odd(grad[name])
            assert got[:at + more + 1].all() and not got[at + more + 63:].any(), (name, at)
        got = odd(other["grad_q"])
        assert got[at:].all() and not got[:max(0, at - 62)].any(), at
        assert not np.isnan(f64(out)[:at]).any()


def test_gradient_along_itself_agrees_with_differences(A):
    """The step is the 64-bit gradient, normalised, so the derivative along it is that gradient's norm: central differences in 64 bits (h = 1e-4) give that to
    1e-6, and the kernel's gradient lies, in norm, within its elements' tolerances.  A gradient of zeros, half of it or its negative is further off than those."""
    print("[case] attention gradient along itself", flush=True)
    q, k, v, go, cu_q, cu_k = make([40, 33], [70, 50], 4, 2, 64, 12)
    out, lse = A.arrol_attention(q, k, v, cu_q, cu_k)
    grad = A.arrol_attention_grad(q, k, v, out, lse, go, cu_q, cu_k)
    torch.cuda.synchronize()
    along_itself({name: f64(x) for name, x in grad.items()}, q, k, v, go, cu_q, cu_k)


def along_itself(grad, q, k, v, go, cu_q, cu_k):
    val, tol = reference(q, k, v, cu_q, cu_k, True, 0.125, go)
    loss = lambda *x: float(np.sum(f64(go) * reference(*x, cu_q, cu_k, True, 0.125)[0]["out"]))
    base = [t.double().cpu() for t in (q, k, v)]
    for which, name, short in ((0, "grad_q", "dq"), (1, "grad_k", "dk"), (2, "grad_v", "dv")):
        norm = float(np.linalg.norm(val[short]))
        step = torch.from_numpy(val[short] / norm)
        side = []
        for sign in (1, -1):
            x = list(base)
            x[which] = base[which] + sign * 1e-4 * step
            side.append(loss(*x))
        assert abs((side[0] - side[1]) / 2e-4 - norm) <= 1e-6 * norm, name
        allowed = float(np.linalg.norm(tol[short]))
        assert np.linalg.norm(grad[name] - val[short]) <= allowed, name
        for wrong in (0.0, 0.5, -1.0):
            assert np.linalg.norm(wrong * val[short] - val[short]) > allowed, (name, wrong)


@pytest.mark.parametrize("H,KV,hd,T", [(4, 2, 64, 300), (2, 1, 128, 900)])
def test_bad_offsets_leave_what_lies_around_the_buffers(A, H, KV, hd, T):
    """Every output and both workspaces inside larger allocations whose other bytes stay as they were."""
    print("[case] attention and its gradient, bad offsets, guarded buffers, T=%d" % T, flush=True)
    q, k, v, go, _, _ = make([T], None, H, KV, hd, 2)
    L, pad, mark = A.lib(), 4096, 0x5A

    def inside(nbytes):
        whole = torch.full((pad + nbytes + pad,), mark, dtype=torch.uint8, device=DEV)
        return whole, whole[pad:pad + nbytes]

    for bad in ([-5, 100, 10 ** 12], [T, 200, 0], [0, -2 ** 62, 2 ** 62, 17], [2 ** 62, -1], [0, T + 1], [T // 2, T // 2, 10 ** 9, 3]):
        offsets = torch.tensor(bad, dtype=torch.int64, device=DEV)
        n = len(bad) - 1
        need = L.arrol_attention_workspace_bytes(T, T, n, H, hd), L.arrol_attention_grad_workspace_bytes(T, T, n, H, KV, hd)
        buffers = [inside(x) for x in (T * H * hd * 2, H * T * 4, need[0], T * H * hd * 2, T * KV * hd * 2, T * KV * hd * 2, need[1])]
        out, lse, ws, gq, gk, gv, gws = (x.data_ptr() if x.numel() else None for _, x in buffers)
        st = torch.cuda.current_stream().cuda_stream
        ends = (offsets.data_ptr(), None, T, T, n, H, KV, hd, 1, 0.125)
        rows = (q.data_ptr(), q.stride(0), k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0))
        assert L.arrol_attention(*rows, *ends, out, lse, ws, need[0], st) == 0
        assert L.arrol_attention_grad(*rows, out, lse, go.data_ptr(), *ends, gq, gk, gv, gws, need[1], st) == 0
        torch.cuda.synchronize()
        for whole, part in buffers:
            assert bool((whole[:pad] == mark).all()) and bool((whole[pad + part.numel():] == mark).all()), bad


def test_batches_past_2_31_elements(A):
    """Rows whose offsets into a fused projection, the output and the gradients pass 2^31 elements (2^32 bytes): the last sequences as if they were alone."""
    print("[case] attention, 6.5e9 elements of a projection", flush=True)
    H, hd, short = 64, 128, [64, 33, 70]
    q, k, v, go, cu_q, _ = make(short, None, H, H, hd, 67)
    want, want_lse = A.arrol_attention(q, k, v, cu_q, workspace=None)
    grads = A.arrol_attention_grad(q, k, v, want, want_lse, go, cu_q)
    n = 4150
    lengths = [64] * n + short
    T, last = sum(lengths), sum(short)
    qkv = torch.zeros(T, 3 * H, hd, dtype=torch.bfloat16, device=DEV)
    many = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
    for x, y in zip(many, (q, k, v)):
        x[T - last:] = y
    many_go = torch.zeros(T, H, hd, dtype=torch.bfloat16, device=DEV)
    many_go[T - last:] = go
    assert T * H * hd > 2 ** 31
    out, lse = A.arrol_attention(*many, cu(lengths))
    got = A.arrol_attention_grad(*many, out, lse, many_go, cu(lengths))
    torch.cuda.synchronize()
    assert torch.equal(out[T - last:], want) and torch.equal(lse[:, T - last:], want_lse) and not out[:T - last].any()
    for name in got:
        assert torch.equal(got[name][T - last:], grads[name]) and not got[name][:T - last].any(), name
