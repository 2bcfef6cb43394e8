"""The gradient of the log-probabilities against a plain implementation in 64 bits and against differences.

Tolerances, element by element (u = 2^-8 for bf16, e = 2^-24 for fp32), derived before the first run:
  z        d products summed in fp32: dz_ = (d + 4) e sum |w||h|
  p        relatively dz_, the argument of the exponential (lse scaled, and the sum: 4 e (|z| + |lse|)) and the exponential, 2^-21: r
  dz       u of itself (rounded to bf16), |g| p r, and at the target 4 e |g|
  dH, dW   what dz is off by times |w|, |h|; n e of the terms' size for n terms (and slabs) summed in fp32; u of the result
and in norm u: the roundings of dz and of the result are off by at most u / sqrt(3) of the values each in the root mean square, and not correlated.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, E = 2.0 ** -8, 2.0 ** -24


@pytest.fixture(scope="module")
def A():
    import paper_2603_24840_amd as pkg
    pkg.lib()
    return pkg


def make(T, V, d, seed=0, sure=8.0, idle=0.2):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    w = (torch.randn(V, d, generator=g, device=DEV) * d ** -0.5).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    h = (torch.randn(T, d, generator=g, device=DEV) + sure * torch.rand(T, 1, generator=g, device=DEV) * w[y.long()].float()).to(torch.bfloat16)
    grad = torch.randn(T, generator=g, device=DEV) * (torch.rand(T, generator=g, device=DEV) >= idle)
    lse = torch.cat([torch.logsumexp(h[a:a + 1024].double() @ w.double().t(), 1) for a in range(0, max(T, 1), 1024)]).float()
    return h, w, y, lse, grad


def reference(h, w, y, lse, g):
    """(dH, its tolerance, dW, its tolerance) in 64 bits, of the tokens that take part."""
    T, V, d = h.shape[0], w.shape[0], h.shape[1]
    on = (g != 0) & (y >= 0) & (y < V)
    w64 = w.double()
    dH, tH = (torch.zeros(T, d, dtype=torch.float64, device=DEV) for _ in range(2))
    dW, tW = (torch.zeros(V, d, dtype=torch.float64, device=DEV) for _ in range(2))
    rows = torch.nonzero(on)[:, 0]
    for some in rows.split(2048):
        x, gg, l, t = h[some].double(), g[some].double()[:, None], lse[some].double()[:, None], y[some].long()
        z = x @ w64.t()
        p = torch.exp(z - l)
        hit = torch.zeros_like(z).scatter_(1, t[:, None], 1.0)
        dz = gg * (hit - p)
        r = (d + 4) * E * (x.abs() @ w64.abs().t()) + 4 * E * (z.abs() + l.abs()) + 2.0 ** -21
        off = U * dz.abs() + gg.abs() * (p * r + 4 * E * hit)
        dH[some] = dz @ w64
        tH[some] = (off + (V + 40) * E * dz.abs()) @ w64.abs()
        dW += dz.t() @ x
        tW += (off + (rows.numel() + 40) * E * dz.abs()).t() @ x.abs()
    return dH, tH + U * dH.abs(), dW, tW + U * dW.abs()


def agree(name, got, val, tol, norm=True):
    got = got.double()
    off = (got - val).abs()
    assert bool((off <= tol + 1e-30).all()), (name, float((off / (tol + 1e-30)).max()), float(off.max()))
    if norm and val.numel() >= 4096 and float(val.norm()) > 0:
        assert float((got - val).norm() / val.norm()) <= U, (name, float((got - val).norm() / val.norm()))


def check(A, h, w, y, lse, g, norm=True):
    got = A.arrol_logprob_grad(h, w, y, lse, g)
    torch.cuda.synchronize()
    dH, tH, dW, tW = reference(h, w, y, lse, g)
    norm = norm and int((g != 0).sum()) >= 64       # of few tokens a single rounding counts, which may be u
    agree("grad_hidden", got["grad_hidden"], dH, tH, norm)
    agree("grad_lm_head", got["grad_lm_head"], dW, tW, norm)
    return got


@pytest.mark.parametrize("T,V,d", [(1, 1, 8), (1, 2, 64), (2, 300, 64), (3, 257, 72), (17, 1000, 8), (64, 255, 128), (70, 1000, 256), (255, 256, 264), (256, 512, 192), (257, 255, 512),
                                   (300, 513, 520), (1000, 4096, 64), (33, 5000, 1024), (513, 1025, 320), (1100, 300, 1088), (5, 20000, 2048), (600, 70, 4096), (12, 40, 16384)])
def test_gradient(A, T, V, d):
    print("[case] logprob_grad T=%d V=%d d=%d" % (T, V, d), flush=True)
    check(A, *make(T, V, d, seed=T + V))


KERNELS = [(1211, 46, 8), (2044, 41, 8), (19579, 39, 8), (3047, 516, 8), (5, 538, 5376), (3, 7073, 408), (811, 43, 4944), (215, 5014, 1216), (984, 1231, 3960), (202, 3792, 2816),
           (1022, 2639, 368), (225, 15340, 664), (467, 9258, 568), (394, 14224, 448), (1152, 11261, 536), (4392, 3092, 192), (4025, 2946, 576), (2579, 3172, 1728), (724, 17984, 384),
           (15386, 6011, 192), (1046, 3757, 8), (131, 51545, 8), (1948, 4612, 8), (146, 6790, 1016), (155, 60441, 280), (74, 58503, 264), (311, 60001, 264), (1, 60000, 264),
           (239, 8272, 3792), (53, 7924, 3992), (9, 140000, 960)]


def kernels(A, T, V, d):
    """What the call takes, as the header numbers it."""
    import ctypes
    out = [ctypes.c_int32() for _ in range(8)]
    assert A.lib().arrol_logprob_grad_kernels(T, V, d, *[ctypes.byref(x) for x in out]) == 0
    names = ("logit_rows", "logit_tokens", "product_columns", "product_tokens", "slabs", "parts", "pieces", "found")
    return dict(zip(names, [x.value for x in out]))


@pytest.mark.parametrize("T,V,d", KERNELS)
def test_gradient_in_every_form(A, T, V, d):
    print("[case] logprob_grad T=%d V=%d d=%d %s" % (T, V, d, kernels(A, T, V, d)), flush=True)
    h, w, y, lse, g = make(T, V, d, seed=T + d)
    check(A, h, w, y, lse, g)
    total = torch.full((V, d), -1.0, device=DEV)
    A.arrol_logprob_grad(h, w, y, lse, g, want_hidden=False, lm_head_sum=total)
    dW, tW = reference(h, w, y, lse, g)[2:]
    agree("lm_head_sum", total, dW - 1, tW + 8 * E * (1 + dW.abs()), norm=False)


def test_every_form_is_reached(A):
    got = [kernels(A, *x) for x in KERNELS]
    tiles = {(256, 256), (128, 160), (128, 128), (128, 64), (64, 64)}
    assert {(k["logit_rows"], k["logit_tokens"]) for k in got} == tiles and {(k["product_columns"], k["product_tokens"]) for k in got} == tiles
    assert {(k["logit_rows"], k["logit_tokens"]) for k in got if k["found"]} == tiles - {(256, 256)} and {(k["logit_rows"], k["logit_tokens"]) for k in got if not k["found"]} == tiles
    assert {(k["slabs"] > 1, k["parts"] > 1) for k in got} == {(a, b) for a in (False, True) for b in (False, True)} and any(k["pieces"] > 1 and k["parts"] > 1 for k in got)
    assert {(k["product_columns"], k["product_tokens"]) for k in got if k["parts"] == 0} == tiles - {(256, 256)}


@pytest.mark.parametrize("target", ["any", "one", "near"])
@pytest.mark.parametrize("T,V,d", [(50, 542, 376), (7, 900, 2048), (320, 9000, 136), (480, 9000, 136), (512, 5000, 256), (320, 700, 1024), (1000, 1000, 512), (60, 60001, 264), (320, 60001, 264)])
def test_few_tokens_are_off_by_the_result_s_rounding_alone(A, T, V, d, target):
    """In norm: u / sqrt(3) of the result, the root mean square of a rounding at worst, and as much of what dz holds elsewhere than at the targets, whose roundings are added back."""
    print("[case] logprob_grad few tokens T=%d V=%d d=%d, targets %s, %s" % (T, V, d, target, kernels(A, T, V, d)), flush=True)
    h, w, y, lse, g = make(T, V, d, seed=21, sure=0.0, idle=0.1)
    if target != "any":
        y = torch.full_like(y, V - 3) if target == "one" else (V - 40 + y % 40)
    got = A.arrol_logprob_grad(h, w, y, lse, g)
    h64, w64 = h.double(), w.double()
    dz = -g.double()[:, None] * torch.exp(h64 @ w64.t() - lse.double()[:, None])
    other = dz * (1 - torch.zeros_like(dz).scatter_(1, y.long()[:, None], 1.0))
    dz.scatter_add_(1, y.long()[:, None], g.double()[:, None])
    for name, want, spread in (("grad_hidden", dz @ w64, other.pow(2) @ w64.pow(2).sum(1)), ("grad_lm_head", dz.t() @ h64, other.pow(2).sum(1) * h64.pow(2).sum(1))):
        if name == "grad_lm_head" and T > 320:
            continue
        bound = U / 3 ** 0.5 * (float(want.norm()) + float(spread.sum()) ** 0.5)
        assert float((got[name].double() - want).norm()) <= bound, (name, float((got[name].double() - want).norm()) / float(want.norm()), bound / float(want.norm()))


FEW = [(724, 17984, 384), (900, 69999, 1984), (330, 140001, 968), (843, 556, 1928), (332, 515, 2848), (934, 27627, 72), (330, 1200001, 120), (771, 270492, 80),           # dL/dh
       (194, 3396, 2816), (202, 3517, 1856), (137, 1113, 2728), (258, 5487, 1064), (72, 79901, 264), (1, 317915, 104), (40, 103018, 296),                                           # both
       (300, 600001, 264), (90, 1134480, 72), (297, 878561, 72), (8, 1065945, 16), (2, 1268440, 144)]                                                            # pieces of the vocabulary


@pytest.mark.parametrize("target", ["any", "one", "near"])
@pytest.mark.parametrize("T,V,d", FEW)
def test_few_tokens_in_the_other_forms(A, T, V, d, target):
    test_few_tokens_are_off_by_the_result_s_rounding_alone(A, T, V, d, target)


def test_every_form_has_few_tokens(A):
    """What the roundings at the targets are added in: dL/dh up to 1,024 tokens, dL/dW up to 320 in tiles of the same, of 128 x 128 for the middle ones, or resident."""
    got = [(T, kernels(A, T, V, d)) for T, V, d in FEW]
    tiles = {(256, 256), (128, 160), (128, 128), (128, 64), (64, 64)}
    form = lambda k: (k["product_columns"], k["product_tokens"])
    assert {form(k) for _, k in got} == tiles and {k["slabs"] > 1 for _, k in got} == {False, True} and all(T <= 1024 for T, _ in got)
    assert {form(k) for T, k in got if T <= 320 and k["parts"] == 1} == tiles and {form(k) for T, k in got if k["parts"] == 0} == tiles - {(256, 256)}
    assert {(T <= 320, k["parts"] == 0) for T, k in got if k["pieces"] > 1} == {(False, False), (True, False), (True, True)}


@pytest.mark.parametrize("target", ["any", "one", "near"])
@pytest.mark.parametrize("T,V,d", [(1100, 5000, 1088), (1153, 11261, 536), (2100, 700, 320), (4025, 2946, 576), (5130, 32000, 512), (16384, 20000, 64), (33000, 1700, 72)])
def test_hidden_gradient_of_many_tokens_is_off_by_its_rounding_alone(A, T, V, d, target):
    """No number of tokens averages out what dz loses at a token's target, which is a row of W of that token's alone."""
    test_few_tokens_are_off_by_the_result_s_rounding_alone(A, T, V, d, target)


@pytest.mark.parametrize("T,V,d", [(320, 60001, 264), (65, 30016, 1000)])
def test_few_tokens_of_a_large_vocabulary(A, T, V, d):
    """The hidden states of all tokens in registers: as many tokens as fit, as few as none, a workspace of NaN, NaN of one that takes part."""
    print("[case] logprob_grad resident T=%d V=%d d=%d" % (T, V, d), flush=True)
    assert kernels(A, T, V, d)["parts"] == 0
    h, w, y, lse, g = make(T, V, d, seed=11, idle=0)
    ws = torch.full((A.lib().arrol_logprob_grad_workspace_bytes(T, V, d, 1),), 255, dtype=torch.uint8, device=DEV)
    want = check(A, h, w, y, lse, g)
    got = A.arrol_logprob_grad(h, w, y, lse, g, workspace=ws)
    assert all(torch.equal(want[x], got[x]) for x in want)
    assert torch.equal(A.arrol_logprob_grad(h, w, y, lse, g, want_hidden=False)["grad_lm_head"], want["grad_lm_head"])
    one = torch.zeros_like(g)
    one[T - 1] = g[T - 1]
    check(A, h, w, y, lse, one)
    total = torch.full((V, d), 2.0, device=DEV)
    got = A.arrol_logprob_grad(h, w, y, lse, torch.zeros_like(g), workspace=ws)
    A.arrol_logprob_grad(h, w, y, lse, torch.zeros_like(g), lm_head_sum=total)
    assert not got["grad_hidden"].any() and not got["grad_lm_head"].any() and bool((total == 2).all())
    x = h.clone()
    x[T // 2, 5] = float("nan")
    got = A.arrol_logprob_grad(x, w, y, lse, g)
    others = torch.arange(T, device=DEV) != T // 2
    assert torch.equal(got["grad_hidden"][others], want["grad_hidden"][others]) and bool(torch.isnan(got["grad_lm_head"]).all())


@pytest.mark.parametrize("T,V,d", [(330, 140001, 968), (900, 69999, 1984), (330, 1200001, 120), (300, 600001, 264)])
def test_gradient_larger_than_the_caches(A, T, V, d):
    """An LM head's gradient that is stored past the caches, of odd sizes and in several forms."""
    print("[case] logprob_grad past the caches T=%d V=%d d=%d %s" % (T, V, d, kernels(A, T, V, d)), flush=True)
    assert V * d > 2 ** 27
    check(A, *make(T, V, d, seed=5))


@pytest.mark.parametrize("T,V,d", [(16385, 300, 64), (16384, 20000, 64), (33000, 17000, 72)])
def test_gradient_in_pieces(A, T, V, d):
    """More than 16,384 tokens, and more than 2^28 values of dz."""
    print("[case] logprob_grad in pieces T=%d V=%d d=%d" % (T, V, d), flush=True)
    h, w, y, lse, g = make(T, V, d, seed=T)
    got = check(A, h, w, y, lse, g)
    total = torch.ones(V, d, device=DEV)
    more = A.arrol_logprob_grad(h, w, y, lse, g, lm_head_sum=total)
    assert more["grad_lm_head"] is None and torch.equal(more["grad_hidden"], got["grad_hidden"])
    dW, tW = reference(h, w, y, lse, g)[2:]
    agree("lm_head_sum", total, dW + 1, tW + 8 * E * (1 + dW.abs()), norm=False)


@pytest.mark.parametrize("scale", [0.0, 20.0, 200.0])
def test_flat_and_certain_distributions(A, scale):
    print("[case] logprob_grad logits x %g" % scale, flush=True)
    h, w, y, lse, g = make(200, 900, 128, seed=9)
    h = (h.float() * scale).to(torch.bfloat16)
    lse = torch.logsumexp(h.double() @ w.double().t(), 1).float()
    check(A, h, w, y, lse, g, norm=scale < 1)       # a rounding of lse of 1,000 is one of 1 - p near 1: the elementwise bound has it


@pytest.mark.parametrize("d", [128, 72])
@pytest.mark.parametrize("share", [0.0, 0.5, 0.97, 1.0])
def test_tokens_that_take_no_part(A, d, share):
    """Zero gradients and targets outside the vocabulary, with NaN and infinities in what belongs to them."""
    print("[case] logprob_grad d=%d, %g of the tokens off" % (d, share), flush=True)
    T, V = 700, 600
    h, w, y, lse, g = make(T, V, d, seed=7, idle=0)
    r = torch.Generator(device=DEV)
    r.manual_seed(3)
    off = torch.rand(T, generator=r, device=DEV) < share
    off[-1] = share > 0
    kind = torch.randint(0, 5, (T,), generator=r, device=DEV)
    g, y, h, lse = g.clone(), y.clone(), h.clone(), lse.clone()
    g[off & (kind < 2)] = 0.0
    for k, bad in ((2, -1), (3, V), (4, -2 ** 31)):
        y[off & (kind == k)] = bad
    g[off & (kind == 3)] = float("nan")
    g[off & (kind == 1)] = -0.0
    h[off] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0], device=DEV).repeat(d // 4).to(torch.bfloat16)
    lse[off & (kind != 0)] = float("nan")
    got = check(A, h, w, y, lse, g)
    assert not got["grad_hidden"][off].any() and bool((got["grad_hidden"][~off] != 0).any(1).all())
    total = torch.full((V, d), 2.0, device=DEV)
    A.arrol_logprob_grad(h, w, y, lse, g, want_hidden=False, lm_head_sum=total)
    assert bool(torch.isfinite(total).all()) and (share < 1 or bool((total == 2).all()))


def test_nan_of_a_token_that_takes_part(A):
    """It reaches its own hidden gradient and the LM head's, as the definition has it, and no other token's."""
    print("[case] logprob_grad NaN", flush=True)
    h, w, y, lse, g = make(300, 400, 64, seed=2, idle=0)
    want = A.arrol_logprob_grad(h, w, y, lse, g)["grad_hidden"]
    for bad in ("hidden", "grad"):
        x, gg = h.clone(), g.clone()
        if bad == "hidden":
            x[77, 5] = float("nan")
        else:
            gg[77] = float("nan")
        got = A.arrol_logprob_grad(x, w, y, lse, gg)
        others = torch.arange(300, device=DEV) != 77
        assert torch.equal(got["grad_hidden"][others], want[others]) and bool(torch.isnan(got["grad_hidden"][77]).all()) and bool(torch.isnan(got["grad_lm_head"]).all())


def test_outputs_one_by_one_and_reproducible(A):
    print("[case] logprob_grad outputs", flush=True)
    h, w, y, lse, g = make(700, 3000, 256, seed=4)
    both, again = A.arrol_logprob_grad(h, w, y, lse, g), A.arrol_logprob_grad(h, w, y, lse, g)
    assert all(torch.equal(both[x], again[x]) for x in both)
    only_h, only_w = A.arrol_logprob_grad(h, w, y, lse, g, want_lm_head=False), A.arrol_logprob_grad(h, w, y, lse, g, want_hidden=False)
    assert only_h["grad_lm_head"] is None and only_w["grad_hidden"] is None
    assert torch.equal(only_h["grad_hidden"], both["grad_hidden"]) and torch.equal(only_w["grad_lm_head"], both["grad_lm_head"])
    # a batch in parts: the same sums in another order
    total = torch.zeros(3000, 256, device=DEV)
    for part in (slice(0, 300), slice(300, 700)):
        A.arrol_logprob_grad(h[part], w, y[part], lse[part], g[part], want_hidden=False, lm_head_sum=total)
    dW, tW = reference(h, w, y, lse, g)[2:]
    agree("lm_head_sum", total, dW, tW + U * dW.abs())
    none = A.arrol_logprob_grad(h[:0], w, y[:0], lse[:0], g[:0])
    assert none["grad_hidden"].shape == (0, 256) and not none["grad_lm_head"].any()
    ws = torch.full((A.lib().arrol_logprob_grad_workspace_bytes(700, 3000, 256, 1),), 255, dtype=torch.uint8, device=DEV)       # NaN in every format
    own = A.arrol_logprob_grad(h, w, y, lse, g, workspace=ws)
    assert all(torch.equal(both[x], own[x]) for x in both)
    with pytest.raises(A.ArrolError):
        A.arrol_logprob_grad(h, w, y, lse, g, workspace=ws[:-1])


@pytest.mark.parametrize("of", ["hidden", "lm_head"])
def test_against_differences(A, of):
    """L = sum g logp, arrol_logprob's, moved along itself: hidden states and LM head on a grid, so that the steps up and down are exact."""
    print("[case] logprob_grad differences, %s" % of, flush=True)
    T, V, d = 150, 500, 64
    r = torch.Generator(device=DEV)
    r.manual_seed(6)
    h = (torch.randint(-60, 61, (T, d), generator=r, device=DEV) / 32).to(torch.bfloat16)
    w = (torch.randint(-60, 61, (V, d), generator=r, device=DEV) / 256).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=r, device=DEV, dtype=torch.int32)
    g = torch.randn(T, generator=r, device=DEV)
    lse = A.arrol_logprob(h, w, y, want_lse=True)[1]
    grad = A.arrol_logprob_grad(h, w, y, lse, g)["grad_" + of].double()
    x, unit = (h, 1 / 32) if of == "hidden" else (w, 1 / 256)
    for trial in range(4):
        step = unit * (torch.randint(0, 2, x.shape, generator=r, device=DEV) * 2 - 1) if trial else unit * torch.sign(grad)
        up, down = ((x.double() + s * step).to(torch.bfloat16) for s in (1, -1))
        assert torch.equal(up.double() - down.double(), 2 * step.double())
        L = [(g.double() * A.arrol_logprob(v if of == "hidden" else h, w if of == "hidden" else v, y).double()).sum() for v in (up, down)]
        moved = (step.double() @ w.double().t() if of == "hidden" else h.double() @ step.double().t()).abs().amax(1)        # of a token's logits, at most
        third = (g.double().abs() * (2 * moved) ** 3 / 3).sum()
        tol = third + 2e-5 * g.double().abs().sum() + 2 * (U * grad.abs() * unit).sum() + 2 * U * float((grad.abs() * unit).sum())
        want = 2 * (grad * step.double()).sum()
        assert abs(float(L[0] - L[1] - want)) <= float(tol), (trial, float(L[0] - L[1]), float(want), float(tol))
        if trial == 0:
            assert float(want) > 4 * float(tol)         # moved along the gradient, L rises by far more than that


@pytest.mark.parametrize("T,V,d", [(300, 700, 128), (100, 60001, 264)])
def test_on_a_stream_and_in_graphs(A, T, V, d):
    """Two graphs that share a workspace, replayed in turn with eager calls between them, on data that changes."""
    print("[case] logprob_grad in graphs T=%d V=%d d=%d" % (T, V, d), flush=True)
    data = [make(T, V, d, seed=s) for s in range(4)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = A.arrol_logprob_grad(*data[0], stream=side)
    side.synchronize()
    want = [A.arrol_logprob_grad(*x) for x in data]
    assert all(torch.equal(got[x], want[0][x]) for x in got)
    buffers = [x.clone() for x in data[0]]
    ws = torch.empty(A.lib().arrol_logprob_grad_workspace_bytes(T, V, d, 1), dtype=torch.uint8, device=DEV)
    total = torch.zeros(V, d, device=DEV)
    graphs = []
    for kw in (dict(), dict(lm_head_sum=total)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = A.arrol_logprob_grad(*buffers, workspace=ws, **kw)
        graphs.append((graph, out))
    for i in (1, 2, 3, 0, 2):
        for b, x in zip(buffers, data[i]):
            b.copy_(x)
        before = total.clone()
        for graph, out in graphs:
            graph.replay()
        eager = A.arrol_logprob_grad(*data[i], workspace=ws)
        torch.cuda.synchronize()
        for x in want[i]:
            assert torch.equal(eager[x], want[i][x]) and torch.equal(graphs[0][1][x], want[i][x])
        assert torch.equal(graphs[1][1]["grad_hidden"], want[i]["grad_hidden"])
        fresh = torch.zeros_like(total)
        A.arrol_logprob_grad(*data[i], want_hidden=False, lm_head_sum=fresh)
        assert torch.equal(total, before + fresh)


def test_past_2_to_the_31_elements(A):
    """An LM head and its gradient of more than 2^31 elements; the tokens' targets are its last rows."""
    print("[case] logprob_grad past 2^31 elements", flush=True)
    V, d, T = 140000, 16384, 6
    w = torch.zeros(V, d, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    w[-300:] = (torch.randn(300, d, generator=g, device=DEV) * d ** -0.5).to(torch.bfloat16)
    h = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
    y = torch.tensor([V - 1, V - 2, V - 299, 0, V - 300, V - 7], dtype=torch.int32, device=DEV)
    grad = torch.randn(T, generator=g, device=DEV)
    z = h.double() @ w[-300:].double().t()
    lse = torch.logsumexp(torch.cat([z, torch.full((T, 1), torch.log(torch.tensor(float(V - 300))), dtype=torch.float64, device=DEV)], 1), 1).float()
    got = A.arrol_logprob_grad(h, w, y, lse, grad)
    p = torch.exp(z - lse.double()[:, None])
    hit = torch.zeros_like(p)
    for t, v in enumerate(y.tolist()):
        if v >= V - 300:
            hit[t, v - (V - 300)] = 1
    dz = grad.double()[:, None] * (hit - p)
    r = (d + 4) * E * (h.double().abs() @ w[-300:].double().abs().t()) + 2.0 ** -20
    off = U * dz.abs() + grad.double().abs()[:, None] * (p * r + 4 * E * hit)
    dH, tail = dz @ w[-300:].double(), dz.t() @ h.double()
    agree("grad_hidden", got["grad_hidden"], dH, (off + 400 * E * dz.abs()) @ w[-300:].double().abs() + U * dH.abs(), norm=False)
    agree("grad_lm_head", got["grad_lm_head"][-300:], tail, (off + 50 * E * dz.abs()).t() @ h.double().abs() + U * tail.abs(), norm=False)
    flat = torch.exp(-lse.double())[:, None] * -grad.double()[:, None] * h.double()
    assert bool(((got["grad_lm_head"][1:5].double() - flat.sum(0)).abs() <= 3 * U * flat.abs().sum(0)).all())
