"""The C++ marshalling of rotary, append and the log-probabilities' gradient against the Python marshalling: the same results bit for bit, and None - so the Python way -
for everything but the ordinary case; the refusals of both."""
import inspect

import pytest
import torch

import paper_2603_24840_amd as A
from paper_2603_24840_amd import binding

DEV = "cuda:0"
NAMES = ["rotary", "append", "logprob_grad"]


def calls(dev):
    g = torch.Generator().manual_seed(5)
    f = lambda *shape: torch.randn(shape, generator=g).to(dev)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).to(dev)
    x = f(30, 8, 64).bfloat16()
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    pos, freq = torch.arange(30, dtype=torch.int32).to(dev) * 3, torch.logspace(0, -4, 24, dtype=torch.float64).to(dev)
    kv, table, start, cu = f(2, 2, 12, 16, 2, 64).bfloat16(), i32(*range(9)).reshape(3, 3), i32(0, 5, 30), torch.tensor([0, 9, 20, 30]).to(dev)
    rows = i32(*range(30)).reshape(30, 1) % 12
    new = lambda t: torch.zeros(t.shape, dtype=torch.bfloat16, device=dev)
    h, w = f(50, 128).bfloat16(), (f(300, 128) / 11).bfloat16()
    y, lse, gr = i32(*range(0, 300, 6)), f(50).abs() + 6, f(50)
    return {
        "rotary": [((q, k, pos, freq), {}), ((q, k, pos, freq), dict(interleaved=True, inverse=True, magnitude=1.5)), ((q, None, pos, freq), dict(magnitude=2)),
                   ((q, k, pos, freq), dict(out_q=new(q), out_k=new(k))), ((q[:1], k[:1], pos[:1], freq), {})],
        "append": [((k, v, kv, 1, table, start, cu), dict(q=q, position=pos, inv_freq=freq, want_k=True)), ((k, v, kv, 0, rows, pos % 16), dict(q=q, inv_freq=freq, interleaved=True)),
                   ((k, v, kv, 0, table, start, cu), {}), ((k, v, kv, 1, table, start, cu), dict(q=q, out_q=new(q), want_k=True, out_k=new(k), inv_freq=freq, magnitude=1.25))],
        "logprob_grad": [((h, w, y, lse, gr), {}), ((h, w, y, lse, gr), dict(want_hidden=False)), ((h, w, y, lse, gr), dict(want_lm_head=False)),
                         ((h, w, y, lse, gr), dict(lm_head_sum=torch.ones(300, 128, device=dev))), ((h, w, y, lse, gr), dict(workspace=torch.zeros(1 << 26, dtype=torch.uint8, device=dev)))],
    }


def native(name, args, kw):
    bound = inspect.signature(getattr(A, "arrol_" + name)).bind(*args, **kw)
    bound.apply_defaults()
    return getattr(binding._load_marshal(), name)(*[v for k, v in bound.arguments.items() if k != "stream"])


def flat(x):
    if isinstance(x, dict):
        return [(k, x[k]) for k in sorted(x)]
    return list(enumerate(x)) if isinstance(x, tuple) else [(0, x)]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_native_marshalling_gives_what_python_gives(name):
    print("[case] marshal", name, flush=True)
    clone = lambda x: x.clone() if isinstance(x, torch.Tensor) and x.is_contiguous() else x
    for args, kw in calls(DEV)[name]:
        results = []
        for way in (lambda a, k: getattr(binding, "_py_" + name)(*a, **k), lambda a, k: getattr(A, "arrol_" + name)(*a, **k), lambda a, k: native(name, a, k)):
            a, k = [clone(x) for x in args], {key: clone(x) for key, x in kw.items()}
            got = way(a, k)
            assert got is not None
            results.append(flat(got) + flat(tuple(a)) + [x for x in flat(k) if x[0] != "workspace"])
        torch.cuda.synchronize()
        for other in results[1:]:
            assert [x for x, _ in other] == [x for x, _ in results[0]]
            for (key, x), (_, y) in zip(results[0], other):
                assert isinstance(x, torch.Tensor) == isinstance(y, torch.Tensor), key
                if isinstance(x, torch.Tensor):
                    assert x.dtype == y.dtype and x.shape == y.shape and torch.equal(x.reshape(-1).contiguous().view(torch.uint8), y.reshape(-1).contiguous().view(torch.uint8)), key


@pytest.mark.gpu
def test_native_marshalling_takes_the_ordinary_case_only():
    c = calls(DEV)
    a, kw = c["rotary"][0]
    for i, x in ((0, a[0].float()), (0, a[0][:, 0]), (0, a[0].cpu()), (0, a[0][:, ::2]), (1, a[1][:5]), (1, a[1][:, :, :32]), (2, a[2][:5]), (2, a[2].long()), (2, None), (3, a[3].float()),
                 (3, a[3][::2])):
        assert native("rotary", [*a[:i], x, *a[i + 1:]], {}) is None, i
    for bad in (dict(interleaved=1), dict(magnitude="1"), dict(out_q=a[0][:, :2]), dict(out_k=a[0])):
        assert native("rotary", a, bad) is None, bad
    assert native("rotary", [a[0], None, *a[2:]], dict(out_k=a[1])) is None
    a, kw = c["append"][0]
    for i, x in ((0, a[0][:5]), (0, a[0].float()), (1, a[1][:, :1]), (2, a[2][0]), (2, a[2].float()), (3, -1), (3, 2 ** 31), (4, a[4].long()), (4, a[4][:2]), (5, a[5][:2]), (6, a[6][:3]), (6, None),
                 (6, a[6].int())):
        assert native("append", [*a[:i], x, *a[i + 1:]], kw) is None, i
    for bad in (dict(q=kw["q"][:5]), dict(position=kw["position"][:5]), dict(position=kw["position"].long()), dict(inv_freq=kw["inv_freq"].float()), dict(want_k=1), dict(want_k=False, out_k=a[0]),
                dict(q=None, out_q=kw["q"])):
        assert native("append", a, {**kw, **bad}) is None, bad
    a, kw = c["logprob_grad"][0]
    for i, x in ((0, a[0][:5]), (0, a[0].float()), (0, a[0][:, ::2]), (1, a[1][:, :64]), (2, a[2].long()), (2, None), (3, a[3][:5]), (3, a[3].double()), (4, None), (4, a[4].cpu())):
        assert native("logprob_grad", [*a[:i], x, *a[i + 1:]], {}) is None, i
    for bad in (dict(want_hidden=False, want_lm_head=False), dict(want_hidden=1), dict(lm_head_sum=torch.zeros(300, 64, device=DEV)), dict(lm_head_sum=torch.zeros(300, 128, dtype=torch.float64, device=DEV)),
                dict(workspace="auto")):
        assert native("logprob_grad", a, bad) is None, bad


@pytest.mark.gpu
def test_refusals():
    """On the GPU's tensors, by the binding and by the library; nothing is launched."""
    c = calls(DEV)
    a, kw = c["rotary"][0]
    for bad, kws in (((a[0], a[1][:5], *a[2:]), {}), ((*a[:2], a[2][:5], a[3]), {}), ((*a[:2], a[2].long(), a[3]), {}), ((*a[:3], a[3].float()), {}), (a, dict(out_q=a[0][:5])), (a, dict(out_k=a[0])),
                     ((a[0], None, *a[2:]), dict(out_k=a[1])), ((*a[:3], torch.zeros(33, dtype=torch.float64, device=DEV)), {}), ((*a[:3], torch.zeros(0, dtype=torch.float64, device=DEV)), {}),
                     ((a[0][:, :, :60].contiguous(), None, *a[2:]), {}), ((a[0].expand(30, 4, 64)[:, :1].transpose(0, 1), None, *a[2:]), {})):
        with pytest.raises((ValueError, TypeError, A.ArrolError)):
            A.arrol_rotary(*bad, **kws)
    a, kw = c["append"][0]
    for bad, kws in (((a[0][:5], *a[1:]), kw), ((*a[:3], 2, *a[4:]), kw), ((*a[:3], -1, *a[4:]), kw), ((*a[:3], 2 ** 32, *a[4:]), kw), ((*a[:4], a[4][:2], *a[5:]), kw), ((*a[:5], a[5][:2], a[6]), kw),
                     ((*a[:6], a[6][:2]), kw), (a[:6], kw), (a, {**kw, "q": kw["q"][:5]}), (a, {**kw, "position": kw["position"][:5]}), (a, {**kw, "inv_freq": torch.zeros(33, dtype=torch.float64, device=DEV)}),
                     (a, {**kw, "want_k": False, "out_k": a[0]}), (a, {**kw, "q": None, "out_q": kw["q"]}), ((a[0], a[1], a[2][:, :, :, :, :1].contiguous(), *a[3:]), kw)):
        with pytest.raises((ValueError, TypeError, A.ArrolError)):
            A.arrol_append(*bad, **kws)
    a, kw = c["logprob_grad"][0]
    for bad, kws in (((a[0][:5], *a[1:]), {}), ((a[0], a[1][:, :64].contiguous(), *a[2:]), {}), (a, dict(want_hidden=False, want_lm_head=False)), (a, dict(lm_head_sum=torch.zeros(5, 128, device=DEV))),
                     ((a[0].float(), *a[1:]), {}), ((a[0], a[1][:, ::2], *a[2:]), {}), (a, dict(workspace=torch.zeros(64, dtype=torch.uint8, device=DEV))),
                     ((a[0][:, :60].contiguous(), a[1][:, :60].contiguous(), *a[2:]), {})):
        with pytest.raises((ValueError, TypeError, A.ArrolError)):
            A.arrol_logprob_grad(*bad, **kws)


def test_native_marshalling_leaves_cpu_tensors_to_python():
    for name, cases in calls("cpu").items():
        with pytest.raises((TypeError, ValueError)):
            getattr(A, "arrol_" + name)(*cases[0][0], **cases[0][1])


@pytest.mark.gpu
def test_the_stride_of_a_single_row_does_not_matter():
    print("[case] marshal, one row of any stride", flush=True)
    a = calls(DEV)["rotary"][0][0]
    far = lambda x: x[:1].as_strided((1, *x.shape[1:]), (2 ** 25 + 4, x.shape[2], 1))
    q, k = a[0][:1].contiguous(), a[1][:1].contiguous()
    want = A.arrol_rotary(q, k, a[2][:1], a[3])
    for got in (A.arrol_rotary(far(q), far(k), a[2][:1], a[3]), binding._py_rotary(far(q), far(k), a[2][:1], a[3])):
        assert all(torch.equal(x, y) for x, y in zip(got, want))
