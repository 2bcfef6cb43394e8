"""The C++ marshalling of the attention calls and the eviction against the Python marshalling: the same results bit for bit, and
None - so the Python way - for everything but the ordinary case."""
import inspect

import pytest
import torch

import paper_2603_24840_amd as A
from paper_2603_24840_amd import binding

DEV = "cuda:0"


def calls(dev):
    g = torch.Generator().manual_seed(5)
    f = lambda *shape: torch.randn(shape, generator=g).to(dev)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).to(dev)
    i64 = lambda *x: torch.tensor(x).to(dev)
    qkv, k2 = f(70, 8, 64).bfloat16(), f(90, 2, 64).bfloat16()
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    cu, cu_k = i64(0, 30, 70), i64(0, 50, 90)
    out, lse, go = f(70, 4, 64).bfloat16(), f(4, 70), f(70, 4, 64).bfloat16()
    kv = f(2, 2, 12, 16, 2, 64).bfloat16()
    table, lens, pt, pl, off = i32(*range(8)).reshape(4, 2), i32(20, 1, 32, 0), i32(8, 9, 10, 11).reshape(2, 2), i32(32, 5), i64(0, 3, 4)
    dq, w, pw = f(4, 8, 64).bfloat16(), f(4, 32).abs(), f(2, 32).abs()
    scratch = lambda: torch.zeros(1 << 20, dtype=torch.uint8, device=dev)
    return {
        "attention": [((q, k, v, cu), {}), ((q, k2, k2, cu, cu_k), dict(causal=False, scale=0.25)), ((q, k, v, cu), dict(out=torch.zeros(70, 4, 64, dtype=torch.bfloat16, device=dev))),
                      ((q[:1], k[:1], v[:1], cu), {}), ((q, f(9000, 2, 64).bfloat16(), f(9000, 2, 64).bfloat16(), cu, i64(0, 4000, 9000)), {}),
                      ((q, k2, k2, cu, cu_k), dict(workspace=None)), ((q, k2, k2, cu, cu_k), dict(workspace=scratch()))],
        "attention_grad": [((q, k, v, out, lse, go, cu), {}), ((q, k2, k2, out, lse, go, cu, cu_k), dict(causal=False, scale=1)), ((q, k, v, out, lse, go, cu), dict(workspace=scratch()))],
        "decode_attention": [((dq, kv, 1, table, lens), {}), ((dq, kv, 0, table, lens, pt, pl, off), {}), ((dq, kv, 1, table, lens, pt, pl, off), dict(want_weight=True, scale=0.2)),
                             ((dq, kv, 1, table, lens), dict(want_weight=True, weight=w)),
                             ((dq, kv, 1, table, lens, pt, pl, off), dict(want_weight=True, weight=w, prefix_weight=pw, out_weight=w, out_prefix_weight=pw, workspace=scratch()))],
        "evict": [((kv, table, lens, w, 16), {}), ((kv, table, lens, w, 16), dict(n_first=2, n_recent=4, position=torch.arange(128, dtype=torch.int32, device=dev).reshape(4, 32))),
                  ((kv, table, lens, w, 40), dict(workspace=scratch()))],
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
@pytest.mark.parametrize("name", ["attention", "attention_grad", "decode_attention", "evict"])
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
    q = c["attention"][0][0][0]
    for name in ("attention", "attention_grad"):
        a = c[name][0][0]
        for i, x in ((0, q.float()), (0, q[:, 0]), (0, q.cpu()), (0, q.transpose(1, 2)), (0, q[:, ::2]), (1, a[1][:, :1]), (1, a[1][:, :, :32]), (2, a[2][:50])):
            assert native(name, [*a[:i], x, *a[i + 1:]], {}) is None, (name, i)
        assert native(name, a, dict(scale="1")) is None and native(name, a, dict(causal=1)) is None
    a = c["attention"][0][0]
    assert native("attention", [*a[:3], a[3].int()], {}) is None and native("attention", a, dict(out=torch.zeros(70, 4, 32, dtype=torch.bfloat16, device=DEV))) is None
    a = c["decode_attention"][2][0]
    for i, x in ((0, a[0][:3]), (0, a[0][:, :, :32]), (1, a[1][0]), (1, a[1].float()), (2, -1), (3, a[3].long()), (4, a[4][:3]), (5, None), (6, a[6][:1]), (7, a[7][:2])):
        assert native("decode_attention", [*a[:i], x, *a[i + 1:]], {}) is None, i
    assert native("decode_attention", a, dict(weight=torch.zeros(4, 32, device=DEV))) is None and native("decode_attention", a, dict(want_weight=True, weight=torch.zeros(4, 16, device=DEV))) is None
    a = c["evict"][0][0]
    for i, x in ((0, a[0][0]), (1, a[1].long()), (2, a[2][:1]), (3, a[3][:, :16]), (4, -1), (4, 2.0)):
        assert native("evict", [*a[:i], x, *a[i + 1:]], {}) is None, i
    for call in (lambda: A.arrol_attention(q[:, :3], *c["attention"][0][0][1:]), lambda: A.arrol_evict(*a[:4], 16, n_first=9, n_recent=9)):
        with pytest.raises(A.ArrolError):       # the library's own refusals
            call()


def test_native_marshalling_leaves_cpu_tensors_to_python():
    for name, cases in calls("cpu").items():
        with pytest.raises((TypeError, ValueError)):
            getattr(A, "arrol_" + name)(*cases[0][0], **cases[0][1])


@pytest.mark.gpu
def test_the_stride_of_a_single_row_does_not_matter():
    """A view of one row of something large: there is no second row that its stride leads to."""
    print("[case] marshal, one row of any stride", flush=True)
    c = calls(DEV)
    q, k, v = (x[:1].contiguous() for x in c["attention"][0][0][:3])
    cu, far = torch.tensor([0, 1], device=DEV), lambda x: x.as_strided(x.shape, (2 ** 25 + 4, x.shape[2], 1))
    want = A.arrol_attention(q, k, v, cu)
    go = q.flip(2).contiguous()
    want_grad = A.arrol_attention_grad(q, k, v, *want, go, cu)
    for got in (A.arrol_attention(far(q), far(k), far(v), cu), binding._py_attention(far(q), far(k), far(v), cu)):
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    for got in (A.arrol_attention_grad(far(q), far(k), far(v), *want, go, cu), binding._py_attention_grad(far(q), far(k), far(v), *want, go, cu)):
        assert all(torch.equal(got[x], want_grad[x]) for x in got)
