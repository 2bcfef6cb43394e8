"""What the rotation by positions and the appending to the pool refuse on the host, before anything is launched, and the frequencies, a host computation."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def A():
    import os
    import paper_2603_24840_amd as pkg
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2603_24840_amd import build
        build.build(verbose=False)
    return pkg


FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1008)


def rotary(A, **kw):
    a = dict(q=FAKE, qs=256, k=FAKE, ks=128, pos=FAKE, f=FAKE, T=10, H=4, KV=2, hd=64, rot=64, inter=0, inverse=0, m=1.0, qo=FAKE, qos=256, ko=FAKE, kos=128)
    a.update(kw)
    return A.lib().arrol_rotary(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=ODD), dict(k=None), dict(k=ODD), dict(pos=None), dict(f=None), dict(T=-1), dict(T=2 ** 25), dict(H=0), dict(H=5), dict(KV=0),
                                 dict(KV=3), dict(KV=-1), dict(hd=0), dict(hd=60), dict(hd=264, qs=2048, ks=1024, qos=2048, kos=1024), dict(rot=0), dict(rot=66), dict(rot=63), dict(rot=-2),
                                 dict(qs=248), dict(qs=260), dict(ks=120), dict(qs=2 ** 24 + 8), dict(qo=None), dict(qo=ODD), dict(qos=248), dict(ko=None), dict(ko=ODD), dict(kos=132)])
def test_rotary_refuses(A, bad):
    assert rotary(A, **bad) == -1


def test_rotary_without_rows_is_a_no_op(A):
    assert rotary(A, T=0, q=None, qo=None, pos=None, f=None) == 0


def append(A, **kw):
    a = dict(k=FAKE, ks=128, v=FAKE, vs=128, q=FAKE, qs=256, cu=FAKE, start=FAKE, pos=None, f=FAKE, T=10, n=3, H=4, rot=64, inter=0, m=1.0, kv=FAKE,
             lay=A.KVLayout(2, 16, 2, 64, 128), layer=1, table=FAKE, width=4, qo=FAKE, qos=256, ko=None, kos=0)
    a.update(kw)
    return A.lib().arrol_append(*a.values(), None)


def test_append_refuses(A):
    lay = lambda **kw: A.KVLayout(*[kw.get(x, y) for x, y in (("layers", 2), ("page", 16), ("KV", 2), ("hd", 64), ("pages", 128))])
    for bad in (dict(k=None), dict(k=ODD), dict(ks=120), dict(ks=132), dict(v=None), dict(v=ODD), dict(vs=120), dict(q=None), dict(q=ODD), dict(qs=248), dict(H=0), dict(H=-1), dict(qo=None),
                dict(qo=ODD), dict(qos=248), dict(ko=ODD, kos=128), dict(ko=FAKE, kos=120), dict(start=None), dict(table=None), dict(width=0), dict(T=-1), dict(T=2 ** 25), dict(n=-1),
                dict(cu=None), dict(rot=0), dict(rot=66), dict(rot=7), dict(kv=None), dict(kv=ODD), dict(layer=-1), dict(layer=2), dict(lay=lay(layers=0)), dict(lay=lay(page=0)),
                dict(lay=lay(KV=0)), dict(lay=lay(KV=3)), dict(lay=lay(hd=60)), dict(lay=lay(hd=264)), dict(lay=lay(pages=-1)), dict(lay=lay(pages=2 ** 27))):
        assert append(A, **bad) == -1, bad
    assert append(A, T=0, k=None, v=None) == 0
    assert append(A, T=0, n=0, cu=None, start=None, table=None) == 0


def test_binding_refuses(A):
    x, kv = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 4, 16, 2, 64, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    f = torch.zeros(32, dtype=torch.float64)
    with pytest.raises(TypeError):
        A.arrol_rotary(x, x, i32(4), f)                       # on the CPU
    with pytest.raises(TypeError):
        A.arrol_append(x, x, kv, 0, i32(4, 1), i32(4))
    gpu_like = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="meta")
    with pytest.raises((TypeError, ValueError)):
        A.arrol_rotary(gpu_like, None, i32(4), f)


def test_binding_refuses_sizes_past_32_bits(A):
    """Of which the library would be handed the lower half: 2^32 + 64 as 64."""
    meta = lambda *s, **kw: torch.empty(*s, device="meta", **kw)
    x, i32 = meta(4, 2, 64, dtype=torch.bfloat16), meta(4, dtype=torch.int32)
    many, f = meta(2 ** 31 + 32, dtype=torch.float64), meta(32, dtype=torch.float64)
    kv = meta(1, 2, 4, 16, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: A.arrol_rotary(x, x, i32, many), lambda: A.arrol_append(x, x, kv, 0, meta(4, 1, dtype=torch.int32), i32, inv_freq=many),
                 lambda: A.arrol_append(x, x, kv, 0, meta(2 ** 32 + 4, 1, dtype=torch.int32), meta(2 ** 32 + 4, dtype=torch.int32), inv_freq=f),
                 lambda: A.arrol_append(x, x, kv, 0, meta(4, 2 ** 32 + 1, dtype=torch.int32), i32, inv_freq=f),
                 lambda: A.arrol_append(x, x, meta(1, 2, 1, 2 ** 32 + 16, 2, 64, dtype=torch.bfloat16), 0, meta(4, 1, dtype=torch.int32), i32, inv_freq=f)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_frequencies(A):
    """Against the definition: unscaled, all divided, and by parts, whose ends and middle are known."""
    plain = A.arrol_rotary_frequencies(64, 5e5, device="cpu")
    want = torch.tensor([5e5 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64)
    assert plain.dtype == torch.float64 and torch.allclose(plain, want, rtol=4 * 2.0 ** -53 * 14, atol=0)       # pow: its argument's rounding times |exponent ln base| < 14
    assert torch.allclose(A.arrol_rotary_frequencies(64, 5e5, factor=8.0, device="cpu"), want / 8, rtol=1e-14, atol=0)
    parts = A.arrol_rotary_frequencies(64, 5e5, factor=8.0, original_context=8192, low=1.0, high=4.0, device="cpu")
    turns = 8192 * want / (2 * math.pi)
    assert torch.equal(parts[turns >= 4], plain[turns >= 4]) and torch.allclose(parts[turns <= 1], want[turns <= 1] / 8, rtol=1e-14, atol=0)
    between = (turns > 1) & (turns < 4)
    assert int(between.sum()) >= 2 and int((turns >= 4).sum()) >= 2 and int((turns <= 1).sum()) >= 2
    s = (turns - 1) / 3
    assert torch.allclose(parts[between], (want * (s + (1 - s) / 8))[between], rtol=1e-13, atol=0)
    step = A.arrol_rotary_frequencies(64, 5e5, factor=8.0, original_context=8192, low=2.0, high=2.0, device="cpu")
    assert torch.allclose(step, torch.where(turns >= 2, want, want / 8), rtol=1e-14, atol=0)
    assert A.arrol_rotary_frequencies(2, device="cpu").tolist() == [1.0]
    nan, inf = math.nan, math.inf
    for bad in (dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=258), dict(rotary_dim=-2), dict(base=0.0), dict(base=nan), dict(base=inf), dict(factor=0.0), dict(factor=nan),
                dict(original_context=-1), dict(original_context=inf), dict(low=2.0, high=1.0), dict(low=nan), dict(high=inf), dict(low=-inf)):
        with pytest.raises(A.ArrolError):
            A.arrol_rotary_frequencies(**{"rotary_dim": 64, "device": "cpu", **bad})
    with pytest.raises(ValueError, match="32 bits"):
        A.arrol_rotary_frequencies(2 ** 32 + 64, device="cpu")
    assert A.lib().arrol_rotary_frequencies(64, 1e4, 1.0, 0.0, 1.0, 4.0, None) == -1
