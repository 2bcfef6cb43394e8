"""What the attention calls and the eviction refuse on the host, before anything is launched, and their workspace queries."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def L():
    import os
    import paper_2603_24840_amd as A
    if not os.path.exists(A.LIB_PATH):
        from paper_2603_24840_amd import build
        build.build(verbose=False)
    return A.lib()


FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1008)


def packed(**kw):
    a = dict(q=FAKE, qs=256, k=FAKE, ks=128, v=FAKE, vs=128, cu=FAKE, cuk=None, Tq=10, Tk=10, n=2, H=4, KV=2, hd=64, causal=1, scale=0.125, out=FAKE, lse=FAKE)
    a.update(kw)
    return list(a.values())


BAD_PACKED = [dict(q=None), dict(k=None), dict(v=None), dict(cu=None), dict(out=None), dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(out=ODD), dict(qs=248), dict(qs=260),
              dict(ks=120), dict(vs=132), dict(Tq=-1), dict(Tk=-1), dict(n=-1), dict(H=3), dict(H=0), dict(KV=0), dict(hd=0), dict(hd=12), dict(hd=136),
              dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(Tq=2 ** 30, H=4096, KV=4096), dict(n=2 ** 24, H=2), dict(Tk=11), dict(Tk=9)]


@pytest.mark.parametrize("bad", BAD_PACKED)
def test_attention_refuses(L, bad):
    assert L.arrol_attention(*packed(**bad), FAKE, 1 << 30, None) == -1


def test_attention_without_rows_is_a_no_op(L):
    assert L.arrol_attention(*packed(Tq=0, Tk=0, q=None, k=None, v=None, out=None, cu=None, n=0), None, 0, None) == 0
    assert L.arrol_attention(*packed(), ODD, 1 << 30, None) == -1
    size = L.arrol_attention_workspace_bytes
    assert size(10, 10, 2, 4, 64) == 0 and size(0, 10, 2, 4, 64) == 0               # nothing to cut
    assert size(1200, 20000, 8, 16, 128) >= 2 * 1200 * 16 * 130 * 4 and size(200000, 200000, 8, 16, 128) == 0


@pytest.mark.parametrize("bad", [b for b in BAD_PACKED if "out" not in b] + [dict(o=None), dict(o=ODD), dict(stat=None), dict(go=None), dict(go=ODD), dict(dq=None), dict(dk=None),
                                                                           dict(dv=None), dict(dq=ODD), dict(dk=ODD), dict(dv=ODD)])
def test_attention_gradient_refuses(L, bad):
    assert grad(L, **bad) == -1


def grad(L, ws=FAKE, nbytes=1 << 30, o=FAKE, stat=FAKE, go=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, **kw):
    a = packed(**kw)
    return L.arrol_attention_grad(*a[:6], o, stat, go, *a[6:16], dq, dk, dv, ws, nbytes, None)


def test_attention_gradient_asks_for_its_workspace(L):
    size = L.arrol_attention_grad_workspace_bytes
    need = size(10, 10, 2, 4, 2, 64)
    assert need >= 2 * 10 * 4 * 4 and size(0, 0, 0, 4, 2, 64) == 0 and size(10, 10, 2, 4, 3, 64) == 0
    assert size(4000, 4000, 1, 4, 1, 64) >= 2 * 4000 * 4 * 4 + 2 * 2 * 4000 * 64 * 4      # one long sequence, few heads: walks in ranges
    assert grad(L, ws=None) == -2 and grad(L, nbytes=need - 1) == -2 and grad(L, ws=ODD) == -2
    assert grad(L, Tq=0, Tk=0, ws=None, nbytes=0) == 0


def decode(L, **kw):
    import paper_2603_24840_amd as A
    a = dict(q=FAKE, n=4, H=8, kv=FAKE, lay=A.KVLayout(2, 16, 2, 64, 128), layer=1, table=FAKE, lens=FAKE, width=4, pt=FAKE, pl=FAKE, pw=3, off=FAKE, groups=2, scale=0.125, out=FAKE,
             lse=None, win=None, pwin=None, wout=None, pwout=None, ws=FAKE, nbytes=1 << 30)
    a.update(kw)
    return L.arrol_decode_attention(*a.values(), None)


def test_decode_refuses(L):
    import paper_2603_24840_amd as A
    lay = lambda **kw: A.KVLayout(*[kw.get(x, y) for x, y in (("layers", 2), ("page", 16), ("KV", 2), ("hd", 64), ("pages", 128))])
    for bad in (dict(q=None), dict(q=ODD), dict(kv=None), dict(kv=ODD), dict(table=None), dict(lens=None), dict(out=None), dict(out=ODD), dict(n=-1), dict(H=7), dict(H=0), dict(layer=2),
                dict(layer=-1), dict(width=0), dict(width=2 ** 31 - 1), dict(pt=None), dict(pl=None), dict(off=None), dict(pw=0), dict(groups=-1), dict(groups=2 ** 20 + 1), dict(scale=0.0),
                dict(scale=float("nan")), dict(win=FAKE), dict(pwin=FAKE), dict(groups=0, pwout=FAKE), dict(n=2 ** 24, wout=FAKE), dict(lay=lay(layers=0)), dict(lay=lay(page=0)), dict(lay=lay(KV=0)),
                dict(lay=lay(KV=3)), dict(lay=lay(hd=12)), dict(lay=lay(hd=256)), dict(lay=lay(pages=-1)), dict(lay=lay(pages=2 ** 31))):
        assert decode(L, **bad) == -1, bad
    assert decode(L, n=0, groups=0, ws=None, nbytes=0, q=None, kv=None) == 0


def test_decode_asks_for_its_workspace(L):
    size = L.arrol_decode_attention_workspace_bytes
    need, more = size(4, 8, 2, 64, 16, 4, 3, 2, 0), size(4, 8, 2, 64, 16, 4, 3, 2, 1)
    assert need >= 4 * 8 * 2 * (64 + 2) * 4 and more >= need + 4 * 8 * (64 + 48) * 4
    assert size(0, 8, 2, 64, 16, 4, 3, 2, 0) == 0 and size(4, 7, 2, 64, 16, 4, 3, 2, 0) == 0
    assert decode(L, ws=None) == -2 and decode(L, nbytes=need - 1) == -2 and decode(L, ws=ODD) == -2 and decode(L, wout=FAKE, nbytes=more - 1) == -2


def evict(L, **kw):
    import paper_2603_24840_amd as A
    a = dict(kv=FAKE, lay=A.KVLayout(2, 16, 2, 64, 128), table=FAKE, lens=FAKE, rows=4, width=4, weight=FAKE, pos=None, budget=32, first=2, recent=8, t=FAKE, n=FAKE, w=FAKE, p=FAKE, ws=FAKE,
             nbytes=1 << 30)
    a.update(kw)
    return L.arrol_evict(*a.values(), None)


def test_evict_refuses(L):
    import paper_2603_24840_amd as A
    for bad in (dict(kv=None), dict(kv=ODD), dict(table=None), dict(lens=None), dict(weight=None), dict(t=None), dict(n=None), dict(w=None), dict(p=None), dict(rows=-1), dict(rows=1 << 22),
                dict(width=0), dict(width=2 ** 31 - 1), dict(budget=-1), dict(first=-1), dict(recent=-1), dict(first=20, recent=13), dict(first=2 ** 31 - 1, recent=2 ** 31 - 1),
                dict(lay=A.KVLayout(2, 16, 1, 4, 128)), dict(lay=A.KVLayout(0, 16, 2, 64, 128)), dict(lay=A.KVLayout(2, 0, 2, 64, 128)), dict(lay=A.KVLayout(2, 16, 2, 64, -1))):
        assert evict(L, **bad) == -1, bad
    assert evict(L, rows=0) == 0
    need = L.arrol_evict_workspace_bytes(4, 4, 16, 32)
    assert need >= 4 * 32 * 24 + 16 and L.arrol_evict_workspace_bytes(0, 4, 16, 32) == 0
    assert evict(L, ws=None) == -2 and evict(L, nbytes=need - 1) == -2 and evict(L, ws=ODD) == -2


def test_binding_refuses(L):
    import paper_2603_24840_amd as A
    q, kv = torch.zeros(4, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 4, 16, 2, 64, dtype=torch.bfloat16)
    off = torch.zeros(2, dtype=torch.int64)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(TypeError):
        A.arrol_attention(q, q, q, off)                                  # on the CPU
    with pytest.raises(TypeError):
        A.arrol_attention_grad(q, q, q, q, torch.zeros(4, 4), q, off)
    with pytest.raises(ValueError):
        A.arrol_decode_attention(q, kv, 0, i32(4, 1), i32(4))
    with pytest.raises(ValueError):
        A.arrol_decode_attention(q, kv, 0, i32(3, 1), i32(4))            # rows of the table
    with pytest.raises(ValueError):
        A.arrol_decode_attention(q, kv, 0, i32(4, 1), i32(4), prefix_table=i32(1, 1))
    with pytest.raises(ValueError):
        A.arrol_decode_attention(q, kv, 0, i32(4, 1), i32(4), weight=torch.zeros(4, 16))
    with pytest.raises(ValueError):
        A.arrol_evict(kv, i32(4, 1), i32(4), torch.zeros(4, 15), 8)
    with pytest.raises(ValueError):
        A.arrol_evict(kv, i32(4, 1), i32(4), torch.zeros(4, 16), 8)      # on the CPU


def test_decode_counts_a_rows_tokens_in_32_bits(L):
    """The kernels look some tokens past a row's end: a table row has to end 4,096 tokens before 2^31."""
    import paper_2603_24840_amd as A
    size = lambda own, pre: L.arrol_decode_attention_workspace_bytes(1, 1, 1, 8, 1, own, pre, 1 if pre else 0, 0)
    most = 2 ** 31 - 4097
    assert size(most, 0) > 0 and size(16, most) > 0
    lay = A.KVLayout(1, 1, 1, 8, 128)
    for own, pre in ((most + 1, 0), (2 ** 31 - 65, 0), (16, most + 1)):
        assert size(own, pre) == 0
        assert decode(L, lay=lay, layer=0, n=1, H=1, width=own, pw=pre, groups=1 if pre else 0) == -1, (own, pre)


def test_attention_gradient_counts_a_launchs_lanes(L):
    """Workgroups of 512 lanes with heads of more than 64: 2^23 of them are 2^32 lanes."""
    for hd, n, rc in ((128, 2 ** 22 - 3, -2), (128, 2 ** 22 - 2, -1), (72, 2 ** 23 - 3, -1), (64, 2 ** 22 - 2, -2), (64, 2 ** 23 - 3, -2), (64, 2 ** 23 - 2, -1)):
        assert grad(L, ws=None, n=n, H=2, KV=2, hd=hd, ks=256, vs=256) == rc, (hd, n)


def test_decode_refuses_what_its_launches_cannot_hold_and_nothing_else(L):
    """Both sides of the limits on workgroups: of the main launch, of the join where there are more than 8 ranges, of the weights' tokens."""
    import paper_2603_24840_amd as A
    size = L.arrol_decode_attention_workspace_bytes

    def takes(n, H, KV, own_pages, pre_pages=0, groups=0, weights=0):
        need = size(n, H, KV, 64, 16, own_pages, pre_pages, groups, weights)
        rc = decode(L, lay=A.KVLayout(1, 16, KV, 64, 128), layer=0, n=n, H=H, width=own_pages, pw=pre_pages, groups=groups, ws=None, wout=FAKE if weights else None)
        assert rc == (-2 if need else -1), (n, H, KV, own_pages, rc, need)       # what has a workspace lacks nothing but that
        return need > 0

    assert takes(2048, 32, 32, 8192, 8192, 256)                     # tables of 131,072 tokens: 5 million workgroups
    assert takes(2 ** 24 - 1, 1, 1, 1) and not takes(2 ** 24, 1, 1, 1)                       # a workgroup a rollout
    assert takes(2 ** 20 - 1, 16, 1, 1152) and not takes(2 ** 20, 16, 1, 1152)               # 9 ranges of 2,048 tokens, a workgroup of the join a query row
    assert takes(2 ** 26 - 1, 1, 1, 1, weights=0) is False
    assert takes(2 ** 16 - 1, 1, 1, 1024, weights=1) and not takes(2 ** 16, 1, 1, 1024, weights=1)      # 2^30 tokens
    assert takes(8, 4, 2, 4, 3, 2 ** 20) and not takes(8, 4, 2, 4, 3, 2 ** 20 + 1)


def test_evict_workspace_of_what_is_refused_is_0(L):
    size = L.arrol_evict_workspace_bytes
    assert size(2 ** 22 - 1, 4, 16, 32) > 0 and size(2 ** 22, 4, 16, 32) == 0 and evict(L, rows=2 ** 22 - 1, ws=None) == -2 and evict(L, rows=2 ** 22, ws=None) == -1
    assert size(1, 2 ** 31 - 1025, 1, 32) > 0 and size(1, 2 ** 31 - 1024, 1, 32) == 0
    assert size(1, 2 ** 27 - 65, 16, 32) > 0 and size(1, 2 ** 27 - 64, 16, 32) == 0


def test_binding_refuses_integers_of_more_than_32_bits():
    """ctypes passes the lower 32 bits on: without a look at them these would run with 0 or 1."""
    import paper_2603_24840_amd as A
    q, kv = torch.zeros(4, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 4, 16, 2, 64, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    for big in (2 ** 32, 2 ** 32 + 1, 2 ** 31, -2 ** 31 - 1):
        with pytest.raises(ValueError, match="32 bits"):
            A.arrol_evict(kv, i32(4, 1), i32(4), torch.zeros(4, 16), big)
        with pytest.raises(ValueError, match="32 bits"):
            A.arrol_evict(kv, i32(4, 1), i32(4), torch.zeros(4, 16), 8, n_first=big)
        with pytest.raises(ValueError, match="32 bits"):
            A.arrol_evict(kv, i32(4, 1), i32(4), torch.zeros(4, 16), 8, n_recent=big)
        with pytest.raises(ValueError, match="32 bits"):
            A.arrol_decode_attention(q, kv, big, i32(4, 1), i32(4))
