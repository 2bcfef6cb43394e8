"""What the gradient of the log-probabilities refuses on the host, before anything is launched, and its workspace query."""
import ctypes

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


def grad(A, **kw):
    a = dict(h=FAKE, w=FAKE, y=FAKE, lse=FAKE, g=FAKE, T=10, V=100, d=64, gh=FAKE, gw=FAKE, sum=None, ws=FAKE, nbytes=1 << 40)
    a.update(kw)
    return A.lib().arrol_logprob_grad(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(h=None), dict(h=ODD), dict(w=None), dict(w=ODD), dict(y=None), dict(lse=None), dict(g=None), dict(T=-1), dict(T=2 ** 40), dict(V=0), dict(V=-1),
                                 dict(V=2 ** 24 + 1), dict(d=0), dict(d=4), dict(d=12), dict(d=16392), dict(gh=None, gw=None), dict(gh=ODD), dict(gw=ODD), dict(sum=FAKE),
                                 dict(gw=None, sum=ODD)])
def test_refuses(A, bad):
    assert grad(A, **bad) == -1


def test_workspace(A):
    size = A.lib().arrol_logprob_grad_workspace_bytes
    need = size(10, 100, 64, 1)
    assert need > 0 and size(0, 100, 64, 1) == 0 and size(-1, 100, 64, 1) == 0 and size(10, 0, 64, 1) == 0 and size(10, 100, 60, 1) == 0
    assert grad(A, ws=None) == -2 and grad(A, ws=ODD) == -2 and grad(A, nbytes=need - 1) == -2
    for V, d in ((100, 64), (4096, 256), (128256, 2048), (151936, 4096)):
        for want in (0, 1):
            sizes = [size(T, V, d, want) for T in (1, 2, 63, 64, 65, 200, 255, 256, 257, 511, 513, 1000, 2049, 4096, 5000, 8192, 12000, 16383, 16384, 16385, 20000, 65536, 10 ** 6, 10 ** 9)]
            assert sizes == sorted(sizes)
            assert size(10 ** 9, V, d, 0) == size(16384, V, d, 0) and size(10 ** 9, V, d, 1) <= size(16384, V, d, 0) + 4 * V * d + 256
    assert size(4096, 151936, 4096, 1) < 4096 * 151936 * 4 // 2        # less than half of the logits in 32 bits
    assert grad(A, T=0, ws=None, nbytes=0, h=None, w=None, y=None, lse=None, g=None, gw=None) == 0


def test_binding_refuses(A):
    h, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(10, 64, dtype=torch.bfloat16)
    y, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for args, kw in (((h, w, y, f, f), {}), ((h, w[:, :32], y, f, f), {}), ((h, w, y[:3], f, f), {}), ((h, w, y, f[:3], f), {}), ((h, w, y, f, f[:3]), {}),
                     ((h, w, y, f, f), dict(lm_head_sum=torch.zeros(9, 64))), ((h, w, y, f, f), dict(want_hidden=False, want_lm_head=False)), ((h[0], w, y, f, f), {})):
        with pytest.raises((TypeError, ValueError)):
            A.arrol_logprob_grad(*args, **kw)


def test_binding_refuses_sizes_past_32_bits(A):
    """Of which the library would be handed the lower half: 2^32 + 10 rows as 10."""
    meta = lambda *s, **kw: torch.empty(*s, device="meta", **kw)
    y, f = meta(4, dtype=torch.int32), meta(4)
    for V, d in ((2 ** 32 + 10, 64), (10, 2 ** 32 + 64)):
        for kw in ({}, dict(want_lm_head=False), dict(want_hidden=False, lm_head_sum=meta(V, d))):
            with pytest.raises(ValueError, match="32 bits"):
                A.arrol_logprob_grad(meta(4, d, dtype=torch.bfloat16), meta(V, d, dtype=torch.bfloat16), y, f, f, **kw)


def test_kernel_query(A):
    out = [ctypes.c_int32(-7) for _ in range(8)]
    ask = lambda T, V, d, n=8: A.lib().arrol_logprob_grad_kernels(T, V, d, *[ctypes.byref(x) for x in out[:n]], *[None] * (8 - n))
    for bad in ((0, 10, 64), (-1, 10, 64), (10, 0, 64), (10, 10, 60), (10, 10, 16392)):
        assert ask(*bad) == -1 and all(x.value == -7 for x in out)
    assert ask(10, 10, 64, 7) == -1
    for T, V, d in ((1, 1, 8), (16384, 151936, 4096), (10 ** 9, 2 ** 24, 16384), (40000, 300, 64), (1024, 5000, 1000)):
        assert ask(T, V, d) == 0
        rows, tokens, columns, product_tokens, slabs, parts, pieces, found = (x.value for x in out)
        assert rows in (64, 128, 256) and columns in (64, 128, 256) and tokens in (64, 128, 256) and product_tokens in (64, 128, 256)
        assert (rows != 256 or d % 64 == 0) and 1 <= slabs <= 32 and 1 <= parts <= 32 and pieces >= 1 and (not found or (T <= 1024 and rows < 256))


def test_kernel_query_has_what_the_header_says(A):
    """Every number of tiles and parts that the header names, and no other, over sizes that meet them all."""
    out = [ctypes.c_int32() for _ in range(8)]
    seen = [set() for _ in out]
    for T, V, d in ((1, 1, 8), (16384, 151936, 4096), (10 ** 9, 2 ** 24, 16384), (40000, 300, 64), (1024, 5000, 1000), (311, 151936, 2048), (60, 60001, 264), (297, 878561, 72), (72, 79901, 264),
                    (640, 32000, 2048), (2579, 3172, 1728), (330, 140001, 968), (346, 4096, 256), (2, 1268440, 144), (332, 515, 2848), (943, 2368, 2360)):
        assert A.lib().arrol_logprob_grad_kernels(T, V, d, *[ctypes.byref(x) for x in out]) == 0
        rows, tokens, columns, product_tokens, slabs, parts, pieces, found = values = [x.value for x in out]
        tiles = {(256, 256), (128, 160), (128, 128), (128, 64), (64, 64)}
        assert (rows, tokens) in tiles and (columns, product_tokens) in tiles and (rows != 256 or d % 64 == 0)
        assert 1 <= slabs <= 32 and 0 <= parts <= 32 and (parts > 0 or (T <= 320 and columns < 256)) and pieces >= 1 and (not found or (T <= 1024 and rows < 256))
        for have, x in zip(seen, values):
            have.add(x)
    assert seen[1] == seen[3] == {64, 128, 160, 256} and seen[0] == seen[2] == {64, 128, 256} and seen[7] == {0, 1}
    assert max(seen[4]) > 1 and {0, 1} < seen[5] and max(seen[6]) > 1
