"""Positions of queries and keys, and new tokens into the paged pool, against a plain implementation in 64 bits.

Tolerance, element by element (u = 2^-8: a rounding to bf16): u |x'| of the result's rounding, and on m (|x| + |y|) what cosine and sine are off by: the angle's
remainder in turns is rounded to 32 bits (pi 2^-24 radians), the function has up to 4 units of 2^-24, m's product and the two products and their sum 2^-24 each, and
the product of position and frequency in 64 bits is off by 2^-52 of the angle: 2^-21 + 2^-51 |angle| in all.
"""
import numpy as np
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


def bits(x):
    return x.detach().contiguous().view(torch.int16).cpu()


def reference(x, position, inv_freq, interleaved, inverse=False, magnitude=1.0):
    """fp64 values and tolerances of rows x [T, heads, hd]; `position` any numbers."""
    x, f = x.detach().cpu().double(), inv_freq.cpu().double()
    angle = torch.as_tensor(position).cpu().double()[:, None] * f
    c, s = (torch.cos(angle) * magnitude)[:, None], (torch.sin(angle) * magnitude)[:, None] * (-1 if inverse else 1)
    n = f.numel()
    i = torch.arange(n)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    val, tol = x.clone(), torch.zeros_like(x)
    val[..., a], val[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    rough = magnitude * (x[..., a].abs() + x[..., b].abs()) * (2.0 ** -21 + 2.0 ** -51 * angle.abs())[:, None]
    tol[..., a], tol[..., b] = rough + U * val[..., a].abs(), rough + U * val[..., b].abs()
    return val, tol


def agree(got, val, tol, name=""):
    off = (got.detach().cpu().double() - val).abs()
    assert bool((off <= tol + 1e-30).all()), (name, float((off - tol).max()))


def rand(*shape, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV).to(torch.bfloat16)


def frequencies(A, rot, base=1e4):
    return A.arrol_rotary_frequencies(rot, base, device=DEV)


SHAPES = [(4, 2, 64, 64), (32, 8, 128, 128), (16, 8, 128, 64), (3, 1, 80, 40), (2, 2, 40, 20), (5, 5, 40, 36), (1, 1, 8, 8), (1, 1, 8, 2), (7, 1, 256, 256), (2, 1, 256, 6), (24, 8, 80, 80)]


@pytest.mark.parametrize("H,KV,hd,rot", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T", [1, 3, 70])
def test_rotary(A, H, KV, hd, rot, interleaved, T):
    print("[case] rotary T=%d heads=%d/%d hd=%d rot=%d interleaved=%d" % (T, H, KV, hd, rot, interleaved), flush=True)
    x = rand(T, H + 2 * KV, hd, seed=T + rot)
    q, k = x[:, :H], x[:, H:H + KV]
    far = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1000003, 65535])
    position = torch.tensor(np.resize(far, T) + (np.arange(T) // len(far)) * (np.resize(far, T) < 2 ** 30) * (np.resize(far, T) > -2 ** 30), dtype=torch.int32, device=DEV)
    f = frequencies(A, rot)
    for inverse, magnitude in ((False, 1.0), (True, 1.25)):
        got = A.arrol_rotary(q, k, position, f, interleaved=interleaved, inverse=inverse, magnitude=magnitude)
        for y, z, name in zip((q, k), got, "qk"):
            assert z.is_contiguous() and z.shape == y.shape
            agree(z, *reference(y, position, f, interleaved, inverse, magnitude), name)
            assert torch.equal(bits(z[..., rot:]), bits(y[..., rot:]))
    only, none = A.arrol_rotary(q, None, position, f, interleaved=interleaved)
    assert none is None and torch.equal(only, A.arrol_rotary(q, k, position, f, interleaved=interleaved)[0])


@pytest.mark.parametrize("T", [2048, 8191, 8193, 20011, 65537])
def test_rotary_of_many_tokens(A, T):
    """A wavefront takes a part of a token's heads where tokens are few, whole tokens beyond 65,536."""
    print("[case] rotary T=%d" % T, flush=True)
    x, f = rand(T, 6, 64, seed=T), frequencies(A, 64)
    position = torch.arange(T, dtype=torch.int32, device=DEV) * 131
    for z, y in zip(A.arrol_rotary(x[:, :4], x[:, 4:], position, f), (x[:, :4], x[:, 4:])):
        agree(z, *reference(y, position, f, False))


@pytest.mark.parametrize("interleaved,rot", [(False, 64), (False, 40), (False, 36), (True, 36)])
def test_rotary_in_place_and_into_strided_rows(A, interleaved, rot):
    print("[case] rotary in place, rot=%d" % rot, flush=True)
    x, f = rand(130, 9, 72, seed=rot), frequencies(A, rot)
    position = torch.arange(130, dtype=torch.int32, device=DEV) * 7 - 100
    want = A.arrol_rotary(x[:, :5], x[:, 5:7], position, f, interleaved=interleaved)
    y = x.clone()
    got = A.arrol_rotary(y[:, :5], y[:, 5:7], position, f, interleaved=interleaved, out_q=y[:, :5], out_k=y[:, 5:7])
    assert got[0].data_ptr() == y.data_ptr() and torch.equal(y[:, :5], want[0]) and torch.equal(y[:, 5:7], want[1]) and torch.equal(y[:, 7:], x[:, 7:])
    room = torch.full((130, 12, 72), 7.0, dtype=torch.bfloat16, device=DEV)
    A.arrol_rotary(x[:, :5], x[:, 5:7], position, f, interleaved=interleaved, out_q=room[:, 2:7], out_k=room[:, 9:11])
    assert torch.equal(room[:, 2:7], want[0]) and torch.equal(room[:, 9:11], want[1])
    assert bool((room[:, :2] == 7).all()) and bool((room[:, 7:9] == 7).all()) and bool((room[:, 11:] == 7).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_keeps_odd_values_to_their_pairs(A, interleaved):
    print("[case] rotary, NaN and infinities", flush=True)
    x, f = rand(40, 3, 64, seed=3), frequencies(A, 32)
    position = torch.arange(1, 41, dtype=torch.int32, device=DEV)
    y = x.clone()
    y[5, 1, 4], y[6, 0, 7], y[7, 2, 40] = float("nan"), float("inf"), float("nan")
    a, b = A.arrol_rotary(x, None, position, f, interleaved=interleaved)[0], A.arrol_rotary(y, None, position, f, interleaved=interleaved)[0]
    odd = torch.zeros_like(x, dtype=torch.bool)
    for t, h, e in ((5, 1, 4), (6, 0, 7)):
        odd[t, h, [e, e ^ 1 if interleaved else e + 16]] = True
    odd[7, 2, 40] = True
    assert torch.equal(bits(a)[~odd.cpu()], bits(b)[~odd.cpu()]) and not bool(torch.isfinite(b[odd].float()).any())


@pytest.mark.parametrize("interleaved,rot", [(False, 64), (True, 64), (False, 24)])
def test_the_inverse_is_the_gradient(A, interleaved, rot):
    """Of L = <g, rotary(x)>: against differences of L, formed in 64 bits from the kernel's outputs, and <g, R x> = <R' g, x>."""
    print("[case] rotary's gradient, rot=%d" % rot, flush=True)
    x, g, f = rand(33, 2, 64, seed=1), rand(33, 2, 64, seed=2), frequencies(A, rot)
    position = torch.arange(33, dtype=torch.int32, device=DEV) * 1000
    turned = A.arrol_rotary(x, None, position, f, interleaved=interleaved, magnitude=1.5)[0].double()
    grad = A.arrol_rotary(g, None, position, f, interleaved=interleaved, magnitude=1.5, inverse=True)[0].double()
    rough = (U * (g.double() * turned).abs() + U * (x.double() * grad).abs()).sum() + 2.0 ** -19 * 3 * (g.double().abs() * x.double().abs().amax()).sum()
    assert abs(float((g.double() * turned).sum() - (grad * x.double()).sum())) <= float(rough)
    for e in (0, 1, 11, 12, 23, 31, 32, 63):        # by one element of every row, 4 up and 4 down
        moved = x.double().clone()
        step = torch.zeros_like(moved)
        step[..., e] = 4
        up, down = ((x.double() + s * step).to(torch.bfloat16) for s in (1, -1))
        L = [(g.double() * A.arrol_rotary(y, None, position, f, interleaved=interleaved, magnitude=1.5)[0].double()).sum(-1) for y in (up, down)]
        width = (up.double() - down.double())[..., e]
        slope = (L[0] - L[1]) / width
        most = sum((g.double().abs() * A.arrol_rotary(y, None, position, f, interleaved=interleaved, magnitude=1.5)[0].double().abs()).sum(-1) for y in (up, down))
        tol = (U * 2 ** -1 * 2 * most + 2.0 ** -18 * most) / width.abs() + U * grad[..., e].abs() + 1e-5
        # moving an element leaves the others of its row bit for bit, so their roundings cancel but for its partner's
        assert bool(((slope - grad[..., e]).abs() <= tol).all()), e


def test_rotary_past_2_to_the_31_elements(A):
    print("[case] rotary, rows past 2^31 elements", flush=True)
    T, f = 2 ** 18 + 5, frequencies(A, 64)
    x = torch.empty(T, 128, 64, dtype=torch.bfloat16, device=DEV)
    x[-6:] = rand(6, 128, 64)
    position = torch.arange(T, dtype=torch.int32, device=DEV)
    q, k = x[:, :2], x[:, 2:3]
    got = A.arrol_rotary(q, k, position, f, out_q=q, out_k=k)
    want = A.arrol_rotary(rand(6, 128, 64)[:, :2], rand(6, 128, 64)[:, 2:3], position[-6:], f)
    assert torch.equal(got[0][-6:], want[0]) and torch.equal(got[1][-6:], want[1]) and torch.equal(x[-6:, 3:], rand(6, 128, 64)[:, 3:])


# ---- append -----------------------------------------------------------------------------------------------------------------------

def pool_reference(kv, layer, table, start, ends, k, v, position, f, interleaved, magnitude):
    """The pool, values and tolerances in 64 bits, and where tokens were written; `ends` the clamped offsets as a list."""
    val, page = kv.detach().cpu().double(), kv.shape[3]
    tol = torch.zeros_like(val)
    table, start = table.cpu().tolist(), start.cpu().tolist()
    places = [None] * k.shape[0]
    for s in range(len(start)):
        for t in range(ends[s], ends[s + 1]):
            places[t] = (s, start[s] + t - ends[s])
    pos = [(0 if p is None else p[1]) for p in places] if position is None else position.cpu().tolist()
    turned = reference(k, torch.tensor(pos), f, interleaved, magnitude=magnitude) if f is not None else (k.cpu().double(), torch.zeros(k.shape, dtype=torch.float64))
    for t, p in enumerate(places):
        if p is None or p[1] < 0 or p[1] // page >= len(table[0]):
            continue
        page_id = table[p[0]][p[1] // page]
        if 0 <= page_id < kv.shape[2]:
            val[layer, 0, page_id, p[1] % page], tol[layer, 0, page_id, p[1] % page] = turned[0][t], turned[1][t]
            val[layer, 1, page_id, p[1] % page] = v[t].cpu().double()
    return val, tol, torch.tensor(pos), torch.tensor([p is not None for p in places])


def check_append(A, H, KV, hd, rot, page, new, start, width, n_pages, interleaved=False, layer=1, table=None, before=0, behind=0, given=True, want_k=True, seed=0, magnitude=1.0, cu=None):
    single = cu is None and new is None
    n = len(start)
    ends = list(range(n + 1)) if single else [before + int(x) for x in np.concatenate([[0], np.cumsum(new)])]
    T = ends[-1] + behind
    x = rand(T, H + 2 * KV, hd, seed=seed)
    q, k, v = x[:, :H], x[:, H:H + KV], x[:, H + KV:]
    g = torch.Generator().manual_seed(seed)
    if table is None:
        table = torch.randperm(max(n_pages, n * width), generator=g)[:n * width].reshape(n, width).to(torch.int32)
        table = torch.where(table < n_pages, table, -1)
    table, start = table.to(DEV), torch.tensor(start, dtype=torch.int32, device=DEV)
    kv = rand(2, 2, n_pages, page, KV, hd, seed=seed + 1)
    position = (torch.arange(T, dtype=torch.int32, device=DEV) * 37 + 5) if given else None
    f = None if rot is None else frequencies(A, rot)
    val, tol, pos, known = pool_reference(kv, layer, table, start, ends, k, v, position, f, interleaved, magnitude)
    got = A.arrol_append(k, v, kv, layer, table, start, None if single else torch.tensor(ends, dtype=torch.int64, device=DEV), q=q, position=position, inv_freq=f,
                         interleaved=interleaved, magnitude=magnitude, want_k=want_k)
    torch.cuda.synchronize()
    written = tol > 0 if f is not None else torch.zeros_like(tol, dtype=torch.bool)
    off = (kv.cpu().double() - val).abs()
    assert bool((off[~written] == 0).all()) and bool((off <= tol + 1e-30).all())
    for y, z in ((q, got["q"]), (k, got["k"])) if want_k else ((q, got["q"]),):
        rows, rough = reference(y, pos, f, interleaved, magnitude=magnitude) if f is not None else (y.cpu().double(), torch.zeros(y.shape, dtype=torch.float64))
        agree(z[known.to(DEV)], rows[known], rough[known])
        assert torch.equal(bits(z)[~known], bits(y)[~known])
    assert want_k or got["k"] is None
    return got, kv


@pytest.mark.parametrize("H,KV,hd,rot", SHAPES[:8] + [(4, 2, 64, None)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_of_single_tokens(A, H, KV, hd, rot, interleaved):
    print("[case] append, heads=%d/%d hd=%d rot=%s" % (H, KV, hd, rot), flush=True)
    for n, given in ((1, True), (9, False), (70, True)):
        check_append(A, H, KV, hd, rot, 16, None, [(i * 7) % 33 for i in range(n)], 3, 3 * n, interleaved, given=given, want_k=n == 9, seed=n, magnitude=1.25)


@pytest.mark.parametrize("new,start", [([5], [0]), ([0, 3, 0, 17, 1], [4, 30, 2, 15, 47]), ([16, 32, 33], [0, 16, 5]), ([1] * 130, list(range(130)))])
@pytest.mark.parametrize("before,behind", [(0, 0), (3, 6)])
def test_append_of_packed_sequences(A, new, start, before, behind):
    print("[case] append, packed %s" % new[:5], flush=True)
    width = max(-(-(a + b) // 16) for a, b in zip(new, start))
    for given in (True, False):
        check_append(A, 4, 2, 64, 64, 16, new, start, width, width * len(new) + 2, before=before, behind=behind, given=given, seed=len(new))


def test_append_among_many_sequences(A):
    """The search for a row's sequence takes 64 offsets at a step: one, two and three steps."""
    for n in (1, 63, 64, 65, 4095, 4097):
        print("[case] append, %d sequences" % n, flush=True)
        new = [(i * 5) % 4 if n < 4000 else int(i % 3 == 0) for i in range(n)]
        check_append(A, 1, 1, 8, 8, 4, new, [i % 3 for i in range(n)], 2, 2 * n, before=2, behind=3, seed=n)


def test_append_leaves_out_what_has_no_place(A):
    print("[case] append, bad pages and slots", flush=True)
    table = torch.tensor([[0, -1, 2], [5, 6, 2 ** 31 - 1], [-2 ** 31, 3, 4], [1, 7, 8]], dtype=torch.int32)
    for page in (8, 16):
        check_append(A, 2, 1, 64, 64, page, [20, 40, 30, 9], [0, 4, -7, 2 * page], 3, 7, table=table, seed=page)
        check_append(A, 2, 1, 64, 32, page, None, [2 ** 31 - 1, -2 ** 31, 3 * page, page], 3, 7, table=table, seed=page)
    # no page at all
    check_append(A, 2, 1, 64, 64, 16, [3], [0], 1, 0, table=torch.zeros(1, 1, dtype=torch.int32))


@pytest.mark.parametrize("cu", [[0, 9, 4, 12], [-5, 3, 8, 100], [7, 7, 7, 7], [2 ** 62, 0, -2 ** 62, 5], [-2 ** 63, 2 ** 63 - 1, 1, 2]])
def test_append_stays_in_bounds_for_any_offsets(A, cu):
    """What a sequence is with offsets that do not ascend is not said; nothing but the table's pages of the layer is written."""
    print("[case] append, offsets %s" % cu, flush=True)
    room = torch.full((2, 2, 12, 8, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    x = rand(12, 8, 64)
    table = torch.tensor([[1, 2], [4, 5], [7, 8]], dtype=torch.int32, device=DEV)
    got = A.arrol_append(x[:, 4:6], x[:, 6:], room, 0, table, torch.tensor([0, 3, 5], dtype=torch.int32, device=DEV), torch.tensor(cu, device=DEV), q=x[:, :4], inv_freq=frequencies(A, 64))
    torch.cuda.synchronize()
    touched = (room != 3).flatten(3).any(-1)
    assert not bool(touched[1].any()) and not bool(touched[:, :, [0, 3, 6, 9, 10, 11]].any()) and bool(torch.isfinite(got["q"].float()).all())


@pytest.mark.parametrize("KV,hd,rot,same", [(1, 8, 2, 3), (2, 64, 64, 40), (5, 80, 40, 2), (8, 128, 128, 17), (3, 40, 36, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_of_tokens_with_one_slot(A, KV, hd, rot, same, interleaved):
    """Every element of the slot is one of its tokens', and nothing else of the pool is touched."""
    print("[case] append, %d tokens a slot, heads=%d hd=%d rot=%d interleaved=%d" % (same, KV, hd, rot, interleaved), flush=True)
    n, f = 6, frequencies(A, rot)
    x = rand(n * same, 1 + 2 * KV, hd, seed=hd)
    k, v = x[:, 1:1 + KV], x[:, 1 + KV:]
    table, start = torch.tensor([[4], [1], [7], [2], [0], [6]], dtype=torch.int32, device=DEV), torch.tensor([3, 15, 0, 8, 9, 1], dtype=torch.int32, device=DEV)
    position = torch.arange(n * same, dtype=torch.int32, device=DEV) * 11
    before = rand(1, 2, 9, 16, KV, hd, seed=4)
    turned = A.arrol_rotary(k, None, position, f, interleaved=interleaved)[0]
    for packed in (False, True):        # a token a row of the table, row s + n i being row s again, or sequences of one token
        kv = before.clone()
        cu = torch.arange(n * same + 1, dtype=torch.int64, device=DEV) if packed else None
        got = A.arrol_append(k, v, kv, 0, table.repeat(same, 1), start.repeat(same), cu, q=x[:, :1], position=position, inv_freq=f, interleaved=interleaved, want_k=True)
        assert torch.equal(got["k"], turned) and torch.equal(got["q"], A.arrol_rotary(x[:, :1], None, position, f, interleaved=interleaved)[0])
        for rows, of in ((turned, 0), (v, 1)):
            there = kv[0, of, table[:, 0].long(), start.long()]
            assert bool((there == rows.view(same, n, KV, hd)).any(0).all())
        kv[0, :, table[:, 0].long(), start.long()] = before[0, :, table[:, 0].long(), start.long()]
        assert torch.equal(kv, before)


def test_append_in_place_and_without_queries(A):
    print("[case] append in place", flush=True)
    x, f = rand(50, 8, 64), frequencies(A, 64)
    table = torch.arange(8, dtype=torch.int32, device=DEV).reshape(2, 4)
    cu, start = torch.tensor([0, 20, 50], device=DEV), torch.tensor([3, 0], dtype=torch.int32, device=DEV)
    kv = [torch.zeros(1, 2, 8, 16, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    want = A.arrol_append(x[:, 4:6], x[:, 6:], kv[0], 0, table, start, cu, q=x[:, :4], inv_freq=f, want_k=True)
    y = x.clone()
    A.arrol_append(y[:, 4:6], y[:, 6:], kv[1], 0, table, start, cu, q=y[:, :4], inv_freq=f, want_k=True, out_q=y[:, :4], out_k=y[:, 4:6])
    assert torch.equal(kv[0], kv[1]) and torch.equal(y[:, :4], want["q"]) and torch.equal(y[:, 4:6], want["k"]) and torch.equal(y[:, 6:], x[:, 6:])
    assert A.arrol_append(x[:, 4:6], x[:, 6:], kv[2], 0, table, start, cu, inv_freq=f) == dict(q=None, k=None)
    assert torch.equal(kv[0], kv[2])


def test_append_past_2_to_the_31_elements(A):
    print("[case] append, a pool past 2^31 elements", flush=True)
    pages = 70000
    kv = torch.empty(1, 2, pages, 16, 8, 128, dtype=torch.bfloat16, device=DEV)
    table = torch.tensor([[pages - 1], [pages - 2]], dtype=torch.int32, device=DEV)
    x, f = rand(2, 16, 128), frequencies(A, 128)
    kv[:, :, -3:] = 0
    A.arrol_append(x[:, :8], x[:, 8:], kv, 0, table, torch.tensor([15, 3], dtype=torch.int32, device=DEV), inv_freq=f)
    turned = A.arrol_rotary(x[:, :8], None, torch.tensor([15, 3], dtype=torch.int32, device=DEV), f)[0]
    assert torch.equal(kv[0, 0, -1, 15], turned[0]) and torch.equal(kv[0, 0, -2, 3], turned[1]) and torch.equal(kv[0, 1, -1, 15], x[0, 8:]) and torch.equal(kv[0, 1, -2, 3], x[1, 8:])
    assert not kv[:, :, -1, :15].any() and not kv[:, :, -3].any()


def test_append_and_rotary_on_a_stream_and_in_a_graph(A):
    """A decode step's call captured once: replays see what the buffers hold then."""
    print("[case] append in a graph", flush=True)
    x, f = rand(6, 8, 64), frequencies(A, 64)
    table, start = torch.arange(12, dtype=torch.int32, device=DEV).reshape(6, 2), torch.arange(6, dtype=torch.int32, device=DEV)
    position = torch.arange(6, dtype=torch.int32, device=DEV) + 40
    kv, side = torch.zeros(1, 2, 12, 16, 2, 64, dtype=torch.bfloat16, device=DEV), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first = A.arrol_append(x[:, 4:6], x[:, 6:], kv, 0, table, start, q=x[:, :4], position=position, inv_freq=f, stream=side)
    side.synchronize()
    eager = torch.zeros_like(kv)
    want = A.arrol_append(x[:, 4:6], x[:, 6:], eager, 0, table, start, q=x[:, :4], position=position, inv_freq=f)
    assert torch.equal(kv, eager) and torch.equal(first["q"], want["q"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = A.arrol_append(x[:, 4:6], x[:, 6:], kv, 0, table, start, q=x[:, :4], position=position, inv_freq=f)
        back = A.arrol_rotary(captured["q"], None, position, f, inverse=True)[0]
        start.add_(1)
        position.add_(1)
    at, where = start.clone(), position.clone()
    for i in range(4):
        x.copy_(rand(6, 8, 64, seed=20 + i))
        graph.replay()
        want = A.arrol_append(x[:, 4:6], x[:, 6:], eager, 0, table, at, q=x[:, :4], position=where, inv_freq=f)
        torch.cuda.synchronize()
        assert torch.equal(kv, eager) and torch.equal(captured["q"], want["q"]) and torch.equal(back, A.arrol_rotary(want["q"], None, where, f, inverse=True)[0])
        at.add_(1), where.add_(1)
