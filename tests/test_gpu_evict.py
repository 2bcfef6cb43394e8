"""Eviction by gathered attention weight, every output and the whole pool bit for bit against a plain implementation."""
import numpy as np
import pytest
import torch

from helpers import npy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def A():
    import paper_2603_24840_amd as pkg
    pkg.lib()
    return pkg


def slots_after(weight, n, budget, first, recent):
    """Which slot each slot's token comes from."""
    left = min(n, budget)
    if n <= budget:
        return list(range(n))
    rank = np.where(np.isnan(weight), -np.inf, weight.astype(np.float64))
    nan = np.isnan(weight)
    order = sorted(range(first, n - recent), key=lambda t: (nan[t], -rank[t], t))
    stay = set(range(first)) | set(range(n - recent, n)) | set(order[:left - first - recent])
    behind = iter(sorted(t for t in stay if t >= left))
    return [t if t in stay else next(behind) for t in range(left)]


def reference(kv, table, lengths, weight, position, budget, first, recent):
    """kv int16 [layers, 2, pages, page, kv, hd] (modified)."""
    page, pages = kv.shape[3], kv.shape[2]
    cap = table.shape[1] * page
    out = dict(block_table=table.copy(), seq_len=np.zeros(len(lengths), np.int32), weight=np.zeros_like(weight),
               position=np.full((len(lengths), cap), -1, np.int32))
    for r, n in enumerate(lengths):
        n = max(0, min(int(n), cap))
        left = min(n, budget)
        source = slots_after(weight[r], n, budget, first, recent)
        before = kv.copy() if any(s != t for t, s in enumerate(source)) else kv
        for t, s in enumerate(source):
            if s != t:
                a, b = table[r][s // page], table[r][t // page]
                if 0 <= a < pages and 0 <= b < pages:
                    kv[:, :, b, t % page] = before[:, :, a, s % page]
        out["block_table"][r, -(-left // page):] = -1
        out["seq_len"][r] = left
        out["weight"][r, :left] = weight[r][source]
        out["position"][r, :left] = np.asarray(source) if position is None else position[r][source]
    return out


def make(lengths, page, KV, hd, layers, seed, spare=0, kind="heavy"):
    rng = np.random.default_rng(seed)
    need = [-(-max(0, x) // page) for x in lengths]
    width, total = max([1] + need) + spare, sum(need) + 2
    pages = list(rng.permutation(total))
    table = np.full((len(lengths), width), -1, np.int32)
    for r, n in enumerate(need):
        table[r, :n] = [pages.pop() for _ in range(n)]
    weight = rng.random((len(lengths), width * page)).astype(np.float32)
    if kind == "heavy":
        weight = np.where(weight < 0.6, 0, weight ** 8).astype(np.float32)
    elif kind == "few":
        weight = np.floor(weight * 3).astype(np.float32)
    elif kind == "equal":
        weight[:] = 0.25
    elif kind == "odd":
        weight = rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -1.0, 1e-45, 3e38], np.float32), weight.shape)
    kv = rng.integers(-2 ** 15, 2 ** 15, (layers, 2, total, page, KV, hd), dtype=np.int16)
    return kv, table, np.asarray(lengths, np.int32), weight


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def check(A, kv, table, lengths, weight, budget, first=0, recent=0, position=None):
    kv_dev = dev(kv).view(torch.bfloat16)
    got = A.arrol_evict(kv_dev, dev(table), dev(lengths), dev(weight), budget, n_first=first, n_recent=recent, position=None if position is None else dev(position))
    torch.cuda.synchronize()
    expect = kv.copy()
    want = reference(expect, table, lengths, weight, position, budget, first, recent)
    assert np.array_equal(npy(kv_dev.view(torch.int16)), expect), "pool"
    for name in want:
        assert np.array_equal(npy(got[name]), want[name], equal_nan=name == "weight"), name
    return got


@pytest.mark.parametrize("kind", ["heavy", "few", "equal", "odd"])
@pytest.mark.parametrize("lengths,budget,first,recent", [
    ([1], 1, 0, 0), ([2, 1, 0], 1, 0, 0), ([64, 63, 33, 32, 31, 1, 0], 32, 2, 8), ([100, 7, 260], 40, 0, 40), ([100, 7, 260], 40, 40, 0),
    ([100, 7, 260], 40, 0, 0), ([1500, 1023, 1024, 1025, 600], 500, 4, 64), ([50, 60], 0, 0, 0), ([3000, 2049], 2048, 1, 1),
])
def test_rows_cut_to_a_budget(A, kind, lengths, budget, first, recent):
    print("[case] evict %s lengths=%s budget=%d first=%d recent=%d" % (kind, lengths, budget, first, recent), flush=True)
    check(A, *make(lengths, 16, 2, 8, 2, len(lengths) + budget, kind=kind), budget, first, recent)


@pytest.mark.parametrize("page,KV,hd,layers", [(1, 1, 8, 1), (5, 3, 24, 3), (16, 8, 128, 2), (32, 1, 64, 5), (7, 8, 1, 2), (16, 8, 64, 1)])
def test_layouts(A, page, KV, hd, layers):
    print("[case] evict page=%d kv=%d hd=%d layers=%d" % (page, KV, hd, layers), flush=True)
    check(A, *make([90, 41, 130, 0, 17], page, KV, hd, layers, page, spare=2), 40, 3, 9)


def test_positions_follow_two_cuts(A):
    print("[case] evict twice, the outputs of one the inputs of the next, in place", flush=True)
    kv, table, lengths, weight = make([300, 90, 200], 16, 2, 16, 2, 5)
    first = check(A, kv, table, lengths, weight, 120, 2, 10)
    expect = kv.copy()
    one = reference(expect, table, lengths, weight, None, 120, 2, 10)
    pool = dev(expect).view(torch.bfloat16)
    two = reference(expect, one["block_table"], one["seq_len"], one["weight"], one["position"], 50, 2, 10)
    got = A.arrol_evict(pool, first["block_table"], first["seq_len"], first["weight"], 50, n_first=2, n_recent=10, position=first["position"], out=first)
    torch.cuda.synchronize()
    assert got is first and np.array_equal(npy(pool.view(torch.int16)), expect)
    for name in two:
        assert np.array_equal(npy(got[name]), two[name]), name
    again = A.arrol_evict(pool, got["block_table"], got["seq_len"], got["weight"], 50, position=got["position"])       # nothing left to do
    torch.cuda.synchronize()
    assert all(torch.equal(again[x], got[x]) for x in got) and np.array_equal(npy(pool.view(torch.int16)), expect)


def test_page_ids_out_of_range_and_lengths_beyond_the_table(A):
    print("[case] evict, bad page ids and lengths", flush=True)
    kv, table, lengths, weight = make([100, 100, 60], 16, 2, 8, 2, 3)
    table[0, 0], table[0, 5], table[1, 6], table[2, 1] = -1, 2 ** 31 - 1, kv.shape[2], -2 ** 31
    lengths[1] = 2 ** 31 - 1
    check(A, kv, table, lengths, weight, 30, 1, 5)
    lengths[2] = -4
    check(A, kv, table, lengths, weight, 30, 1, 5)


def test_pool_past_32_bit_offsets(A):
    print("[case] evict, a 10 GB pool", flush=True)
    page, KV, hd = 16, 8, 128
    P = (5 << 30) // (KV * hd * page * 2)
    kv, table, lengths, weight = make([90, 64], page, KV, hd, 1, 7)
    n = kv.shape[2]
    pool = torch.zeros(1, 2, P, page, KV, hd, dtype=torch.bfloat16, device=DEV)
    pool[:, :, P - n:] = dev(kv).view(torch.bfloat16)
    A.arrol_evict(pool, dev(np.where(table >= 0, table + P - n, table).astype(np.int32)), dev(lengths), dev(weight), 30, n_first=1, n_recent=5)
    torch.cuda.synchronize()
    reference(kv, table, lengths, weight, None, 30, 1, 5)
    assert np.array_equal(npy(pool[:, :, P - n:].contiguous().view(torch.int16)), kv) and not pool[:, :, :P - n].any()


def test_side_stream_and_graph(A):
    print("[case] evict on a side stream, captured", flush=True)
    kv, table, lengths, weight = make([300, 90, 200], 16, 2, 16, 2, 15)
    side = torch.cuda.Stream()
    pool, t, n, w = dev(kv).view(torch.bfloat16), dev(table), dev(lengths), dev(weight)
    side.wait_stream(torch.cuda.current_stream())
    got = A.arrol_evict(pool, t, n, w, 100, stream=side)
    junk = [torch.full((3, w.shape[1]), 7, device=DEV) for _ in range(8)]
    side.synchronize()
    expect = kv.copy()
    want = reference(expect, table, lengths, weight, None, 100, 0, 0)
    assert np.array_equal(npy(pool.view(torch.int16)), expect) and all(np.array_equal(npy(got[x]), want[x]) for x in want)
    del junk
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = A.arrol_evict(pool, t, n, w, 100)
    for seed in (16, 17, 18):
        kv2, _, _, weight2 = make([300, 90, 200], 16, 2, 16, 2, seed)
        pool.copy_(dev(kv2).view(torch.bfloat16))
        w.copy_(dev(weight2))
        graph.replay()
        torch.cuda.synchronize()
        want = reference(kv2, table, lengths, weight2, None, 100, 0, 0)
        assert np.array_equal(npy(pool.view(torch.int16)), kv2) and all(np.array_equal(npy(held[x]), want[x]) for x in want), seed
