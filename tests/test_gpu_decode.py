"""Attention of single tokens over the paged pool with shared prefixes, and the weights it gathers, against a plain implementation in 64 bits.

Tolerances (u = 2^-8 for bf16, e = 2^-24 for fp32), derived before the first run: a score is off by dz = (hd + 4) e scale sum |q||k|; a weight by
2 dz + 2^-20 (exp2, its argument, the joined sum) + tokens * e relatively; the output by u |o| + (u + that) sum p |v|; lse by that and 4 e |lse|; a gathered weight
by that times the sum of what was added, and 2 e of the result per addition."""
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


def tables(lengths, page, pages, width=None):
    """Block table rows cut from the list `pages` (consumed), -1 behind a row's length."""
    need = [-(-x // page) for x in lengths]
    width = max([1] + need) if width is None else width
    table = np.full((len(lengths), width), -1, np.int32)
    for r, n in enumerate(need):
        table[r, :n] = [pages.pop() for _ in range(n)]
    return table


class Batch:
    def __init__(self, sizes, prefix, lengths, H, KV, hd, page, seed, layers=2, extra=3, before=0, spread=1.0, spare=0):
        rng = np.random.default_rng(seed)
        self.n, self.page = len(lengths), page
        total = sum(-(-x // page) for x in list(prefix) + list(lengths)) + extra
        pages = list(rng.permutation(total))
        self.prefix, self.lengths, self.sizes = list(prefix), list(lengths), list(sizes)
        width = max([1] + [-(-x // page) for x in prefix]) + spare
        self.ptable = tables(prefix, page, pages, width) if prefix else None
        self.table = tables(lengths, page, pages, max([1] + [-(-x // page) for x in lengths]) + spare)
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.kv = torch.randn(layers, 2, total, page, KV, hd, generator=g, device=DEV).to(torch.bfloat16)
        self.q = (spread * torch.randn(self.n, H, hd, generator=g, device=DEV)).to(torch.bfloat16)
        self.offsets = np.concatenate([[before], before + np.cumsum(sizes)]).astype(np.int64)
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
        self.args = [dev(self.table), dev(np.asarray(lengths, np.int32))]
        self.shared = [dev(self.ptable), dev(np.asarray(prefix, np.int32)), dev(self.offsets)] if prefix else [None, None, None]

    def run(self, A, layer=1, **kw):
        got = A.arrol_decode_attention(self.q, self.kv, layer, *self.args, *self.shared, **kw)
        torch.cuda.synchronize()
        return got

    def places(self, table, row, length):
        t = np.arange(length)
        return table[row][t // self.page].astype(np.int64), t % self.page

    def reference(self, layer=1, scale=None):
        kv, q = self.kv[layer].cpu().double().numpy(), self.q.cpu().double().numpy()
        n, H, hd = q.shape
        KV = kv.shape[3]
        scale = hd ** -0.5 if scale is None else scale
        out, lse, tol_out, tol_lse = np.zeros_like(q), np.full((n, H), -np.inf), np.zeros_like(q), np.zeros((n, H))
        cap = self.table.shape[1] * self.page
        w, tw = np.zeros((n, cap)), np.zeros((n, cap))
        pw = tpw = None
        if self.prefix:
            pcap = self.ptable.shape[1] * self.page
            pw, tpw = np.zeros((len(self.prefix), pcap)), np.zeros((len(self.prefix), pcap))
        for r in range(n):
            group = [g for g in range(len(self.prefix)) if self.offsets[g] <= r < self.offsets[g + 1]]
            P = self.prefix[group[0]] if group else 0
            where = [self.places(self.ptable, group[0], P)] if group else []
            where.append(self.places(self.table, r, self.lengths[r]))
            ids, at = np.concatenate([x[0] for x in where]), np.concatenate([x[1] for x in where])
            there = (ids >= 0) & (ids < kv.shape[1])
            k, v = kv[0][np.where(there, ids, 0), at], kv[1][np.where(there, ids, 0), at]
            if not there.any():
                continue
            for h in range(H):
                x, y, z = q[r, h], k[there, h * KV // H], v[there, h * KV // H]
                s = scale * (y @ x)
                rel = 2 * np.max((hd + 4) * E * scale * (np.abs(y) @ np.abs(x))) + 2.0 ** -20 + len(s) * E + np.abs(s).max() * 4 * E
                p = np.exp(s - s.max())
                lse[r, h] = s.max() + np.log(p.sum())
                p /= p.sum()
                out[r, h] = p @ z
                tol_out[r, h] = U * np.abs(out[r, h]) + (U + rel) * (p @ np.abs(z))
                tol_lse[r, h] = rel + 4 * E * abs(lse[r, h])
                full = np.zeros(len(there))
                full[there] = p
                if group:
                    pw[group[0], :P] += full[:P]
                    tpw[group[0], :P] += (rel + 512 * E) * full[:P]
                w[r, :self.lengths[r]] += full[P:]
                tw[r, :self.lengths[r]] += (rel + 512 * E) * full[P:]
        return dict(out=(out, tol_out), lse=(lse, tol_lse), weight=(w, tw), prefix_weight=(pw, tpw))

    def check(self, A, layer=1, scale=None, **kw):
        got, want = self.run(A, layer, scale=scale, **kw), self.reference(layer, scale)
        for name, (val, tol) in want.items():
            if val is None or got[name] is None:
                continue
            x = got[name].cpu().double().numpy()
            assert np.array_equal(np.isneginf(x), np.isneginf(val)), name
            fine = np.isfinite(val)
            off, allowed = np.abs(x[fine] - val[fine]), tol[fine] + 1e-30
            assert np.all(off <= allowed), (name, float((off / allowed).max()), float(off.max()))
        return got


@pytest.mark.parametrize("H,KV,hd,page", [(4, 2, 64, 16), (8, 1, 128, 8), (6, 6, 40, 5), (32, 8, 128, 16), (40, 2, 72, 32), (48, 1, 64, 1)])
@pytest.mark.parametrize("sizes,prefix,lengths", [
    ([1], [1], [1]),
    ([3, 0, 5], [100, 7, 33], [1, 31, 32, 33, 64, 65, 200, 17]),
    ([9], [700], [0, 1, 2, 3, 4, 90, 600, 5, 6]),
    ([2, 2], [0, 129], [0, 5, 0, 64]),
    ([], [], [1, 77, 1025]),
])
def test_shared_prefixes_and_own_tokens(A, sizes, prefix, lengths, H, KV, hd, page):
    print("[case] decode sizes=%s prefix=%s lengths=%s heads=%d/%d hd=%d page=%d" % (sizes, prefix, lengths, H, KV, hd, page), flush=True)
    b = Batch(sizes, prefix, lengths, H, KV, hd, page, len(lengths) + hd)
    got = b.check(A, want_weight=True)
    plain = b.run(A)
    assert torch.equal(plain["out"], got["out"]) and torch.equal(plain["lse"], got["lse"]) and plain["weight"] is None


@pytest.mark.parametrize("hd", [8, 24, 32, 96, 120])
def test_head_sizes(A, hd):
    print("[case] decode hd=%d" % hd, flush=True)
    Batch([4, 2], [50, 90], [3, 40, 70, 1, 9, 33], 6, 2, hd, 16, hd).check(A, want_weight=True)


def test_no_tokens_at_all(A):
    print("[case] decode, rollouts without a token", flush=True)
    got = Batch([2, 1], [0, 40], [0, 5, 0], 4, 2, 64, 16, 1).check(A, want_weight=True)
    assert not got["out"][0].any() and bool(torch.all(got["lse"][0] == -float("inf"))) and got["out"][2].any()


def test_rollouts_of_no_group_see_their_own_tokens_alone(A):
    print("[case] decode, rollouts before and behind the groups", flush=True)
    b = Batch([2, 3], [60, 45], [9, 20, 33, 5, 70, 1, 64, 12], 4, 2, 64, 16, 4, before=2)
    b.check(A, want_weight=True)
    for bad in (np.array([-5, 3, 10 ** 12]), np.array([8, 4, 0]), np.array([0, 2 ** 62, -2 ** 62])):      # clamped; what comes out of disorder is not defined
        b.shared[2] = torch.from_numpy(bad.astype(np.int64)).to(DEV)
        b.run(A, want_weight=True)
    b.offsets = np.array([0, 3, 8])
    b.shared[2] = torch.tensor([-5, 3, 10 ** 12], dtype=torch.int64, device=DEV)
    b.check(A, want_weight=True)


def test_nan_past_the_lengths_and_bad_page_ids(A):
    """Page tails, pages of nobody and page ids out of range hold nothing that counts."""
    print("[case] decode, NaN behind the lengths, page ids out of range", flush=True)
    for hd, H, KV in ((64, 4, 2), (128, 20, 1)):
        b = Batch([3, 2], [37, 90], [5, 33, 64, 100, 17], H, KV, hd, 16, 8, spare=2)
        clean = b.check(A, want_weight=True)
        used = torch.zeros(b.kv.shape[2], 16, dtype=torch.bool)
        for table, lens in ((b.ptable, b.prefix), (b.table, b.lengths)):
            for r, n in enumerate(lens):
                ids, at = b.places(table, r, n)
                used[torch.from_numpy(ids), torch.from_numpy(at)] = True
        for bad in (float("nan"), float("inf")):
            b.kv[:, :, ~used.to(DEV)] = bad
            got = b.run(A, want_weight=True)
            for name in clean:
                assert torch.equal(got[name], clean[name]), name
        b.kv.nan_to_num_(0.0, 0.0, 0.0)
        for table, dev in ((b.ptable, b.shared[0]), (b.table, b.args[0])):
            table[0, 0] = -7
            table[1, 1] = 2 ** 31 - 1
            table[-1, 0] = b.kv.shape[2]
            dev.copy_(torch.from_numpy(table))
        got = b.check(A, want_weight=True)
        assert not got["weight"][0, :16].any()


def test_lengths_are_clamped_to_the_table(A):
    print("[case] decode, lengths beyond the table and below zero", flush=True)
    b = Batch([2, 2], [64, 32], [48, 48, 48, 48], 4, 2, 64, 16, 3)
    want = b.check(A, want_weight=True)
    b.args[1] = torch.tensor([2 ** 31 - 1, 49, 48, 60], dtype=torch.int32, device=DEV)
    b.shared[1] = torch.tensor([10 ** 9, 32], dtype=torch.int32, device=DEV)
    got = b.run(A, want_weight=True)
    assert all(torch.equal(got[x], want[x]) for x in want)
    b.args[1].fill_(-3)
    b.lengths = [0] * 4
    b.check(A, want_weight=True)


@pytest.mark.parametrize("spread", [0.0, 12.0])
def test_flat_and_peaked_weights(A, spread):
    print("[case] decode spread=%g" % spread, flush=True)
    Batch([5, 3], [300, 1000], [500, 3, 64, 200, 1, 90, 33, 700], 8, 2, 128, 16, 6, spread=spread).check(A, want_weight=True, scale=0.5)


def test_weights_gather_over_layers_and_tokens(A):
    """The _out may be the _in; behind a row's length the weight is 0, so that the next token starts from nothing."""
    print("[case] decode, weights gathered in place", flush=True)
    b = Batch([3, 4], [130, 20], [1, 40, 70, 33, 64, 2, 129], 8, 2, 64, 16, 14, spare=1)
    want = {name: 0.0 for name in ("weight", "prefix_weight")}
    tol = dict(want)
    for layer in (0, 1):
        ref = b.reference(layer)
        for name in want:
            want[name], tol[name] = want[name] + ref[name][0], tol[name] + ref[name][1]
    w, pw = torch.full((7, b.table.shape[1] * 16), 0.0, device=DEV), torch.zeros(2, b.ptable.shape[1] * 16, device=DEV)
    for r, n in enumerate(b.lengths):
        w[r, n:] = float("nan")
    b.run(A, 0, want_weight=True, weight=w, prefix_weight=pw, out_weight=w, out_prefix_weight=pw)
    b.run(A, 1, want_weight=True, weight=w, prefix_weight=pw, out_weight=w, out_prefix_weight=pw)
    for name, got in (("weight", w), ("prefix_weight", pw)):
        x = got.cpu().double().numpy()
        assert np.all(np.abs(x - want[name]) <= tol[name] + 4 * E * want[name]), name


def test_long_cache_past_32_bit_offsets(A):
    """A pool of more than 2^32 bytes a slab and 2^31 elements: the last pages against the first of a small one."""
    print("[case] decode, a 10 GB pool", flush=True)
    KV, hd, page = 8, 128, 16
    P = (5 << 30) // (KV * hd * page * 2)
    kv = torch.zeros(1, 2, P, page, KV, hd, dtype=torch.bfloat16, device=DEV)
    b = Batch([2], [200], [70, 33], 16, KV, hd, page, 2, layers=1)
    small = b.run(A, 0, want_weight=True)
    n = b.kv.shape[2]
    kv[:, :, P - n:] = b.kv
    shift = lambda t: torch.where(t >= 0, t + (P - n), t)
    b.kv, b.args[0], b.shared[0] = kv, shift(b.args[0]), shift(b.shared[0])
    got = b.run(A, 0, want_weight=True)
    for name in small:
        assert torch.equal(got[name], small[name]), name


def test_many_ranges(A):
    print("[case] decode, one rollout over 70,000 tokens", flush=True)
    Batch([1], [30000], [40001], 2, 1, 64, 16, 2).check(A, want_weight=True)


@pytest.mark.parametrize("hd", [64, 128])
def test_groups_of_many_query_rows(A, hd):
    """64 query rows and more of a kv head read a prefix: tiles of 64 rows, some with wavefronts that have none, groups of very different sizes."""
    print("[case] decode, large groups hd=%d" % hd, flush=True)
    b = Batch([16, 3, 21], [500, 1, 2100], [1 + 7 * i for i in range(40)], 16, 4, hd, 16, 50)
    b.check(A, want_weight=True)
    b.check(A, layer=0)


def test_ranges_longer_than_the_table_of_places(A):
    """More than 128 x 2,048 tokens: a workgroup's range is looked up in parts; 20 query rows for the parts' shared path, and 2 for the other."""
    for H in (20, 2):
        print("[case] decode, 270,000 tokens, heads=%d" % H, flush=True)
        Batch([1], [270000], [300], H, 1, 16, 16, 51, layers=1).check(A, layer=0, want_weight=True)


def test_single_tokens_are_the_last_rows_of_the_packed_form(A):
    """The same keys through arrol_attention (nq = 1): both forms are held to the same reference within their tolerances."""
    print("[case] decode against the packed form", flush=True)
    b = Batch([4], [150], [30, 1, 64, 99], 8, 2, 64, 16, 31)
    got, want = b.run(A), b.reference()
    rows = []
    for r, n in enumerate(b.lengths):
        ids, at = (np.concatenate(x) for x in zip(b.places(b.ptable, 0, 150), b.places(b.table, r, n)))
        rows.append(b.kv[1][:, torch.from_numpy(ids).to(DEV), torch.from_numpy(at).to(DEV)])
    k, v = torch.cat(rows, 1)
    cu = torch.tensor(np.concatenate([[0], np.cumsum([150 + n for n in b.lengths])]), dtype=torch.int64, device=DEV)
    out, lse = A.arrol_attention(b.q, k.contiguous(), v.contiguous(), torch.arange(5, dtype=torch.int64, device=DEV), cu)
    for x, y, (val, tol) in ((out, got["out"], want["out"]), (lse.t(), got["lse"], want["lse"])):
        assert np.all(np.abs(x.cpu().double().numpy() - val) <= tol) and np.all(np.abs(y.cpu().double().numpy() - val) <= tol)


def test_calls_repeat_bit_for_bit_on_a_side_stream_and_in_a_graph(A):
    print("[case] decode repeated, on a side stream, captured", flush=True)
    b = Batch([4, 3], [333, 20], [100, 1, 64, 200, 7, 40, 3], 8, 2, 128, 16, 40)
    want = b.run(A, want_weight=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = A.arrol_decode_attention(b.q, b.kv, 1, *b.args, *b.shared, want_weight=True, stream=side)
    junk = [torch.full((7, 8, 128), float("nan"), device=DEV) for _ in range(8)]
    side.synchronize()
    assert all(torch.equal(got[x], want[x]) for x in want)
    del junk
    q, kv, lens = b.q.clone(), b.kv.clone(), b.args[1].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = A.arrol_decode_attention(q, kv, 1, b.args[0], lens, *b.shared, want_weight=True)
    for seed in (40, 41, 42):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        b.q.copy_(torch.randn(q.shape, generator=g, device=DEV))
        b.args[1].copy_(torch.tensor([100, 1, 64, 200, 7, 40, 3], device=DEV) - (seed - 40))
        want = b.run(A, want_weight=True)
        q.copy_(b.q)
        lens.copy_(b.args[1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[x], want[x]) for x in want), seed


def test_empty_batches(A):
    print("[case] decode, no rollouts", flush=True)
    b = Batch([2], [40], [3, 4], 4, 2, 64, 16, 1)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    got = A.arrol_decode_attention(b.q[:0], b.kv, 0, b.args[0][:0], none, b.shared[0], b.shared[1], torch.zeros(2, dtype=torch.int64, device=DEV), want_weight=True)
    torch.cuda.synchronize()
    assert got["out"].shape == (0, 4, 64) and not got["prefix_weight"].any()
    got = A.arrol_decode_attention(b.q, b.kv, 0, *b.args)
    assert got["prefix_weight"] is None


def close(got, clean, rows):
    """Rows that a spoiled one shares a wavefront with: the maximum they are scaled by may move on at other places."""
    x, y = got[rows].float(), clean[rows].float()
    assert bool(torch.isfinite(x).all()) and bool(((x - y).abs() <= 2 * U * y.abs() + U * 4.0).all())


@pytest.mark.parametrize("sizes,prefix,H,KV,hd", [([2, 2], [60, 300], 4, 2, 64), ([2, 2], [700, 2600], 20, 1, 128)])
def test_nan_reaches_the_rollout_that_sees_it(A, sizes, prefix, H, KV, hd):
    """A query, or a key alone in its range of tokens, whose scores are all NaN: no number comes out, not what a rollout without tokens gets."""
    print("[case] decode, NaN queries and keys, prefix=%s heads=%d/%d" % (prefix, H, KV), flush=True)
    nan = float("nan")
    b = Batch(sizes, prefix, [1, 400, 33, 1], H, KV, hd, 16, 61)
    clean = b.run(A, want_weight=True)
    q = b.q.clone()
    b.q[0, 1], b.q[2] = nan, nan                 # one head of the first rollout, all of the third
    got = b.run(A, want_weight=True)
    for name in ("out", "lse"):
        assert bool(torch.isnan(got[name][0, 1]).all()) and bool(torch.isnan(got[name][2]).all()), name
    others = torch.ones(4, H, dtype=torch.bool, device=DEV)
    others[0, 1], others[2] = False, False
    close(got["out"], clean["out"], others)
    assert bool(((got["lse"] - clean["lse"])[others].abs() <= 1e-4).all())
    for name, row, n in (("weight", 0, 1), ("weight", 2, 33), ("prefix_weight", 0, prefix[0]), ("prefix_weight", 1, prefix[1])):
        assert bool(torch.isnan(got[name][row, :n]).all()) and not got[name][row, n:].any(), (name, row)
    b.q.copy_(q)
    kv = b.kv.clone()
    for row in (0, 3):                           # these rollouts' only tokens
        ids, at = b.places(b.table, row, 1)
        b.kv[1, 0, ids[0], at[0]] = nan
    got = b.run(A, want_weight=True)
    for name in ("out", "lse"):
        assert bool(torch.isnan(got[name][[0, 3]]).all()), name
        assert torch.equal(got[name][[1, 2]], clean[name][[1, 2]]), name
    b.kv.copy_(kv)
    ids, at = b.places(b.ptable, 1, prefix[1])   # a whole prefix
    b.kv[1, 0, torch.from_numpy(ids).to(DEV), torch.from_numpy(at).to(DEV)] = nan
    got = b.run(A, want_weight=True)
    assert bool(torch.isnan(got["out"][2:]).all()) and bool(torch.isnan(got["lse"][2:]).all()) and torch.equal(got["out"][:2], clean["out"][:2])


@pytest.mark.parametrize("bad", [float("inf"), -float("inf")])
@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("sizes,prefix,H", [([2, 1], [33, 65], 4), ([2, 1], [1000, 545], 40)])
def test_an_infinite_value_gives_an_infinite_output(A, sizes, prefix, H, hd, bad):
    """Also where it is the one token whose place the missing ones of a step of 32 take: their weight is 0, and 0 times infinity would be NaN."""
    print("[case] decode, infinite values, hd=%d heads=%d" % (hd, H), flush=True)
    b = Batch(sizes, prefix, [1, 33, 40], H, 2, hd, 16, 63)
    want = b.reference()["out"]
    expect = np.zeros((3, H, hd), bool)
    spoiled = [(b.table, 0, 1, 0, [0]), (b.table, 1, 33, 32, [1]), (b.ptable, 1, prefix[1], prefix[1] // 32 * 32, [2])]      # row, its length, token, who sees it
    for table, row, n, token, seen_by in spoiled:
        ids, at = b.places(table, row, n)
        b.kv[1, 1, ids[token], at[token], 1, 3::5] = bad            # the second kv head's
        for r in seen_by:
            expect[r, H // 2:, 3::5] = True
    got = b.run(A, want_weight=True)["out"].cpu().double().numpy()
    assert np.array_equal(np.isinf(got), expect) and np.all(got[expect] == bad)
    rest = ~expect
    assert np.all(np.abs(got[rest] - want[0][rest]) <= want[1][rest])


@pytest.mark.parametrize("hd", [8, 40, 64, 72, 120, 128])
@pytest.mark.parametrize("sizes,prefix,H", [([2, 1], [50, 90], 4), ([2, 1], [700, 90], 40)])
def test_a_key_of_minus_infinity_has_no_weight(A, sizes, prefix, H, hd):
    """Its score is -inf, and nothing else: what a head is padded with counts 0 in the products."""
    print("[case] decode, keys of -inf, hd=%d heads=%d" % (hd, H), flush=True)
    b = Batch(sizes, prefix, [3, 40, 70], H, 2, hd, 16, 62)
    b.q[:, :, hd - 1] = b.q[:, :, hd - 1].abs() + 0.5
    for table, lens in ((b.table, b.lengths), (b.ptable, b.prefix)):
        for row, n in enumerate(lens):
            ids, at = b.places(table, row, n)
            b.kv[1, 0, ids[-1], at[-1], :, hd - 1] = -float("inf")
    got = b.run(A, want_weight=True)
    b.lengths, b.prefix = [n - 1 for n in b.lengths], [n - 1 for n in b.prefix]      # as if the last tokens were not there
    for name, (val, tol) in b.reference().items():
        assert np.all(np.abs(got[name].cpu().double().numpy() - val) <= tol + 1e-30), name


@pytest.mark.parametrize("H,KV,hd", [(8, 2, 64), (40, 2, 128)])
def test_tables_much_wider_than_their_rows(A, H, KV, hd):
    """Ranges are cut from what a table could hold; a row takes part in as many as its length reaches."""
    print("[case] decode, tables of 40,000 tokens, heads=%d/%d" % (H, KV), flush=True)
    Batch([3, 2], [700, 33], [1, 500, 64, 2500, 129], H, KV, hd, 16, 68, spare=2500).check(A, want_weight=True)
