"""What a call of the log-prob gradient takes fits the workspace that it asks for, whatever its tiles cost: the host's choice, compiled by itself with the costs it was measured with and
with others, on sizes from one token to many pieces."""
import os
import shlex
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_24840_amd", "csrc")

PROGRAM = r"""
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <random>
#include "logprob_grad_plan.h"
using namespace logprob_grad;

int main() {
    std::mt19937_64 random(1);
    auto uniform = [&](double a, double b) { return a + (b - a) * (random() >> 11) / 9007199254740992.0; };
    auto size = [&](double a, double b) { return std::max<int64_t>(1, std::llround(std::exp(uniform(std::log(a), std::log(b))))); };
    long parts = 0, slabs = 0, resident = 0, pieces_v = 0, pieces_t = 0, none = 0;
    for (int trial = 0; trial < 150000; ++trial) {
        const int64_t T = trial % 2 ? size(1, 2e5) : size(1985, 70000), V = size(1, 1 << 24), d = 8 * size(1, trial % 2 ? 2048 : 64);
        Size costs[kForms];
        for (int f = 0; f < kForms; ++f) {
            costs[f] = kSize[f];
            if (trial % 3)
                for (double* c : {&costs[f].tile, &costs[f].step, &costs[f].lone, &costs[f].tile_w, &costs[f].step_w, &costs[f].lone_w}) *c *= std::exp(uniform(-2, 2));
        }
        const Pieces p = pieces(T, V, d, costs);
        const char* wrong = nullptr;
        for (int lm_head = 0; lm_head < 2; ++lm_head) {
            const Workspace w = workspace(T, V, d, lm_head != 0);
            const int64_t token = p.rows * 4, v = std::min(V, p.v);
            auto holds = [&](const char* what, size_t from, size_t to, int64_t need) { if (to < from || static_cast<int64_t>(to - from) < need) wrong = what; };
            holds("count", w.n_active, w.g, 4);
            holds("g", w.g, w.lse, token), holds("lse", w.lse, w.target, token), holds("target", w.target, w.row, token), holds("row", w.row, w.rest, token), holds("rest", w.rest, w.H, token);
            holds("hidden states", w.H, w.dz, p.rows * d * 2);
            holds("dz", w.dz, w.slabs, up256(p.rows) * p.v * 2);
            if (p.slabs > 1 || p.n_v > 1) holds("slabs", w.slabs, w.slabs_w, p.slabs * p.rows * d * 4);
            if (p.parts > 1) holds("parts", w.slabs_w, w.sum, p.parts * v * d * 4);
            if (lm_head && p.n_rows > 1) holds("sum", w.sum, w.bytes, V * d * 4);
        }
        const int64_t k64 = (std::min(V, p.v) + 63) / 64;
        if (p.rows < 1 || p.rows > kPieceRows || p.rows * (p.n_rows - 1) >= T || p.rows * p.n_rows < T) wrong = "pieces of tokens";
        if (p.v % 256 || p.v * (p.n_v - 1) >= up256(V) || p.v * p.n_v < V) wrong = "pieces of the vocabulary";
        if (p.slabs < 1 || p.slabs > kMaxSlabs || static_cast<int64_t>(p.slabs) * p.k64_per_slab < k64 || static_cast<int64_t>(p.slabs - 1) * p.k64_per_slab >= k64) wrong = "parts of the vocabulary";
        if (p.parts < 1 || p.parts > kMaxSlabs || (p.parts > 1 && V * d > kCachedElements)) wrong = "parts of the tokens";
        if (p.blocks && (p.blocks > 16 || p.products == kRing || p.rows > kResidentTokens || p.parts > 1)) wrong = "resident form";
        if (p.dz == kRing && d % 64) wrong = "tiles of dz";
        if (wrong) return std::printf("%s: T = %lld, V = %lld, d = %lld, costs %s\n", wrong, (long long)T, (long long)V, (long long)d, trial % 3 ? "others" : "measured"), 1;
        parts += p.parts > 1, slabs += p.slabs > 1, resident += p.blocks > 0, pieces_v += p.n_v > 1, pieces_t += p.n_rows > 1;
        none += part_floats(T, V, d) == 0 && p.n_v > 1 && p.v * d * 2 <= kSlabFloats && p.rows >= 2048;
    }
    std::printf("%ld %ld %ld %ld %ld %ld\n", parts, slabs, resident, pieces_v, pieces_t, none);
    return 0;
}
"""


def test_what_a_call_takes_fits_its_workspace(tmp_path):
    cxx = shlex.split(os.environ.get("CXX") or "g++")
    if not shutil.which(cxx[0]):
        pytest.skip("no C++ compiler")
    source, program = tmp_path / "plan.cpp", tmp_path / "plan"
    source.write_text(PROGRAM)
    subprocess.run(cxx + ["-O2", "-std=c++17", "-I", CSRC, str(source), "-o", str(program)], check=True)
    got = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True, timeout=100)
    assert got.returncode == 0, got.stdout
    assert all(int(n) > 200 for n in got.stdout.split()), got.stdout        # each of what it is about came up
