"""Which tokens and heads the warps of the norm and rotation kernels take, by the kernels' own host-compiled rule (CPU)."""
import os
import subprocess

import pytest

from paper_2512_10411_b200.build import CSRC, INCLUDE

SOURCE = r"""
#include <cstdio>
#include <vector>
#include "swaa.h"
#include "swaa_rope.cuh"
using namespace swaa;

// Every index into `positions` is that of a token, and every (token, head) of queries, keys and values is taken once.
template <int D, int kRows>
static bool sound(int T, int Hq, int Hkv, bool values, int sms) {
    const RopeSplit split(Hq, Hkv, D, kRows, values);
    const unsigned warps = rope_blocks(T, split, sms) * kRopeWarps;
    std::vector<int> taken((size_t)T * (Hq + 2 * Hkv), 0);
    for (unsigned w = 0; w < warps; ++w) {
        const RopeWarp<D, kRows> me(split, w, warps);
        if (!me.works(T)) continue;
        if (me.stream >= T) return false;  // the first position that the warp loads
        for (long long t = me.stream; t < T; t += me.streams)
            for (int u = 0; u < me.groups; ++u)
                for (int i = 0; i < RopeWarp<D, kRows>::kHeads; ++i) {
                    const int h = me.head(split, u) + i, heads = me.keys ? Hkv : Hq;
                    if (h < heads) ++taken[t * (Hq + 2 * Hkv) + (!me.keys ? h : Hq + (me.value(split, u) ? Hkv : 0) + h)];
                }
    }
    for (int t = 0; t < T; ++t)
        for (int h = 0; h < Hq + 2 * Hkv; ++h)
            if (taken[(size_t)t * (Hq + 2 * Hkv) + h] != (h < Hq + Hkv || values ? 1 : 0)) return false;
    return true;
}

int main() {
    const int heads[][2] = {{1, 1}, {4, 2}, {5, 1}, {7, 7}, {16, 4}, {28, 4}, {32, 8}, {64, 8}, {9, 3}, {200, 100}};
    int bad = 0, cases = 0;
    for (const auto& h : heads)
        for (int T : {1, 2, 3, 4, 5, 6, 7, 8, 9, 17, 37, 300, 2500})
            for (int values = 0; values < 2; ++values)
                for (int sms : {1, 148}) {
                    const bool ok = sound<64, kRopeRows>(T, h[0], h[1], values, sms) && sound<128, kRopeRows>(T, h[0], h[1], values, sms) &&
                                    sound<64, kRopeBwdRows>(T, h[0], h[1], values, sms) && sound<128, kRopeBwdRows>(T, h[0], h[1], values, sms);
                    ++cases;
                    if (!ok) printf("%d tokens, %d + %d heads, values %d, %d SMs\n", T, h[0], h[1], values, sms), ++bad;
                }
    printf("%d of %d cases wrong\n", bad, cases);
    return bad != 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    where = tmp_path_factory.mktemp("rope_split")
    src, exe = where / "rope_split.cu", where / "rope_split"
    src.write_text(SOURCE)
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", INCLUDE, "-I", CSRC, "-o", str(exe), str(src)],
                   check=True, capture_output=True, text=True)
    return exe


def test_warps_take_every_token_once_and_no_other(program):
    """In short calls the grid has more streams of tokens than there are tokens (one token of 4 + 2 heads of 64: four)."""
    got = subprocess.run([str(program)], capture_output=True, text=True)
    assert got.returncode == 0, got.stdout
