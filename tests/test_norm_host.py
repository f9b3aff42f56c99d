"""Layer norm without a GPU: where its kernels read and write, and what they hold."""
import os
import re
import subprocess

import numpy as np
import pytest

from block_util import kernels, norm_graph

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2012_02732_amd", "csrc")


def test_offsets_of_a_norm_stay_in_their_image(tmp_path):
    """Every channel that exists is where it belongs, and what does not exist, channel or token, is outside for a load, which is checked by the
    thread's own part alone, and for a store, whose parts are added up in 32 bits: for workgroups of every size and form over images of up to
    2^29 values, few channels of millions of tokens among them (8 of 4096 x 4096: a turn of the channels is 2^31 bytes)."""
    src = tmp_path / "offsets.cpp"
    src.write_text(r"""
#include <cstdio>
#include <initializer_list>
#include "ng_device.h"
using u64 = unsigned long long;
static int check(int threads, int K, int lanes, u64 C, u64 T) {
    const int rows = threads / lanes;
    const u64 bytes = 4 * C * T;
    for (int k = 0; k < K; ++k) {
        const unsigned shared = (unsigned)k * ng::norm_turn(rows, (int)T);
        for (int row = 0; row < rows; ++row) {
            const u64 c = row + (u64)k * rows;
            for (u64 t : {(u64)0, T / 2, T - 1}) {
                const unsigned own = ng::norm_lane(c < C, row, (int)T, (int)t), sum = ng::norm_store_at(own, shared);
                if (c < C ? !(own < bytes && sum == 4 * (c * T + t) && (u64)own + shared < bytes) : !(own >= bytes && sum >= bytes)) return 1;
            }
            const unsigned none = ng::norm_lane(false, row, (int)T, 0);
            if (none < bytes || ng::norm_store_at(none, shared) < bytes) return 2;
        }
    }
    return 0;
}
int main() {
    const u64 most = 1ull << 29;
    for (int threads : {256, 512, 1024})
        for (int K : {8, 16})
            for (int lanes : {1, 2, 4, 8})
                for (u64 C : {1, 2, 3, 7, 8, 31, 32, 33, 64, 127, 128, 129, 520, 1000, 1023, 1024, 2047, 4096, 8192, 16384}) {
                    if (C > (u64)K * threads / lanes) continue;
                    for (u64 T : {(u64)1, (u64)3, (u64)4, (u64)333, (u64)65536, (u64)1000000, (u64)1 << 22, (u64)2500000, (u64)1 << 24, most / C - 1, most / C})
                        if (T > 0 && C * T <= most)
                            if (const int what = check(threads, K, lanes, C, T)) return std::printf("%d: %d threads of %d channels, %d side by side, %llu x %llu\n", what, threads, K, lanes, C, T), 1;
                }
    std::puts("ok");
}
""")
    exe = str(tmp_path / "offsets")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", CSRC, str(src), "-o", exe], check=True)
    done = subprocess.run([exe], capture_output=True, text=True)
    assert (done.returncode, done.stdout.strip()) == (0, "ok")
    # and the kernels take their offsets from nowhere else
    kernels = open(os.path.join(CSRC, "ng_block_tiles.inc")).read()
    calls = re.findall(r"norm_(?:load|store)<V(?:, FIN)?>\(\w+, (.*)\);", kernels)
    assert len(calls) == 7 and all(re.match(r"(on \? |\w*row \+ k \* rows < a\.C \? )?(lane_at|store_at|at)( : kOutside)?, (k|\(first \+ j\)) \* turn", call) for call in calls), calls
    assert kernels.count("lane_at = norm_lane(in, row, a.T, t0),") + kernels.count("lane_at = norm_lane(in, row, a.T, t0);") == kernels.count("turn = norm_turn(rows, a.T);") == 1
    assert kernels.count("const unsigned at = norm_store_at(lane, shared);") == 1


HELD = {"8": (256, 8), "16": (256, 16), "few": (256, 16), "half": (512, 8), "half_16": (512, 16), "wide": (1024, 8), "wide_16": (1024, 16)}      # threads, channels of each


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 9, 33, 260, 5000])
def test_the_kernel_of_a_norm_holds_its_channels(tokens):
    """What a workgroup has in registers is at least all channels of its tokens: with one to three tokens, 1, 2 and 4 threads side by side (three
    tokens of 1025 to 1365 channels are 3075 to 4095 values, but 1024 channels are all that 64 threads have)."""
    side_by_side = {1: 1, 2: 2, 3: 4}.get(tokens, 1)
    for n in (1, 16):
        for c in (1, 8, 255, 520, 1023, 1024, 1025, 1100, 1365, 1366, 2047, 2048, 2049, 4095, 4096, 4097, 8192, 8193, 16384, 16385):
            g = norm_graph(*(np.zeros(s, np.float32) for s in ((1, 1, 1, 1), 1, 1, (1, 1, 1, 1))), 1e-5)
            for name in ("x", "dy"):                            # the shapes alone
                g.nodes[g.names[name]].params = dict(n=n, c=c, h=1, w=tokens)
            for name, kernel in kernels(g).items():
                how = re.fullmatch("layer_norm_(?:dgrad_|wgrad_)?(.*)", kernel).group(1)
                most = 16 * (256 // side_by_side) if tokens < 4 else 16384
                if how == "many":                               # read again for each sum: any number
                    assert c > most, (n, c, tokens, kernel)
                else:
                    threads, turns = HELD[how]
                    assert c <= min(most, turns * (threads // side_by_side)), (n, c, tokens, kernel)
