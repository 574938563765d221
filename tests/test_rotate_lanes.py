"""CPU checks of which vectors of a row a lane of the rotation has (csrc/pp_rotate_lanes.h, compiled by
itself): every lane reads places of its own group, and the lanes that belong to no group none at all."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_01655_gb300", "csrc")

MAIN = r"""
#include <cstdio>
#include "pp_rotate_lanes.h"
using namespace pp;

// Faults of all threads of a CTA with heads of `dim`, `rotated` of them in `turned` lanes of stretches (-1: without).
static long faults(int dim, int rotated, int turned)
{
    const int lanes = rotate_lanes(dim), per_head = dim / 8, pairs = rotated / 2;
    long bad = lanes < 1 || 2 * lanes < per_head;
    for (int thread = 0; thread < 128; ++thread) {
        const RotateLane r = rotate_lane(thread, lanes, per_head, turned);
        const bool in = thread % 32 < 32 / lanes * lanes;
        for (int x = 0; x < 2; ++x) {
            if (r.at[x] >= per_head) continue;
            bad += !in || r.at[x] < 0;
            if (turned >= 0) continue;
            for (int d = 8 * r.at[x]; d < 8 * r.at[x] + 8 && d < rotated; ++d) {
                const int v = (d < pairs ? d + pairs : d - pairs) / 8;       // the other one's of the pair
                const int holder = rotate_holder(thread, lanes, v), which = rotate_which(lanes, v);
                if (holder < 0 || holder >= 128 || which < 0 || which > 1) {
                    ++bad;
                    continue;
                }
                const RotateLane other = rotate_lane(holder, lanes, per_head, turned);
                bad += holder / 32 != thread / 32 || other.of_warp != r.of_warp || other.at[which] != v;
            }
        }
        if (!in || r.lane) continue;
        // all vectors of a row are had once by the group's lanes, and the first ones of pairs with the second ones
        int count[64] = {};
        for (int l = 0; l < lanes; ++l) {
            const RotateLane o = rotate_lane(thread + l, lanes, per_head, turned);
            bad += o.of_warp != r.of_warp || o.lane != l;
            for (int x = 0; x < 2; ++x)
                if (o.at[x] < per_head) ++count[o.at[x]];
            if (turned >= 0 && o.at[0] < turned) bad += o.at[1] != o.at[0] + turned;
        }
        for (int v = 0; v < per_head; ++v) bad += count[v] != 1;
    }
    return bad;
}
int main()
{
    long all = 0;
    for (int dim = 8; dim <= 128; dim += 8)
        for (int rotated = 0; rotated <= dim; rotated += 2) {
            const long without = faults(dim, rotated, -1), with = rotated % 16 ? 0 : faults(dim, rotated, rotated / 16);
            if (without || with) printf("%d of %d: %ld %ld\n", rotated, dim, without, with);
            ++all;
        }
    printf("%ld\n", all);
}
"""


def test_lanes_have_and_read_rows_of_their_own_group(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    (tmp_path / "main.cpp").write_text(MAIN)
    subprocess.run([gxx, "-std=c++17", "-Wall", "-Werror", "-I" + CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")],
                   check=True)
    out = subprocess.run([str(tmp_path / "main")], check=True, capture_output=True, text=True).stdout
    assert out == f"{sum(dim // 2 + 1 for dim in range(8, 129, 8))}\n"
