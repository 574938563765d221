// Which vectors (8 elements) of a head's row a lane of the rotation has: plain C++, no device.
#pragma once

#ifdef __CUDACC__
#define PP_LANES_FN __host__ __device__ __forceinline__
#else
#define PP_LANES_FN inline
#endif

namespace pp {

// Lanes of a group for heads of `dim` elements: two vectors each, and as few lanes as do.
constexpr int rotate_lanes(int dim) { return dim > 96 ? 8 : dim > 80 ? 6 : dim > 64 ? 5 : dim > 32 ? 4 : dim > 16 ? 2 : 1; }

// A thread's group and its vectors of a row of `per_head`; from per_head on: none.
struct RotateLane {
    int lane, of_warp;                  // of the group, of the warp's 32 / lanes; the lanes left over are in none
    int at[2];
};

// turned: lanes whose two vectors hold the two halves of 8 pairs (half layout of whole
// vectors); the others have the row's rest in two stretches.  Without those (-1) vectors
// go round the lanes.
PP_LANES_FN RotateLane rotate_lane(int thread, int lanes, int per_head, int turned)
{
    RotateLane r;
    r.lane = thread % 32 % lanes;
    r.of_warp = thread % 32 / lanes;
    if (r.of_warp >= 32 / lanes) {
        r.at[0] = r.at[1] = per_head;
    } else if (turned >= 0) {
        const int others = (per_head - 2 * turned + 1) / 2;
        r.at[0] = r.lane < turned + others ? r.lane + (r.lane < turned ? 0 : turned) : per_head;
        r.at[1] = r.lane < turned + others ? r.at[0] + (r.lane < turned ? turned : others) : per_head;
    } else {
        r.at[0] = r.lane;
        r.at[1] = r.lane + lanes;
    }
    return r;
}

// Without stretches: the thread that has vector v of the row of `thread`'s group, and which of its two that is.
PP_LANES_FN int rotate_holder(int thread, int lanes, int v) { return thread - thread % 32 % lanes + v % lanes; }
PP_LANES_FN int rotate_which(int lanes, int v) { return v / lanes; }

}  // namespace pp
