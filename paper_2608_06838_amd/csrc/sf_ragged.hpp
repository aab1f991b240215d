// sf_ragged.hpp -- sequences of a ragged batch, as the kernels see them.
#pragma once
#include "sf_chunk.hpp"

namespace sf {

// A sequence's rows [begin, end) and slot; end <= begin or slot < 0: nothing to do.
struct Seq {
    int64_t begin, end;
    int slot;
};
__device__ __forceinline__ int64_t clamp_row(int64_t x, int64_t T) { return x < 0 ? 0 : x > T ? T : x; }
__device__ __forceinline__ Seq seq_of(const RaggedArgs &r, int i) {
    Seq s;
    s.begin = clamp_row(r.cu[i], r.T);
    s.end = clamp_row(r.cu[i + 1], r.T);
    s.slot = r.slot ? r.slot[i] : i;
    if (s.slot >= r.n_slots) s.slot = -1;
    return s;
}

// Runs of `run` tokens, none across a sequence's end.  Run numbers of sequence i start
// at cu[i] / run + i, which leaves it room for its own ceil(n / run) runs (its last one
// may be short, and one number may stay unused), so a launch of T / run + N numbers
// needs neither the lengths on the host nor a table.
// the last sequence i in [0, N) whose first run is <= id; 64 candidates a step
__device__ __forceinline__ int find_seq(const RaggedArgs &r, int run, int64_t id) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = r.N;
    while (n > 1) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const bool in = lane * step < n && clamp_row(r.cu[lane * step < n ? i : lo], r.T) / run + i <= id;
        const int m = __popcll(__ballot(in));
        const int at = m > 0 ? (m - 1) * step : 0;
        lo += at;
        n = n - at < step ? n - at : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
__device__ __forceinline__ int64_t first_run(const Seq &s, int run, int i) { return s.begin / run + i; }

}  // namespace sf
