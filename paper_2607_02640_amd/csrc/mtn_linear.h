// Internal launch interface of the linear-attention layers (mtn_linear.hip).
#pragma once
#include <algorithm>

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mtn {

// One sequence of a plan, or one segment of it: {first io row, tokens, state slot
// (2 * session + which of its two), with kLinFresh where the session holds no
// token yet, segment | segments << 16}.  A sequence's segments follow one another;
// all but its last hold the same multiple of kLinTile tokens.
constexpr int kLinItem = 4;
constexpr int32_t kLinFresh = 1 << 30;
constexpr int kLinTile = 64;
// e^(m log_decay), m = 0 .. kLinTile, in two fp32 terms: the larger of each, then
// what those leave
constexpr int kLinDecays = 2 * (kLinTile + 1);
constexpr int kLinMaxSeg = 1024;  // segments of a plan that cuts sequences, at most

struct LinArgs {
    const int32_t *items;     // device [n_items][kLinItem]
    const void *q, *k, *v;    // [rows][Hq | Hkv | Hkv][D]
    void *out;                // [rows][Hq][D]
    float *state;             // the layer's states in slot 0: [Hkv][value D][key D]
    int64_t slot_stride;      // floats from a slot to the next
    float *seg;               // segments' states [item][Hkv][D][D]
    const double *log2_decay;  // device [Hkv]
    const float *decay;       // device [Hkv][kLinDecays]
    float scale;
    int32_t hq, hkv, d, n_items;
    int32_t parts;            // chunk form: workgroups that share a KV head's query heads
};

// Tokens of a segment of a plan of n_seq sequences and n_tok tokens; 0: nothing is cut.
// Sequences are cut where they leave compute units idle: two workgroups a CU, half of that
// where a KV head's query heads can share one's work (linear_parts), of at least two
// tiles.  Each segment's state is written, scanned and read, 4 D^2 floats of
// traffic (32 heads of 8192 tokens, D = 128: 8 segments 153 us, 12 147, 16 124, 24 149;
// 4 heads of G = 8: 16 segments 103 us, 32 79, 64 72).
inline int64_t linear_segment(int64_t n_seq, int64_t n_tok, int64_t hq, int64_t hkv, int64_t n_cu) {
    if (n_cu < 1 || n_seq * hkv >= n_cu) return 0;
    const int64_t want = std::min<int64_t>((hq > hkv ? 1 : 2) * n_cu / hkv, kLinMaxSeg);
    const int64_t len = (n_tok + want - 1) / want;
    return std::max<int64_t>((len + kLinTile - 1) / kLinTile, 2) * kLinTile;
}
// (segment, KV head) pairs of such a plan, per compute unit, that it stays under: each
// sequence adds one segment to n_tok / len <= want, n_seq + want segments in all, of
// which n_seq hkv < n_cu and want hkv <= 2 n_cu pairs.
constexpr int kLinSegUnits = 3;

// Tokens of a chunk workgroup's tiles: 32 take chunks up to 32 tokens and fp32.
inline int linear_tile(int dtype, int max_tok) { return dtype == 1 && max_tok > 32 ? 64 : 32; }
// Workgroups that share a KV head's query heads in the chunk form, each with the state,
// where that fills the CUs: with a workgroup of eight waves each (tiles of 32), or two of
// four (one session of 25 tokens, G = 4, 4 KV heads 14.5 us whole, 11.0 in four
// parts; 32 sessions 16.6, 15.2 in two, 18.9 in four; 8192 tokens of G = 8, 4 KV
// heads, 64 segments 84.5 whole, 72.8 in two, 86.2 in four).
inline int linear_parts(int64_t units, int g, int tile, int n_cu) {
    int parts = 1;
    while (2 * parts * units <= (tile == 64 ? 2 : 1) * (int64_t)n_cu && g % (2 * parts) == 0) parts *= 2;
    return parts;
}
// Workgroups that share the rows of a state in the single-token form, where states are
// few (32 sessions, G = 4, 4 heads 9.0 us whole, 7.2 in four slices; 512 states of
// G = 8 17.6 whole, 18.4 in two).
inline int linear_slices(int64_t units, int d, int n_cu) {
    int sl = 1;
    while (sl < d / 32 && sl * units <= n_cu) sl *= 2;
    return sl;
}

bool linear_supported(int dtype, int d, int g);
// Plans of one token per sequence
hipError_t launch_linear_decode(int dtype, const LinArgs &a, int n_cu, hipStream_t s);
// Plans of any lengths; max_tok: the longest item, split: some sequence has segments
hipError_t launch_linear_chunk(int dtype, LinArgs a, int max_tok, bool split, int n_cu, hipStream_t s);
// Debug: NaN into every state slot with dead[slot] != 0 (slots of slot_stride floats)
hipError_t launch_linear_poison(float *states, int64_t slot_stride, int32_t n_slots, const uint8_t *dead,
                                hipStream_t s);

}  // namespace mtn
