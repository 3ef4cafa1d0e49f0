// gfx950 kernels that move whole pages of the pool: the fork of a session into
// copies, and the move of every session's pages into another buffer; of int8
// pools also the sessions' tails.
//
// A page is one block of one layer (every KV head's tiles), `block_stride`
// contiguous bytes of any cache type.  Bound by memory alone: a fork reads a
// page once and writes it once per copy, a move reads and writes it once (6.0 TB/s
// of both at the sizes below; the streaming copy reaches 4.8 on 2 GiB).  A
// workgroup takes up to 8 KiB of a page, its loads all in flight, non-temporal
// both ways like the streaming copy.
//
// A session's assigned logical blocks are a prefix of its sinks and a prefix of
// its ring (slots fill from the first on), so a page's logical block follows
// from its number, and its physical block from the device's own table: what a
// launch needs from the host besides that travels in its kernel arguments.
// Nothing is staged and nothing is waited for.
#include "mtn_kernels.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

namespace mtn {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
constexpr int kPageThreads = 256;
constexpr int64_t kMaxGrid = UINT32_MAX / kPageThreads;  // a dimension's threads are counted in 32 bits
// 16-byte loads in flight per thread.  One session of 48 layers (411 MB) forked:
// 136 us with 2, 138 with 4 or 5, 200 with 8; 24 int8 sessions of 12 layers (1.15 GB)
// moved: 381, 402 and 383, 727.
constexpr int kLoads = 2;

// A page of n vectors is cut into `parts` workgroups of `per` vectors (the last may
// have fewer): as few as kLoads per thread allow, of equal size.  (With whole 16 KiB
// parts an int8 page of four heads, 16512 bytes, was one workgroup and a sliver:
// the move above took 463 us.)
struct Parts {
    uint32_t parts;
    int32_t per, n;
};
Parts page_parts(int64_t bytes) {
    const int64_t n = bytes / 16;
    const int64_t parts = (n + kLoads * kPageThreads - 1) / (kLoads * kPageThreads);
    return Parts{(uint32_t)parts, (int32_t)((n + parts - 1) / parts), (int32_t)n};
}

// logical block of a session's page i
__device__ __forceinline__ int page_lb(int i, int n_sink_pages, int n_sink_blocks) {
    return i < n_sink_pages ? i : n_sink_blocks + (i - n_sink_pages);
}

// part `part` of a page into every destination
template <class Dst>
__device__ __forceinline__ void copy_part(const u32x4_t *src, const Parts &p, uint32_t part, int n_dst, Dst &&dst) {
    const int v0 = (int)part * p.per, end = min(v0 + p.per, p.n);
    u32x4_t x[kLoads];
    const int i = v0 + (int)threadIdx.x;
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
        if (i + u * kPageThreads < end) x[u] = __builtin_nontemporal_load(src + i + u * kPageThreads);
    for (int c = 0; c < n_dst; ++c) {
        u32x4_t *d = dst(c);
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (i + u * kPageThreads < end) __builtin_nontemporal_store(x[u], d + i + u * kPageThreads);
    }
}

// workgroup (page x part, layer): pages first .. first + m - 1 of the source
// session into every copy; the first layer's also enter the copies' tables.
// (No workgroup reads the rows that another writes: copies are new sessions.)
__global__ __launch_bounds__(kPageThreads) void k_fork(ForkArgs a, Parts p) {
    const uint32_t i = blockIdx.x / p.parts, part = blockIdx.x - i * p.parts;
    const int lb = page_lb(a.first + (int)i, a.n_sink_pages, a.n_sink_blocks);
    const int64_t from = a.table[(int64_t)a.src * a.row_len + lb];
    uint8_t *layer = a.kv + (int64_t)blockIdx.y * a.layer_stride;
    copy_part((const u32x4_t *)(layer + from * a.block_stride), p, part, a.copies, [&](int c) { return (u32x4_t *)(layer + (int64_t)a.block[c * a.m + (int)i] * a.block_stride); });
    if (blockIdx.y == 0 && part == 0 && (int)threadIdx.x < a.copies)
        a.table[(int64_t)a.sid[threadIdx.x] * a.row_len + lb] = a.block[threadIdx.x * a.m + i];
}

// workgroup (page x part, session, layer): the session's page i becomes block
// base + i of the other buffer
__global__ __launch_bounds__(kPageThreads) void k_move(MoveArgs a, Parts p) {
    const MoveSession s = a.s[blockIdx.y];
    const uint32_t i = blockIdx.x / p.parts, part = blockIdx.x - i * p.parts;
    if ((int)i >= s.pages) return;
    const int lb = page_lb((int)i, s.n_sink_pages, a.n_sink_blocks);
    const int64_t from = a.table[(int64_t)s.sid * a.row_len + lb];
    const uint8_t *src = a.kv + (int64_t)blockIdx.z * a.layer_stride + from * a.block_stride;
    uint8_t *dst = a.to + (int64_t)blockIdx.z * a.to_layer_stride + ((int64_t)s.base + i) * a.block_stride;
    copy_part((const u32x4_t *)src, p, part, 1, [&](int) { return (u32x4_t *)dst; });
}

// the tables after the move, in a launch of its own: every layer's copy reads the old ones
__global__ __launch_bounds__(kPageThreads) void k_move_table(MoveArgs a) {
    const MoveSession s = a.s[blockIdx.x];
    for (int i = threadIdx.x; i < s.pages; i += kPageThreads)
        a.table[(int64_t)s.sid * a.row_len + page_lb(i, s.n_sink_pages, a.n_sink_blocks)] = s.base + i;
}

// workgroup (part, copy): an int8 pool's tails, every layer of one at a time
__global__ __launch_bounds__(kPageThreads) void k_copy_tails(TailArgs a, Parts p) {
    const u32x4_t *src = (const u32x4_t *)(a.from + (int64_t)a.src[blockIdx.y] * a.stride);
    u32x4_t *dst = (u32x4_t *)(a.to + (int64_t)a.dst[blockIdx.y] * a.stride);
    copy_part(src, p, blockIdx.x, 1, [&](int) { return dst; });
}

}  // namespace

hipError_t launch_fork(const ForkArgs &a, int32_t n_layers, hipStream_t s) {
    const Parts p = page_parts(a.block_stride);
    const int64_t x = (int64_t)a.m * p.parts;
    if (a.m < 1 || a.copies < 1 || a.copies > kForkCopies || a.m * a.copies > kForkBlocks || x > kMaxGrid ||
        n_layers > 65535 || a.block_stride % 16 || a.block_stride / 16 > INT32_MAX)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_fork, dim3((unsigned)x, (unsigned)n_layers), dim3(kPageThreads), 0, s, a, p);
    return hipGetLastError();
}

hipError_t launch_move(const MoveArgs &a, int32_t n_layers, hipStream_t s) {
    const Parts p = page_parts(a.block_stride);
    int64_t pages = 0;
    for (int i = 0; i < a.n; ++i) pages = std::max<int64_t>(pages, a.s[i].pages);
    const int64_t x = pages * p.parts;
    if (a.n < 1 || a.n > kMoveSessions || x < 1 || x > kMaxGrid || n_layers > 65535 ||
        a.block_stride % 16 || a.block_stride / 16 > INT32_MAX)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_move, dim3((unsigned)x, (unsigned)a.n, (unsigned)n_layers), dim3(kPageThreads), 0, s, a, p);
    return hipGetLastError();
}

hipError_t launch_copy_tails(const TailArgs &a, hipStream_t s) {
    if (a.n < 1 || a.n > kTailCopies || a.stride < 1 || a.stride % 16 || a.stride / 16 > INT32_MAX)
        return hipErrorInvalidValue;
    const Parts p = page_parts(a.stride);
    hipLaunchKernelGGL(k_copy_tails, dim3(p.parts, (unsigned)a.n), dim3(kPageThreads), 0, s, a, p);
    return hipGetLastError();
}

hipError_t launch_move_table(const MoveArgs &a, hipStream_t s) {
    if (a.n < 1 || a.n > kMoveSessions) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_move_table, dim3((unsigned)a.n), dim3(kPageThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace mtn
