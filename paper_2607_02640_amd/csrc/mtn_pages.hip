// gfx950 kernels that move whole pages of the pool: the fork of a session into
// copies, and the move of every session's pages into another buffer; of int8
// pools also the sessions' tails.
//
// A page is one block of one layer (every KV head's tiles), `block_stride`
// contiguous bytes of any cache type.  Bound by memory alone: a fork reads a
// page once and writes it once per copy, a move reads and writes it once.  A
// workgroup takes 16 KiB of a page, four 16-byte loads in flight per thread,
// non-temporal both ways like the streaming copy.
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
constexpr int64_t kPart = 4 * 16 * kPageThreads;  // bytes of a page per workgroup

// logical block of a session's page i
__device__ __forceinline__ int page_lb(int i, int n_sink_pages, int n_sink_blocks) {
    return i < n_sink_pages ? i : n_sink_blocks + (i - n_sink_pages);
}

// vectors [v0, v0 + 4 * kPageThreads) of a page of n into every destination
template <class Dst>
__device__ __forceinline__ void copy_part(const u32x4_t *src, int64_t v0, int64_t n, int n_dst, Dst &&dst) {
    u32x4_t x[4];
    const int64_t i = v0 + threadIdx.x;
    if (v0 + 4 * kPageThreads <= n) {
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = __builtin_nontemporal_load(src + i + u * kPageThreads);
        for (int c = 0; c < n_dst; ++c) {
            u32x4_t *d = dst(c);
#pragma unroll
            for (int u = 0; u < 4; ++u) __builtin_nontemporal_store(x[u], d + i + u * kPageThreads);
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (i + u * kPageThreads < n) x[u] = __builtin_nontemporal_load(src + i + u * kPageThreads);
    for (int c = 0; c < n_dst; ++c) {
        u32x4_t *d = dst(c);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * kPageThreads < n) __builtin_nontemporal_store(x[u], d + i + u * kPageThreads);
    }
}

// workgroup (page x part, layer): pages first .. first + m - 1 of the source
// session into every copy; the first layer's also enter the copies' tables.
// (No workgroup reads the rows that another writes: copies are new sessions.)
__global__ __launch_bounds__(kPageThreads) void k_fork(ForkArgs a, uint32_t parts) {
    const uint32_t i = blockIdx.x / parts, part = blockIdx.x - i * parts;
    const int lb = page_lb(a.first + (int)i, a.n_sink_pages, a.n_sink_blocks);
    const int64_t from = a.table[(int64_t)a.src * a.row_len + lb];
    uint8_t *layer = a.kv + (int64_t)blockIdx.y * a.layer_stride;
    copy_part((const u32x4_t *)(layer + from * a.block_stride), (int64_t)part * (kPart / 16), a.block_stride / 16,
              a.copies, [&](int c) { return (u32x4_t *)(layer + (int64_t)a.block[c * a.m + (int)i] * a.block_stride); });
    if (blockIdx.y == 0 && part == 0 && (int)threadIdx.x < a.copies)
        a.table[(int64_t)a.sid[threadIdx.x] * a.row_len + lb] = a.block[threadIdx.x * a.m + i];
}

// workgroup (page x part, session, layer): the session's page i becomes block
// base + i of the other buffer
__global__ __launch_bounds__(kPageThreads) void k_move(MoveArgs a, uint32_t parts) {
    const MoveSession s = a.s[blockIdx.y];
    const uint32_t i = blockIdx.x / parts, part = blockIdx.x - i * parts;
    if ((int)i >= s.pages) return;
    const int lb = page_lb((int)i, s.n_sink_pages, a.n_sink_blocks);
    const int64_t from = a.table[(int64_t)s.sid * a.row_len + lb];
    const uint8_t *src = a.kv + (int64_t)blockIdx.z * a.layer_stride + from * a.block_stride;
    uint8_t *dst = a.to + (int64_t)blockIdx.z * a.to_layer_stride + ((int64_t)s.base + i) * a.block_stride;
    copy_part((const u32x4_t *)src, (int64_t)part * (kPart / 16), a.block_stride / 16, 1,
              [&](int) { return (u32x4_t *)dst; });
}

// the tables after the move, in a launch of its own: every layer's copy reads the old ones
__global__ __launch_bounds__(kPageThreads) void k_move_table(MoveArgs a) {
    const MoveSession s = a.s[blockIdx.x];
    for (int i = threadIdx.x; i < s.pages; i += kPageThreads)
        a.table[(int64_t)s.sid * a.row_len + page_lb(i, s.n_sink_pages, a.n_sink_blocks)] = s.base + i;
}

// workgroup (part, copy): an int8 pool's tails, every layer of one at a time
__global__ __launch_bounds__(kPageThreads) void k_copy_tails(TailArgs a) {
    const u32x4_t *src = (const u32x4_t *)(a.from + (int64_t)a.src[blockIdx.y] * a.stride);
    u32x4_t *dst = (u32x4_t *)(a.to + (int64_t)a.dst[blockIdx.y] * a.stride);
    copy_part(src, (int64_t)blockIdx.x * (kPart / 16), a.stride / 16, 1, [&](int) { return dst; });
}

uint32_t page_parts(int64_t block_stride) { return (uint32_t)((block_stride + kPart - 1) / kPart); }

}  // namespace

hipError_t launch_fork(const ForkArgs &a, int32_t n_layers, hipStream_t s) {
    const uint32_t parts = page_parts(a.block_stride);
    const int64_t x = (int64_t)a.m * parts;
    if (a.m < 1 || a.copies < 1 || a.copies > kForkCopies || a.m * a.copies > kForkBlocks || x > INT32_MAX ||
        n_layers > 65535 || a.block_stride % 16)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_fork, dim3((unsigned)x, (unsigned)n_layers), dim3(kPageThreads), 0, s, a, parts);
    return hipGetLastError();
}

hipError_t launch_move(const MoveArgs &a, int32_t n_layers, hipStream_t s) {
    const uint32_t parts = page_parts(a.block_stride);
    int64_t pages = 0;
    for (int i = 0; i < a.n; ++i) pages = std::max<int64_t>(pages, a.s[i].pages);
    const int64_t x = pages * parts;
    if (a.n < 1 || a.n > kMoveSessions || x < 1 || x > INT32_MAX || n_layers > 65535 || a.block_stride % 16)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_move, dim3((unsigned)x, (unsigned)a.n, (unsigned)n_layers), dim3(kPageThreads), 0, s, a, parts);
    return hipGetLastError();
}

hipError_t launch_copy_tails(const TailArgs &a, hipStream_t s) {
    const int64_t x = (a.stride + kPart - 1) / kPart;
    if (a.n < 1 || a.n > kTailCopies || a.stride < 1 || a.stride % 16 || x > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_copy_tails, dim3((unsigned)x, (unsigned)a.n), dim3(kPageThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_move_table(const MoveArgs &a, hipStream_t s) {
    if (a.n < 1 || a.n > kMoveSessions) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_move_table, dim3((unsigned)a.n), dim3(kPageThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace mtn
