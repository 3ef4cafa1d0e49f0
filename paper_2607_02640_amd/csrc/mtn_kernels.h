// Internal launch interface between the host library (mtn_host.cpp) and the
// gfx950 kernels (mtn_kernels.hip).  Not part of the public C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mtn {

// Geometry of the paged pool as the kernels see it.  Byte strides; the pool
// layout is [layer][block][kv_head]{K tile [16][D], V^T tile [D][16]}.
struct PoolGeom {
    const uint8_t *kv;       // pool base (device)
    int64_t layer_stride;    // bytes per layer
    int64_t block_stride;    // bytes per (layer, block)
    int64_t head_stride;     // bytes per (layer, block, kv head) = 2 tiles
    int64_t tile_bytes;      // bytes of one K (or V^T) tile
    const int32_t *table;    // [max_sessions][row_len] physical block ids
    int32_t row_len;
    int32_t n_sink;          // S (0 when unbounded)
    int32_t window;          // W, or -1 when unbounded
    int32_t ring;            // R tokens (unbounded: row_len * 16)
    int32_t n_sink_blocks;   // ceil(S / 16)
    int32_t hq, hkv;
    // (packed: with eight bytes more of kernel arguments a lone session's frame
    // of 768 decode launches took 9.83 ms instead of 9.67)
    uint16_t d;
    // Rotation pairs: pair i of a row (i < D/2) takes elements 2i and 2i + 1
    // (rope_il), or i and i + rope_half for i < rope_half and the rest, which
    // the table leaves alone, in order.  The kernels hold pair i in dims i and
    // i + D/2, queries and stored keys alike: scores do not depend on the order.
    uint8_t rope_half;       // rotary_dim / 2
    uint8_t rope_il;         // kRopeInterleaved | kRopeNorm
};
constexpr uint8_t kRopeInterleaved = 1, kRopeNorm = 2;

// Norm weights lie in front of the rotary table (PlanView::rope), layer l at
// float offset -(l + 1) * norm_stride(D): the query's D, the key's D, eps.
constexpr int norm_stride(int d) { return 2 * d + 4; }

// One planned token: which session, absolute position, io row, slot.
struct PlanView {
    const int32_t *tok_sid;
    const int32_t *tok_pos;
    const int32_t *tok_row;
    const int32_t *tok_block;
    const int32_t *tok_off;
    const float2  *rope;     // [T][D/2] (cos, sin) of pos * theta^(-2i/D)
    int32_t n_tok;
};

struct AttnArgs {
    PoolGeom g;
    PlanView p;
    int32_t layer;
    const void *q;           // [rows][Hq][D], row = tok_row[t]
    void *out;               // [rows][Hq][D]
    float *lse;              // [rows][Hq] or null
    float *part;             // split partials (acc [unit][G][D] then ml [unit][G][2])
    int32_t n_split;
    float scale_log2;        // softmax scale * log2(e)
    const uint8_t *zero_page;  // 16 KiB of zeros (DMA source of absent blocks)
    // decode with a fused append (or null): [rows][Hkv][D] keys / values of
    // the planned tokens, each the newest position of its own query
    const void *k_new;
    const void *v_new;
};

// Tails of an int8 pool (the rows of every session's open block): per (session,
// one of two), `stride` bytes: [layer][kv head]{K [16][D], V [16][D] bf16}.
struct TailView {
    uint8_t *base;
    int64_t stride;
};
struct I8Args {
    AttnArgs a;
    TailView tails;
    int32_t ahead;  // a wave issues its next block before it waits for the current one
};

// dtype codes match the public MTN_F32 / MTN_BF16 / MTN_FP8_E4M3 / MTN_INT8_BLOCK
// src non-null: pinned host words, first copied to dst (both 16-byte aligned,
// whole 16-byte vectors allocated); the other arrays may lie in src.
hipError_t launch_plan_apply(const int32_t *src, int32_t *dst, int32_t n_words,
                             const int32_t *upd_idx, const int32_t *upd_val, int32_t n_upd,
                             int32_t *table, const int32_t *tok_pos, int32_t n_tok,
                             const double *inv_freq, int32_t half_d, float2 *rope,
                             hipStream_t s);  // inv_freq: [2][half_d], frequencies, then factors

// Append (fp32 / bf16 pools) over runs: run r covers planned tokens
// run_tok0[r] .. + run_len[r] - 1, consecutive slots of one block.
hipError_t launch_append(int dtype, const PoolGeom &g, const PlanView &p, int32_t layer,
                         const void *k, const void *v, const int32_t *run_tok0,
                         const int32_t *run_len, int32_t n_runs, hipStream_t s);

// Vector (VALU) decode attention over items = planned tokens.  Returns
// hipErrorInvalidValue for shapes with no instance.
hipError_t launch_attn_valu(int dtype, const AttnArgs &a, hipStream_t s);
hipError_t launch_merge(int dtype, const AttnArgs &a, hipStream_t s);

// MFMA chunk-prefill attention (bf16 and int8 pools, D = 128 or 64; fp8 pool, D = 128): one
// workgroup per (sequence, row pass, kv head, key segment of a.n_split).  items: n_items records of kPfItem int32 (32-byte
// aligned), one per row pass: {pass, first planned token t0, tokens, session
// id, position of t0, io row of t0, tail (int8 pools: which of the session's two
// holds its open block once the plan is appended), 0}; token t0 + j of the sequence uses
// io row (row of t0) + j (multi-token plans always do); pass p covers the
// sequence's query rows [p, p + 1) * pass_rows (rows are token * G + group
// head).  pass_rows: prefill_rows_per_pass() or, to spread few sequences over
// more workgroups, 128 (prefill_pass_rows_valid).  zero_page: 16 KiB of
// device zeros, the DMA source of blocks a pass does not see.  a.k_new /
// a.v_new (both or neither; fp8 pool only; [rows][Hkv][D] bf16): the launch
// also appends the planned tokens (RoPE on K, quantized), which the caller may
// ask for only when every sequence takes exactly one row pass.
constexpr int kPfItem = 8;
int prefill_rows_per_pass();
bool prefill_pass_rows_valid(int rows);
hipError_t launch_prefill_mfma(int dtype, const AttnArgs &a, const int32_t *items, int32_t n_items,
                               int32_t pass_rows, const uint8_t *zero_page, const TailView &tails,
                               hipStream_t s);

// The same over fp32 pools (D = 64 or 128), a.zero_page the zero page:
// passes of prefill_f32_rows_per_pass() rows.
int prefill_f32_rows_per_pass();
hipError_t launch_prefill_f32(const AttnArgs &a, const int32_t *items, int32_t n_items,
                              hipStream_t s);

hipError_t launch_poison(int dtype, const PoolGeom &g, int32_t n_layers, int64_t n_blocks,
                         const uint16_t *live_mask, hipStream_t s);

hipError_t launch_copy(const void *src, void *dst, size_t bytes, hipStream_t s);
// streaming read of the whole 8 KiB chunks of `bytes` into LDS (nothing
// computed or written)
hipError_t launch_read(const void *src, size_t bytes, uint32_t *out, hipStream_t s);

// Fork: pages first .. first + m - 1 of session src into `copies` new sessions;
// copy c of page first + i is block[c * m + i].  n_sink_pages: how many of the
// session's pages are sink blocks (the rest are its ring's, from the first on).
constexpr int kForkCopies = 32, kForkBlocks = 896;  // per launch (kernel arguments hold at most 4 KiB)
struct ForkArgs {
    uint8_t *kv;
    int64_t layer_stride, block_stride;
    int32_t *table;
    int32_t row_len, n_sink_blocks;
    int32_t src, n_sink_pages, first, m, copies;
    int32_t sid[kForkCopies];
    int32_t block[kForkBlocks];
};
hipError_t launch_fork(const ForkArgs &a, int32_t n_layers, hipStream_t s);

// Move: page i of session s[k] becomes block s[k].base + i of the buffer `to`;
// launch_move copies, launch_move_table then rewrites the block tables.
constexpr int kMoveSessions = 240;
struct MoveSession {
    int32_t sid, base, pages, n_sink_pages;
};
struct MoveArgs {
    const uint8_t *kv;
    uint8_t *to;
    int64_t layer_stride, to_layer_stride, block_stride;
    int32_t *table;
    int32_t row_len, n_sink_blocks;
    int32_t n;
    MoveSession s[kMoveSessions];
};
hipError_t launch_move(const MoveArgs &a, int32_t n_layers, hipStream_t s);
hipError_t launch_move_table(const MoveArgs &a, hipStream_t s);

// Tails: slot src[i] of one buffer's tails to slot dst[i] of another's (or the same's).
constexpr int kTailCopies = 480;
struct TailArgs {
    const uint8_t *from;
    uint8_t *to;
    int64_t stride;  // bytes of a slot
    int32_t n;
    int32_t src[kTailCopies], dst[kTailCopies];
};
hipError_t launch_copy_tails(const TailArgs &a, hipStream_t s);

// The library's static device workspace for split partials (a file-scope
// array, no allocation): its address on the current device and its size in
// floats.
hipError_t scratch_buffer(float **ptr, size_t *floats);

// FP8 (E4M3) KV cache, D = 128, bf16 io: bytes per (layer, block, kv head)
// region (0 for an unsupported head dim), the fused RoPE + quantize + append,
// the MFMA decode (k_new / v_new in AttnArgs select the fused append) and the
// debug poison.
int fp8_head_stride(int d);
bool attn_fp8_supported(int d, int g);
int attn_fp8_resident_per_cu(int g);
hipError_t launch_append_fp8(const PoolGeom &g, const PlanView &p, int32_t layer, const void *k,
                             const void *v, hipStream_t s);
hipError_t launch_attn_fp8(const AttnArgs &a, hipStream_t s);
hipError_t launch_poison_fp8(const PoolGeom &g, int32_t n_layers, int64_t n_blocks,
                             const uint16_t *live_mask, hipStream_t s);

// The same MFMA decode over bf16 blocks (D = 128 or 64, bf16 io), append fusable.
bool attn_mfma_bf16_supported(int d, int g);
int attn_mfma_bf16_resident_per_cu(int d, int g);
hipError_t launch_attn_mfma_bf16(const AttnArgs &a, hipStream_t s);

// int8 KV cache (bf16 io, D = 128 or 64): tok_off of its plans holds the slot
// in bits 0 .. 7 and which of the session's tails the token's block uses (while
// open) in bit 8.
bool attn_i8_supported(int d, int g);
int attn_i8_groups();  // waves that share a unit's keys
hipError_t launch_append_i8(const PoolGeom &g, const PlanView &p, int32_t layer, const void *k,
                            const void *v, const TailView &tails, const int32_t *run_tok0,
                            const int32_t *run_len, int32_t n_runs, hipStream_t s);
hipError_t launch_attn_i8(const AttnArgs &a, const TailView &tails, int n_cu, hipStream_t s);
hipError_t launch_poison_i8(const PoolGeom &g, const TailView &tails, int32_t n_layers,
                            int64_t n_blocks, int32_t n_tails, const uint16_t *live_mask,
                            const uint8_t *tail_rows, hipStream_t s);

bool attn_valu_supported(int dtype, int d, int g);
// workgroups of the vector attention kernel resident per CU (occupancy query)
int attn_valu_resident_per_cu(int dtype, int d, int g);
// wave groups that share a unit's keys in the vector and matrix-core decode
int attn_valu_groups(int g);
int attn_mfma_groups(int g);
bool prefill_mfma_supported(int dtype, int d, int g);

constexpr int kBlock = 16;      // tokens per KV block
constexpr int kMaxSplit = 64;   // decode split cap

}  // namespace mtn
