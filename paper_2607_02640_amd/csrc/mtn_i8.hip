// gfx950 kernels of the int8 KV cache: codes under one fp32 scale per block of
// 16 tokens, KV head and tensor.  Fused RoPE + append (with the quantization of
// the blocks it completes), decode attention with the append fusable, and the
// debug poison.  (The chunk prefill over these blocks is an instance of the
// common one.)
//
// A block is complete once the last of its positions has been appended, and
// open before.  A complete block holds code = rne(x / s), s = max|x| / 127 over
// its rows (1 where all are zero, NaN where an element is not finite), and
// reads as code * s; the rows of the open block are kept as they are (bf16,
// keys rotated) in a tail of 16 rows per session, layer and KV head, so that
// every row is rounded to 8 bits once, whatever chunks brought it.
//
// Region of one (layer, block, KV head), 32 D + 16 bytes (a layer's block padded to
// 128):
//   [0, 16 D)      K codes + 128 (unsigned), [16 keys][D]
//   [16 D, 32 D)   V codes (signed) in key quads: byte ((key / 4) * D + d) * 4 + key % 4
//   [32 D, + 8)    the scales {K, V}, fp32
// The scales lie right behind their codes: gathered behind the block's last head
// instead, a second place to wait for with every block, they cost 128 sessions of
// G = 8 98.8 us a launch against 87.5 without any.  A tail is K [16][D], V [16][D]
// bf16.
#include "mtn_kernels.h"
#include "mtn_device.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

namespace mtn {
namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4_t;

__device__ __forceinline__ f32x4_t mfma_pv16(const uint2 &a, const uint2 &b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, a),
                                                      __builtin_bit_cast(s16x4_t, b), c, 0, 0, 0);
}
// codes of a row or block: nearest integer to x / s (the correctly rounded
// quotient), within [-127, 127]
__device__ __forceinline__ int i8_code(float x, float s) {
    return (int)fminf(fmaxf(rintf(x / s), -127.f), 127.f);
}
// scale of a block from its largest magnitude (NaN or infinite: NaN)
__device__ __forceinline__ float i8_scale(float amax) {
    if (!(amax < INFINITY)) return __builtin_nanf("");
    return amax > 0.f ? amax / 127.f : 1.f;
}
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// positions that the block of the token at `pos`, slot `off`, holds
__device__ __forceinline__ int block_rows(const PoolGeom &g, int pos, int off) {
    return pos < g.n_sink ? min(kBlock, g.n_sink - (pos - off)) : kBlock;
}
__device__ __forceinline__ uint8_t *tail_of(const TailView &t, const PoolGeom &g, int sid, int slot,
                                            int layer, int h, int D) {
    return t.base + ((int64_t)sid * 2 + slot) * t.stride + ((int64_t)layer * g.hkv + h) * (64 * D);
}

// ---------------------------------------------------------------------------
// fused RoPE + append: one workgroup per (run, KV head), a run being one
// sequence's tokens in consecutive slots of one block
// ---------------------------------------------------------------------------
// Thread (j, c) holds row j of the block, K pairs P c .. P c + P - 1 (dims i and
// i + D/2) and V dims 2 P c .. + 2 P - 1, P = D / 32.  A run that completes its
// block takes the rows before it from the session's tail, finds the largest
// magnitudes over the block and writes codes and scales; any other run's rows
// go to the tail.  (A plan that opens a block uses the session's other tail: the
// one that holds the rows committed before it stays whole, so the plan can be
// abandoned.)  Moves a few KiB per workgroup: bound by its chain of
// round trips (metadata, rows, two barriers); 10.4 us for 128 x 25 tokens of 4
// heads.
template <int D, int RF>
__global__ __launch_bounds__(256) void k_append_i8(PoolGeom g, PlanView p, int32_t layer,
                                                   const bf16_t *__restrict__ k,
                                                   const bf16_t *__restrict__ v, TailView tails,
                                                   const int32_t *__restrict__ run_tok0,
                                                   const int32_t *__restrict__ run_len) {
    constexpr int P = D / 32;        // pairs per thread: 4 or 2
    constexpr int NW = P / 2;        // ... in words of two bf16
    __shared__ uint8_t sv[kBlock * D];
    __shared__ float smax[2][4];
    const int tid = threadIdx.x, j = tid >> 4, c = tid & 15, w = tid >> 6;
    const int h = (int)(blockIdx.x % (uint32_t)g.hkv), r = (int)(blockIdx.x / (uint32_t)g.hkv);
    const int t0 = run_tok0[r], len = run_len[r];
    const int off0 = p.tok_off[t0] & 255, slot = p.tok_off[t0] >> 8;
    const int rows = block_rows(g, p.tok_pos[t0], off0);
    const bool complete = off0 + len == rows;
    uint8_t *tail = tail_of(tails, g, p.tok_sid[t0], slot, layer, h, D);
    bf16_t *tk = (bf16_t *)tail + j * D, *tv = tk + kBlock * D;
    const bool mine = j >= off0 && j < off0 + len;  // a new row
    uint32_t ka[NW], kb[NW], vw[2 * NW];            // bf16 pairs: dims P c .., P c + D/2 .., V
#pragma unroll
    for (int e = 0; e < NW; ++e) ka[e] = kb[e] = vw[2 * e] = vw[2 * e + 1] = 0u;
    if (mine) {
        const int t = t0 + j - off0;
        const int64_t row = p.tok_row[t];
        const bf16_t *kr = k + (row * g.hkv + h) * D;
        const uint32_t *vr = (const uint32_t *)(v + (row * g.hkv + h) * D + 2 * P * c);
        const float2 *rp = p.rope + (int64_t)t * (D / 2) + P * c;
        const RopeSrc o = rope_src<RF>(g, P * c, P, D);
#pragma unroll
        for (int e = 0; e < NW; ++e) {
            ka[e] = ((const uint32_t *)(kr + o.x))[e];
            kb[e] = ((const uint32_t *)(kr + o.y))[e];
        }
#pragma unroll
        for (int e = 0; e < 2 * NW; ++e) vw[e] = vr[e];
        if (RF && rope_il<RF>(g)) {
            // in memory order: words 0 .. 2 NW - 1 hold (a, b) each
            uint32_t m[2 * NW];
#pragma unroll
            for (int e = 0; e < NW; ++e) m[e] = ka[e], m[NW + e] = kb[e];
#pragma unroll
            for (int e = 0; e < NW; ++e) {
                ka[e] = m[2 * e];
                kb[e] = m[2 * e + 1];
                rope_split(ka[e], kb[e], false);
            }
        }
        float nr = 1.f;
        NormView nw{};
        if constexpr (RF == 2) {  // the row's sixteen lanes are all here
            nw = norm_view(p, layer, D);
            nr = norm_factor(D, nw.eps, [&](float f) __attribute__((always_inline)) {
                float ss[NW];  // (the order of wave_norm_factor)
#pragma unroll
                for (int e = 0; e < NW; ++e)
                    ss[e] = pair_square(__uint_as_float(ka[e] << 16), __uint_as_float(kb[e] << 16), f) +
                            pair_square(__uint_as_float(ka[e] & 0xFFFF0000u), __uint_as_float(kb[e] & 0xFFFF0000u), f);
                return row16_sum(NW == 2 ? ss[0] + ss[NW - 1] : ss[0]);
            });
        }
#pragma unroll
        for (int e = 0; e < NW; ++e) {
            const float2 c0 = rp[2 * e], c1 = rp[2 * e + 1];
            float a0 = __uint_as_float(ka[e] << 16), a1 = __uint_as_float(ka[e] & 0xFFFF0000u);
            float b0 = __uint_as_float(kb[e] << 16), b1 = __uint_as_float(kb[e] & 0xFFFF0000u);
            if constexpr (RF == 2) {
                const float *wa = nw.k + P * c + 2 * e, *wb = wa + D / 2;
                a0 = normed(a0, nr, wa[0]), a1 = normed(a1, nr, wa[1]);
                b0 = normed(b0, nr, wb[0]), b1 = normed(b1, nr, wb[1]);
            }
            ka[e] = pack_bf16x2(fmaf(a0, c0.x, -b0 * c0.y), fmaf(a1, c1.x, -b1 * c1.y));
            kb[e] = pack_bf16x2(fmaf(b0, c0.x, a0 * c0.y), fmaf(b1, c1.x, a1 * c1.y));
        }
    } else if (complete && j < off0) {
#pragma unroll
        for (int e = 0; e < NW; ++e) {
            ka[e] = ((const uint32_t *)(tk + P * c))[e];
            kb[e] = ((const uint32_t *)(tk + D / 2 + P * c))[e];
        }
#pragma unroll
        for (int e = 0; e < 2 * NW; ++e) vw[e] = ((const uint32_t *)(tv + 2 * P * c))[e];
    }
    if (!complete) {
        if (mine) {
#pragma unroll
            for (int e = 0; e < NW; ++e) {
                ((uint32_t *)(tk + P * c))[e] = ka[e];
                ((uint32_t *)(tk + D / 2 + P * c))[e] = kb[e];
            }
#pragma unroll
            for (int e = 0; e < 2 * NW; ++e) ((uint32_t *)(tv + 2 * P * c))[e] = vw[e];
        }
        return;  // uniform over the workgroup
    }
    auto lo = [](uint32_t x) { return __uint_as_float(x << 16); };
    auto hi = [](uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); };
    float mk = 0.f, mv = 0.f;
#pragma unroll
    for (int e = 0; e < NW; ++e) {
        mk = vmaxabs3(lo(ka[e]), hi(ka[e]), mk);
        mk = vmaxabs3(lo(kb[e]), hi(kb[e]), mk);
        mv = vmaxabs3(lo(vw[2 * e]), hi(vw[2 * e]), mv);
        mv = vmaxabs3(lo(vw[2 * e + 1]), hi(vw[2 * e + 1]), mv);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        mk = max_nan(mk, __shfl_xor(mk, m, 64));
        mv = max_nan(mv, __shfl_xor(mv, m, 64));
    }
    if ((tid & 63) == 0) {
        smax[0][w] = mk;
        smax[1][w] = mv;
    }
    __syncthreads();
    mk = max_nan(max_nan(smax[0][0], smax[0][1]), max_nan(smax[0][2], smax[0][3]));
    mv = max_nan(max_nan(smax[1][0], smax[1][1]), max_nan(smax[1][2], smax[1][3]));
    const float ks = i8_scale(mk), vs = i8_scale(mv);
    uint8_t *region = (uint8_t *)g.kv + (int64_t)layer * g.layer_stride +
                      (int64_t)p.tok_block[t0] * g.block_stride;
    uint8_t *codes = region + (int64_t)h * g.head_stride;
    // (a row of NaN scale: the codes are never looked at)
    uint32_t wa = 0, wb = 0;
#pragma unroll
    for (int e = 0; e < NW; ++e) {
        wa |= (uint32_t)((i8_code(lo(ka[e]), ks) + 128) & 255) << (16 * e);
        wa |= (uint32_t)((i8_code(hi(ka[e]), ks) + 128) & 255) << (16 * e + 8);
        wb |= (uint32_t)((i8_code(lo(kb[e]), ks) + 128) & 255) << (16 * e);
        wb |= (uint32_t)((i8_code(hi(kb[e]), ks) + 128) & 255) << (16 * e + 8);
        *(uint32_t *)&sv[j * D + 2 * P * c + 4 * e] =
            (uint32_t)(i8_code(lo(vw[2 * e]), vs) & 255) | (uint32_t)(i8_code(hi(vw[2 * e]), vs) & 255) << 8 |
            (uint32_t)(i8_code(lo(vw[2 * e + 1]), vs) & 255) << 16 |
            (uint32_t)(i8_code(hi(vw[2 * e + 1]), vs) & 255) << 24;
    }
    if constexpr (NW == 2) {
        *(uint32_t *)(codes + j * D + P * c) = wa;
        *(uint32_t *)(codes + j * D + D / 2 + P * c) = wb;
    } else {
        *(uint16_t *)(codes + j * D + P * c) = (uint16_t)wa;
        *(uint16_t *)(codes + j * D + D / 2 + P * c) = (uint16_t)wb;
    }
    if (tid == 0) *(float2 *)(codes + 2 * kBlock * D) = make_float2(ks, vs);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < NW; ++e) {  // quad words, memory order
        const int q = tid + 256 * e, kq = q / D, d = q % D;
        uint32_t x = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) x |= (uint32_t)sv[(4 * kq + i) * D + d] << (8 * i);
        ((uint32_t *)(codes + kBlock * D))[q] = x;
    }
}

// ---------------------------------------------------------------------------
// MFMA decode attention over int8 blocks
// ---------------------------------------------------------------------------
// Units, waves, rings and the lane layout are those of the bf16 / FP8 decode:
// one workgroup of NG waves per (query token, KV head, split segment), each
// wave streaming its own segment of the keys through its own LDS ring; per
// block and wave S = K . Q^T on D / 32 16x16x32 MFMAs and O^T += V^T . P on D / 16
// 16x16x16 ones, lane (n, g4) holding head n, keys 4 g4 .. + 3.
//
// K codes become f16 (exact) against the query in f16, scaled per head by a
// power of two to at most 1 (11 bits against bf16's 8; what a head's largest
// element leaves below 2^-24 is lost); V codes become bf16 (exact) against
// probability * V scale in bf16, which has the range of the scales.  The K scale
// multiplies scores: no product of codes is rounded before it.
//
// The query's newest block, where it is open, is taken from the session's tail
// in bf16, by the wave of the unit's last segment, before its ring; with the
// append fused that wave also rotates the newest key, keeps it and its value in
// the tail, or, where they complete the block, quantizes the block, uses and
// stores it.
//
// Bound by the stream of codes (5.8 TB/s at 128 sessions of G = 8, 4100 keys: 93 to
// 95 us a launch, the FP8 kernel 89; D = 64, 128 sessions of G = 8, 256 units, 38.7
// us, 3.5 TB/s: a CU's one workgroup waits for copies of 2 KiB; 256 sessions 52.8,
// 5.1 TB/s).  Per block a wave converts 4096 codes in 80 vector instructions (K 32, V
// 48), against 32 of the FP8 kernel.
// Launch shape: four waves a workgroup with two-block rings at every group size.
// (Eight waves, which the FP8 kernel takes below G = 8: 8 KV heads, G = 4, 60
// sessions of 2048 keys 50.3 us against 48.9, 32 sessions 32.1 against 29.7; 200
// sessions of 1000 keys, D = 64, G = 1, 48.9 against 43.6; only 64 sessions of G = 1,
// 2048 units, are faster, 179.1 against 180.3.  Three-block rings: 128 sessions of
// G = 8 98.1 against 93.8.)
constexpr int kI8Waves = 4, kI8Ring = 2;
// What the tail takes its wave, in blocks of the ring: that wave's segment is
// shorter by as many where segments are at least 8 blocks.  0, 3, 5, 8: 64 sessions
// of G = 8 60.2, 58.2, 57.3, 57.0 us; 8 sessions 23.6, 21.9, 20.7, 23.4 (at 8 the rule
// no longer applied to them).
constexpr int kTailBlocks = 5;

template <int D, int G, int RF>
__global__ __launch_bounds__(64 * kI8Waves) void k_attn_i8(I8Args ia) {
    constexpr int NG = kI8Waves, NBUF = kI8Ring;
    constexpr int ND = D / 32;   // QK MFMAs per block
    constexpr int NJ = D / 16;   // PV MFMAs per block
    constexpr int VD = D / 64;   // dims per lane of a row
    constexpr int CODES = 2 * kBlock * D;
    constexpr int BLK = CODES + 16;      // ring slot: the head's region, codes and scales
    constexpr int NFI = CODES / 1024;    // 1 KiB copies per block
    constexpr int NIW = NFI + 1;
    static_assert(NBUF * BLK >= 16 * D * 4, "merge scratch fits one wave's ring");
    __shared__ __attribute__((aligned(16))) uint8_t ring[NG][NBUF][BLK];
    __shared__ float sM[NG][16], sL[NG][16];

    const AttnArgs &a = ia.a;
    const int lane = threadIdx.x & 63;
    const int n = lane & 15, g4 = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PoolGeom &g = a.g;
    const uint32_t ns = (uint32_t)a.n_split;
    const UnitIdx ui = decode_unit(blockIdx.x, ns, (uint32_t)g.hkv);
    const int split = ui.split, kvh = ui.kvh, t = ui.t;
    const int sid = __builtin_amdgcn_readfirstlane(a.p.tok_sid[t]);
    const int pos = __builtin_amdgcn_readfirstlane(a.p.tok_pos[t]);
    const int64_t row = __builtin_amdgcn_readfirstlane(a.p.tok_row[t]);
    const int off_slot = __builtin_amdgcn_readfirstlane(a.p.tok_off[t]);
    const int toff = off_slot & 255, tslot = off_slot >> 8;  // the newest key's slot, its block's tail
    const bool complete = toff + 1 == block_rows(g, pos, toff);
    const bool fused = a.k_new != nullptr;
    // the wave that takes the last block from the tail
    const bool tail_wave = (fused || !complete) && split == a.n_split - 1 && wv == NG - 1;

    const VisRange vr = vis_range(g, pos);
    const int nv = vr.n_sb + vr.n_rb;
    const uint32_t nseg = ns * NG, seg = (uint32_t)split * NG + wv;
    // the tail counts as kTailBlocks more where segments are long
    const int nw = nv + ((fused || !complete) && nv >= 8 * (int)nseg ? kTailBlocks : 0);
    const int v0 = __builtin_amdgcn_readfirstlane(seg_begin(seg, nseg, nw));
    const int v1 = __builtin_amdgcn_readfirstlane(min(seg_begin(seg + 1, nseg, nw), nv));
    const int nblk = v1 - v0 - (tail_wave ? 1 : 0);  // blocks from the pool (the last segment holds the last block)
    const uint8_t *head_base = g.kv + (int64_t)a.layer * g.layer_stride + (int64_t)kvh * BLK;
    const int32_t *trow = g.table + (int64_t)sid * g.row_len;
    const uint32_t ring0 = lds_addr(&ring[wv][0][0]);

    // the segment's blocks in the order they are issued; the table entry of the
    // next one is loaded one issue ahead
    const int ring_blocks = g.ring / kBlock;
    int vi = v0;
    int rb = vr.first / kBlock;
    if (v0 > vr.n_sb) rb = (rb + (v0 - vr.n_sb)) % ring_blocks;
    auto next_phys = [&]() {
        const int lb = vi < vr.n_sb ? vi : g.n_sink_blocks + rb;
        if (vi >= vr.n_sb) rb = rb + 1 == ring_blocks ? 0 : rb + 1;
        ++vi;
        return scalar_ld(trow, __builtin_amdgcn_readfirstlane(lb));
    };
    uint32_t doff[NFI];
#pragma unroll
    for (int j = 0; j < NFI; ++j) doff[j] = (uint32_t)swz(j * 64 + lane) * 16;
    int ph = nblk > 0 ? next_phys() : 0;  // of the next block to issue
    auto issue = [&](int i) {
        const uint8_t *src = head_base + (int64_t)max(ph, 0) * g.block_stride;
        const uint32_t dst = ring0 + (uint32_t)((i % NBUF) * BLK);
#pragma unroll
        for (int j = 0; j < NFI; ++j) dma16_s(doff[j], src, dst + j * 1024);
        if (lane < 1) dma16_s(CODES, src, dst + CODES);
        if (i + 1 < nblk) ph = next_phys();
    };
    for (int i = 0; i < min(nblk, NBUF - 1); ++i) issue(i);

    // How far a score may exceed the head's reference (log2 units) before the
    // reference moves; it starts at the lowest finite float: the first finite
    // score sets it, masked (-inf) scores give 0
    constexpr float kLag = 8.f;
    float m_ref = -3.402823466e38f, lsum = 0.f;
    f32x4_t acc[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // One block's softmax and PV: sc[r] the scores of keys 4 g4 + r, visible where
    // ok (all, if not MASKED), vop(j) the PV A operand of MFMA j, vs the V scale.
    auto softmax_pv = [&](auto masked_c, float (&sc)[4], const bool (&ok)[4], float vs, auto &&vop)
                          __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(masked_c)::value;
        const float mx = rows_max(vmax3(vmax3(sc[0], sc[1], sc[2]), sc[3], sc[0]));
        const bool bump = mx > m_ref + kLag;
        if (__builtin_amdgcn_ballot_w64(bump)) {
            const float mnew = bump ? mx : m_ref;
            const float alpha = mnew == m_ref ? 1.f : __builtin_amdgcn_exp2f(m_ref - mnew);
            m_ref = mnew;
            lsum *= alpha;
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[j] *= alpha;
        }
        float pv[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) pv[r] = __builtin_amdgcn_exp2f(sc[r] - m_ref);
        lsum += (pv[0] + pv[1]) + (pv[2] + pv[3]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            pv[r] *= vs;
            if constexpr (MASKED) pv[r] = ok[r] ? pv[r] : 0.f;  // (the scale of an unseen row may be NaN)
        }
        const uint2 pb = make_uint2(pack_bf16x2(pv[0], pv[1]), pack_bf16x2(pv[2], pv[3]));
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] = mfma_pv16(vop(j), pb, acc[j]);
    };

    // ---- q prologue: rotate at pos, fold the softmax scale (log2 domain), scale
    // to f16 by a power of two per head: lane (n, g4) holds dims D/4 g4 + 8 s .. + 7
    // of head n
    const int d0 = D / 4 * g4;
    const float2 *rp = a.p.rope + (int64_t)t * (D / 2) + (d0 & (D / 2 - 1));
    const float sgn = g4 < 2 ? -1.f : 1.f;
    // elements of slice s of an input row and their partners
    auto load_pair = [&](const bf16_t *r, int s, float (&x)[8], float (&z)[8]) __attribute__((always_inline)) {
        const RopeSrc o = rope_src<RF>(g, d0 + 8 * s, 8, D);
        uint4 xv = *(const uint4 *)(r + o.x), pv = *(const uint4 *)(r + o.y);
        if constexpr (RF)
            if (rope_il<RF>(g)) rope_split(xv, pv, g4 >= 2);
        unpack8(xv, x);
        unpack8(pv, z);
    };
    NormView norms{};
    if constexpr (RF == 2) norms = norm_view(a.p, a.layer, D);
    auto row_factor = [&](const bf16_t *r) __attribute__((always_inline)) {
        return norm_factor(D, norms.eps, [&](float c) __attribute__((always_inline)) {
            float ss = 0.f;
#pragma unroll
            for (int s = 0; s < ND; ++s) {
                float x[8], z[8];
                load_pair(r, s, x, z);
                ss += sum_square8(x, c);
            }
            return rows_sum(ss);
        });
    };
    // ... of the newest key, in the order of wave_norm_factor
    auto key_factor = [&](const bf16_t *r) __attribute__((always_inline)) {
        return norm_factor(D, norms.eps, [&](float c) __attribute__((always_inline)) {
            float s8[ND];
#pragma unroll
            for (int s = 0; s < ND; ++s) {
                float x[8], z[8], y[4];
                load_pair(r, s, x, z);
#pragma unroll
                for (int e = 0; e < 4; ++e)  // dims 2 e and 2 e + 1, each with its partner
                    y[e] = pair_square(x[2 * e], z[2 * e], c) + pair_square(x[2 * e + 1], z[2 * e + 1], c);
                s8[s] = (y[0] + y[1]) + (y[2] + y[3]);
            }
            float ss = s8[0];
            if constexpr (ND == 2) ss = s8[0] + s8[1];
            if constexpr (ND == 4) ss = (s8[0] + s8[1]) + (s8[2] + s8[3]);
            return rows_pair<true, false>(ss);  // (rows two apart hold the partners)
        });
    };
    // 8 rotated elements of slice s of an input row (w, f: its norm)
    auto rotate8 = [&](const bf16_t *r, int s, const float *w, float f, float (&y)[8]) __attribute__((always_inline)) {
        float x[8], z[8];
        load_pair(r, s, x, z);
        if constexpr (RF == 2) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = normed(x[e], f, w[d0 + 8 * s + e]);
                z[e] = normed(z[e], f, w[(d0 ^ (D / 2)) + 8 * s + e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 cs = rp[8 * s + e];
            y[e] = fmaf(x[e], cs.x, sgn * z[e] * cs.y);
        }
    };
    uint4 qh[ND], qb[ND];  // the query in f16 (scaled) for codes, in bf16 for the tail
    float qscale;
    {
        const bool hv = n < G;
        const bf16_t *qr = (const bf16_t *)a.q + (row * g.hq + (int64_t)kvh * G + (hv ? n : 0)) * D;
        float q[ND][8], mx = 0.f, f = 1.f;
        if constexpr (RF == 2) f = row_factor(qr);
#pragma unroll
        for (int s = 0; s < ND; ++s) {
            rotate8(qr, s, norms.q, f, q[s]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                q[s][e] = hv ? q[s][e] * a.scale_log2 : 0.f;
                mx = fmaxf(mx, fabsf(q[s][e]));
            }
        }
        const int eq = min(__builtin_amdgcn_frexp_expf(rows_max(mx)), 127);  // 0 for zero and for infinities
        qscale = ldexpf(1.f, eq);
#pragma unroll
        for (int s = 0; s < ND; ++s) {
            qh[s] = make_uint4(pack_f16x2(ldexpf(q[s][0], -eq), ldexpf(q[s][1], -eq)),
                               pack_f16x2(ldexpf(q[s][2], -eq), ldexpf(q[s][3], -eq)),
                               pack_f16x2(ldexpf(q[s][4], -eq), ldexpf(q[s][5], -eq)),
                               pack_f16x2(ldexpf(q[s][6], -eq), ldexpf(q[s][7], -eq)));
            qb[s] = make_uint4(pack_bf16x2(q[s][0], q[s][1]), pack_bf16x2(q[s][2], q[s][3]),
                               pack_bf16x2(q[s][4], q[s][5]), pack_bf16x2(q[s][6], q[s][7]));
        }
    }
    // ---- the newest block from the tail: keys to scores, then values, so that
    // the registers of one are free before the other's are used
    if (tail_wave) {
        uint8_t *tail = tail_of(ia.tails, g, sid, tslot, a.layer, kvh, D);
        bf16_t *tk = (bf16_t *)tail, *tv = tk + kBlock * D;
        uint8_t *region = (uint8_t *)g.kv + (int64_t)a.layer * g.layer_stride +
                          (int64_t)__builtin_amdgcn_readfirstlane(a.p.tok_block[t]) * g.block_stride;
        uint8_t *codes = region + (int64_t)kvh * BLK;
        const bool keep = fused && complete;  // the block is quantized, stored and used so
        int lb, lo, hi;
        vblock(g, vr, nv - 1, &lb, &lo, &hi);  // slots the query sees: hi - 1 is the newest key
        auto lo16 = [](uint32_t x) { return __uint_as_float(x << 16); };
        auto hi16 = [](uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); };
        auto wave_max = [](float x) {
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) x = max_nan(x, __shfl_xor(x, m, 64));
            return x;
        };
        // K row n, dims d0 .. + D/4 - 1; V rows 4 g4 + r, dims NJ n .. (NJ / 2 words)
        uint4 kr[ND];
        uint32_t vv[4][NJ / 2];
#pragma unroll
        for (int s = 0; s < ND; ++s) kr[s] = *(const uint4 *)(tk + n * D + d0 + 8 * s);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int x = 0; x < NJ / 2; x += 2)
                *(uint2 *)&vv[r][x] = *(const uint2 *)(tv + (4 * g4 + r) * D + NJ * n + 2 * x);
        uint32_t vn[NJ / 2];
        if (fused) {
            const bf16_t *kh = (const bf16_t *)a.k_new + (row * g.hkv + kvh) * D;
            const bf16_t *vh = (const bf16_t *)a.v_new + (row * g.hkv + kvh) * D + NJ * n;
#pragma unroll
            for (int x = 0; x < NJ / 2; x += 2) *(uint2 *)&vn[x] = *(const uint2 *)(vh + 2 * x);
            float f = 1.f;
            if constexpr (RF == 2) f = key_factor(kh);
#pragma unroll
            for (int s = 0; s < ND; ++s) {
                float y[8];
                rotate8(kh, s, norms.k, f, y);
                const uint4 kn = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]),
                                            pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
                if (n == toff) {
                    kr[s] = kn;
                    if (!complete) *(uint4 *)(tk + toff * D + d0 + 8 * s) = kn;  // for later launches
                }
            }
        }
        // rows past the newest one hold nothing (or NaN)
#pragma unroll
        for (int s = 0; s < ND; ++s) kr[s] = n <= toff ? kr[s] : make_uint4(0, 0, 0, 0);
        float ks = 1.f, vs = 1.f;
        if (keep) {
            float mk = 0.f;
#pragma unroll
            for (int s = 0; s < ND; ++s) {
                const uint32_t w[4] = {kr[s].x, kr[s].y, kr[s].z, kr[s].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) mk = vmaxabs3(lo16(w[e]), hi16(w[e]), mk);
            }
            ks = i8_scale(wave_max(mk));
            uint32_t kc[2 * ND];  // the lane's K codes, four a word
#pragma unroll
            for (int s = 0; s < ND; ++s) {
                uint32_t w[4] = {kr[s].x, kr[s].y, kr[s].z, kr[s].w};
                kc[2 * s] = kc[2 * s + 1] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c0 = i8_code(lo16(w[e]), ks), c1 = i8_code(hi16(w[e]), ks);
                    kc[2 * s + e / 2] |= (uint32_t)((c0 + 128) & 255) << (16 * (e & 1)) |
                                         (uint32_t)((c1 + 128) & 255) << (16 * (e & 1) + 8);
                    w[e] = pack_bf16x2((float)c0, (float)c1);
                }
                kr[s] = make_uint4(w[0], w[1], w[2], w[3]);
            }
#pragma unroll
            for (int x = 0; x < 2 * ND; x += 4)
                *(uint4 *)(codes + n * D + d0 + 4 * x) = make_uint4(kc[x], kc[x + 1], kc[x + 2], kc[x + 3]);
        }
        f32x4_t c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < ND; ++s) c = mfma16x16x32(kr[s], qb[s], c);
        // values: the newest one's row, nothing past it
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int key = 4 * g4 + r;
#pragma unroll
            for (int x = 0; x < NJ / 2; ++x)
                vv[r][x] = fused && key == toff ? vn[x] : key <= toff ? vv[r][x] : 0u;
        }
        if (fused && !complete && g4 == (toff >> 2))
#pragma unroll
            for (int x = 0; x < NJ / 2; x += 2)
                *(uint2 *)(tv + toff * D + NJ * n + 2 * x) = *(const uint2 *)&vn[x];
        if (keep) {
            float mv = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int x = 0; x < NJ / 2; ++x) mv = vmaxabs3(lo16(vv[r][x]), hi16(vv[r][x]), mv);
            vs = i8_scale(wave_max(mv));
            uint32_t vc[NJ];  // V codes: keys 4 g4 .. + 3 of dim NJ n + j
#pragma unroll
            for (int j = 0; j < NJ; ++j) vc[j] = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int x = 0; x < NJ / 2; ++x) {
                    const int c0 = i8_code(lo16(vv[r][x]), vs), c1 = i8_code(hi16(vv[r][x]), vs);
                    vc[2 * x] |= (uint32_t)(c0 & 255) << (8 * r);
                    vc[2 * x + 1] |= (uint32_t)(c1 & 255) << (8 * r);
                    vv[r][x] = pack_bf16x2((float)c0, (float)c1);
                }
#pragma unroll
            for (int x = 0; x < NJ; x += 4)
                *(uint4 *)(codes + kBlock * D + (g4 * D + NJ * n + x) * 4) =
                    make_uint4(vc[x], vc[x + 1], vc[x + 2], vc[x + 3]);
            if (lane == 0) *(float2 *)(codes + CODES) = make_float2(ks, vs);
        }
        float sc[4];
        bool ok[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            ok[r] = 4 * g4 + r >= lo && 4 * g4 + r < hi;
            sc[r] = ok[r] ? c[r] * ks : -INFINITY;
            // (0 * NaN: rows that are not seen must not bring their values)
#pragma unroll
            for (int x = 0; x < NJ / 2; ++x) vv[r][x] = ok[r] ? vv[r][x] : 0u;
        }
        softmax_pv(std::true_type{}, sc, ok, vs, [&](int j) __attribute__((always_inline)) {
            const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
            return make_uint2(__builtin_amdgcn_perm(vv[1][j / 2], vv[0][j / 2], sel),
                              __builtin_amdgcn_perm(vv[3][j / 2], vv[2][j / 2], sel));
        });
    }

    // per-lane LDS chunks of the K and V fragments inside a ring slot: K row n,
    // D/4 bytes from d0 on; V quad row g4, dims NJ n ..
    int ko[VD], vo[VD];
#pragma unroll
    for (int x = 0; x < VD; ++x) {
        ko[x] = swz(n * NJ + g4 * VD + x) * 16;
        vo[x] = swz(D + g4 * (D / 4) + n * VD + x) * 16;
    }
    // one block of the ring; MASKED: it may hold slots that the query cannot
    // see; AHEAD: the next block is issued before the wait for this one
    auto step = [&](int i, auto ahead_c, auto masked_c) __attribute__((always_inline)) {
        constexpr bool AHEAD = decltype(ahead_c)::value, MASKED = decltype(masked_c)::value;
        if constexpr (AHEAD) {
            if (i + NBUF - 1 < nblk) issue(i + NBUF - 1);
            vm_wait_blocks<NIW, NBUF - 1>(min(NBUF - 1, nblk - 1 - i));
        } else {
            vm_wait_blocks<NIW, NBUF - 2>(min(NBUF - 2, nblk - 1 - i));
            if (i + NBUF - 1 < nblk) issue(i + NBUF - 1);
        }
        const uint8_t *blk = &ring[wv][i % NBUF][0];
        uint32_t kw[2 * ND], vw[NJ];
#pragma unroll
        for (int x = 0; x < VD; ++x) {
            const uint4 k4 = *(const uint4 *)(blk + ko[x]), v4 = *(const uint4 *)(blk + vo[x]);
            kw[4 * x] = k4.x; kw[4 * x + 1] = k4.y; kw[4 * x + 2] = k4.z; kw[4 * x + 3] = k4.w;
            vw[4 * x] = v4.x; vw[4 * x + 1] = v4.y; vw[4 * x + 2] = v4.z; vw[4 * x + 3] = v4.w;
        }
        const float2 sc2 = *(const float2 *)(blk + CODES);
        f32x4_t c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < ND; ++s)
            c = mfma16x16x32_f16(make_uint4(i8_f16x2<false>(kw[2 * s]), i8_f16x2<true>(kw[2 * s]),
                                       i8_f16x2<false>(kw[2 * s + 1]), i8_f16x2<true>(kw[2 * s + 1])), qh[s], c);
        const float ks = sc2.x * qscale;
        float sc[4];
        bool ok[4] = {true, true, true, true};
        int lo = 0, hi = kBlock;
        if constexpr (MASKED) {
            int lb;
            vblock(g, vr, v0 + i, &lb, &lo, &hi);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            sc[r] = c[r] * ks;
            if constexpr (MASKED) {
                ok[r] = 4 * g4 + r >= lo && 4 * g4 + r < hi;
                sc[r] = ok[r] ? sc[r] : -INFINITY;
            }
        }
        softmax_pv(masked_c, sc, ok, sc2.y, [&](int j) __attribute__((always_inline)) {
            const float f0 = (float)(int8_t)vw[j], f1 = (float)(int8_t)(vw[j] >> 8);
            const float f2 = (float)(int8_t)(vw[j] >> 16), f3 = (float)(int8_t)(vw[j] >> 24);
            auto top = [](float x, float y) {  // two bf16 (exact: 8 bits at most)
                return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
            };
            return make_uint2(top(f0, f1), top(f2, f3));
        });
    };
    // sinks and the window's first block, the blocks between, its last one
    const int m_a = max(0, min(nblk, vr.n_sb + 1 - v0));
    const int m_b = max(m_a, v0 + nblk == nv ? nblk - 1 : nblk);
    // A wave issues its next block before it waits for the current one where
    // segments are short, a chain of round trips, and where a CU has one
    // workgroup, whose four waves' single copies would not cover the memory's
    // latency (64 sessions of G = 8, a workgroup per CU, 49.0 us against 57.4 in
    // two segments each); with more workgroups per CU after the wait (128 sessions
    // 93.9 against 96.7).  One choice per unit: its waves, one block apart, would
    // end apart with different ones.
    auto run = [&](auto ahead_c) __attribute__((always_inline)) {
        int i = 0;
        for (; i < m_a; ++i) step(i, ahead_c, std::true_type{});
        for (; i < m_b; ++i) step(i, ahead_c, std::false_type{});
        for (; i < nblk; ++i) step(i, ahead_c, std::true_type{});
    };
    if (ia.ahead || nv <= 20 * (int)nseg)
        run(std::true_type{});
    else
        run(std::false_type{});

    const float L = rows_sum(lsum);
    const int hq0 = kvh * G;
    // every wave hands (m, l, acc) over through its own drained ring; then all
    // threads merge them by log-sum-exp, VD output dims per thread and step
    static_assert(NG > 1, "the waves merge through LDS");
    float *scr = (float *)&ring[wv][0][0] + n * D + d0;  // [16][D]
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NJ; j += 4)
            *(float4 *)(scr + NJ * i + j) = make_float4(acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]);
    if (g4 == 0) {
        sM[wv][n] = m_ref;
        sL[wv][n] = L;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < G * 64; e += 64 * NG) {
        const int h = e >> 6, d = VD * (e & 63);
        float M = sM[0][h];
#pragma unroll
        for (int q = 1; q < NG; ++q) M = fmaxf(M, sM[q][h]);
        float l = 0.f, o[VD];
#pragma unroll
        for (int r = 0; r < VD; ++r) o[r] = 0.f;
#pragma unroll
        for (int q = 0; q < NG; ++q) {
            const float wq = __builtin_amdgcn_exp2f(sM[q][h] - M);
            const float *x = (const float *)&ring[q][0][0] + h * D + d;
            l = fmaf(sL[q][h], wq, l);
#pragma unroll
            for (int r = 0; r < VD; ++r) o[r] = fmaf(wq, x[r], o[r]);
        }
        if (a.n_split == 1) {
            const float inv = 1.f / l;
            bf16_t *ob = (bf16_t *)a.out + (row * g.hq + hq0 + h) * D + d;
            if constexpr (VD == 2)
                *(uint32_t *)ob = pack_bf16x2(o[0] * inv, o[1] * inv);
            else
                *ob = from_f32<bf16_t>(o[0] * inv);
            if (a.lse && d == 0) a.lse[row * g.hq + hq0 + h] = row_lse(M, l);
        } else {
            const int64_t base = ((int64_t)t * g.hq + hq0 + h) * ns + split;
            float *po = a.part + base * D + d;
            if constexpr (VD == 2)
                *(float2 *)po = make_float2(o[0], o[1]);
            else
                *po = o[0];
            if (d == 0) {
                float *pml = a.part + (int64_t)a.p.n_tok * g.hq * ns * D;
                pml[base * 2] = M;
                pml[base * 2 + 1] = l;
            }
        }
    }
}

// ---------------------------------------------------------------------------
// debug poison: codes of +127 in every slot whose live bit is clear, NaN scales
// where a block has none set; NaN rows past `rows` in every tail
// ---------------------------------------------------------------------------
__global__ void k_poison_i8(PoolGeom g, TailView tails, int32_t n_layers, int64_t n_blocks,
                            int32_t n_tails, const uint16_t *__restrict__ live,
                            const uint8_t *__restrict__ rows) {
    const int D = g.d;
    const int64_t n_items = (int64_t)n_layers * n_blocks * g.hkv;
    for (int64_t it = blockIdx.x; it < n_items; it += gridDim.x) {
        const int h = (int)(it % g.hkv);
        const int64_t b = (it / g.hkv) % n_blocks;
        const int l = (int)(it / ((int64_t)g.hkv * n_blocks));
        const uint16_t lm = live[b];
        if (lm == 0xFFFF) continue;
        uint8_t *region = (uint8_t *)g.kv + (int64_t)l * g.layer_stride + b * g.block_stride;
        uint8_t *codes = region + (int64_t)h * g.head_stride;
        for (int e = threadIdx.x; e < kBlock * D; e += blockDim.x) {
            const int key = e / D, d = e % D;
            if ((lm >> key) & 1) continue;
            codes[e] = 0xFF;
            codes[kBlock * D + ((key >> 2) * D + d) * 4 + (key & 3)] = 0x7F;
        }
        if (lm == 0 && threadIdx.x < 2)
            ((float *)(codes + 2 * kBlock * D))[threadIdx.x] = __builtin_nanf("");
    }
    const int64_t n_rows = (int64_t)n_tails * n_layers * g.hkv * kBlock;
    for (int64_t it = blockIdx.x; it < n_rows; it += gridDim.x) {
        const int key = (int)(it % kBlock);
        const int64_t th = it / kBlock;  // (tail, layer, head)
        const int64_t tail = th / ((int64_t)n_layers * g.hkv);
        if (key < rows[tail]) continue;
        uint16_t *r = (uint16_t *)(tails.base + tail * tails.stride +
                                   (th - tail * n_layers * g.hkv) * (64 * D)) + key * D;
        for (int e = threadIdx.x; e < D; e += blockDim.x) r[e] = r[kBlock * D + e] = 0x7FC0;
    }
}

template <int D, int G>
hipError_t launch_i8_g(const I8Args &ia, hipStream_t s) {
    const int64_t units = (int64_t)ia.a.p.n_tok * ia.a.g.hkv * ia.a.n_split;
    if (units == 0) return hipSuccess;
    if (units > INT32_MAX) return hipErrorInvalidValue;  // one grid dimension, 32-bit unit index
    const dim3 grid((unsigned)units), block(64 * kI8Waves);
    with_form(ia.a.g, [&](auto rf) {
        hipLaunchKernelGGL((k_attn_i8<D, G, decltype(rf)::value>), grid, block, 0, s, ia);
    });
    return hipGetLastError();
}
template <class F>
auto with_shape(int d, int g, F &&f) {
    auto by_g = [&](auto dc) {
        switch (g) {
            case 1: return f(dc, std::integral_constant<int, 1>{});
            case 2: return f(dc, std::integral_constant<int, 2>{});
            case 4: return f(dc, std::integral_constant<int, 4>{});
            default: return f(dc, std::integral_constant<int, 8>{});
        }
    };
    return d == 128 ? by_g(std::integral_constant<int, 128>{}) : by_g(std::integral_constant<int, 64>{});
}

}  // namespace

bool attn_i8_supported(int d, int g) {
    return (d == 128 || d == 64) && (g == 1 || g == 2 || g == 4 || g == 8);
}
int attn_i8_groups() { return kI8Waves; }

hipError_t launch_append_i8(const PoolGeom &g, const PlanView &p, int32_t layer, const void *k, const void *v,
                            const TailView &tails, const int32_t *run_tok0, const int32_t *run_len,
                            int32_t n_runs, hipStream_t s) {
    if (g.d != 128 && g.d != 64) return hipErrorInvalidValue;
    const int64_t groups = (int64_t)n_runs * g.hkv;
    if (groups == 0) return hipSuccess;
    if (groups > INT32_MAX) return hipErrorInvalidValue;
    auto launch = [&](auto dc, auto rf) {
        hipLaunchKernelGGL((k_append_i8<decltype(dc)::value, decltype(rf)::value>), dim3((unsigned)groups), dim3(256),
                           0, s, g, p, layer, (const bf16_t *)k, (const bf16_t *)v, tails, run_tok0, run_len);
    };
    auto by_d = [&](auto rf) {
        g.d == 128 ? launch(std::integral_constant<int, 128>{}, rf) : launch(std::integral_constant<int, 64>{}, rf);
    };
    with_form(g, by_d);
    return hipGetLastError();
}

hipError_t launch_attn_i8(const AttnArgs &a, const TailView &tails, int n_cu, hipStream_t s) {
    const int G = a.g.hq / a.g.hkv;
    if (!attn_i8_supported(a.g.d, G) || (a.k_new == nullptr) != (a.v_new == nullptr)) return hipErrorInvalidValue;
    const I8Args ia{a, tails, (int64_t)a.p.n_tok * a.g.hkv * a.n_split <= n_cu};
    return with_shape(a.g.d, G, [&](auto dc, auto gc) { return launch_i8_g<decltype(dc)::value, decltype(gc)::value>(ia, s); });
}

hipError_t launch_poison_i8(const PoolGeom &g, const TailView &tails, int32_t n_layers, int64_t n_blocks,
                            int32_t n_tails, const uint16_t *live, const uint8_t *rows, hipStream_t s) {
    hipLaunchKernelGGL(k_poison_i8, dim3(8192), dim3(256), 0, s, g, tails, n_layers, n_blocks, n_tails, live, rows);
    return hipGetLastError();
}

}  // namespace mtn
