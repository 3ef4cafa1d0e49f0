// Linear attention with a decay per head on gfx950: the chunk form for plans of any
// lengths and the recurrent form for single tokens.
//
//   S_t = lambda S_(t-1) + v_t k_t^T,   o_t = scale S_t q_t
//
// S is value dims by key dims in fp32, one per session, layer and KV head, shared by
// the G query heads of the KV head.  A plan reads each session's state from the
// slot that holds the committed one and writes the session's other slot, so that
// an abandoned plan, or a captured one that is replayed, changes nothing that
// a later plan reads.
#include "mtn_device.h"
#include "mtn_linear.h"

#include <algorithm>

namespace mtn {
namespace {

constexpr int kLinWaves = 4;
constexpr int kLinThreads = 64 * kLinWaves;

// ---------------------------------------------------------------------------
// recurrent form: one token per sequence
// ---------------------------------------------------------------------------
// One workgroup per (sequence, KV head, slice of D / SL value rows of the state): row
// e holds S[e][0 .. D - 1].  Eight lanes share a row (16-byte vectors side by side,
// whole 128-byte lines per load instruction), 32 rows per step of the workgroup;
// every load of a thread's part of the state goes out before the first is used.
// Each element takes one product and one multiply-add for its update and one
// more per query head: bound by the state's bytes, read and written once.
template <typename T, int D, int G, int SL>
__global__ __launch_bounds__(kLinThreads) void k_linear_decode(LinArgs a) {
    constexpr int RW = D / SL;         // rows of the workgroup
    constexpr int NP = RW / 32;        // steps
    constexpr int NC = D / 32;         // vectors per thread and row
    __shared__ __align__(16) float sq[G][D], sk[D], so[G][RW];
    const int tid = threadIdx.x, lane = tid & 63;
    const uint32_t u = blockIdx.x / SL;
    const int sl = (int)(blockIdx.x - u * SL);
    const int i = (int)(u / (uint32_t)a.hkv), h = (int)(u - (uint32_t)i * a.hkv);
    const int64_t row = scalar_ld(a.items, kLinItem * i);
    const int32_t rec = scalar_ld(a.items, kLinItem * i + 2);
    const int32_t slot = rec & (kLinFresh - 1);
    const int64_t off = (int64_t)h * D * D + sl * RW * D;
    const float *src = a.state + (int64_t)slot * a.slot_stride + off;
    float *dst = a.state + (int64_t)(slot ^ 1) * a.slot_stride + off;
    const int e0 = tid >> 3, c0 = 4 * (tid & 7);  // first row, first column
    f32x4_t S[NP][NC];
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int c = 0; c < NC; ++c)
            S[p][c] = rec & kLinFresh ? f32x4_t{0.f, 0.f, 0.f, 0.f}
                                      : *(const f32x4_t *)(src + (e0 + 32 * p) * D + c0 + 32 * c);
    const T *vr = (const T *)a.v + (row * a.hkv + h) * D + sl * RW;
    float v[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) v[p] = to_f32(vr[e0 + 32 * p]);
    const T *qr = (const T *)a.q + (row * a.hq + (int64_t)h * G) * D;
    const T *kr = (const T *)a.k + (row * a.hkv + h) * D;
    for (int x = tid; x < G * D; x += kLinThreads) (&sq[0][0])[x] = to_f32(qr[x]);
    if (tid < D) sk[tid] = to_f32(kr[tid]);
    const float lam = __builtin_amdgcn_exp2f(a.log2_decay[h]);
    __syncthreads();
    float acc[NP][G];
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int g = 0; g < G; ++g) acc[p][g] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const f32x4_t kk = *(const f32x4_t *)&sk[c0 + 32 * c];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
#pragma unroll
            for (int e = 0; e < 4; ++e) S[p][c][e] = fmaf(lam, S[p][c][e], v[p] * kk[e]);
            *(f32x4_t *)(dst + (e0 + 32 * p) * D + c0 + 32 * c) = S[p][c];
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const f32x4_t qq = *(const f32x4_t *)&sq[g][c0 + 32 * c];
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[p][g] = fmaf(S[p][c][e], qq[e], acc[p][g]);
        }
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float x = acc[p][g];
            x += dpp<kQuadXor1>(x);
            x += dpp<kQuadXor2>(x);
            x += dpp<kRowHalfMirror>(x);
            if ((lane & 7) == g) so[g][e0 + 32 * p] = x;
        }
    __syncthreads();
    T *out = (T *)a.out + (row * a.hq + (int64_t)h * G) * D + sl * RW;
    for (int x = tid; x < G * RW; x += kLinThreads)
        out[(x / RW) * D + x % RW] = from_f32<T>(a.scale * so[x / RW][x % RW]);
}

// ---------------------------------------------------------------------------
// matrix operands
// ---------------------------------------------------------------------------
// A fragment is a lane's share of a 16 x 32 operand (or 32 x 16: the two are
// alike): lane (n, g) with n = lane % 16, g = lane / 16 holds row n and eight
// depth elements.  Which eight is free as long as both operands agree; a
// product over tokens takes tokens 4 g .. + 3 of two tiles of 16, which is how a
// lane holds the results of two earlier products, so that those feed the next
// without moving.  split: fp32 numbers as that many terms of 8 bits, the last one
// rounded (three hold all 24 bits).
template <typename T>
struct Ops;
template <>
struct Ops<bf16_t> {
    using Frag = uint4;
    // The state takes all 24 bits of a weighted value, in three terms (two would
    // leave it 2^-15 off, in fp32 whose other roundings are 2^-24); the products that
    // only make an output, rounded by up to 2^-8, take 16 bits of state and of
    // scores (2^-15).
    static constexpr int kOut = 2, kState = 3;
    static __device__ __forceinline__ Frag row(const bf16_t *p) { return *(const uint4 *)p; }
    // rows (tokens) of p0 and p1, a column a lane: see tr()
    static __device__ __forceinline__ uint2 tr(const bf16_t *p) {
        typedef __attribute__((ext_vector_type(4))) short s16x4;
        return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                             (__attribute__((address_space(3))) s16x4 *)(
                                                 const __attribute__((address_space(3))) void *)p));
    }
    // Four tokens of two tiles for column n: lane (n, g) hands in the address of
    // columns 4 (n % 4) .. + 3 (wherever those lie) of token 4 g + n / 4 and
    // receives column n of tokens 4 g .. + 3.
    static __device__ __forceinline__ Frag cols(const bf16_t *p, int tile_stride, int, int) {
        const uint2 x = tr(p), y = tr(p + tile_stride);
        return make_uint4(x.x, x.y, y.x, y.y);
    }
    static __device__ __forceinline__ f32x4_t mma(const Frag &a, const Frag &b, f32x4_t c) {
        return mfma16x16x32(a, b, c);
    }
    static __device__ __forceinline__ void unpack(const Frag &f, float (&x)[8]) { unpack8(f, x); }
    template <int N>
    static __device__ __forceinline__ void split(float (&x)[8], Frag (&f)[N]) {
#pragma unroll
        for (int p = 0; p < N; ++p) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float &a = x[2 * e], &b = x[2 * e + 1];
                if (p == N - 1) {
                    w[e] = pack_bf16x2(a, b);
                } else {  // the upper halves; the rest is exact
                    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
                    w[e] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
                    a -= __uint_as_float(ua & 0xFFFF0000u);
                    b -= __uint_as_float(ub & 0xFFFF0000u);
                }
            }
            f[p] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    // largest magnitude's bits reach the exponent of infinities
    static __device__ __forceinline__ bool bad(const Frag &f) {
        const uint32_t w[4] = {f.x, f.y, f.z, f.w};
        bool b = false;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            b |= (w[e] & 0x7F80u) == 0x7F80u || (w[e] & 0x7F800000u) == 0x7F800000u;
        return b;
    }
    static __device__ __forceinline__ bool bad_at(const Frag &f, int e) {
        const uint32_t w[4] = {f.x, f.y, f.z, f.w};
        return e & 1 ? (w[e / 2] & 0x7F800000u) == 0x7F800000u : (w[e / 2] & 0x7F80u) == 0x7F80u;
    }
    static __device__ __forceinline__ void clear_at(Frag &f, int e) {
        uint32_t w[4] = {f.x, f.y, f.z, f.w};
        w[e / 2] &= e & 1 ? 0xFFFFu : 0xFFFF0000u;
        f = make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ void store4(bf16_t *p, const f32x4_t &x) {
        *(uint2 *)p = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    }
    static __device__ __forceinline__ void store8(bf16_t *p, const f32x4_t &x, const f32x4_t &y) {
        *(uint4 *)p = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(y[0], y[1]),
                                 pack_bf16x2(y[2], y[3]));
    }
};
template <>
struct Ops<float> {
    struct Frag {
        float x[8];
    };
    static constexpr int kOut = 1, kState = 1;
    static __device__ __forceinline__ Frag row(const float *p) {
        Frag f;
        *(float4 *)&f.x[0] = *(const float4 *)p;
        *(float4 *)&f.x[4] = *(const float4 *)(p + 4);
        return f;
    }
    // the lane's own column (n % 4 of those handed in), token by token
    static __device__ __forceinline__ Frag cols(const float *p, int tile_stride, int ld, int n) {
        Frag f;
        const float *c = p - (n >> 2) * ld;  // token 4 g
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f.x[e] = c[e * ld];
            f.x[4 + e] = c[tile_stride + e * ld];
        }
        return f;
    }
    static __device__ __forceinline__ f32x4_t mma(const Frag &a, const Frag &b, f32x4_t c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[e], b.x[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ void unpack(const Frag &f, float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = f.x[e];
    }
    template <int N>
    static __device__ __forceinline__ void split(float (&x)[8], Frag (&f)[N]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[0].x[e] = x[e];
    }
    static __device__ __forceinline__ bool bad_at(const Frag &f, int e) { return !(fabsf(f.x[e]) < INFINITY); }
    static __device__ __forceinline__ bool bad(const Frag &f) {
        bool b = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) b |= bad_at(f, e);
        return b;
    }
    static __device__ __forceinline__ void clear_at(Frag &f, int e) { f.x[e] = 0.f; }
    static __device__ __forceinline__ void store4(float *p, const f32x4_t &x) { *(f32x4_t *)p = x; }
    static __device__ __forceinline__ void store8(float *p, const f32x4_t &x, const f32x4_t &y) {
        *(f32x4_t *)p = x;
        *(f32x4_t *)(p + 4) = y;
    }
};

// ---------------------------------------------------------------------------
// chunk form
// ---------------------------------------------------------------------------
// One workgroup of four waves per (item, KV head), tiles of B tokens one after the
// other.  With S before the tile, i and j tokens of the tile, n its length:
//   o_i  = scale (lambda^(i+1) S q_i + sum_{j <= i} lambda^(i-j) (k_j . q_i) v_j)
//   S'   = lambda^n S + sum_j (lambda^(n-1-j) v_j) k_j^T
// A wave owns D / 4 value dims: their rows of S stay in its accumulators from the
// first tile to the last, and serve as an operand of S q as they lie (two
// accumulators make a fragment's depth).  Scores are formed transposed (keys by
// queries), each wave those of one 16-query tile, and go through LDS to
// the other waves; they too feed the product with V as they lie.  K and V
// are contracted over tokens by transposing reads of LDS.  Decays multiply scores,
// rows of S q, and values in fp32, never as rounded operands.
//
// LOCAL: a segment's own state, from zero, into a.seg (no queries, no outputs).
// Otherwise an unsegmented item starts from its session's state and leaves the
// new one, a segment starts from what k_linear_scan left for it.
//
// A value that is not finite reaches the outputs from its token on and no others, as
// in the recurrence (though an infinity may read NaN there): masked scores are 0,
// and 0 * inf is NaN, so a wave whose values hold one clears it, and writes
// NaN into that dim's outputs from that token on.
template <typename T, int D, int B, bool LOCAL>
__global__ __launch_bounds__(kLinThreads, 1) void k_linear_chunk(LinArgs a) {
    using O = Ops<T>;
    using Frag = typename O::Frag;
    constexpr int NT = D / 64, NS = D / 32, MT = D / 16, JT = B / 16, KS = B / 32;
    constexpr int EPV = 16 / (int)sizeof(T), LD = D + EPV;  // row pitch in LDS
    constexpr int VPR = D / EPV;                            // vectors of a row
    constexpr int CH = B * VPR / kLinThreads;
    static_assert(B * VPR % kLinThreads == 0 && JT <= kLinWaves, "tile shape");
    __shared__ __align__(16) T sk[B * LD], sv[B * LD], sq[LOCAL ? EPV : B * LD];
    __shared__ Frag sp[LOCAL ? 1 : JT * KS * O::kOut * 64];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, n = lane & 15, g = lane >> 4;
    const int it_ = (int)(blockIdx.x / (uint32_t)a.hkv), h = (int)(blockIdx.x - (uint32_t)it_ * a.hkv);
    const int row0 = scalar_ld(a.items, kLinItem * it_), ntok = scalar_ld(a.items, kLinItem * it_ + 1);
    const int rec = scalar_ld(a.items, kLinItem * it_ + 2);
    const int nseg = scalar_ld(a.items, kLinItem * it_ + 3) >> 16;
    if (LOCAL && nseg == 1) return;  // the whole workgroup
    const int slot = rec & (kLinFresh - 1), G = a.hq / a.hkv;
    const float l2 = a.log2_decay[h];
    auto power = [&](int e) { return __builtin_amdgcn_exp2f((float)e * l2); };

    // this wave's value dims: lane n of tile nt is dim dv0 + dvn + 4 nt, result row
    // 4 g + r dim dv0 + 8 g + 4 nt + r (one tile: n and 4 g + r)
    const int dv0 = wv * 16 * NT;
    const int dvn = NT == 2 ? 8 * (n >> 2) + (n & 3) : n;
    // S as the products make it: result row 4 g + r of tile mt = 2 s + t is key dim
    // 32 s + 8 g + 4 t + r, column n the value dim above
    f32x4_t S[MT][NT];
    float *const seg = a.seg + ((int64_t)it_ * a.hkv + h) * D * D;
    {
        const float *src = nseg > 1 ? seg : a.state + (int64_t)slot * a.slot_stride + (int64_t)h * D * D;
        const bool zero = LOCAL || (nseg == 1 && (rec & kLinFresh));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int m = 0; m < MT; ++m)
                S[m][nt] = zero ? f32x4_t{0.f, 0.f, 0.f, 0.f}
                                : *(const f32x4_t *)(src + (dv0 + dvn + 4 * nt) * D + 32 * (m / 2) + 8 * g + 4 * (m & 1));
    }
    // decays of this wave's scores (queries 16 wv + n) and of the outputs' rows
    float wp[JT][4], wr[JT];
    if constexpr (!LOCAL) {
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) {
#pragma unroll
            for (int r = 0; r < 4; ++r) wp[jt][r] = power(max(16 * (wv - jt) + n - 4 * g - r, 0));
            wr[jt] = power(16 * jt + n + 1);
        }
    }
    // 16 bytes of token row, vector col of a tile, per thread and step
    auto load = [&](const void *base, int heads, int head, int t0, int nb, uint4 (&x)[CH]) __attribute__((always_inline)) {
        const T *p = (const T *)base + ((int64_t)(row0 + t0) * heads + head) * D;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int v = tid + c * kLinThreads, r = v / VPR;
            x[c] = r < nb ? *(const uint4 *)(p + (int64_t)r * heads * D + v % VPR * EPV) : make_uint4(0, 0, 0, 0);
        }
    };
    auto put = [&](T *dst, const uint4 (&x)[CH]) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int v = tid + c * kLinThreads;
            *(uint4 *)(dst + v / VPR * LD + v % VPR * EPV) = x[c];
        }
    };
    uint4 xk[CH], xv[CH], xq[CH];
    {
        const int nb = min(B, ntok);
        load(a.k, a.hkv, h, 0, nb, xk);
        load(a.v, a.hkv, h, 0, nb, xv);
        if constexpr (!LOCAL) load(a.q, a.hq, h * G, 0, nb, xq);
    }
    for (int t0 = 0; t0 < ntok; t0 += B) {
        const int nb = min(B, ntok - t0);
        put(sk, xk);
        put(sv, xv);
        if constexpr (!LOCAL) put(sq, xq);
        __syncthreads();
        auto next_tile = [&]() __attribute__((always_inline)) {
            if (t0 + B >= ntok) return;
            const int nx = min(B, ntok - t0 - B);
            load(a.k, a.hkv, h, t0 + B, nx, xk);
            load(a.v, a.hkv, h, t0 + B, nx, xv);
            if constexpr (!LOCAL) load(a.q, a.hq, h * G, t0 + B, nx, xq);
        };
        // values of this wave's dims, tokens deep
        Frag vf[KS][NT];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                vf[ks][nt] = O::cols(sv + (32 * ks + 4 * g + (n >> 2)) * LD + dv0 +
                                         (NT == 2 ? 8 * (n & 3) + 4 * nt : 4 * (n & 3)) * (sizeof(T) == 2 ? 1 : 0) +
                                         (sizeof(T) == 2 ? 0 : dvn + 4 * nt),
                                     16 * LD, LD, n);
        if constexpr (LOCAL) next_tile();
        if constexpr (!LOCAL) {
            bool bad = false;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) bad |= O::bad(vf[ks][nt]);
            const bool any_bad = __builtin_amdgcn_ballot_w64(bad) != 0;
            for (int gh = 0; gh < G; ++gh) {
                if (gh + 1 < G)
                    load(a.q, a.hq, h * G + gh + 1, t0, nb, xq);
                else
                    next_tile();
                // ---- scores of queries 16 wv .. + 15, keys by queries
                if (wv < JT && 16 * wv < nb) {
                    f32x4_t sc[JT];
#pragma unroll
                    for (int jt = 0; jt < JT; ++jt) sc[jt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const Frag qf = O::row(sq + (16 * wv + n) * LD + 32 * s + 8 * g);
#pragma unroll
                        for (int jt = 0; jt < JT; ++jt)
                            if (jt <= wv) sc[jt] = O::mma(O::row(sk + (16 * jt + n) * LD + 32 * s + 8 * g), qf, sc[jt]);
                    }
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        if (2 * ks > wv) break;
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int jt = 2 * ks + e / 4, r = e & 3;
                            x[e] = 16 * jt + 4 * g + r <= 16 * wv + n ? sc[jt][r] * wp[jt][r] : 0.f;
                        }
                        Frag pf[O::kOut];
                        O::template split<O::kOut>(x, pf);
#pragma unroll
                        for (int p = 0; p < O::kOut; ++p) sp[((wv * KS + ks) * O::kOut + p) * 64 + lane] = pf[p];
                    }
                }
                // ---- S q, value dims by queries
                f32x4_t o[JT][NT];
#pragma unroll
                for (int it = 0; it < JT; ++it)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) o[it][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    Frag sf[NT][O::kOut];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = S[2 * s + e / 4][nt][e & 3];
                        O::template split<O::kOut>(x, sf[nt]);
                    }
#pragma unroll
                    for (int it = 0; it < JT; ++it) {
                        const Frag qf = O::row(sq + (16 * it + n) * LD + 32 * s + 8 * g);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int p = 0; p < O::kOut; ++p) o[it][nt] = O::mma(sf[nt][p], qf, o[it][nt]);
                    }
                }
                __syncthreads();  // every score is there, nobody reads these queries any more
                if (gh + 1 < G) put(sq, xq);
                // ---- plus V times the scores
                T *ob = (T *)a.out + ((int64_t)(row0 + t0) * a.hq + h * G + gh) * D + dv0;
                auto finish = [&](auto bad_c) __attribute__((always_inline)) {
                    constexpr bool BAD = decltype(bad_c)::value;
                    int first[NT];  // BAD: the first token whose value of the lane's dim is not finite
                    Frag vc[BAD ? KS : 1][NT];
                    if constexpr (BAD) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            first[nt] = B;
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks) {
                                vc[ks][nt] = vf[ks][nt];
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    if (O::bad_at(vf[ks][nt], e)) {
                                        O::clear_at(vc[ks][nt], e);
                                        first[nt] = min(first[nt], 32 * ks + 16 * (e / 4) + 4 * g + (e & 3));
                                    }
                            }
                            first[nt] = min(first[nt], __shfl_xor(first[nt], 16, 64));
                            first[nt] = min(first[nt], __shfl_xor(first[nt], 32, 64));
                        }
                    }
#pragma unroll
                    for (int it = 0; it < JT; ++it) {
                        if (16 * it >= nb) break;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) o[it][nt] *= wr[it];
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            if (2 * ks > it) break;
#pragma unroll
                            for (int p = 0; p < O::kOut; ++p) {
                                const Frag pf = sp[((it * KS + ks) * O::kOut + p) * 64 + lane];
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
                                    o[it][nt] = O::mma(BAD ? vc[BAD ? ks : 0][nt] : vf[ks][nt], pf, o[it][nt]);
                            }
                        }
                        const int i = 16 * it + n;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            o[it][nt] *= a.scale;
                            if constexpr (BAD) {
#pragma unroll
                                for (int r = 0; r < 4; ++r)
                                    if (i >= __shfl(first[nt], 4 * g + r, 64)) o[it][nt][r] = __builtin_nanf("");
                            }
                        }
                        if (i < nb) {
                            T *p = ob + (int64_t)i * a.hq * D;
                            if constexpr (NT == 2)
                                O::store8(p + 8 * g, o[it][0], o[it][NT - 1]);
                            else
                                O::store4(p + 4 * g, o[it][0]);
                        }
                    }
                };
                if (__builtin_expect(any_bad, 0))
                    finish(std::true_type{});
                else
                    finish(std::false_type{});
                if (gh + 1 < G) __syncthreads();  // the next queries are there, the scores read
            }
        }
        // ---- the state after the tile
        if (LOCAL || nseg == 1 || t0 + B < ntok) {
            const float dec = power(nb);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) S[m][nt] *= dec;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (32 * ks >= nb) break;
                Frag vw[NT][O::kState];
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = power(max(nb - 1 - (32 * ks + 16 * (e / 4) + 4 * g + (e & 3)), 0));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float x[8];
                    O::unpack(vf[ks][nt], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= w[e];
                    O::template split<O::kState>(x, vw[nt]);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const Frag kf = O::cols(sk + (32 * ks + 4 * g + (n >> 2)) * LD + 32 * (m / 2) + 4 * (m & 1) +
                                                (sizeof(T) == 2 ? 8 * (n & 3) : 8 * (n >> 2) + (n & 3)),
                                            16 * LD, LD, n);
#pragma unroll
                    for (int p = 0; p < O::kState; ++p)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) S[m][nt] = O::mma(kf, vw[nt][p], S[m][nt]);
                }
            }
        }
        __syncthreads();  // K, V, Q and scores may be overwritten
    }
    if (!LOCAL && nseg > 1) return;
    float *dst = LOCAL ? seg : a.state + (int64_t)(slot ^ 1) * a.slot_stride + (int64_t)h * D * D;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int m = 0; m < MT; ++m)
            *(f32x4_t *)(dst + (dv0 + dvn + 4 * nt) * D + 32 * (m / 2) + 8 * g + 4 * (m & 1)) = S[m][nt];
}

// ---------------------------------------------------------------------------
// segments: every segment's own state becomes the state it starts from
// ---------------------------------------------------------------------------
// Thread per four elements of a sequence's state, segment after segment, the loads
// of eight segments ahead of their use.  The last state is the session's new one.
template <int D>
__global__ __launch_bounds__(256) void k_linear_scan(LinArgs a) {
    const int u = blockIdx.y, it = u / a.hkv, h = u - it * a.hkv;
    const int w = scalar_ld(a.items, kLinItem * it + 3), nseg = w >> 16;
    if (nseg == 1 || (w & 0xFFFF)) return;
    const int rec = scalar_ld(a.items, kLinItem * it + 2), slot = rec & (kLinFresh - 1);
    const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const int64_t st = (int64_t)slot * a.slot_stride + (int64_t)h * D * D + e;
    f32x4_t cur = rec & kLinFresh ? f32x4_t{0.f, 0.f, 0.f, 0.f} : *(const f32x4_t *)(a.state + st);
    float *p = a.seg + ((int64_t)it * a.hkv + h) * D * D + e;
    const int64_t step = (int64_t)a.hkv * D * D;
    const float l2 = a.log2_decay[h];
    for (int s0 = 0; s0 < nseg; s0 += 8) {
        f32x4_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (s0 + j < nseg) x[j] = *(const f32x4_t *)(p + (s0 + j) * step);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (s0 + j < nseg) {
                *(f32x4_t *)(p + (s0 + j) * step) = cur;
                const float d = __builtin_amdgcn_exp2f((float)scalar_ld(a.items, kLinItem * (it + s0 + j) + 1) * l2);
#pragma unroll
                for (int r = 0; r < 4; ++r) cur[r] = fmaf(d, cur[r], x[j][r]);
            }
    }
    *(f32x4_t *)(a.state + st + (((slot ^ 1) - slot) * a.slot_stride)) = cur;
}

__global__ __launch_bounds__(256) void k_linear_poison(float *states, int64_t slot_stride, int32_t n_slots,
                                                       const uint8_t *__restrict__ dead) {
    for (int s = blockIdx.y; s < n_slots; s += gridDim.y) {
        if (!dead[s]) continue;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < slot_stride; i += (int64_t)gridDim.x * 256)
            states[s * slot_stride + i] = __builtin_nanf("");
    }
}

// f(D as an integral constant, an element of the type)
template <class F>
hipError_t by_shape(int dtype, int d, F &&f) {
    auto by_d = [&](auto elt) {
        if (d == 128)
            f(std::integral_constant<int, 128>{}, elt);
        else
            f(std::integral_constant<int, 64>{}, elt);
    };
    if (dtype == 1)
        by_d(bf16_t{});
    else
        by_d(0.f);
    return hipGetLastError();
}

}  // namespace

bool linear_supported(int dtype, int d, int g) {
    return (dtype == 0 || dtype == 1) && (d == 64 || d == 128) && (g == 1 || g == 2 || g == 4 || g == 8);
}

hipError_t launch_linear_decode(int dtype, const LinArgs &a, int n_cu, hipStream_t s) {
    if (!linear_supported(dtype, a.d, a.hq / a.hkv) || a.n_items < 1) return hipErrorInvalidValue;
    const int64_t units = (int64_t)a.n_items * a.hkv;
    if (2 * units > INT32_MAX) return hipErrorInvalidValue;
    return by_shape(dtype, a.d, [&](auto dc, auto elt) {
        constexpr int D = decltype(dc)::value;
        using T = decltype(elt);
        auto go = [&](auto gc) {
            hipLaunchKernelGGL((k_linear_decode<T, D, decltype(gc)::value, 1>), dim3((unsigned)units),
                               dim3(kLinThreads), 0, s, a);
        };
        switch (a.hq / a.hkv) {
            case 1: go(std::integral_constant<int, 1>{}); break;
            case 2: go(std::integral_constant<int, 2>{}); break;
            case 4: go(std::integral_constant<int, 4>{}); break;
            default: go(std::integral_constant<int, 8>{}); break;
        }
    });
}

hipError_t launch_linear_chunk(int dtype, const LinArgs &a, int max_tok, bool split, hipStream_t s) {
    if (!linear_supported(dtype, a.d, a.hq / a.hkv) || a.n_items < 1 || (split && !a.seg)) return hipErrorInvalidValue;
    const int64_t units = (int64_t)a.n_items * a.hkv;
    if (units > (split ? 65535 : INT32_MAX)) return hipErrorInvalidValue;  // (the scan's second grid dimension)
    return by_shape(dtype, a.d, [&](auto dc, auto elt) {
        constexpr int D = decltype(dc)::value;
        using T = decltype(elt);
        auto go = [&](auto bc) {
            constexpr int B = decltype(bc)::value;
            const dim3 grid((unsigned)units), block(kLinThreads);
            if (split) {
                hipLaunchKernelGGL((k_linear_chunk<T, D, B, true>), grid, block, 0, s, a);
                hipLaunchKernelGGL((k_linear_scan<D>), dim3(D * D / 1024, (unsigned)units), dim3(256), 0, s, a);
            }
            hipLaunchKernelGGL((k_linear_chunk<T, D, B, false>), grid, block, 0, s, a);
        };
        if constexpr (sizeof(T) == 2) {
            if (max_tok > 32) return go(std::integral_constant<int, 64>{});
        }
        go(std::integral_constant<int, 32>{});
    });
}

hipError_t launch_linear_poison(float *states, int64_t slot_stride, int32_t n_slots, const uint8_t *dead,
                                hipStream_t s) {
    hipLaunchKernelGGL(k_linear_poison, dim3(64, (unsigned)std::min(n_slots, 1024)), dim3(256), 0, s, states,
                       slot_stride, n_slots, dead);
    return hipGetLastError();
}

}  // namespace mtn
