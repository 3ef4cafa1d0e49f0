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

constexpr int kLinThreads = 256;  // of the single-token form
// Waves of a chunk workgroup with tiles of B tokens.  Four with 64-token tiles: at
// eight, a wave's operands served half as many products, and its registers (128 for
// two workgroups a CU) spilled in the loop (one prompt of 8192 tokens of 32 heads
// 5 % longer than with four).  With 32-token tiles eight at D = 128 end sooner where
// few workgroups run (32 sessions of 25 tokens, G = 4, 4 KV heads 16.5 us, four 18.0).
constexpr int lin_waves(int d, int b) { return b == 64 ? 4 : d / 16; }

// ---------------------------------------------------------------------------
// recurrent form: one token per sequence
// ---------------------------------------------------------------------------
// One workgroup per (sequence, KV head, slice of D / SL value rows of the state): row
// e holds S[e][0 .. D - 1].  Eight lanes share a row (16-byte vectors side by side,
// whole 128-byte lines per load instruction), 32 rows per step of the workgroup;
// every load of a thread's part of the state goes out before the first is used.
// Each element takes one product and two multiply-adds for its update and one
// more per query head: bound by the state's bytes, read and written once.
// The decay comes in two fp32 terms: one that is rounded is off the same way token
// after token (lambda = 1 - 2^-14 and a steady input: 2^-25 of lambda are 2^-11 of the
// state it comes to), which roundings of the state are not.
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
    const float *dec = a.decay + h * kLinDecays;
    const float lam = dec[1], lam1 = dec[kLinTile + 2];
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
            for (int e = 0; e < 4; ++e) S[p][c][e] = fmaf(lam, S[p][c][e], fmaf(lam1, S[p][c][e], v[p] * kk[e]));
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
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    static __device__ __forceinline__ s16x4 tr(const bf16_t *p) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)(const __attribute__((address_space(3))) void *)p);
    }
    // Four tokens of two tiles for column n: lane (n, g) hands in the address of
    // columns 4 (n % 4) .. + 3 (wherever those lie) of token 4 g + n / 4 and
    // receives column n of tokens 4 g .. + 3.
    // p(row, column): where an element of the token array lies
    template <class P>
    static __device__ __forceinline__ Frag cols(P &&p, int t0, int g, int n, int col4, int) {
        const s16x4 x = tr(p(t0 + 4 * g + (n >> 2), col4)), y = tr(p(t0 + 16 + 4 * g + (n >> 2), col4));
        return __builtin_bit_cast(uint4, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
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
    // is some element not finite?
    template <int N>
    static __device__ __forceinline__ bool bad(const Frag (&f)[N]) {
        typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
        u16x2 m = {0, 0};
#pragma unroll
        for (int i = 0; i < N; ++i)
            for (const uint32_t w : {f[i].x, f[i].y, f[i].z, f[i].w})
                m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu));
        return m[0] >= 0x7F80 || m[1] >= 0x7F80;
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
    // the lane's own column, token by token
    template <class P>
    static __device__ __forceinline__ Frag cols(P &&p, int t0, int g, int, int, int col) {
        Frag f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f.x[e] = *p(t0 + 4 * g + e, col);
            f.x[4 + e] = *p(t0 + 16 + 4 * g + e, col);
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
    template <int N>
    static __device__ __forceinline__ bool bad(const Frag (&f)[N]) {
        bool b = false;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) b |= bad_at(f[i], e);
        return b;
    }
    static __device__ __forceinline__ void clear_at(Frag &f, int e) { f.x[e] = 0.f; }
    static __device__ __forceinline__ void store4(float *p, const f32x4_t &x) { *(f32x4_t *)p = x; }
    static __device__ __forceinline__ void store8(float *p, const f32x4_t &x, const f32x4_t &y) {
        *(f32x4_t *)p = x;
        *(f32x4_t *)(p + 4) = y;
    }
};

// (a vector times a scalar keeps four copies of the scalar)
__device__ __forceinline__ void scale4(f32x4_t &x, float f) {
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] *= f;
}

// ---------------------------------------------------------------------------
// chunk form
// ---------------------------------------------------------------------------
// One workgroup per (item, KV head), tiles of B tokens one after the
// other.  With S before the tile, i and j tokens of the tile, n its length:
//   o_i  = scale (lambda^(i+1) S q_i + sum_{j <= i} lambda^(i-j) (k_j . q_i) v_j)
//   S'   = lambda^n S + sum_j (lambda^(n-1-j) v_j) k_j^T
// A wave owns 16 or 32 value dims: their rows of S stay in its accumulators from the
// first tile to the last, and serve as an operand of S q as they lie (two
// accumulators make a fragment's depth).  Scores are formed transposed (keys by
// queries), each wave those of one 16-query tile, and go through LDS to
// the other waves; they too feed the product with V as they lie.  K and V
// are contracted over tokens by transposing reads of LDS.  Decays multiply scores,
// rows of S q, and values in fp32, never as rounded operands.
//
// The tile's products are summed from zero, and S' is formed of them by two
// multiply-adds with two fp32 terms of lambda^n, as in the recurrent form.  With one
// term, and the products summed onto lambda^n S, states were off the same way plan
// after plan: one that nothing is added to by 2e-5 of it after 600 tokens at lambda =
// 1 - 1.1e-6, one of a steady input by 2^-14.5 of it in rms (lambda = 1 - 2^-12, plans of two
// tokens; a sum of the same addend and a number on S's grid is rounded alike every
// time).  An addend that joins before the one rounding of S' leaves 2^-20.5.  It costs
// a multiply-add per element and tile (one prompt of 8192 tokens, 32 heads, 2.6 %).
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
__global__ __launch_bounds__(64 * lin_waves(D, B), lin_waves(D, B) / 2) void k_linear_chunk(LinArgs a) {
    using O = Ops<T>;
    using Frag = typename O::Frag;
    constexpr int NW = lin_waves(D, B), kThreads = 64 * NW;
    constexpr int NT = D / (16 * NW), NS = D / 32, MT = D / 16, JT = B / 16, KS = B / 32;
    constexpr int KW = NW >= 2 * JT ? 1 : KS;  // 32-key slices of scores per wave
    constexpr int kMG = LOCAL && sizeof(T) == 2 ? 4 : 2;  // tiles of S updated side by side
    constexpr int EPV = 16 / (int)sizeof(T);  // elements of a vector
    constexpr int VPR = D / EPV;              // vectors of a row
    constexpr int LD = sizeof(T) == 2 ? D : D + EPV;  // pitch of a row in LDS
    constexpr int CH = B * VPR / kThreads;
    static_assert(B * VPR % kThreads == 0 && JT <= NW && (NT == 1 || NT == 2), "tile shape");
    __shared__ __align__(256) T sk[B * LD], sv[B * LD], sq[LOCAL ? EPV : B * LD];
    __shared__ Frag sp[LOCAL ? 1 : JT * KS * O::kOut * 64];
    __shared__ __align__(16) float pw[B + 1], pr[B];  // lambda^m; lambda^(B - 1 - m)
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (item, KV head, part of its query heads)
    const uint32_t unit = LOCAL ? blockIdx.x : blockIdx.x / (uint32_t)a.parts;
    const int part = LOCAL ? 0 : (int)(blockIdx.x - unit * (uint32_t)a.parts);
    const int it_ = (int)(unit / (uint32_t)a.hkv), h = (int)(unit - (uint32_t)it_ * a.hkv);
    const int row0 = scalar_ld(a.items, kLinItem * it_), ntok = scalar_ld(a.items, kLinItem * it_ + 1);
    const int rec = scalar_ld(a.items, kLinItem * it_ + 2);
    const int nseg = scalar_ld(a.items, kLinItem * it_ + 3) >> 16;
    if (LOCAL && nseg == 1) return;  // the whole workgroup
    const int slot = rec & (kLinFresh - 1);
    const int G = a.hq / a.hkv / a.parts, hq0 = (h * a.parts + part) * G;  // this workgroup's query heads
    const float *const dtab = a.decay + h * kLinDecays;
    for (int m = tid; m <= B; m += kThreads) {
        const float x = dtab[m];
        pw[m] = x;
        if (m < B) pr[B - 1 - m] = x;
    }
    // Token rows in LDS, laid so that sixteen rows' vectors of one column, a
    // fragment's, lie in different banks: bf16 vector x of a row at x ^ its swizzle,
    // fp32 rows a vector apart (their single elements are read by column, too).
    auto at = [](T *base, int row, int col) {
        const int sw = sizeof(T) == 4 ? 0 : VPR == 16 ? row & 15 : (row >> 1) & 7;
        return base + row * LD + ((col / EPV) ^ sw) * EPV + col % EPV;
    };
    // this wave's value dims: lane n of tile nt is dim dv0 + dvn + 4 nt, result row
    // 4 g + r dim dv0 + 8 g + 4 nt + r (one tile: n and 4 g + r)
    const int dv0 = wv * 16 * NT;
    const int dvn = NT == 2 ? 8 * (n >> 2) + (n & 3) : n;
    // this wave's scores: queries of tile wv % JT, key slices wv / JT + kk
    const int pit = wv % JT, pks = wv / JT;
    const int pd = 16 * pit + n - 32 * pks - 4 * g;  // query - key of the lane's first score
    auto key = [](int e) { return 16 * (e / 4) + (e & 3); };  // ... and its others, from there
    // A thread's vectors of the nb tokens from t0 (the last token's in place of those
    // behind it), and into LDS (zeros behind the last token).
    auto load = [&](const void *base, int heads, int head, int t0, int nb, uint4 (&x)[CH]) __attribute__((always_inline)) {
        const T *p = (const T *)base + ((int64_t)(row0 + t0) * heads + head) * D;
        uint32_t t = tid;
        asm volatile("" : "+v"(t));  // (what it makes is not kept over the loop, in registers)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t v = t + c * kThreads;
            x[c] = *(const uint4 *)(p + (min(v / VPR, (uint32_t)nb - 1) * (uint32_t)(heads * D) + v % VPR * EPV));
        }
    };
    auto put = [&](T *dst, uint4 (&x)[CH], int nb) __attribute__((always_inline)) {
        const uint32_t t = tid;
        if (nb < B) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if ((t + c * kThreads) / VPR >= (uint32_t)nb) x[c] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t v = t + c * kThreads;
            *(uint4 *)at(dst, v / VPR, v % VPR * EPV) = x[c];
        }
    };
    uint4 xk[CH], xv[CH], xq[CH];
    {
        const int nb = min(B, ntok);
        load(a.k, a.hkv, h, 0, nb, xk);
        load(a.v, a.hkv, h, 0, nb, xv);
        if constexpr (!LOCAL) load(a.q, a.hq, hq0, 0, nb, xq);
    }
    // (behind the rows, which are needed first)
    // S as the products make it: result row 4 g + r of tile mt = 2 s + t is key dim
    // 32 s + 8 g + 4 t + r, column n the value dim above
    f32x4_t S[MT][NT];
    float *const seg = a.seg + ((int64_t)it_ * a.hkv + h) * D * D;
    {
        const float *src = nseg > 1 ? seg : a.state + (int64_t)slot * a.slot_stride + (int64_t)h * D * D;
        if (LOCAL || (nseg == 1 && (rec & kLinFresh))) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int m = 0; m < MT; ++m) S[m][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        } else {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    S[m][nt] = *(const f32x4_t *)(src + (dv0 + dvn + 4 * nt) * D + 32 * (m / 2) + 8 * g + 4 * (m & 1));
        }
    }
    for (int t0 = 0; t0 < ntok; t0 += B) {
        const int nb = min(B, ntok - t0);
        put(sk, xk, nb);
        put(sv, xv, nb);
        if constexpr (!LOCAL) put(sq, xq, nb);
        __syncthreads();
        // values of this wave's dims, tokens deep
        Frag vf[KS][NT];
        auto values = [&]() __attribute__((always_inline)) {
            int n1 = n, g1 = g;
            asm volatile("" : "+v"(n1), "+v"(g1));  // (what they make is not kept over the loop, in registers)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    vf[ks][nt] = O::cols([&](int r, int c) { return at(sv, r, c); }, 32 * ks, g1, n1,
                                         dv0 + (NT == 2 ? 8 * (n1 & 3) + 4 * nt : 4 * (n1 & 3)),
                                         dv0 + 4 * nt + (NT == 2 ? 8 * (n1 >> 2) + (n1 & 3) : n1));
        };
        values();
        bool any_bad = false;
        // the next tile's keys and values, in flight through this one (nothing to keep
        // where there is none)
        uint4 yk[CH], yv[CH], yq[CH];
        if (t0 + B < ntok) {
            load(a.k, a.hkv, h, t0 + B, min(B, ntok - t0 - B), yk);
            load(a.v, a.hkv, h, t0 + B, min(B, ntok - t0 - B), yv);
        }
        if constexpr (!LOCAL) {
            // a value that is not finite: out of the products with scores, and into
            // the outputs from its token on
            bool bad = false;
            int first[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) first[nt] = B;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) bad |= O::bad(vf[ks]);
            any_bad = __builtin_amdgcn_ballot_w64(bad) != 0;
            if (__builtin_expect(any_bad, 0)) {
                int g1 = g;
                asm volatile("" : "+v"(g1));  // (as above)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (O::bad_at(vf[ks][nt], e)) {
                                O::clear_at(vf[ks][nt], e);
                                first[nt] = min(first[nt], 32 * ks + 4 * g1 + key(e));
                            }
                    first[nt] = min(first[nt], __shfl_xor(first[nt], 16, 64));
                    first[nt] = min(first[nt], __shfl_xor(first[nt], 32, 64));
                }
            }
            for (int gh = 0; gh < G; ++gh) {
                {   // the next head's queries, or the next tile's (or, last, these once more)
                    const bool more = gh + 1 < G;
                    const int tq = !more && t0 + B < ntok ? t0 + B : t0;
                    load(a.q, a.hq, hq0 + (more ? gh + 1 : 0), tq, min(B, ntok - tq), yq);
                }
                // ---- scores, keys by queries
                int pdl = pd, n1 = n;
                asm volatile("" : "+v"(pdl), "+v"(n1));  // (what they make is not kept over the loop, in registers)
#pragma unroll
                for (int kk = 0; kk < KW; ++kk) {
                    const int ks = pks + kk;
                    if (2 * ks > pit || 16 * pit >= nb) break;
                    f32x4_t sc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const Frag qf = O::row(at(sq, 16 * pit + n1, 32 * s + 8 * g));
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            sc[j] = O::mma(O::row(at(sk, 32 * ks + 16 * j + n1, 32 * s + 8 * g)), qf, sc[j]);
                    }
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = pdl >= 32 * kk + key(e) ? sc[e / 4][e & 3] * pw[max(pdl - 32 * kk - key(e), 0)] : 0.f;
                    Frag pf[O::kOut];
                    O::template split<O::kOut>(x, pf);
#pragma unroll
                    for (int p = 0; p < O::kOut; ++p) sp[((pit * KS + ks) * O::kOut + p) * 64 + lane] = pf[p];
                }
                // ---- S q, value dims by queries
                asm volatile("" : "+v"(n1));
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
                        for (int e = 0; e < 8; ++e) {
                            // (split anew for every head: kept, the terms of all of S
                            // would take as many registers as S)
                            asm volatile("" : "+v"(S[2 * s + e / 4][nt][e & 3]));
                            x[e] = S[2 * s + e / 4][nt][e & 3];
                        }
                        O::template split<O::kOut>(x, sf[nt]);
                    }
                    // (each term over all tiles: products in a row that do not wait for
                    // one another)
                    Frag qf[JT];
#pragma unroll
                    for (int it = 0; it < JT; ++it) qf[it] = O::row(at(sq, 16 * it + n1, 32 * s + 8 * g));
#pragma unroll
                    for (int p = 0; p < O::kOut; ++p)
#pragma unroll
                        for (int it = 0; it < JT; ++it)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) o[it][nt] = O::mma(sf[nt][p], qf[it], o[it][nt]);
                }
                __syncthreads();  // every score is there, nobody reads these queries any more
                if (gh + 1 < G) put(sq, yq, nb);
                // ---- plus V times the scores
                T *ob = (T *)a.out + ((int64_t)(row0 + t0) * a.hq + hq0 + gh) * D + dv0;
                int i1 = n + 1;  // (as above)
                asm volatile("" : "+v"(i1));
                const uint32_t oo = (uint32_t)((i1 - 1) * a.hq * D + (NT == 2 ? 8 : 4) * g);
#pragma unroll
                for (int it = 0; it < JT; ++it)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) scale4(o[it][nt], pw[16 * it + i1]);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if (32 * ks >= nb) break;
#pragma unroll
                    for (int p = 0; p < O::kOut; ++p) {
                        Frag pf[JT];
#pragma unroll
                        for (int it = 2 * ks; it < JT; ++it) pf[it] = sp[((it * KS + ks) * O::kOut + p) * 64 + lane];
#pragma unroll
                        for (int it = 2 * ks; it < JT; ++it)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) o[it][nt] = O::mma(vf[ks][nt], pf[it], o[it][nt]);
                    }
                }
#pragma unroll
                for (int it = 0; it < JT; ++it) {
                    if (16 * it >= nb) break;
                    const int i = 16 * it + i1 - 1;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) scale4(o[it][nt], a.scale);
                    if (__builtin_expect(any_bad, 0)) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (i >= __shfl(first[nt], 4 * g + r, 64)) o[it][nt][r] = __builtin_nanf("");
                    }
                    if (i < nb) {
                        T *p = ob + (int64_t)16 * it * a.hq * D + oo;
                        if constexpr (NT == 2)
                            O::store8(p, o[it][0], o[it][NT - 1]);
                        else
                            O::store4(p, o[it][0]);
                    }
                }
                if (gh + 1 < G) __syncthreads();  // the next queries are there, the scores read
            }
        }
        // ---- the state after the tile
        if (LOCAL || (nseg == 1 && part == 0) || t0 + B < ntok) {
            if (__builtin_expect(any_bad, 0)) values();  // as they are
            const float dec = __int_as_float(scalar_ld((const int32_t *)dtab, nb));
            const float dec1 = __int_as_float(scalar_ld((const int32_t *)dtab, kLinTile + 1 + nb));
            int left = nb - 1 - 4 * g;  // tokens after the lane's first
            int n1 = n, g1 = g;
            asm volatile("" : "+v"(left), "+v"(n1), "+v"(g1));  // (as above)
            Frag vw[KS][NT][O::kState];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                float w[8];
                if (nb == B) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) *(f32x4_t *)&w[4 * u] = *(const f32x4_t *)&pr[32 * ks + 16 * u + 4 * g];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = pw[max(left - 32 * ks - key(e), 0)];
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float x[8];
                    O::unpack(vf[ks][nt], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= w[e];
                    O::template split<O::kState>(x, vw[ks][nt]);
                }
            }
#pragma unroll
            for (int m0 = 0; m0 < MT; m0 += kMG) {
                f32x4_t add[kMG][NT];
#pragma unroll
                for (int j = 0; j < kMG; ++j)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) add[j][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    Frag kf[kMG];
#pragma unroll
                    for (int j = 0; j < kMG; ++j) {
                        const int c = 32 * ((m0 + j) / 2) + 4 * (j & 1);
                        kf[j] = O::cols([&](int r, int c) { return at(sk, r, c); }, 32 * ks, g1, n1, c + 8 * (n1 & 3),
                                        c + 8 * (n1 >> 2) + (n1 & 3));
                    }
#pragma unroll
                    for (int p = 0; p < O::kState; ++p)
#pragma unroll
                        for (int j = 0; j < kMG; ++j)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) add[j][nt] = O::mma(kf[j], vw[ks][nt][p], add[j][nt]);
                }
#pragma unroll
                for (int j = 0; j < kMG; ++j)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float x = S[m0 + j][nt][r];
                            const float t = fmaf(dec1, x, add[j][nt][r]);
                            S[m0 + j][nt][r] = fmaf(dec, x, t);
                            // (alive past the sum, which is then formed where S lies and
                            // not in t's place and moved)
                            asm volatile("" ::"v"(t));
                        }
            }
        }
        __syncthreads();  // K, V, Q and scores may be overwritten
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            xk[c] = yk[c];
            xv[c] = yv[c];
            if constexpr (!LOCAL) xq[c] = yq[c];
        }
    }
    if (!LOCAL && (nseg > 1 || part)) return;
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
    // the decay of a segment in two terms; all but the last are as long as the first
    const double l2 = a.log2_decay[h];
    const double df = exp2(l2 * scalar_ld(a.items, kLinItem * it + 1));
    const double dl = exp2(l2 * scalar_ld(a.items, kLinItem * (it + nseg - 1) + 1));
    const float full = (float)df, last = (float)dl, full1 = (float)(df - full), last1 = (float)(dl - last);
    for (int s0 = 0; s0 < nseg; s0 += 8) {
        f32x4_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (s0 + j < nseg) x[j] = *(const f32x4_t *)(p + (s0 + j) * step);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (s0 + j < nseg) {
                *(f32x4_t *)(p + (s0 + j) * step) = cur;
                const bool l = s0 + j == nseg - 1;
                const float d = l ? last : full, d1 = l ? last1 : full1;
#pragma unroll
                for (int r = 0; r < 4; ++r) cur[r] = fmaf(d, cur[r], fmaf(d1, cur[r], x[j][r]));
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
    if (4 * units > INT32_MAX) return hipErrorInvalidValue;
    return by_shape(dtype, a.d, [&](auto dc, auto elt) {
        constexpr int D = decltype(dc)::value;
        using T = decltype(elt);
        auto go = [&](auto gc) {
            constexpr int G = decltype(gc)::value, kMost = D / 32;
            auto sliced = [&](auto sc) {
                constexpr int SL = decltype(sc)::value;
                hipLaunchKernelGGL((k_linear_decode<T, D, G, SL>), dim3((unsigned)(units * SL)), dim3(kLinThreads), 0,
                                   s, a);
            };
            const int sl = linear_slices(units, D, n_cu);
            if (sl == 1) return sliced(std::integral_constant<int, 1>{});
            if (sl == 2 || kMost == 2) return sliced(std::integral_constant<int, 2>{});
            sliced(std::integral_constant<int, kMost>{});
        };
        switch (a.hq / a.hkv) {
            case 1: go(std::integral_constant<int, 1>{}); break;
            case 2: go(std::integral_constant<int, 2>{}); break;
            case 4: go(std::integral_constant<int, 4>{}); break;
            default: go(std::integral_constant<int, 8>{}); break;
        }
    });
}

hipError_t launch_linear_chunk(int dtype, LinArgs a, int max_tok, bool split, int n_cu, hipStream_t s) {
    if (!linear_supported(dtype, a.d, a.hq / a.hkv) || a.n_items < 1 || (split && !a.seg)) return hipErrorInvalidValue;
    const int64_t units = (int64_t)a.n_items * a.hkv;
    if (units > (split ? 65535 : INT32_MAX)) return hipErrorInvalidValue;  // (the scan's second grid dimension)
    const int tile = linear_tile(dtype, max_tok);
    a.parts = linear_parts(units, a.hq / a.hkv, tile, n_cu);
    return by_shape(dtype, a.d, [&](auto dc, auto elt) {
        constexpr int D = decltype(dc)::value;
        using T = decltype(elt);
        auto go = [&](auto bc) {
            constexpr int B = decltype(bc)::value;
            const dim3 grid((unsigned)units), block(64 * lin_waves(D, B));
            const dim3 grid2((unsigned)(units * a.parts));
            if (split) {
                hipLaunchKernelGGL((k_linear_chunk<T, D, B, true>), grid, block, 0, s, a);
                hipLaunchKernelGGL((k_linear_scan<D>), dim3(D * D / 1024, (unsigned)units), dim3(256), 0, s, a);
            }
            hipLaunchKernelGGL((k_linear_chunk<T, D, B, false>), grid2, block, 0, s, a);
        };
        if constexpr (sizeof(T) == 2) {
            if (tile == 64) return go(std::integral_constant<int, 64>{});
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
