// Linear attention with a decay for each head, chunked on matrix instructions.
//
//   S_t = e^{g_h} S_{t-1} + k_t v_t^T          y_t = S_t^T q_t          (per batch and head)
//
// One kernel serves the forward and the three gradients of the backward, because with
//   run(Q, K, V)_t = sum_{s <= t} e^{g (t-s)} (Q_t . K_s) V_s  (+ what a start state adds)
// they are y = run(q, k, v), dq = run(dy, v, k), and, walking the tokens backwards,
// dk = run(v, dy, q) and dv = run(k, q, dy).  In a chunk of kLC = 32 tokens (positions i, j):
//   Y  = (Q K^T o D) V + diag(e^{g (i+o)}) Q R            D_ij = e^{g (i-j)} for j <= i, else 0
//   R <- e^{g n} R + K^T diag(e^{g (n-j-o)}) V            n: the chunk's tokens
// R is the state before the chunk (o = 1), or, walking backwards, that state already decayed once
// (o = 0): the gradient of the final state enters undecayed, and the last R is the gradient of the
// start state.  All exponents are at least 0, so no factor exceeds 1 for g <= 0; e^{-inf * 0} is 1.  What is
// formed on the way are products q . k and q . R of undecayed values: where those leave fp32's range, so may
// the outputs that decay away from them, and nothing else does.
//
// A wave owns CW value columns of one sequence (or segment of one) and their state, in registers, or half of
// the state's rows, and then, the sums over the rows exchanged, the outputs of half of the chunk's tokens;
// the waves of a workgroup share the chunk's Q, K and V in LDS, loaded a chunk ahead.  Accumulators are
// operands as they stand: over tokens, lane group g holds {4g .. 4g+3} u {16+4g .. 16+4g+3} of a 32-deep
// product, and the 32 rows of two tiles of the state are dealt so that g holds 8g .. 8g+7 (slot_of),
// which a lane reads of a row of Q or K with one access.  Q's fragments serve Q K^T and Q R, V's
// (Q K^T) V and K^T V.  Rows are stored in 16-byte pieces, piece p of row r at p ^ f(r), which
// spreads both the reads along rows and those across rows over the LDS banks.
//
// bf16: v_mfma_f32_16x16x32_bf16.  q, k, v are exact operands; fp32 factors (the masked scores, the
// state, the decayed values) are split into three bf16 parts, all of their 24 bits, so that outputs are
// fp32 sums rounded once.  (Two parts of scores and state, 16 bits, take 11% off a training step, but round
// one output in 500 the other way, and what cancels against a large state keeps their error.)
// fp32: v_mfma_f32_16x16x4_f32.
#include <atomic>

#include "kla_buf.hpp"
#include "kla_internal.hpp"
#include "kla_mfma.hpp"

namespace kla {
namespace {

constexpr int kLC = 32;   // tokens per chunk

__host__ __device__ constexpr int ilog2(int x) { return x <= 1 ? 0 : 1 + ilog2(x / 2); }

// A tile of rows of W elements in LDS.
template <typename E, int W>
struct Tile {
    static constexpr int NC = W * (int)sizeof(E) / 16;   // 16-byte pieces per row
    static constexpr int UNITS = kLC * NC / 64;          // wave loads per tile
    static constexpr int BYTES = kLC * NC * 16;
    // byte offset of piece c of row r: rows are 16 NC bytes, and 16 rows read at one piece, or 4 at
    // two, touch different 16-byte columns of the banks
    __device__ static int piece(int r, int c) {
        constexpr int SH = NC >= 16 ? 0 : ilog2(16 / NC);
        constexpr int MASK = NC >= 16 ? 15 : NC - 1;
        return r * NC * 16 + ((c ^ ((r >> SH) & MASK)) << 4);
    }
    __device__ static int piece_at(int r, int place) { return piece(r, place) / 16 - r * NC; }   // its own inverse
    __device__ static int at(int r, int col) {
        constexpr int PER = 16 / (int)sizeof(E);
        return piece(r, col / PER) + (col % PER) * (int)sizeof(E);
    }
};

// Slot n of the state's row (tile rt, row m of 16): 32 slots over two tiles, 8g + 4 (rt & 1) + rr at row
// 4g + rr; a width of 16 is one tile.
template <int N>
__device__ __forceinline__ int slot_of(int rt, int m) {
    return N == 16 ? m : 32 * (rt >> 1) + 8 * (m >> 2) + 4 * (rt & 1) + (m & 3);
}

// Operands of a 32-deep product: eight values per lane.
template <typename E>
struct Op;

template <>
struct Op<uint16_t> {
    bf16x8 x;
    template <int W>
    __device__ static Op row(const unsigned char* t, int r, int ks, int g4) {   // slots of row r for step ks
        using TL = Tile<uint16_t, W>;
        if constexpr (W == 16) {
            const uint2 a = *reinterpret_cast<const uint2*>(t + TL::at(r, 4 * g4));
            return {__builtin_bit_cast(bf16x8, uint4{a.x, a.y, 0u, 0u})};
        } else {
            return {__builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(t + TL::piece(r, 4 * ks + g4)))};
        }
    }
    template <int W>
    __device__ static Op slots(const unsigned char* t, int rt, int g4, int l16) {   // down the slots of state tile rt
        return W == 16 ? tr<W>(t, 4 * (l16 & 3), g4, l16) : tr<W>(t, 32 * (rt >> 1) + 8 * (l16 & 3) + 4 * (rt & 1), g4, l16);
    }
    template <int W>
    __device__ static Op col(const unsigned char* t, int col0, int g4, int l16) {   // down column col0 + l16
        return tr<W>(t, col0 + 4 * (l16 & 3), g4, l16);
    }
    // lane i of 16 gets, over the tokens, column i % 4 of the four that lane i / 4 addresses at c
    template <int W>
    __device__ static Op tr(const unsigned char* t, int c, int g4, int l16) {
        using TL = Tile<uint16_t, W>;
        const int r = 4 * g4 + (l16 >> 2);
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)(t + TL::at(r, c)));
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)(t + TL::at(r + 16, c)));
        return {__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
    }
};

template <>
struct Op<float> {
    float x[8];
    template <int W>
    __device__ static Op row(const unsigned char* t, int r, int ks, int g4) {
        using TL = Tile<float, W>;
        if constexpr (W == 16) {
            const float4 a = *reinterpret_cast<const float4*>(t + TL::piece(r, g4));
            return {{a.x, a.y, a.z, a.w, 0.f, 0.f, 0.f, 0.f}};
        } else {
            const float4 a = *reinterpret_cast<const float4*>(t + TL::piece(r, 8 * ks + 2 * g4));
            const float4 b = *reinterpret_cast<const float4*>(t + TL::piece(r, 8 * ks + 2 * g4 + 1));
            return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
        }
    }
    template <int W>
    __device__ static Op slots(const unsigned char* t, int rt, int g4, int l16) {
        return col<W>(t, slot_of<W>(rt, l16) - l16, g4, l16);
    }
    template <int W>
    __device__ static Op col(const unsigned char* t, int col0, int g4, int l16) {
        Op o;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            o.x[e] = *reinterpret_cast<const float*>(t + Tile<float, W>::at(4 * g4 + (e & 3) + (e & 4) * 4, col0 + l16));
        return o;
    }
};

// Accumulators (rows 4 g4 + rr of two 16-row tiles) as operands.  bf16: three parts, each the upper half of what
// the ones before leave, which is exact: 24 bits.  What a part leaves is formed by the matrix cores, tile - pick
// part with pick[u] minus the unit that takes tile u's rows out of the operand (one product a sum); on the vector
// units the same takes four instructions for each pair of elements (backward of B = 8, T = 2048, H = 16, 128 wide:
// 241 us, with both on the vector units 244, of B = 4 145 and 152).
template <typename E>
struct Acc;
template <>
struct Acc<uint16_t> {
    static constexpr int BYTES = 24;   // of a lane of one tile
    bf16x8 p[3];
    struct Pick {
        bf16x8 of[2];
        __device__ Pick(int g4, int l16) {
            uint32_t w[2][4];   // two elements a word
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = 2 * i - 4 * u;   // element 2 i is row 4 g4 + e of tile u
                    w[u][i] = e >= 0 && e < 4 ? (4 * g4 + e == l16 ? 0xbf80u : 4 * g4 + e + 1 == l16 ? 0xbf800000u : 0u) : 0u;
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) of[u] = __builtin_bit_cast(bf16x8, uint4{w[u][0], w[u][1], w[u][2], w[u][3]});
        }
    };
    __device__ Acc() {}
    template <bool HALF>
    __device__ static bf16x8 upper(const f32x4& a, const f32x4& b) {
        auto two = [](float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u); };
        return __builtin_bit_cast(bf16x8, uint4{two(a[0], a[1]), two(a[2], a[3]), HALF ? 0u : two(b[0], b[1]),
                                                HALF ? 0u : two(b[2], b[3])});
    }
    template <bool HALF = false>   // HALF: b is zero
    __device__ static Acc from(f32x4 a, f32x4 b, const Pick& pick) {
        Acc o;
#pragma unroll
        for (int s = 0; s < 3; ++s) {
            o.p[s] = upper<HALF>(a, b);
            if (s == 2) break;
            a = mfma_bf16(pick.of[0], o.p[s], a);
            if (!HALF) b = mfma_bf16(pick.of[1], o.p[s], b);
        }
        return o;
    }
    // One tile in LDS, at: the lane's place, and the operands of (tile, nothing) or two tiles from there.
    __device__ static void put(const f32x4& a, const Pick& pick, uint2* at) {
        const Acc o = from<true>(a, zero4(), pick);
#pragma unroll
        for (int s = 0; s < 3; ++s) {
            const uint4 u = __builtin_bit_cast(uint4, o.p[s]);
            at[64 * s] = uint2{u.x, u.y};
        }
    }
    __device__ static Acc get(const uint2* a, const uint2* b) {
        Acc o;
#pragma unroll
        for (int s = 0; s < 3; ++s) {
            const uint2 x = a[64 * s], y = b ? b[64 * s] : uint2{0u, 0u};
            o.p[s] = __builtin_bit_cast(bf16x8, uint4{x.x, x.y, y.x, y.y});
        }
        return o;
    }
};
template <>
struct Acc<float> {
    static constexpr int BYTES = 16;
    float x[8];
    struct Pick {
        __device__ Pick(int, int) {}
    };
    __device__ Acc() {}
    template <bool HALF = false>
    __device__ static Acc from(const f32x4& a, const f32x4& b, const Pick&) {
        Acc o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o.x[e] = a[e];
            o.x[4 + e] = b[e];
        }
        return o;
    }
    __device__ static void put(const f32x4& a, const Pick&, uint2* at) {
        const uint4 u = __builtin_bit_cast(uint4, a);
        at[0] = uint2{u.x, u.y};
        at[64] = uint2{u.z, u.w};
    }
    __device__ static Acc get(const uint2* a, const uint2* b) {
        const uint2 none{0u, 0u}, x = a[0], y = a[64], z = b ? b[0] : none, w = b ? b[64] : none;
        return from(__builtin_bit_cast(f32x4, uint4{x.x, x.y, y.x, y.y}), __builtin_bit_cast(f32x4, uint4{z.x, z.y, w.x, w.y}),
                    Pick(0, 0));
    }
};

// v scaled by w, as an operand of the state's update.
template <typename E>
struct Scaled;
template <>
struct Scaled<uint16_t> {
    bf16x8 p[3];   // 24 bits
    __device__ Scaled() {}
    __device__ Scaled(const Op<uint16_t>& v, const float* w) {
        const uint4 u = __builtin_bit_cast(uint4, v.x);
        const uint32_t in[4] = {u.x, u.y, u.z, u.w};
        uint32_t o[3][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float a = __uint_as_float(in[e] << 16) * w[2 * e], b = __uint_as_float(in[e] & 0xffff0000u) * w[2 * e + 1];
#pragma unroll
            for (int s = 0; s < 3; ++s) {
                o[s][e] = cvt_pk_bf16(a, b);
                a -= __uint_as_float(o[s][e] << 16);
                b -= __uint_as_float(o[s][e] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int s = 0; s < 3; ++s) p[s] = __builtin_bit_cast(bf16x8, uint4{o[s][0], o[s][1], o[s][2], o[s][3]});
    }
};
template <>
struct Scaled<float> {
    float x[8];
    __device__ Scaled() {}
    __device__ Scaled(const Op<float>& v, const float* w) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v.x[e] * w[e];
    }
};

__device__ __forceinline__ f32x4 mfma_f32(float a, float b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// c += a b; STEPS: values per lane that are not zero by construction (4 or 8)
template <int STEPS = 8>
__device__ __forceinline__ f32x4 mma(const Op<uint16_t>& a, const Op<uint16_t>& b, f32x4 c) {
    return mfma_bf16(a.x, b.x, c);
}
template <int STEPS = 8>
__device__ __forceinline__ f32x4 mma(const Op<uint16_t>& a, const Acc<uint16_t>& b, f32x4 c) {
#pragma unroll
    for (int s = 2; s >= 0; --s) c = mfma_bf16(a.x, b.p[s], c);
    return c;
}
// c[i][j] += a[i] b[j], part after part, so that no product waits for the one before it
template <int STEPS, int NI>
__device__ __forceinline__ void mma_each(const Acc<uint16_t> (&a)[NI], const Op<uint16_t> (&b)[2], f32x4 (&c)[NI][2]) {
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) c[i][j] = mfma_bf16(a[i].p[s], b[j].x, c[i][j]);
}
template <int NI, int NJ>
__device__ __forceinline__ void mma_each(const Op<uint16_t> (&a)[NI], const Scaled<uint16_t> (&b)[NJ], f32x4 (*c)[NJ]) {
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) c[i][j] = mfma_bf16(a[i].x, b[j].p[s], c[i][j]);
}
template <int STEPS>
__device__ __forceinline__ f32x4 mma_f32(const float* a, const float* b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < STEPS; ++e) c = mfma_f32(a[e], b[e], c);
    return c;
}
template <int STEPS = 8>
__device__ __forceinline__ f32x4 mma(const Op<float>& a, const Op<float>& b, f32x4 c) {
    return mma_f32<STEPS>(a.x, b.x, c);
}
template <int STEPS = 8>
__device__ __forceinline__ f32x4 mma(const Op<float>& a, const Acc<float>& b, f32x4 c) {
    return mma_f32<STEPS>(a.x, b.x, c);
}
template <int STEPS, int NI>
__device__ __forceinline__ void mma_each(const Acc<float> (&a)[NI], const Op<float> (&b)[2], f32x4 (&c)[NI][2]) {
#pragma unroll
    for (int e = 0; e < STEPS; ++e)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) c[i][j] = mfma_f32(a[i].x[e], b[j].x[e], c[i][j]);
}
template <int NI, int NJ>
__device__ __forceinline__ void mma_each(const Op<float> (&a)[NI], const Scaled<float> (&b)[NJ], f32x4 (*c)[NJ]) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) c[i][j] = mfma_f32(a[i].x[e], b[j].x[e], c[i][j]);
}

// Four output values of one token.
__device__ __forceinline__ void store4(uint16_t, const f32x4& y, rsrc_t r, uint32_t voff) {
    buf_st64(uint2{cvt_pk_bf16(y[0], y[1]), cvt_pk_bf16(y[2], y[3])}, r, voff);
}
__device__ __forceinline__ void store4(float, const f32x4& y, rsrc_t r, uint32_t voff) {
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, y), r, voff, 0, 0);
}

// e^{g n}, 1 for n = 0 whatever g is.  The exponent is formed in fp64, where g n keeps its digits, and its
// fraction is an argument of at most 1/2 of the hardware's 2^x (1 ulp): every workgroup begins with these.
__device__ __forceinline__ float decay_pow(float g, int n) {
    double x = (double)g * (double)n * 1.4426950408889634;
    x = x < -300.0 ? -300.0 : x > 300.0 ? 300.0 : x;   // NaN stays
    const double i = rint(x);
    return n == 0 ? 1.f : ldexpf(__builtin_amdgcn_exp2f((float)(x - i)), x == x ? (int)i : 0);
}

__device__ __forceinline__ float lds_val(uint16_t, const unsigned char* p) {
    return bf16_to_f32(*reinterpret_cast<const uint16_t*>(p));
}
__device__ __forceinline__ float lds_val(float, const unsigned char* p) { return *reinterpret_cast<const float*>(p); }

// (Q K^T o D) V of a chunk again, where it was not finite: the mask and the matrix instruction multiply
// later tokens' scores and values by zero, and what is not finite must not reach the tokens before it.
template <typename E, int N, int DT>
__device__ __forceinline__ f32x4 masked_sums(const unsigned char* sQ, const unsigned char* sK, const unsigned char* sV,
                                             const float* pw, int col0, int i, int g4) {
    f32x4 y = zero4();
#pragma unroll 1
    for (int j = 0; j <= i; ++j) {
        float s = 0.f;
#pragma unroll 1
        for (int n = 0; n < N; ++n)
            s += lds_val(E(), sQ + Tile<E, N>::at(i, n)) * lds_val(E(), sK + Tile<E, N>::at(j, n));
        s *= pw[i - j];
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) y[rr] += s * lds_val(E(), sV + Tile<E, DT>::at(j, col0 + 4 * g4 + rr));
    }
    return y;
}

// One pass: Q, K [B, T, H, N] and V, Y [B, T, H, D].
struct LinJob {
    const void *q, *k, *v;
    const float* start;   // start states, or none (0): by sequence, or with ns > 1 by sequence and segment
    void* y;
    float* end;           // final states, or none; NOY: the segments' own, by sequence and segment
    int rev;              // tokens from the last to the first
    int flip;             // bit 0: the start states, bit 1: the final ones are stored [D][N] instead of [N][D]
};

struct LinArgs {
    LinJob job[3];        // passes run side by side
    const float* g;       // [H]
    const int* len;       // [B] or none
    int B, T, H, jobs;
    int ns, lc, run;      // segments per sequence, chunks in one, segments run
};

// Tokens of sequence b.
__device__ __forceinline__ int seq_len(const LinArgs& a, int b) {
    return a.len ? min(max(a.len[b], 0), a.T) : a.T;
}

// A workgroup takes DT of the D columns, a wave CW of them and one of RS shares of the state's rows.  Where the
// rows of Q and K are long and the waves that compute (NCW RS) few, others help with the loads.  64 columns in
// waves of 16 with all rows take 133 registers and 45 KiB of LDS, so three workgroups of 128-wide bf16 passes
// share a CU (B = 8, T = 2048, H = 16: forward 108 us and backward 243, against 225 and 316 with 128 columns
// in waves of 32, whose scores are formed half as often but which one wave a SIMD has to hide).  The states' pass
// forms no scores: all columns.
template <typename E, int N, int D, bool NOY, int RS>
struct LinCfg {
    static constexpr int CW = NOY && D == 128 ? 32 : 16, DT = NOY || D <= 64 ? D : 64, NTILE = D / DT, NCW = DT / CW;
    static constexpr int ROW = N * (int)sizeof(E), LW = ROW >= 256 ? 4 : ROW >= 128 ? 2 : 1,
                         NW = NCW * RS > LW ? NCW * RS : LW;
    static constexpr int BUF = 2 * Tile<E, N>::BYTES + Tile<E, DT>::BYTES, SCORE = 64 * Acc<E>::BYTES,
                         LDS = 2 * BUF + 2 * kLC * (int)sizeof(float) + 3 * SCORE + (RS > 1 ? NCW * RS * (CW / 16) * 1024 : 0);
    // waves per SIMD: of fp32 rows of 128 slots, LDS holds one workgroup a CU
    static constexpr int OCC = sizeof(E) == 4 && N == 128 ? 2 : RS > 1 ? 4 : 3;
};

// Workgroup `block` of `jobs` passes from job[j0] on; NW: its waves.
template <typename E, int N, int D, bool NOY, int RS, int NW>
__device__ __forceinline__ void linattn_pass(const LinArgs& a, int block, int j0, int jobs) {
    using Cfg = LinCfg<E, N, D, NOY, RS>;
    constexpr int CW = Cfg::CW, NDT = CW / 16;
    // a wave's tiles of state rows, steps over them, tiles of tokens
    constexpr int NRT = N / 16 / RS, KS = (N + 31) / 32 / RS, NIT = 2 / RS;
    constexpr int ES = (int)sizeof(E);
    using TQ = Tile<E, N>;
    constexpr int DT = Cfg::DT, NTILE = Cfg::NTILE;
    using TV = Tile<E, DT>;
    constexpr int UQ = NOY ? 0 : TQ::UNITS, UK = TQ::UNITS, UNITS = UQ + UK + TV::UNITS;
    constexpr int NL = (UNITS + NW - 1) / NW;   // a wave's loads per chunk
    constexpr int NST = NOY ? 0 : NIT * NDT;      // and stores, of one that computes
    constexpr int BUF = Cfg::BUF;
    extern __shared__ __align__(16) unsigned char smem[];
    float* pw = reinterpret_cast<float*>(smem + 2 * BUF);   // e^{g n}
    constexpr int SCORE = Cfg::SCORE / 8;
    uint2* scores = reinterpret_cast<uint2*>(pw + 2 * kLC);   // of the chunk, three tiles
    f32x4* part = reinterpret_cast<f32x4*>(scores + 3 * SCORE);  // of Q R, for the wave with the other rows

    int vi, ji, tile;   // the passes and tiles of one sequence on one XCD: they read the same rows
    {
        const int i = block, nv = a.B * a.H * a.run, each = jobs * NTILE;
        const int slot = nv % 8 == 0 ? i / 8 : i;
        vi = nv % 8 == 0 ? slot / each * 8 + i % 8 : slot / each;
        ji = j0 + slot % each / NTILE;
        tile = slot % NTILE;
    }
    const LinJob job = a.job[ji];
    const bool rev = job.rev;
    const int O = rev ? 0 : 1;
    const int bh = vi / a.run, seg = vi % a.run, b = bh / a.H, h = bh % a.H, H = a.H;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g4 = lane >> 4;
    const float g = a.g[h];
    const int Tb = __builtin_amdgcn_readfirstlane(seq_len(a, b));
    const int u0 = seg * a.lc * kLC, nu = min(max(Tb - u0, 0), a.lc * kLC);   // this segment's tokens, in walk order
    const int nchunk = (nu + kLC - 1) / kLC;
    const int sh = RS == 1 ? 0 : wave / Cfg::NCW % 2;   // its share of the state's rows, and of the outputs' tokens
    const int dl0 = (RS == 1 ? wave : wave % Cfg::NCW) * CW, dm0 = tile * DT + dl0;   // first column, in the tile and of all
    const bool works = NW == Cfg::NCW * RS || wave < Cfg::NCW * RS;

    if (threadIdx.x < 2 * kLC) pw[threadIdx.x] = decay_pow(g, threadIdx.x);

    // Chunk c has n = min(nu - 32 c, 32) tokens.  Row r of a full one lies at r, walking backwards at 31 - r,
    // rows after a place that moves on from chunk to chunk (at); a last one of fewer tokens starts `miss`
    // rows later there when walking backwards.  Rows past the chunk's tokens fall outside the buffer: behind
    // its end, or, walking backwards, before its start and so past 2^31.
    const uint32_t sn = (uint32_t)(H * N * ES), sd = (uint32_t)(H * D * ES);   // bytes from token to token
    auto row_off = [&](int r, uint32_t stride) { return (uint32_t)(rev ? kLC - 1 - r : r) * stride; };
    const size_t t0 = (size_t)b * a.T + (rev ? Tb - u0 - kLC : u0);   // may wrap for a short sequence; used with n rows
    auto at = [&](const void* p, uint32_t stride, int w) {
        return reinterpret_cast<uintptr_t>(p) + t0 * stride + (uint32_t)(h * w * ES);
    };
    auto tokens = [&](int c) { return min(nu - c * kLC, kLC); };
    // cols: bytes of a row that are read or written
    auto rsrc_of = [&](uintptr_t p, uint32_t stride, int n, uint32_t cols) {
        const uint32_t miss = (uint32_t)(kLC - n) * stride;
        return make_rsrc(reinterpret_cast<const void*>(p + (rev ? miss : 0u)), (kLC - 1) * stride + cols - miss);
    };
    auto words_of = [&](uintptr_t p, uint32_t stride, int n, uint32_t cols) {   // the same, for load_lds
        const uint32_t miss = (uint32_t)(kLC - n) * stride;
        const uintptr_t q = p + (rev ? miss : 0u);
        return words_t{(uint32_t)q, (uint32_t)(q >> 32) & 0xffffu, (kLC - 1) * stride + cols - miss, 0x00020000u};
    };
    auto shift_of = [&](uint32_t stride, int n) { return rev ? (uint32_t)(kLC - n) * stride : 0u; };
    uintptr_t pq = at(job.q, sn, N), pk = at(job.k, sn, N), pv = at(job.v, sd, D) + tile * DT * ES, py = at(job.y, sd, D) + dm0 * ES;
    const intptr_t step_n = rev ? -(intptr_t)(kLC * (size_t)sn) : (intptr_t)(kLC * (size_t)sn);
    const intptr_t step_d = rev ? -(intptr_t)(kLC * (size_t)sd) : (intptr_t)(kLC * (size_t)sd);

    // Wave load i: 64 pieces of Q, K or V; which, is known at compile time where the tiles are whole rounds
    // of the workgroup's loads.
    constexpr bool EVEN = UQ % NW == 0 && UK % NW == 0, FULL = UNITS % NW == 0;
    auto part_of = [&](int i) { return EVEN ? i * NW : i * NW + wave; };
    uint32_t goff[NL];   // in a full chunk; the piece that belongs at the lane's place in the tile
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int u = i * NW + wave;
        if (part_of(i) < UQ + UK) {
            const int x = (part_of(i) < UQ ? u : u - UQ) * 64 + lane;
            goff[i] = row_off(x / TQ::NC, sn) + (uint32_t)TQ::piece_at(x / TQ::NC, x % TQ::NC) * 16;
        } else {
            const int x = (u - UQ - UK) * 64 + lane;
            goff[i] = row_off(x / TV::NC, sd) + (uint32_t)TV::piece_at(x / TV::NC, x % TV::NC) * 16;
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    int into = 0;                // the buffer of the next load
    auto load = [&](int c) {     // chunks in order, each once
        const int n = tokens(c);
        const words_t rk = words_of(pk, sn, n, N * ES), rq = NOY ? rk : words_of(pq, sn, n, N * ES);
        const words_t rv = words_of(pv, sd, n, DT * ES);
        const uint32_t hn = shift_of(sn, n), hd = shift_of(sd, n);
        pq += step_n;
        pk += step_n;
        pv += step_d;
        const uint32_t dst = lds0 + (NOY ? TQ::BYTES : 0) + into * BUF + wave * 1024;   // tiles follow each other
        into ^= 1;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            if (part_of(i) < UQ)
                load_lds(rq, dst + i * NW * 1024, goff[i] - hn);
            else if (part_of(i) < UQ + UK)
                load_lds(rk, dst + i * NW * 1024, goff[i] - hn);
            else if (FULL || i * NW + wave < UNITS)
                load_lds(rv, dst + i * NW * 1024, goff[i] - hd);
        }
    };

    // state R[n, d], n = slot_of(sh NRT + rt, 4 g4 + rr), d = dm0 + 16 dt + l16
    const size_t srow = (size_t)bh * a.ns + seg;
    f32x4 R[NRT][NDT];
    auto state_at = [&](int rt, int dt, int rr, bool flip) {
        const int n = slot_of<N>(sh * NRT + rt, 4 * g4 + rr), d = dm0 + 16 * dt + l16;
        return flip ? d * N + n : n * D + d;
    };
    if (nchunk > 0) load(0);
    {
        const float* s0 = NOY || !job.start || !works ? nullptr : job.start + srow * (size_t)(N * D);
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) R[rt][dt][rr] = s0 ? s0[state_at(rt, dt, rr, job.flip & 1)] : 0.f;
    }
    __syncthreads();   // pw
    float dia[4], off[4], rd[NIT], kw[8];
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
        const int lag = l16 - 4 * g4 - rr;
        dia[rr] = lag >= 0 ? pw[max(lag, 0)] : 0.f;
        off[rr] = pw[16 + lag];
    }
    uint32_t yoff[NIT];
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
        const int i = 16 * (sh + it) + l16;
        rd[it] = pw[i + O];
        yoff[it] = row_off(i, sd) + (uint32_t)(4 * g4 * ES);
    }
    auto weights = [&](int n) {   // of the state's update; values past the chunk's tokens are zero
#pragma unroll
        for (int e = 0; e < 8; ++e) kw[e] = pw[max(n - O - (4 * g4 + (e & 3) + (e & 4) * 4), 0)];
    };
    const typename Acc<E>::Pick pick(g4, l16);
    weights(kLC);
    // The state is rho R, so that its decay is one product a chunk and not one an element.  rho falls from kRho
    // to 1 and is then set back: R is the state or up to kRho times smaller, so it is finite where the state is;
    // what it loses are bits of states within 2^8 of fp32's smallest.  Uniform: the branches on them are the wave's.
    auto uniform = [](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); };
    constexpr float kRho = 0x1p8f;
    float gn = uniform(pw[kLC]), rho = nchunk > 0 ? kRho : 1.f;
    auto scale = [&](float f) {
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) R[rt][dt][rr] *= f;
    };
    if (job.start) scale(1.f / rho);
    // the start state has arrived: without this the loop would wait at the state's first use for every
    // access in flight, in each round
    wait_vm_all();

    int from = 0;   // this chunk's buffer
    for (int c = 0; c < nchunk; ++c) {
        const int n = tokens(c);
        // this chunk's loads have ended, of this wave and behind the barrier of all: younger are the last
        // chunk's stores
        if (works) wait_vm_le<NST>();
        else wait_vm_le<0>();
        __syncthreads();
        if (c + 1 < nchunk) load(c + 1);   // into the last chunk's buffer
        const unsigned char* buf = smem + from * BUF;
        from ^= 1;
        const unsigned char *sQ = buf, *sK = buf + TQ::BYTES, *sV = buf + 2 * TQ::BYTES;
        if (n < kLC) {
            weights(n);
            gn = uniform(pw[n]);
        }
        constexpr int ST = N == 16 ? 4 : 8;
        if constexpr (!NOY) {
            // the waves share the scores S^T[j, i] = K_j . Q_i, masked: tiles (jt, it) = (0,0), (0,1), (1,1)
            for (int t = wave; t < 3; t += NW) {
                f32x4 s = zero4();
#pragma unroll
                for (int ks = 0; ks < KS * RS; ++ks)
                    s = mma<ST>(Op<E>::template row<N>(sK, (t == 2 ? 16 : 0) + l16, ks, g4),
                                Op<E>::template row<N>(sQ, (t > 0 ? 16 : 0) + l16, ks, g4), s);
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) s[rr] *= t == 1 ? off[rr] : dia[rr];
                Acc<E>::put(s, pick, scores + t * SCORE + lane);
            }
        }
        Op<E> vf[NDT];
        f32x4 y[NDT][2];
        const float was = rho;
        if (works) {
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) vf[dt] = Op<E>::template col<DT>(sV, dl0 + 16 * dt, g4, l16);
            if constexpr (!NOY) {   // Y^T[d, i] from the state
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) y[dt][0] = y[dt][1] = zero4();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const Op<E> qs[2] = {Op<E>::template row<N>(sQ, l16, sh * KS + ks, g4),
                                         Op<E>::template row<N>(sQ, 16 + l16, sh * KS + ks, g4)};
                    Acc<E> r[NDT];
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt)
                        r[dt] = Acc<E>::template from<N == 16>(R[2 * ks][dt], N == 16 ? zero4() : R[N == 16 ? 0 : 2 * ks + 1][dt], pick);
                    mma_each<ST>(r, qs, y);
                }
                if constexpr (RS > 1)
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt) {
                        part[(wave * NDT + dt) * 64 + lane] = sh ? y[dt][0] : y[dt][1];
                        if (sh) y[dt][0] = y[dt][1];
                    }
            }

            // R <- e^{g n} R + K^T (w V)
            float w[8];
            rho *= gn;
            if (!(rho >= 1.f)) {
                scale(rho * (1.f / kRho));
                rho = kRho;
            }
            const float inv = 1.f / rho;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = kw[e] * inv;
            Scaled<E> vs[NDT];
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) vs[dt] = Scaled<E>(vf[dt], w);
            constexpr int RT = NRT >= 2 ? 2 : 1;
#pragma unroll
            for (int rt = 0; rt < NRT; rt += RT) {
                Op<E> kt[RT];
#pragma unroll
                for (int i = 0; i < RT; ++i) kt[i] = Op<E>::template slots<N>(sK, sh * NRT + rt + i, g4, l16);
                mma_each<RT, NDT>(kt, vs, R + rt);
            }
        }
        if constexpr (!NOY) {
            __syncthreads();   // the scores are there
            if (works) {
                f32x4 in[NDT][NIT];
                float sum = 0.f;   // not finite where a value is not
#pragma unroll
                for (int it = 0; it < NIT; ++it) {
                    const int at = RS > 1 ? sh : it;   // one tile of earlier tokens, or two
                    const Acc<E> p = at ? Acc<E>::get(scores + SCORE + lane, scores + 2 * SCORE + lane) : Acc<E>::get(scores + lane, nullptr);
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt) {
                        in[dt][it] = RS > 1 || it ? mma<8>(vf[dt], p, zero4()) : mma<4>(vf[dt], p, zero4());
#pragma unroll
                        for (int rr = 0; rr < 4; ++rr) sum += in[dt][it][rr];
                    }
                }
                if (__any(!(fabsf(sum) <= 3.4e38f)))
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                        for (int it = 0; it < NIT; ++it)
                            in[dt][it] = masked_sums<E, N, DT>(sQ, sK, sV, pw, dl0 + 16 * dt, 16 * (sh + it) + l16, g4);
                if constexpr (RS > 1)
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt) {
                        const f32x4 other = part[((wave ^ Cfg::NCW) * NDT + dt) * 64 + lane];
#pragma unroll
                        for (int rr = 0; rr < 4; ++rr) y[dt][0][rr] += other[rr];
                    }
                const rsrc_t ry = rsrc_of(py, sd, n, CW * ES);
                const uint32_t hd = shift_of(sd, n);
                py += step_d;
#pragma unroll
                for (int it = 0; it < NIT; ++it) {
                    const uint32_t to = yoff[it] - hd;
                    const float f = rd[it] * was;
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt) {
#pragma unroll
                        for (int rr = 0; rr < 4; ++rr) y[dt][it][rr] = y[dt][it][rr] * f + in[dt][it][rr];
                        store4(E(), y[dt][it], ry, to + 16 * dt * ES);
                    }
                }
            }
        }
    }

    if (works && job.end && (NOY || seg == a.ns - 1)) {
        scale(rho);
        float* o = job.end + (NOY ? srow : (size_t)bh) * (size_t)(N * D);
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) o[state_at(rt, dt, rr, !NOY && (job.flip & 2))] = R[rt][dt][rr];
    }
    if constexpr (!NOY) {   // rows past the sequence's length are zero
        const int z1 = min(a.T, u0 + a.lc * kLC);
        constexpr int PV = DT * ES / 16;
        char* y0 = static_cast<char*>(job.y);
        for (size_t x = (size_t)max(Tb, u0) * PV + threadIdx.x; x < (size_t)z1 * PV; x += NW * 64)
            *reinterpret_cast<uint4*>(y0 + ((((size_t)b * a.T + x / PV) * H + h) * D + tile * DT) * ES + (x % PV) * 16) =
                uint4{0u, 0u, 0u, 0u};
    }
}

template <typename E, int N, int D, bool NOY, int RS>
__global__ __launch_bounds__((LinCfg<E, N, D, NOY, RS>::NW * 64),
                             (LinCfg<E, N, D, NOY, RS>::OCC)) void linattn_kernel(LinArgs a) {
    linattn_pass<E, N, D, NOY, RS, LinCfg<E, N, D, NOY, RS>::NW>(a, blockIdx.x, 0, a.jobs);
}

// A backward with dk != dv: two passes with N = dv, D = dk and one the other way round in one launch, R0 and R1
// waves for their state rows.  Side by side they fill what each leaves idle (us in two launches and in one, dk/dv:
// bf16, B = 8, T = 2048, H = 16, 64/128 195 and 156, 128/64 197 and 176; B = 16, T = 512, 16/64 46 and 27; B = 3,
// T = 777, H = 5, 64/128 40 and 34; fp32, B = 8, T = 1024, H = 16, 32/64 125 and 94, 64/128 200 and 189).
template <typename E, int N, int D, int R0, int R1>
struct PairCfg {
    using A = LinCfg<E, N, D, false, R0>;
    using B = LinCfg<E, D, N, false, R1>;
    static constexpr int NW = A::NW > B::NW ? A::NW : B::NW, LDS = A::LDS > B::LDS ? A::LDS : B::LDS,
                         OCC = A::OCC < B::OCC ? A::OCC : B::OCC;
};
template <typename E, int N, int D, int R0, int R1>
__global__ __launch_bounds__((PairCfg<E, N, D, R0, R1>::NW * 64),
                             (PairCfg<E, N, D, R0, R1>::OCC)) void linattn_pair_kernel(LinArgs a) {
    using Cfg = PairCfg<E, N, D, R0, R1>;
    const int two = a.B * a.H * a.run * 2 * Cfg::A::NTILE;
    if ((int)blockIdx.x < two) linattn_pass<E, N, D, false, R0, Cfg::NW>(a, blockIdx.x, 0, 2);
    else linattn_pass<E, D, N, false, R1, Cfg::NW>(a, blockIdx.x - two, 2, 1);
}

// Start states of the segments from their own end states, in place: a workgroup takes 256 elements of
// one sequence's state through its segments.  job.k: the states before the first segments.
__global__ __launch_bounds__(256) void linattn_join_kernel(LinArgs a, int N, int D) {
    const int per = N * D / 256, nbh = a.B * a.H;
    const int bh = blockIdx.x / per % nbh, x = (blockIdx.x % per) * 256 + threadIdx.x;
    const LinJob& job = a.job[blockIdx.x / per / nbh];
    const float* s0 = static_cast<const float*>(job.k);
    const int Tb = seq_len(a, bh / a.H), L = a.lc * kLC;
    const float g = a.g[bh % a.H];
    float* e = job.end + (size_t)bh * a.ns * N * D + x;
    float R = s0 ? s0[(size_t)bh * N * D + x] : 0.f;
    const float whole = decay_pow(g, L);
    constexpr int U = 8;   // segments in flight: the states are read and written in place
    for (int s1 = 0; s1 < a.ns; s1 += U) {
        float own[U];
#pragma unroll
        for (int i = 0; i < U; ++i) own[i] = s1 + i < a.ns - 1 ? e[(size_t)(s1 + i) * N * D] : 0.f;
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (s1 + i < a.ns) {
                e[(size_t)(s1 + i) * N * D] = R;
                const int n = min(max(Tb - (s1 + i) * L, 0), L);
                R = (n == L ? whole : decay_pow(g, n)) * R + own[i];
            }
    }
}

template <auto KERN, int LDS>
hipError_t launch_kernel(const LinArgs& a, size_t grid, int threads, hipStream_t st) {
    if constexpr (LDS > 64 * 1024) {   // must be opted into, once per kernel and device
        static std::atomic<uint64_t> done{0};
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        const uint64_t bit = 1ull << (dev & 63);
        if (!(done.load() & bit)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERN), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
            if (e != hipSuccess) return e;
            done.fetch_or(bit);
        }
    }
    hipLaunchKernelGGL(KERN, dim3((unsigned)grid), dim3(threads), LDS, st, a);
    return hipGetLastError();
}

template <typename E, int N, int D, bool NOY, int RS = 1>
hipError_t launch(const LinArgs& a, hipStream_t st) {
    using Cfg = LinCfg<E, N, D, NOY, RS>;
    return launch_kernel<linattn_kernel<E, N, D, NOY, RS>, Cfg::LDS>(a, (size_t)a.B * a.H * a.run * a.jobs * Cfg::NTILE,
                                                                     Cfg::NW * 64, st);
}

template <typename E, int N, int D, int R0, int R1>
hipError_t launch_pair(const LinArgs& a, hipStream_t st) {
    using Cfg = PairCfg<E, N, D, R0, R1>;
    return launch_kernel<linattn_pair_kernel<E, N, D, R0, R1>, Cfg::LDS>(
        a, (size_t)a.B * a.H * a.run * (2 * Cfg::A::NTILE + Cfg::B::NTILE), Cfg::NW * 64, st);
}

// One or two waves for a column group's state rows.  Two shorten the chain of a chunk's products and fill the
// SIMDs where there are fewer than two workgroups a CU, but both convert V.  128 rows, us with one and two
// (workgroups): bf16, 128/128, H = 16, T = 2048, forward 118 and 108 (256), T = 1024, forward 97 and 98 (512), 122 and
// 136 (640), backward 84 and 80 (384), 90 and 89 (480), 107 and 119 (576); backward of both shapes, H = 8,
// T = 1024, 128/64 77 and 69 (480), 92 and 98 (640), 64/128 81 and 79 (480), 100 and 114 (640); fp32, whose LDS holds
// one workgroup a CU, 128/128, T = 1024, forward 127 and 117, backward 369 and 339 (B = 8), 735 and 674 (B = 16).
// With 32 columns or fewer two win beyond that too (backward of 128/16, 640: 77 and 67, 1920: 198 and 192).  Of 64
// rows two take the forward of an uncut sequence from 81 to 75 (128 workgroups), where segments take it to 41, and
// the backward from 175 to 201 (768).
constexpr size_t kTwoWaves = 512;   // two workgroups a CU: fewer take two waves
template <typename E, int N, int D>
hipError_t run_rows(const LinArgs& a, hipStream_t st) {
    constexpr int RS = N == 128 ? 2 : 1;
    if constexpr (sizeof(E) == 2 && RS > 1)
        if ((size_t)a.B * a.H * a.run * a.jobs * LinCfg<E, N, D, false, 1>::NTILE >= kTwoWaves)
            return launch<E, N, D, false, 1>(a, st);
    return launch<E, N, D, false, RS>(a, st);
}

template <typename E>
hipError_t run(const LinArgs& a, int N, int D, bool noy, hipStream_t st) {
#define KLA_LIN(N_, D_) \
    if (N == N_ && D == D_) return noy ? launch<E, N_, D_, true>(a, st) : run_rows<E, N_, D_>(a, st);
#define KLA_LIN_ROW(N_) KLA_LIN(N_, 16) KLA_LIN(N_, 32) KLA_LIN(N_, 64) KLA_LIN(N_, 128)
    KLA_LIN_ROW(16) KLA_LIN_ROW(32) KLA_LIN_ROW(64) KLA_LIN_ROW(128)
#undef KLA_LIN_ROW
#undef KLA_LIN
    return hipErrorInvalidValue;
}

template <typename E, int N, int D>
hipError_t pair_rows(const LinArgs& a, hipStream_t st) {   // by the same rule as run_rows
    constexpr int R0 = N == 128 ? 2 : 1, R1 = D == 128 ? 2 : 1;
    using Cfg = PairCfg<E, N, D, R0, R1>;
    if constexpr (sizeof(E) == 2 && R0 + R1 > 2)
        if ((size_t)a.B * a.H * a.run * (2 * Cfg::A::NTILE + Cfg::B::NTILE) >= kTwoWaves)
            return launch_pair<E, N, D, 1, 1>(a, st);
    return launch_pair<E, N, D, R0, R1>(a, st);
}

template <typename E>
hipError_t run_pair(const LinArgs& a, int N, int D, hipStream_t st) {
#define KLA_LIN(N_, D_) \
    if (N == N_ && D == D_) return pair_rows<E, N_, D_>(a, st);
    KLA_LIN(16, 32) KLA_LIN(16, 64) KLA_LIN(16, 128) KLA_LIN(32, 16) KLA_LIN(32, 64) KLA_LIN(32, 128)
    KLA_LIN(64, 16) KLA_LIN(64, 32) KLA_LIN(64, 128) KLA_LIN(128, 16) KLA_LIN(128, 32) KLA_LIN(128, 64)
#undef KLA_LIN
    return hipErrorInvalidValue;
}

hipError_t run(const Shape& s, const LinArgs& a, int N, int D, bool noy, hipStream_t st) {
    return s.bf16 ? run<uint16_t>(a, N, D, noy, st) : run<float>(a, N, D, noy, st);
}

// One token: state <- e^g state + k v^T in place, y = state^T q.  A workgroup of 256 threads takes CT
// columns of one sequence and head, CT / 4 threads a row of 16-byte accesses; bound by the state's
// traffic, so every load is issued before the first is used.
template <typename E, int DK, int CT>
__global__ __launch_bounds__(256) void linattn_step_kernel(int H, int dv, const E* __restrict__ q, const E* __restrict__ k,
                                                           const E* __restrict__ v, const float* __restrict__ g,
                                                           float* __restrict__ state, E* __restrict__ y) {
    constexpr int LR = CT / 4, RP = 256 / LR, NR = (DK + RP - 1) / RP;   // lanes per row, rows per pass, passes
    __shared__ float4 part[256];
    const int nt = dv / CT, sh = blockIdx.x / nt, d0 = (blockIdx.x % nt) * CT;
    const int row = threadIdx.x / LR, c = 4 * (threadIdx.x % LR);
    float* s = state + (size_t)sh * DK * dv + d0 + c;
    float4 x[NR];
    float kv[NR], qv[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int n = row + i * RP;
        const bool in = DK % RP == 0 || n < DK;
        x[i] = in ? *reinterpret_cast<const float4*>(s + (size_t)n * dv) : float4{0.f, 0.f, 0.f, 0.f};
        kv[i] = in ? ld(k, (size_t)sh * DK + n) : 0.f;
        qv[i] = in ? ld(q, (size_t)sh * DK + n) : 0.f;
    }
    const float gam = expf(g[sh % H]);
    float vv[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) vv[e] = ld(v, (size_t)sh * dv + d0 + c + e);
    float4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        x[i].x = gam * x[i].x + kv[i] * vv[0];
        x[i].y = gam * x[i].y + kv[i] * vv[1];
        x[i].z = gam * x[i].z + kv[i] * vv[2];
        x[i].w = gam * x[i].w + kv[i] * vv[3];
        const int n = row + i * RP;
        if (DK % RP == 0 || n < DK) *reinterpret_cast<float4*>(s + (size_t)n * dv) = x[i];
        acc.x += qv[i] * x[i].x;
        acc.y += qv[i] * x[i].y;
        acc.z += qv[i] * x[i].z;
        acc.w += qv[i] * x[i].w;
    }
    part[threadIdx.x] = acc;
    __syncthreads();
    if (threadIdx.x < CT) {   // column threadIdx.x, over the row groups in a fixed order
        const float* p = reinterpret_cast<const float*>(part) + threadIdx.x;
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < RP; ++r) t += p[r * CT];
        st(y, (size_t)sh * dv + d0 + threadIdx.x, t);
    }
}

template <typename E, int DK>
hipError_t launch_step(const Shape& s, const void* q, const void* k, const void* v, const float* g, float* state, void* y,
                       hipStream_t st) {
    const E *q_ = static_cast<const E*>(q), *k_ = static_cast<const E*>(k), *v_ = static_cast<const E*>(v);
    E* y_ = static_cast<E*>(y);
    const unsigned n = (unsigned)((size_t)s.B * s.H);
#define KLA_STEP(CT_) \
    linattn_step_kernel<E, DK, CT_><<<dim3(n * (unsigned)(s.dv / CT_)), dim3(256), 0, st>>>(s.H, s.dv, q_, k_, v_, g, state, y_)
    // Whole rows of dv = 128, but quarters of them while those are no more than two workgroups a CU (us a step
    // in quarters and whole, dk = dv = 128: 16 of sequence and head 2.6 and 3.3, 64 3.0 and 3.7, 128 3.8 and 4.2,
    // 256 5.6 and 5.2, 8192 212 and 207; of dv = 64 halves gain nothing, 2.4 and 2.3).
    if (s.dv == 128 && n > 128) KLA_STEP(128);
    else if (s.dv == 64) KLA_STEP(64);
    else if (s.dv >= 32) KLA_STEP(32);
    else KLA_STEP(16);
#undef KLA_STEP
    return hipGetLastError();
}

template <typename E>
hipError_t step(const Shape& s, const void* q, const void* k, const void* v, const float* g, float* state, void* y,
                hipStream_t st) {
    switch (s.dk) {
        case 16: return launch_step<E, 16>(s, q, k, v, g, state, y, st);
        case 32: return launch_step<E, 32>(s, q, k, v, g, state, y, st);
        case 64: return launch_step<E, 64>(s, q, k, v, g, state, y, st);
        default: return launch_step<E, 128>(s, q, k, v, g, state, y, st);
    }
}

// Segments per sequence and chunks in one, for passes of `groups` workgroups where no sequence is cut, to
// make `want`, or `more` where segments would be longer than 96 chunks.  Segments cost a pass over K and V for
// their states and two launches more, so a sequence of fewer than 16 chunks is not cut, nor where there is a
// workgroup for every CU (dk = dv = 128, bf16, B = 8, T = 2048, H = 16, us whole and in two: forward, 256
// workgroups, 110 and 145; backward, 768, 250 and 322).
// Otherwise the forward makes two workgroups a CU and the backward, whose passes share their reads,
// three (us in 4, 8, 16, 24 segments, B = 1, T = 16384, H = 16, forward 317, 175, 137, 137, backward 428,
// 330, 327, 349; in 2, 4, 8, 16, B = 4, T = 4096, H = 8, forward 165, 96, 78, 81, backward 220, 171, 175, 198), but
// none shorter than two chunks; where they are long, one and three workgroups a CU more (T = 65536 in 8, 16, 24,
// 32: forward 629, 513, 501, 505, backward 1267, 1225, 1266, 1233).
void segments(const Shape& s, long groups, long want, long more, int& ns, int& lc) {
    const int nc = (s.T + kLC - 1) / kLC;
    ns = 1;
    lc = nc;
    if (nc < 16 || groups >= 256) return;
    ns = (int)((want + groups - 1) / groups);
    if (nc > 96 * ns) ns = (int)((more + groups - 1) / groups);
    if (ns > nc / 2) ns = nc / 2;
    lc = (nc + ns - 1) / ns;
    ns = (nc + lc - 1) / lc;
}

long tiles(int D) { return D > 64 ? 2 : 1; }   // workgroups of a pass over one sequence
void fwd_segments(const Shape& s, int& ns, int& lc) { segments(s, (long)s.B * s.H * tiles(s.dv), 512, 768, ns, lc); }
void bwd_segments(const Shape& s, int& ns, int& lc) {
    segments(s, (long)s.B * s.H * (2 * tiles(s.dk) + tiles(s.dv)), 768, 1536, ns, lc);
}

LinArgs args_of(const Shape& s, const float* g, const int* len, bool backward) {
    LinArgs a{};
    a.g = g;
    a.len = len;
    a.B = s.B;
    a.T = s.T;
    a.H = s.H;
    if (backward) bwd_segments(s, a.ns, a.lc);
    else fwd_segments(s, a.ns, a.lc);
    return a;
}

// States before the segments of `jobs` passes over [dk][dv] states, from q, k, v and start states as in job:
// into st0[j], by sequence and segment.
hipError_t start_states(const Shape& s, const LinArgs& a, const LinJob* job, float* const* st0, int jobs, hipStream_t st) {
    LinArgs p = a;
    p.jobs = jobs;
    p.run = a.ns - 1;
    for (int j = 0; j < jobs; ++j) {
        p.job[j] = job[j];
        p.job[j].end = st0[j];
    }
    hipError_t e = run(s, p, s.dk, s.dv, true, st);
    if (e != hipSuccess) return e;
    for (int j = 0; j < jobs; ++j) p.job[j].k = job[j].start;
    const size_t grid = (size_t)s.B * s.H * (s.dk * s.dv / 256) * jobs;
    linattn_join_kernel<<<dim3((unsigned)grid), dim3(256), 0, st>>>(p, s.dk, s.dv);
    return hipGetLastError();
}

size_t states_bytes(const Shape& s, int ns) {
    return ns > 1 ? (size_t)s.B * s.H * ns * s.dk * s.dv * sizeof(float) : 0;
}

}  // namespace

size_t linattn_workspace(const Shape& s, bool backward) {
    const LinArgs a = args_of(s, nullptr, nullptr, backward);
    return (backward ? 2 : 1) * states_bytes(s, a.ns);
}

hipError_t launch_linattn_fwd(const Shape& s, const void* q, const void* k, const void* v, const float* g, const float* s0,
                              const int* len, void* y, float* sT, void* ws, hipStream_t st) {
    LinArgs a = args_of(s, g, len, false);
    a.jobs = 1;
    a.run = a.ns;
    a.job[0] = LinJob{q, k, v, s0, y, sT, 0, 0};
    if (a.ns > 1) {
        float* st0 = static_cast<float*>(ws);
        const hipError_t e = start_states(s, a, a.job, &st0, 1, st);
        if (e != hipSuccess) return e;
        a.job[0].start = st0;
    }
    return run(s, a, s.dk, s.dv, false, st);
}

hipError_t launch_linattn_bwd(const Shape& s, const void* q, const void* k, const void* v, const float* g, const float* s0,
                              const int* len, const void* dy, const float* dsT, void* dq, void* dk, void* dv, float* ds0,
                              void* ws, hipStream_t st) {
    LinArgs a = args_of(s, g, len, true);
    a.run = a.ns;
    const float *first = s0, *last = dsT;
    if (a.ns > 1) {   // the states before the segments, and their adjoints behind them
        float* st0[2] = {static_cast<float*>(ws), static_cast<float*>(ws) + states_bytes(s, a.ns) / sizeof(float)};
        const LinJob j[2] = {{nullptr, k, v, s0, nullptr, nullptr, 0, 0}, {nullptr, q, dy, dsT, nullptr, nullptr, 1, 0}};
        const hipError_t e = start_states(s, a, j, st0, 2, st);
        if (e != hipSuccess) return e;
        first = st0[0];
        last = st0[1];
    }
    // the states of dq and dk are the transposes [dv][dk]
    a.job[0] = LinJob{dy, v, k, first, dq, nullptr, 0, 1};
    a.job[1] = LinJob{v, dy, q, last, dk, nullptr, 1, 1};
    a.job[2] = LinJob{k, q, dy, last, dv, ds0, 1, 0};
    a.jobs = 3;
    if (s.dk == s.dv) return run(s, a, s.dk, s.dv, false, st);
    return s.bf16 ? run_pair<uint16_t>(a, s.dv, s.dk, st) : run_pair<float>(a, s.dv, s.dk, st);
}

hipError_t launch_linattn_step(const Shape& s, const void* q, const void* k, const void* v, const float* g, float* state,
                               void* y, hipStream_t st) {
    return s.bf16 ? step<uint16_t>(s, q, k, v, g, state, y, st) : step<float>(s, q, k, v, g, state, y, st);
}

}  // namespace kla
