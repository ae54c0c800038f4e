// Softmax attention with a sliding window and first tokens that stay visible, on matrix instructions.
//
//   y_i = sum_j P_ij v_j,   P_i = softmax over the visible j of scale q_i . k_j
//
// j is visible to the query at position p iff j <= p and (j > p - W or j < sinks).  H query heads share Hk heads
// of keys and values.  Queries are the last T of Tk tokens; a sequence ends at len.
//
// Forward and dq: a wave owns 32 queries of a head, the workgroup's four 128.  Tiles of 32 or 64 tokens' keys and
// values go through LDS, loaded a tile ahead.  Scores are formed transposed, S^T = K Q^T (tokens x queries), so
// that a query is a lane's column: its running reference and sum are one value a lane and one exchange between the
// wave's halves, and S^T, rounded to the operands' type, is the operand of O^T += V^T P^T as it stands.
//   m, l: a reference near the largest score and the sum of exponentials about it.
//   dS = P (dy . v - D),  D = dy . y,  dq = scale dS K
// dk, dv: a wave owns 32 tokens and walks the queries that see them, of all heads that share them, with
// S = Q K^T (queries x tokens) in the same way: dV^T += dy^T P, dK^T += Q^T dS.  No sum has more than one
// writer, so results do not depend on the order of workgroups.  First tokens are seen by all later queries:
// the queries behind the window of the first 128 tokens are cut into segments, whose sums over those tokens are
// joined.
//
// What bounds it.  Long windows: matrix work; a prompt of B1 T65536 H16 Hk4 d128 window 2048 takes 1.10 ms, 985
// TFLOP/s of its 1085 GFLOP (a large product reaches 1240), at a clock that the card's power holds to 1.9 GHz, the matrix
// cores busy for half of the time; a wave's 32 rows read every product's other operand from LDS.  B8 T2048 H16 d128
// window 512: 119 us forward (two products of a tile), 161 dq (three), 202 dk and dv (four), the matrix cores busy for a
// quarter of the time at 2.4 GHz: reckoned from the prompt's time a tile, the forward's workgroups, of 22 tiles, spend more than
// a third of their time outside the loop over them, on the first reads, the vote on sums that are not finite and the
// stores, those of a round all at once.  fp32: its matrix instructions, 153 TFLOP/s, busy for 0.3 to 0.5 of the time and
// CUs for 0.7 where workgroups are few.  The step: HBM, 5.6 TB/s (S512 Hk4 d128 over 1028 slots, 190 us).
//
// v_mfma_f32_32x32x16_bf16 (lane l, half h = l / 32): A row l % 32 and B column l % 32, contraction 8 h .. 8 h + 7;
// C column l % 32, register r at row 8 (r / 4) + 4 h + r % 4.  Over the contraction of a C used as B, half h
// therefore has rows 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 of 16, and A is read with the same.  fp32:
// v_mfma_f32_32x32x2_f32, one contraction index a half.
//
// bf16: q, k, v, dy are exact operands; scores, references, sums and accumulators stay in fp32; P and dS are rounded to
// bf16, which adds as much as the rounding of the outputs.  Where a few tokens take most of a row, D, which is common to a
// row's dS, is as large as dy . v, and what y is off by is many times dS.  So y is divided by the sum of the weights as
// rounded, which takes a heavy weight's rounding out again, and saved with 8 more bits for D.  Errors over those of exact
// outputs rounded once (T1024 d128 window 512, rows from 256 on; scores of deviation 1, 6 and 20, whose largest weights
// are 0.03, 0.6 and 0.9): y 1.4, 1.05, 1.02; dq and dk 1.4, 1.5, 1.55; dv 1.4, 1.3, 1.2; with the sum of the weights
// themselves and y as stored dq would be off by 1.4, 3.1 and 5.3.  Calls whose rows all see few tokens (fewer than kFew), and
// the first kRows positions, take P and dS in two parts: 1.0 (window 200, deviations 1 and 6).  fp32 inputs keep fp32
// operands throughout.
//
// Values that are not finite: scores of masked places are left out by selection, but the products with a zero weight
// are not, and an infinity or NaN there would reach rows that do not see it.  So a workgroup whose sums are not finite
// walks its tiles once more, its products element by element without the masked places.
#include <type_traits>

#include "kla_buf.hpp"
#include "kla_internal.hpp"
#include "kla_mfma.hpp"

namespace kla {
namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

constexpr int kRows = 128;   // queries, or tokens in the dk, dv pass, a workgroup
// The exponents' reference lies this far above the largest score (times c, rounded up) that moved it: weights are at
// most 1, and a row is rescaled only when a score passes the reference, not whenever the maximum grows, which one of
// a wave's 32 rows does in nearly every tile.  The backward takes it lower by as much, with the sum multiplied
// accordingly (context): small weights then end where exp2's range does below the largest, not 2^8 above.
constexpr float kAhead = 8.f;
constexpr int kFew = 256;    // a call whose rows see fewer tokens than this sees few
constexpr uint32_t kMasked = 0x80000000u;   // the weight of a masked place: -0, which seen() keeps apart from others

// A visible place's weight where masked ones are left out: dS is signed, and its zeros are +0.
__device__ __forceinline__ float seen(float w) { return w == 0.f ? 0.f : w; }

// Rows of D elements in LDS, in 16-byte pieces: piece c of row r lies at c ^ key(r), so that 16 rows read at one
// piece, 4 rows of bf16 read across at four pieces, and rows of fp32 read across at eight, 4 rows apart, touch
// different columns of 64 banks.  256-byte rows of bf16 have every four of them 16 bytes further on instead of half
// of the key: reads then need four addresses a lane, and constant offsets, instead of eight.  16 columns are
// padded with zeros to 32.
template <typename E, int D>
struct Rows {
    static constexpr int DP = D < 32 ? 32 : D, NC = DP * (int)sizeof(E) / 16, NR = D * (int)sizeof(E) / 16;
    static constexpr bool APART = sizeof(E) == 2 && NC == 16;
    static constexpr int UNIT = 1024 + (APART ? 16 : 0);   // bytes of a wave's load, 1024 / (16 NC) rows
    static constexpr int bytes(int rows) { return rows * NC / 64 * UNIT; }
    __device__ static int key(int r) {
        if (APART) return (r & 3) << 2;
        if (sizeof(E) == 4) return NC >= 16 ? ((r & 4) << 1) | ((r & 8) >> 1) | (r & 3) : (r >> 1) & 7;
        return NC == 8 ? ((r & 2) << 1) | ((r >> 2) & 3) : (r >> 2) & 3;
    }
    __device__ static int row(int r) { return r * NC * 16 + (APART ? (r >> 2) * 16 : 0); }
    __device__ static int at(int r, int col) {
        constexpr int PER = 16 / (int)sizeof(E);
        return row(r) + (((col / PER) ^ key(r)) << 4) + (col % PER) * (int)sizeof(E);
    }
    // piece 2 k + h of row l32, k a constant; rows a multiple of 16 further on lie row() of that further
    __device__ static int row_at(int l32, int h, int k) {
        if (APART) return row(l32) + (((k >> 1) ^ (l32 & 3)) << 6) + h * 16 + (k & 1) * 32;
        return row(l32) + (((2 * k + h) ^ key(l32)) << 4);
    }
    // for a read across (bf16): lane s of 16 addresses row 4 h + s / 4 (second: 8 further on) at column
    // 32 t + (l32 & 16) + 4 (s % 4)
    __device__ static int col_at(int l32, int h, int t, bool second) {
        const int s = l32 & 15, r = 4 * h + (s >> 2);
        if (APART)
            return row(4) * h + (s >> 2) * NC * 16 + ((t ^ (s >> 2)) << 6) + ((l32 & 16) << 1) + ((s & 2) << 3) + ((s & 1) << 3) +
                   (second ? row(8) : 0);
        return at(r + (second ? 8 : 0), 32 * t + (l32 & 16) + 4 * (s & 3));
    }
};

// C tiles over the columns of a row, 32 each
template <typename E, int D>
using Acc = f32x16[Rows<E, D>::DP / 32];

// What rounding to bf16 left of four values, in 1/254 of each one's last place: with it D = dy . y has 16 bits of
// y.  D is common to a row's dS = P (dy . v - D), and where a row sees few tokens, or a few of them take most of it, as
// large as dy . v: y's rounding alone would be as much as that of dS, or many times as much.  Differences of bit
// patterns, which go on past a power of two; an infinity and a zero leave 0.
__device__ __forceinline__ uint32_t rest_of(const float (&x)[4], const uint2& y) {
    const uint32_t b[4] = {y.x << 16, y.x & 0xffff0000u, y.y << 16, y.y & 0xffff0000u};
    uint32_t t[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = (uint32_t)(__mul24((int)(__float_as_uint(x[e]) - b[e]), 254) + 0x8000);   // byte 2
    return __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0602u) | __builtin_amdgcn_perm(t[3], t[2], 0x06020c0cu);
}
__device__ __forceinline__ float rest_add(float y, uint32_t w, int e) {
    return __uint_as_float(__float_as_uint(y) + (uint32_t)__mul24((int)(int8_t)(w >> (8 * e)), 258));   // 2^16 / 254
}

// One row of a lane (A's or B's 32 rows): half h has every second piece.
template <typename E, int D>
struct Row;
template <int D>
struct Row<uint16_t, D> {
    static constexpr int K = D / 16;
    bf16x8 x[K];
    __device__ void load(const void* p, bool live, int h) {   // p: the row
#pragma unroll
        for (int k = 0; k < K; ++k)
            x[k] = __builtin_bit_cast(bf16x8, live ? reinterpret_cast<const uint4*>(p)[2 * k + h] : uint4{0, 0, 0, 0});
    }
    __device__ float dot(const Row& y, const int8_t* rest, int h) const {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint2 w = rest ? *reinterpret_cast<const uint2*>(rest + 16 * k + 8 * h) : uint2{0, 0};
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf((float)x[k][e], rest_add((float)y.x[k][e], e < 4 ? w.x : w.y, e % 4), s);
        }
        return s;
    }
};
template <int D>
struct Row<float, D> {
    static constexpr int K = D / 8;
    f32x4 x[K];
    __device__ void load(const void* p, bool live, int h) {
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] = live ? reinterpret_cast<const f32x4*>(p)[2 * k + h] : zero4();
    }
    __device__ float dot(const Row& y, const int8_t*, int) const {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = fmaf(x[k][e], y.x[k][e], s);
        return s;
    }
};

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}

// N products whose operands come from LDS, read AHEAD products before.  The scheduler, left alone, sinks each read to
// its product and waits for it (backward 395 us, 370 this way; 3 to 7 ahead are alike); the barriers let only other
// arithmetic (0x6) pass.
template <int N, int AHEAD, typename Read, typename Mul>
__device__ __forceinline__ void stream(Read read, Mul mul) {
    constexpr int A = AHEAD < N ? AHEAD : N;
    bf16x8 f[A];
#pragma unroll
    for (int i = 0; i < A; ++i) f[i] = read(i);
    __builtin_amdgcn_sched_barrier(0x6);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        mul(i, f[i % A]);
        if (i + A < N) f[i % A] = read(i + A);
        __builtin_amdgcn_sched_barrier(0x6);
    }
}

__device__ __forceinline__ bf16x8 read16(const unsigned char* p) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(p));
}

// C = (rows row0 .. row0 + 31 of the tile) (row b of each lane)^T
template <int D>
__device__ __forceinline__ f32x16 rows_dot(const unsigned char* t, int row0, const Row<uint16_t, D>& b, int l32, int h) {
    using R = Rows<uint16_t, D>;
    f32x16 c = zero16();
    stream<D / 16, 4>([&](int k) { return read16(t + R::row(row0) + R::row_at(l32, h, k)); },
                      [&](int k, const bf16x8& a) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b.x[k], c, 0, 0, 0); });
    return c;
}
// Two of them in turn, which do not wait for each other's sums.
template <int D>
__device__ __forceinline__ void rows_dot_two(const unsigned char* t0, const unsigned char* t1, int row0, const Row<uint16_t, D>& b0,
                                             const Row<uint16_t, D>& b1, f32x16& c0, f32x16& c1, int l32, int h) {
    using R = Rows<uint16_t, D>;
    c0 = c1 = zero16();
    stream<D / 8, 4>([&](int i) { return read16((i % 2 ? t1 : t0) + R::row(row0) + R::row_at(l32, h, i / 2)); },
                     [&](int i, const bf16x8& a) {
                         f32x16& c = i % 2 ? c1 : c0;
                         c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, (i % 2 ? b1 : b0).x[i / 2], c, 0, 0, 0);
                     });
}
template <int D>
__device__ __forceinline__ f32x16 rows_dot(const unsigned char* t, int row0, const Row<float, D>& b, int l32, int h) {
    f32x16 c = zero16();
#pragma unroll
    for (int k = 0; k < D / 8; ++k) {
        using R = Rows<float, D>;
        const f32x4 a = *reinterpret_cast<const f32x4*>(t + R::row(row0) + R::row_at(l32, h, k));
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b.x[k][e], c, 0, 0, 0);
    }
    return c;
}

template <int D>
__device__ __forceinline__ void rows_dot_two(const unsigned char* t0, const unsigned char* t1, int row0, const Row<float, D>& b0,
                                             const Row<float, D>& b1, f32x16& c0, f32x16& c1, int l32, int h) {
    c0 = rows_dot<D>(t0, row0, b0, l32, h);
    c1 = rows_dot<D>(t1, row0, b1, l32, h);
}

// The same with b0's rows in LDS, l32 of them from p on.
struct RowsAt {
    const unsigned char* p;
};
template <int D>
__device__ __forceinline__ void rows_dot_two(const unsigned char* t0, const unsigned char* t1, int row0, const RowsAt& b0,
                                             const Row<uint16_t, D>& b1, f32x16& c0, f32x16& c1, int l32, int h) {
    using R = Rows<uint16_t, D>;
    c0 = c1 = zero16();
    bf16x8 q{};
    stream<3 * D / 16, 5>(   // a row of t0, of b0, of t1 in turn
        [&](int i) {
            const int at = R::row_at(l32, h, i / 3);
            return read16(i % 3 == 1 ? b0.p + at : (i % 3 ? t1 : t0) + R::row(row0) + at);
        },
        [&](int i, const bf16x8& a) {
            if (i % 3 == 0)
                q = a;
            else if (i % 3 == 1)
                c0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, a, c0, 0, 0, 0);
            else
                c1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b1.x[i / 3], c1, 0, 0, 0);
        });
}

// Weights of 32 rows (a C, register r at row 8 (r / 4) + 4 h + r % 4) as the operand of a product over them.
template <typename E>
struct Weights;
template <>
struct Weights<uint16_t> {
    bf16x8 b[2];
    __device__ explicit Weights(const f32x16& w) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            b[k] = __builtin_bit_cast(bf16x8, uint4{cvt_pk_bf16(w[8 * k], w[8 * k + 1]), cvt_pk_bf16(w[8 * k + 2], w[8 * k + 3]),
                                                    cvt_pk_bf16(w[8 * k + 4], w[8 * k + 5]),
                                                    cvt_pk_bf16(w[8 * k + 6], w[8 * k + 7])});
    }
};
template <>
struct Weights<float> {
    const f32x16& w;
    __device__ explicit Weights(const f32x16& w) : w(w) {}
};

// s + the sum of a lane's weights as rounded, two at once
__device__ __forceinline__ float pairs_sum(const bf16x8& w, float s) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 pair_t;
#pragma unroll
    for (int r = 0; r < 8; r += 2)
        s = __builtin_amdgcn_fdot2_f32_bf16(pair_t{w[r], w[r + 1]}, pair_t{(__bf16)1.f, (__bf16)1.f}, s, false);
    return s;
}

// o[t] += (columns 32 t .. 32 t + 31 of rows row0 .. row0 + 31)^T w
template <int D>
__device__ __forceinline__ void cols_dot(Acc<uint16_t, D>& o, const unsigned char* x, int row0, const Weights<uint16_t>& w, int l32,
                                         int h) {
    using R = Rows<uint16_t, D>;
    constexpr int DT = R::DP / 32;
    stream<2 * DT, 4>(
        [&](int i) {
            const unsigned char* p = x + R::row(row0 + 16 * (i / DT));
            const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)(p + R::col_at(l32, h, i % DT, false)));
            const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)(p + R::col_at(l32, h, i % DT, true)));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        },
        [&](int i, const bf16x8& a) {
            o[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w.b[i / DT], o[i % DT], 0, 0, 0);
        });
}
template <int D>
__device__ __forceinline__ void cols_dot(Acc<float, D>& o, const unsigned char* x, int row0, const Weights<float>& w, int l32, int h) {
    using R = Rows<float, D>;
#pragma unroll
    for (int t = 0; t < R::DP / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float a = *reinterpret_cast<const float*>(x + R::row(row0) + R::at(8 * (r / 4) + 4 * h + r % 4, 32 * t + l32));
            o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w.w[r], o[t], 0, 0, 0);
        }
}

__device__ __forceinline__ float elem(const unsigned char* p, uint16_t) {
    return bf16_to_f32(*reinterpret_cast<const uint16_t*>(p));
}
__device__ __forceinline__ float elem(const unsigned char* p, float) { return *reinterpret_cast<const float*>(p); }

// The same element by element, without the rows whose weight is masked.  scratch: 128 floats of the wave's own.
template <typename E, int D>
__device__ __forceinline__ void cols_apart(f32x16& c, const unsigned char* x, int row0, int t, const f32x16& w, float* scratch,
                                           int l32, int h) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {   // rows 4 k .. 4 k + 3, of half k % 2
        if (h == k % 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) scratch[e * 32 + l32] = w[4 * (k / 2) + e];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            const float f = scratch[i * 32 + l32];
            if (__float_as_uint(f) == kMasked) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                c[r] = fmaf(f, elem(x + Rows<E, D>::at(row0 + 4 * k + i, 32 * t + 8 * (r / 4) + 4 * h + r % 4), E{}), c[r]);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// What the operands' rounding left of the weights.
__device__ __forceinline__ f32x16 left_of(const f32x16& w, const Weights<uint16_t>& b) {
    f32x16 x;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = w[r] - (float)b.b[r / 8][r % 8];
    return x;
}

// o += (rows row0 .. row0 + 31)^T w.  TWO: bf16 weights enter in two parts.  sum: takes the weights as rounded, where
// they enter in one.
template <bool CAREFUL, bool TWO, typename E, int D>
__device__ __forceinline__ void add_cols(Acc<E, D>& o, const unsigned char* x, int row0, const f32x16& w, float* scratch, int l32,
                                         int h, float* sum = nullptr) {
    if constexpr (CAREFUL) {
#pragma unroll
        for (int t = 0; t < Rows<E, D>::DP / 32; ++t) cols_apart<E, D>(o[t], x, row0, t, w, scratch, l32, h);
    } else {
        const Weights<E> b(w);
        if constexpr (sizeof(E) == 2 && !TWO)
            if (sum) *sum = pairs_sum(b.b[0], 0.f) + pairs_sum(b.b[1], *sum);
        cols_dot<D>(o, x, row0, b, l32, h);
        if constexpr (sizeof(E) == 2 && TWO) cols_dot<D>(o, x, row0, Weights<E>(left_of(w, b)), l32, h);
    }
}

template <int N>
__device__ __forceinline__ bool finite(const f32x16 (&o)[N]) {
    float z = 0.f;   // NaN where one is not
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) z = fmaf(o[t][r], 0.f, z);
    return z == 0.f;
}

// Whether any thread of the workgroup says so.  Orders LDS before and after.
__device__ __forceinline__ bool any_of(bool x, int* flag) {
    __syncthreads();
    if (threadIdx.x == 0) *flag = 0;
    __syncthreads();
    if (x) *flag = 1;
    __syncthreads();
    return *flag != 0;
}

// A row's sum l about the reference m.  The largest score lies within 9 of a reference below 2^24; past that by half of
// fp32's steps more, 64 between 2^30 and 2^31.  A sum that says more is lost: NaN, where its row would else be zeros or
// wrong.  (m = -inf: no score, or NaN.)
__device__ __forceinline__ float sum_of(float l, float m) {
    return m == -INFINITY || (l > 0x1p-64f && l < 0x1p64f) ? l : __uint_as_float(0x7fc00000u);
}

// What the backward takes of a row with reference m and sum l: the reference less kAhead, and the sum about that.  m is a
// whole number, but past 2^27 fp32 has no step of 8: the sum is multiplied by 2 to the distance that came out (0, 8 or
// 16), exactly.  Rows without a score have zeros.
__device__ __forceinline__ float2 context(float m, float l) {
    if (l == 0.f) return float2{0.f, 0.f};
    const float low = m - kAhead;
    return float2{low, ldexpf(l, (int)(m - low))};
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// The value of the lane 32 away: of two copies the instruction swaps one's upper half with the other's lower one.
__device__ __forceinline__ void both_halves(float x, float& lower, float& upper) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    lower = __uint_as_float(p[0]);
    upper = __uint_as_float(p[1]);
}
__device__ __forceinline__ float halves_sum(float x) {
    float a, b;
    both_halves(x, a, b);
    return a + b;
}
__device__ __forceinline__ float halves_max(float x) {
    float a, b;
    both_halves(x, a, b);
    return fmaxf(a, b);
}

struct WinArgs {
    const void *q, *k, *v, *y, *dy;
    void *o, *dq, *dk, *dv;   // o: y of the forward
    const int* len;
    float2* stat;             // [B, T, H]: the exponents' reference less kAhead and the sum of exponentials about it
    int8_t* rest;             // bf16: [B, T, H, D], what the rounding of y left (rest_of)
    float* part;              // forward: partial O [nsplit][B T H][D]; dk, dv: the first tokens' sums
    float2* pstat;            // forward: [nsplit][B T H]
    float* rows;              // backward: [3][B H][T64] m, 1 / l, D
    float* kpart;             // dk, dv: [B Hk][ksplit][2][Tk][D], where a workgroup's queries are dealt to several
    int B, T, Tk, H, Hk, W, sinks, blocks, nsplit, nseg, seg, ksplit, T64;
    float scale, c;           // c = scale log2(e)
    bool few;                 // rows see few tokens
    bool sums;                // forward: the weights' own sums too, for the backward's P and for joining parts
};

// Workgroups go around the chip's 8 dies: a run of neighbours, which read the same keys, on one of them.
__device__ __forceinline__ int block_of(int n) {
    const int per = (n + 7) / 8;
    return (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
}

// Whether token j is visible to the query at position p.  Without branches: selections of single registers of a
// matrix tile by control flow have come out wrong (the compiler lost the copy of a branch's tile), and cost more.
__device__ __forceinline__ bool visible(const WinArgs& a, int j, int p) {
    return ((uint32_t)(p - j) < (uint32_t)a.W) | ((j <= p) & (j < a.sinks));
}

// C tiles U from tokens j0 on, of the query at p: what it does not see is set to `none`.
template <int U>
__device__ __forceinline__ void hide(const WinArgs& a, f32x16 (&s)[U], int j0, int p, int h, float none) {
    const int d = p - j0 - 4 * h;
    if (j0 < a.sinks) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[u][r] = visible(a, j0 + 32 * u + 8 * (r / 4) + 4 * h + r % 4, p) ? s[u][r] : none;
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[u][r] = (uint32_t)(d - (32 * u + 8 * (r / 4) + r % 4)) < (uint32_t)a.W ? s[u][r] : none;
    }
}

__device__ __forceinline__ int end_of(const WinArgs& a, int b) {
    return a.len ? min(max(a.len[b], 0), a.Tk) : a.Tk;
}

// A tile of TT rows from row r0 on of `rows` into LDS, by the four waves; rows past them are zero.
template <typename E, int D, int TT>
struct Loader {
    using R = Rows<E, D>;
    static constexpr int N = TT * R::NC / 64 / 4;   // loads a wave
    uint32_t off[N];
    uint32_t stride;
    __device__ Loader(uint32_t stride, int wave, int lane) : stride(stride) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int x = (i * 4 + wave) * 64 + lane, r = x / R::NC, c = (x % R::NC) ^ R::key(r);
            off[i] = c < R::NR ? r * stride + c * 16 : 0x80000000u;
        }
    }
    __device__ void load(const void* base, int r0, int rows, uint32_t dst, int wave) const {
        const uintptr_t p = reinterpret_cast<uintptr_t>(base) + (size_t)r0 * stride;
        const int n = min(rows - r0, TT);
        const words_t rs{(uint32_t)p, (uint32_t)(p >> 32) & 0xffffu, n > 0 ? (uint32_t)(n - 1) * stride + D * (uint32_t)sizeof(E) : 0u,
                         0x00020000u};
#pragma unroll
        for (int i = 0; i < N; ++i) load_lds(rs, dst + (uint32_t)(i * 4 + wave) * R::UNIT, off[i]);
    }
};

__device__ __forceinline__ uint32_t lds_of(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)p;
}

__device__ __forceinline__ void store4(uint16_t* p, const float (&x)[4], int8_t* rest) {
    const uint2 y{cvt_pk_bf16(x[0], x[1]), cvt_pk_bf16(x[2], x[3])};
    *reinterpret_cast<uint2*>(p) = y;
    if (rest) *reinterpret_cast<uint32_t*>(rest) = rest_of(x, y);
}
__device__ __forceinline__ void store4(float* p, const float (&x)[4], int8_t*) {
    *reinterpret_cast<float4*>(p) = float4{x[0], x[1], x[2], x[3]};
}

// A lane's column of a C over columns 32 t + 8 (r / 4) + 4 h + r % 4 of row p, 16 bytes at a time.
template <typename E, int D>
__device__ __forceinline__ void store_row(E* p, const Acc<E, D>& o, float f, int h, int8_t* rest = nullptr) {
#pragma unroll
    for (int t = 0; t < Rows<E, D>::DP / 32; ++t)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            if (32 * t + 8 * j >= D) continue;
            float x[2][4];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i / 4][i % 4] = o[t][4 * j + i] * f;
            if constexpr (sizeof(E) == 4) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    *reinterpret_cast<float4*>(p + 32 * t + 8 * (j + i) + 4 * h) = float4{x[i][0], x[i][1], x[i][2], x[i][3]};
            } else {   // the lower half takes both halves' columns of j, the upper one those of j + 1
                const uint2 y[2] = {{cvt_pk_bf16(x[0][0], x[0][1]), cvt_pk_bf16(x[0][2], x[0][3])},
                                    {cvt_pk_bf16(x[1][0], x[1][1]), cvt_pk_bf16(x[1][2], x[1][3])}};
                const auto a = __builtin_amdgcn_permlane32_swap(y[0].x, y[1].x, false, false);
                const auto b = __builtin_amdgcn_permlane32_swap(y[0].y, y[1].y, false, false);
                const int col = 32 * t + 8 * (j + h);
                *reinterpret_cast<uint4*>(p + col) = uint4{a[0], b[0], a[1], b[1]};
                if (rest) {
                    const auto r = __builtin_amdgcn_permlane32_swap(rest_of(x[0], y[0]), rest_of(x[1], y[1]), false, false);
                    *reinterpret_cast<uint2*>(rest + col) = uint2{r[0], r[1]};
                }
            }
        }
}
template <typename E, int D>
__device__ __forceinline__ void store_zero(E* p, int h) {
#pragma unroll
    for (int c = 0; c < D * (int)sizeof(E) / 32; ++c) reinterpret_cast<uint4*>(p)[2 * c + h] = uint4{0, 0, 0, 0};
}

// How a pass (forward, dq, or dk and dv) goes over its tiles: TT tokens (queries for dk, dv) a tile, NB tiles in LDS
// (one worked on, the others on their way), U halves of 32 at once, WAVES a SIMD.  At 128 bf16 columns tiles of 32
// leave the forward registers for three waves a SIMD (B8 T2048 H16 window 512: with tiles of 64 and two waves 13% more;
// three tiles in LDS instead of two gain nothing there); of its 168 the walk without masked places stores five.  fp32: as
// many waves as registers allow (B64 T512 H4 d32: forward 40 us, 50 with one a SIMD).
enum Pass { kFwd, kDq, kDkv };
template <typename E, int D, Pass P>
struct Geo {
    static constexpr bool BF = sizeof(E) == 2;
    static constexpr int TT = Rows<E, D>::NC < 8 || (BF ? D < 128 : D < 64 || (D == 128 && P != kFwd)) ? 64 : 32;
    static constexpr int U = BF && P != kDkv ? TT / 32 : 1;
    static constexpr int PAIR = 2 * Rows<E, D>::bytes(TT);
    static constexpr int WAVES = !BF ? (D < 128 ? 2 : 1) : D == 128 && P == kFwd ? 3 : 2;
    static constexpr int NB = BF && D < 128 && P != kFwd ? 3 : 2;
    // dk, dv at 128 bf16 columns: the tokens' keys stay in LDS; with them in registers, beside their values and both
    // sums, some of each were stored and loaded again around every tile (backward 447 us, 390 with the keys in LDS).
    static constexpr bool KEYS = BF && D == 128 && P == kDkv;
};

template <typename E, int D, Pass P>
struct Shared {
    using G = Geo<E, D, P>;
    alignas(16) unsigned char tile[G::NB][G::PAIR];   // of keys and values, or of queries and dy
    alignas(16) float row[P == kDkv ? G::NB : 1][3][P == kDkv ? G::TT : 1];   // the queries' m, 1 / l, D
    alignas(16) unsigned char keys[G::KEYS ? Rows<E, D>::bytes(kRows) : 16];
    float scratch[4][128];
    int flag;
};

// Before tile i of n: waits until it is there, L loads a tile and wave, the tiles up to NB - 2 after it under way.
template <int NB, int L>
__device__ __forceinline__ void wait_tile(int i, int n) {
    if (i + NB - 2 < n)
        wait_vm_le<(NB - 2) * L>();
    else
        wait_vm_all();
    barrier_lds();
}

// The tiles that a workgroup of queries p0 .. p1 reads: the window's, after the first tokens' where they lie apart.
template <int TT>
struct Tiles {
    int t0, n;
    int first;
    __device__ Tiles(const WinArgs& a, int p0, int p1) {
        t0 = max(0, p0 - a.W + 1) / TT;
        first = min(t0, (a.sinks + TT - 1) / TT);   // tiles before it that hold first tokens
        n = p1 / TT - t0 + 1 + first;
    }
    __device__ int operator[](int i) const { return i < first ? i : t0 + i - first; }
};

// TWO: weights enter in two parts.
template <typename E, int D, bool TWO>
__device__ __forceinline__ void win_fwd(const WinArgs& a, Shared<E, D, kFwd>& sh, int split, int qb, int head, int b) {
    using R = Rows<E, D>;
    using G = Geo<E, D, kFwd>;
    constexpr int DT = R::DP / 32, TT = G::TT, NB = G::NB, BYTES = R::bytes(TT);
    constexpr bool ROUNDED = sizeof(E) == 2 && !TWO;   // y is divided by the sum of the weights as they entered
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, l32 = lane % 32, h = lane / 32;
    const int kh = head / (a.H / a.Hk), past = a.Tk - a.T, end = end_of(a, b);
    const int q0 = qb * kRows, p0 = past + q0, p1 = min(past + min(q0 + kRows, a.T), end) - 1;
    const int qi = q0 + 32 * wave + l32, pos = past + qi;
    const bool live = qi < a.T && pos < end;
    const size_t row = ((size_t)b * a.T + min(qi, a.T - 1)) * a.H + head;
    const uint32_t stride = (uint32_t)(a.Hk * D * (int)sizeof(E));
    const E* kb = (const E*)a.k + ((size_t)b * a.Tk * a.Hk + kh) * D;
    const E* vb = (const E*)a.v + ((size_t)b * a.Tk * a.Hk + kh) * D;

    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = zero16();
    float mc = -INFINITY, l = 0.f, lr = 0.f;   // the exponents' reference, the lane's shares of the sum and of that as rounded
    if (p1 >= p0) {
        const Tiles<TT> tiles(a, p0, p1);
        const int per = (tiles.n + a.nsplit - 1) / a.nsplit, i0 = split * per, i1 = min(i0 + per, tiles.n);
        const Loader<E, D, TT> ld(stride, wave, lane);
        const uint32_t lds0 = lds_of(sh.tile);
        int into = 0;   // the place of the next tile
        auto issue = [&](int i) {
            const int r0 = tiles[i] * TT;
            const uint32_t to = lds0 + (uint32_t)into * 2 * BYTES;
            into = into + 1 < NB ? into + 1 : 0;
            ld.load(kb, r0, end, to, wave);
            ld.load(vb, r0, end, to + BYTES, wave);
        };
        Row<E, D> q;
        q.load((const E*)a.q + row * D, live, h);
        const int w0 = p0 + 32 * wave, w1 = min(w0 + 31, p1);   // the wave's positions
        // U: 32 tokens each at once, from u0 on
        auto step = [&](auto careful, bool masked, const unsigned char* K, int u0, int j0) {
            constexpr bool CAREFUL = decltype(careful)::value;
            constexpr int U = CAREFUL ? 1 : G::U;
            const unsigned char* V = K + BYTES;
            f32x16 s[U];
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] = rows_dot<D>(K, u0 + 32 * u, q, l32, h);
            if (masked) hide<U>(a, s, j0, pos, h, -INFINITY);
            float top = s[0][0];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
            top = halves_max(top) * a.c;
            if (__any(top > mc)) {
                const float now = top > mc ? ceilf(top) + kAhead : mc, f = now == -INFINITY ? 0.f : exp2_hw(mc - now);
                mc = now;
                l *= f;
                lr *= f;
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[t][r] *= f;
            }
            const float base = mc == -INFINITY ? 0.f : mc;   // nothing visible yet: weights 2^-inf
            float sum[4] = {l, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[u][r] = exp2_hw(fmaf(s[u][r], a.c, -base));
                    if (CAREFUL || !ROUNDED) sum[r % 4] += s[u][r];
                }
            if constexpr (!CAREFUL && ROUNDED) {
                if (a.sums) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int r = 0; r < 16; ++r) sum[r % 4] += s[u][r];
                }
            }
            if constexpr (CAREFUL) hide<U>(a, s, j0, pos, h, __uint_as_float(kMasked));
            l = (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
            for (int u = 0; u < U; ++u) add_cols<CAREFUL, TWO, E, D>(o, V, u0 + 32 * u, s[u], sh.scratch[wave], l32, h, &lr);
            if constexpr (CAREFUL || !ROUNDED) lr = l;
        };
        auto walk = [&](auto careful) {
            constexpr bool CAREFUL = decltype(careful)::value;
            constexpr int US = CAREFUL ? 32 : 32 * G::U;
            into = 0;
            for (int i = i0; i < min(i0 + NB - 1, i1); ++i) issue(i);
            int at = 0;
            for (int i = i0; i < i1; ++i) {
                wait_tile<NB, 2 * Loader<E, D, TT>::N>(i, i1);
                if (i + NB - 1 < i1) issue(i + NB - 1);
                const unsigned char* K = sh.tile[at];
                at = at + 1 < NB ? at + 1 : 0;
#pragma unroll 1
                for (int u0 = 0; u0 < TT; u0 += US) {
                    const int j0 = tiles[i] * TT + u0;
                    if (j0 > w1 || w1 < w0 || (j0 + US - 1 <= w0 - a.W && j0 >= a.sinks)) continue;
                    step(careful, j0 + US - 1 > w0 || j0 <= w1 - a.W, K, u0, j0);
                }
            }
        };
        walk(std::false_type{});
        if (any_of(live && !finite(o), &sh.flag)) {
            mc = -INFINITY, l = lr = 0.f;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] = zero16();
            walk(std::true_type{});
        }
        l = sum_of(halves_sum(l), mc);
        lr = ROUNDED ? sum_of(halves_sum(lr), mc) : l;
        if (ROUNDED && !a.sums) l = lr;
    }
    if (qi >= a.T) return;
    if (a.nsplit > 1) {
        const size_t at = (size_t)split * a.B * a.T * a.H + row;
        if (!live) l = 0.f, mc = -INFINITY;
        if (live) store_row<float, D>(a.part + at * D, o, ROUNDED ? l / lr : 1.f, h);
        if (h == 0) a.pstat[at] = float2{mc, l};
        return;
    }
    E* y = (E*)a.o + row * D;
    if (live && l != 0.f)
        store_row<E, D>(y, o, 1.f / lr, h, a.rest ? a.rest + row * D : nullptr);
    else
        store_zero<E, D>(y, h);
    if (a.stat && h == 0) a.stat[row] = context(mc, live ? l : 0.f);
}

// Workgroup id's block of queries, head and sequence.  Heads that share keys go side by side, then blocks in order, where
// the window makes most alike, since they read on in the tiles that the last ones left in L2 (B1 T65536 H16 Hk4 window
// 2048: head after head takes 6% more, the blocks backwards 10%), or the longest first where they are not alike (B2
// T4096 window 4096: 179 us, in order 191).
__device__ __forceinline__ void place_of(const WinArgs& a, int id, int& qb, int& head, int& b) {
    const int nq = (a.T + kRows - 1) / kRows, G = a.H / a.Hk, at = id / G % nq, rest = id / G / nq;
    qb = 2 * (int64_t)a.W > a.T ? nq - 1 - at : at;
    head = rest % a.Hk * G + id % G;
    b = rest / a.Hk;
}

template <typename E, int D>
__global__ __launch_bounds__(256, (Geo<E, D, kFwd>::WAVES)) void win_fwd_kernel(WinArgs a) {
    __shared__ Shared<E, D, kFwd> sh;
    int id = block_of(a.blocks);
    if (id >= a.blocks) return;
    const int split = id % a.nsplit;
    id /= a.nsplit;
    int qb, head, b;
    place_of(a, id, qb, head, b);
    if (sizeof(E) == 2 && (a.few || a.Tk - a.T + qb * kRows < kRows))
        win_fwd<E, D, sizeof(E) == 2>(a, sh, split, qb, head, b);
    else
        win_fwd<E, D, false>(a, sh, split, qb, head, b);
}

// Joins nsplit (at most 64) partial rows: y = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  Four columns a thread,
// for many rows.
template <typename E, int D>
__global__ __launch_bounds__(256) void win_join_rows_kernel(size_t rows, int nsplit, const float* __restrict__ part,
                                                            const float2* __restrict__ pstat, E* __restrict__ y,
                                                            float2* __restrict__ stat, int8_t* __restrict__ rest) {
    const size_t x = (size_t)blockIdx.x * 256 + threadIdx.x, row = x / (D / 4);
    const int col = (int)(x % (D / 4)) * 4;
    if (row >= rows) return;
    float m = -INFINITY;
#pragma unroll 4
    for (int s = 0; s < nsplit; ++s) m = fmaxf(m, pstat[s * rows + row].x);
    float l = 0.f;
    f32x4 o = zero4();
#pragma unroll 2
    for (int s = 0; s < nsplit; ++s) {
        const float2 st = pstat[s * rows + row];
        if (st.y == 0.f) continue;   // a row that is not there, or saw nothing: its part was not written
        const float f = exp2_hw(st.x - m);
        l = fmaf(f, st.y, l);
        const f32x4 p = *reinterpret_cast<const f32x4*>(part + (s * rows + row) * D + col);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(f, p[e], o[e]);
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const float x4[4] = {o[0] * f, o[1] * f, o[2] * f, o[3] * f};
    store4(y + row * D + col, x4, rest ? rest + row * D + col : nullptr);
    if (stat && col == 0) stat[row] = context(m, l);
}

// The same for few rows, a workgroup each: its lanes read the parts' m and l at once, its column groups the parts' O,
// eight at once: two readings after another (one sequence's token over 4100 slots in 32 parts: 3.4 us where the one
// above takes 12.9).
template <typename E, int D>
__global__ __launch_bounds__(2 * D) void win_join_kernel(size_t rows, int nsplit, const float* __restrict__ part,
                                                         const float2* __restrict__ pstat, E* __restrict__ y,
                                                         float2* __restrict__ stat, int8_t* __restrict__ rest) {
    constexpr int G = D / 4;   // column groups
    __shared__ float f[64];
    __shared__ f32x4 sum[8][G];
    __shared__ float2 ml;
    const size_t row = blockIdx.x;
    const int c = threadIdx.x % G, part0 = threadIdx.x / G;
    if (threadIdx.x < 64) {   // fewer threads than 64 (D = 16): each lane takes several parts
        const int n = 2 * D < 64 ? 2 * D : 64;
        float m = -INFINITY, l = 0.f;
        for (int s = threadIdx.x; s < nsplit; s += n) m = fmaxf(m, pstat[s * rows + row].x);
        for (int x = n / 2; x > 0; x /= 2) m = fmaxf(m, __shfl_xor(m, x));
        for (int s = threadIdx.x; s < nsplit; s += n) {
            const float2 st = pstat[s * rows + row];
            const float e = st.y == 0.f ? 0.f : exp2_hw(st.x - m);
            f[s] = e;
            if (st.y != 0.f) l = fmaf(e, st.y, l);
        }
        for (int x = n / 2; x > 0; x /= 2) l += __shfl_xor(l, x);
        if (threadIdx.x == 0) ml = float2{m, l};
    }
    __syncthreads();
    f32x4 o = zero4();
    for (int s = part0; s < nsplit; s += 8) {
        const float e = f[s];
        if (e == 0.f) continue;   // rows that are not there, or saw nothing
        const f32x4 p = *reinterpret_cast<const f32x4*>(part + (s * rows + row) * D + 4 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(e, p[i], o[i]);
    }
    sum[part0][c] = o;
    __syncthreads();
    if (part0 > 0) return;
#pragma unroll
    for (int s = 1; s < 8; ++s) o += sum[s][c];
    const float m = ml.x, l = ml.y, r = l == 0.f ? 0.f : 1.f / l;
    const float x[4] = {o[0] * r, o[1] * r, o[2] * r, o[3] * r};
    store4(y + row * D + 4 * c, x, rest ? rest + row * D + 4 * c : nullptr);
    if (stat && c == 0) stat[row] = context(m, l);
}

// The ring caches after the last token of each sequence: slot < sinks holds that token, slot sinks + x the last
// token t >= sinks with (t - sinks) mod W = x; slots without a token are zero.  16 bytes a thread.
template <typename E, int D>
__global__ __launch_bounds__(256) void win_cache_kernel(WinArgs a, uint4* __restrict__ ck, uint4* __restrict__ cv) {
    const int per = a.Hk * D * (int)sizeof(E) / 16, slots = a.sinks + a.W;
    const size_t n = (size_t)a.B * slots * per;
    for (size_t x = (size_t)blockIdx.x * 256 + threadIdx.x; x < n; x += (size_t)gridDim.x * 256) {
        const int c = (int)(x % per), slot = (int)(x / per % slots), b = (int)(x / per / slots), end = end_of(a, b);
        int tok = slot;
        if (slot >= a.sinks && end - 1 > slot) tok = end - 1 - (end - 1 - slot) % a.W;
        const bool held = tok < end;
        const size_t at = ((size_t)b * a.Tk + (held ? tok : 0)) * per + c;
        ck[x] = held ? ((const uint4*)a.k)[at] : uint4{0, 0, 0, 0};
        cv[x] = held ? ((const uint4*)a.v)[at] : uint4{0, 0, 0, 0};
    }
}

template <typename E, int D, bool TWO>
__device__ __forceinline__ void win_dq(const WinArgs& a, Shared<E, D, kDq>& sh, int qb, int head, int b) {
    using R = Rows<E, D>;
    using G = Geo<E, D, kDq>;
    constexpr int DT = R::DP / 32, TT = G::TT, NB = G::NB, BYTES = R::bytes(TT);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, l32 = lane % 32, h = lane / 32;
    const int kh = head / (a.H / a.Hk), past = a.Tk - a.T, end = end_of(a, b);
    const int q0 = qb * kRows, p0 = past + q0, p1 = min(past + min(q0 + kRows, a.T), end) - 1;
    const int qi = q0 + 32 * wave + l32, pos = past + qi;
    const bool live = qi < a.T && pos < end;
    const size_t row = ((size_t)b * a.T + min(qi, a.T - 1)) * a.H + head;
    const uint32_t stride = (uint32_t)(a.Hk * D * (int)sizeof(E));
    const E* kb = (const E*)a.k + ((size_t)b * a.Tk * a.Hk + kh) * D;
    const E* vb = (const E*)a.v + ((size_t)b * a.Tk * a.Hk + kh) * D;
    E* dq = (E*)a.dq + row * D;
    const size_t nrow = (size_t)a.B * a.H * a.T64, at = ((size_t)b * a.H + head) * a.T64 + qi;

    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = zero16();
    bool scored = false;   // a row without a score has no gradient
    if (p1 >= p0) {
        const Tiles<TT> tiles(a, p0, p1);
        const Loader<E, D, TT> ld(stride, wave, lane);
        const uint32_t lds0 = lds_of(sh.tile);
        int into = 0;   // the place of the next tile
        auto issue = [&](int i) {
            const int r0 = tiles[i] * TT;
            const uint32_t to = lds0 + (uint32_t)into * 2 * BYTES;
            into = into + 1 < NB ? into + 1 : 0;
            ld.load(kb, r0, end, to, wave);
            ld.load(vb, r0, end, to + BYTES, wave);
        };
        Row<E, D> q, g;
        q.load((const E*)a.q + row * D, live, h);
        g.load((const E*)a.dy + row * D, live, h);
        const float2 st = live ? a.stat[row] : float2{0.f, 0.f};
        scored = st.y != 0.f;
        float Dq;
        {
            Row<E, D> y;
            y.load((const E*)a.y + row * D, live, h);
            Dq = g.dot(y, scored ? a.rest + row * D : nullptr, h);   // other rows' y are zeros, with no rest
            Dq = halves_sum(Dq);
        }
        const float li = scored ? 1.f / st.y : 0.f, Dl = Dq * li;
        if (h == 0 && qi < a.T64) {
            a.rows[at] = st.x;
            a.rows[nrow + at] = li;
            a.rows[2 * nrow + at] = Dq;
        }
        const int w0 = p0 + 32 * wave, w1 = min(w0 + 31, p1);
        // U: 32 tokens each at once, from u0 on
        auto step = [&](auto careful, bool masked, const unsigned char* K, int u0, int j0) {
            constexpr bool CAREFUL = decltype(careful)::value;
            constexpr int U = CAREFUL ? 1 : G::U;
            const unsigned char* V = K + BYTES;
            f32x16 s[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                f32x16 dp;
                rows_dot_two<D>(K, V, u0 + 32 * u, q, g, s[u], dp, l32, h);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[u][r] = exp2_hw(fmaf(s[u][r], a.c, -st.x)) * fmaf(dp[r], li, -Dl);
                    if constexpr (CAREFUL) s[u][r] = seen(s[u][r]);
                }
            }
            if (masked) hide<U>(a, s, j0, pos, h, __uint_as_float(kMasked));
#pragma unroll
            for (int u = 0; u < U; ++u) add_cols<CAREFUL, TWO, E, D>(o, K, u0 + 32 * u, s[u], sh.scratch[wave], l32, h);
        };
        auto walk = [&](auto careful) {
            constexpr bool CAREFUL = decltype(careful)::value;
            constexpr int US = CAREFUL ? 32 : 32 * G::U;
            into = 0;
            for (int i = 0; i < min(NB - 1, tiles.n); ++i) issue(i);
            int at = 0;
            for (int i = 0; i < tiles.n; ++i) {
                wait_tile<NB, 2 * Loader<E, D, TT>::N>(i, tiles.n);
                if (i + NB - 1 < tiles.n) issue(i + NB - 1);
                const unsigned char* K = sh.tile[at];
                at = at + 1 < NB ? at + 1 : 0;
#pragma unroll 1
                for (int u0 = 0; u0 < TT; u0 += US) {
                    const int j0 = tiles[i] * TT + u0;
                    if (j0 > w1 || w1 < w0 || (j0 + US - 1 <= w0 - a.W && j0 >= a.sinks)) continue;
                    step(careful, j0 + US - 1 > w0 || j0 <= w1 - a.W, K, u0, j0);
                }
            }
        };
        walk(std::false_type{});
        if (any_of(scored && !finite(o), &sh.flag)) {
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] = zero16();
            walk(std::true_type{});
        }
    } else if (h == 0 && qi < a.T64) {
        a.rows[at] = a.rows[nrow + at] = a.rows[2 * nrow + at] = 0.f;
    }
    if (qi >= a.T) return;
    if (scored)
        store_row<E, D>(dq, o, a.scale, h);
    else
        store_zero<E, D>(dq, h);
}

template <typename E, int D>
__global__ __launch_bounds__(256, (Geo<E, D, kDq>::WAVES)) void win_dq_kernel(WinArgs a) {
    __shared__ Shared<E, D, kDq> sh;
    const int id = block_of(a.blocks);
    if (id >= a.blocks) return;
    int qb, head, b;
    place_of(a, id, qb, head, b);
    if (sizeof(E) == 2 && (a.few || a.Tk - a.T + qb * kRows < kRows))
        win_dq<E, D, sizeof(E) == 2>(a, sh, qb, head, b);
    else
        win_dq<E, D, false>(a, sh, qb, head, b);
}

// dk, dv.  Workgroup (b, kh, kb, split): 128 tokens and a share of the queries that see them; after those, nseg segments
// of the queries behind the first 128 tokens' window for each (b, kh), whose waves take (32 of the first tokens, every
// second 32 queries).
template <typename E, int D, bool TWO>
__device__ __forceinline__ void win_dkv(const WinArgs& a, Shared<E, D, kDkv>& sh, int job, int split, int nk, int bk, int kh, int b) {
    using R = Rows<E, D>;
    using Gm = Geo<E, D, kDkv>;
    constexpr int DT = R::DP / 32, TT = Gm::TT, NB = Gm::NB, BYTES = R::bytes(TT);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, l32 = lane % 32, h = lane / 32;
    const bool seg = job >= nk;
    const int k0 = seg ? 0 : job * kRows, w0 = k0 + 32 * (seg ? wave / 2 : wave);   // the wave's first token
    const int G = a.H / a.Hk, past = a.Tk - a.T, end = end_of(a, b);
    const int tok = w0 + l32;
    const bool live = tok < end;
    // positions of the queries: those that the window reaches, or a segment of those behind
    const int behind = max(past, kRows - 1 + min(a.W, a.Tk));
    const int plo = seg ? behind + (job - nk) * a.seg : max(past, k0);
    const int phi = min(seg ? plo + a.seg - 1 : k0 + kRows - 2 + min(a.W, a.Tk), end - 1);
    const bool works = !seg || w0 < a.sinks;

    f32x16 ok[DT], ov[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) ok[t] = ov[t] = zero16();
    if (phi >= plo) {
        const size_t krow = ((size_t)b * a.Tk + min(tok, a.Tk - 1)) * a.Hk + kh;
        const uint32_t stride = (uint32_t)(a.H * D * (int)sizeof(E));
        const Loader<E, D, TT> ld(stride, wave, lane);
        const uint32_t lds0 = lds_of(sh.tile), row0 = lds_of(sh.row);
        const int t0 = (plo - past) / TT, nt = (phi - past) / TT - t0 + 1, all = nt * G;
        // this workgroup's n of all tiles, from i0 on
        const int share = seg ? all : (all + a.ksplit - 1) / a.ksplit, i0 = seg ? 0 : min(split * share, all), n = min(share, all - i0);
        const size_t nrow = (size_t)a.B * a.H * a.T64;
        int into, next_t, next_h;   // the next tile: its place, its queries and head
        auto issue = [&]() {
            const int r0 = next_t * TT;
            const uint32_t to = lds0 + (uint32_t)into * 2 * BYTES;
            const size_t first = ((size_t)b * a.T * a.H + next_h) * D;
            ld.load((const E*)a.q + first, r0, end - past, to, wave);
            ld.load((const E*)a.dy + first, r0, end - past, to + BYTES, wave);
            // m, 1 / l or D of the tile's rows, 16 bytes a lane; the fourth wave as the third
            const int of = min(wave, 2);
            const uintptr_t p = reinterpret_cast<uintptr_t>(a.rows + of * nrow + ((size_t)b * a.H + next_h) * a.T64 + r0);
            const words_t rs{(uint32_t)p, (uint32_t)(p >> 32) & 0xffffu, TT * 4u, 0x00020000u};
            if (lane < TT / 4) load_lds(rs, row0 + (uint32_t)(into * 3 + of) * TT * 4, (uint32_t)lane * 16);
            into = into + 1 < NB ? into + 1 : 0;
            if (++next_t == t0 + nt) next_t = t0, ++next_h;
        };
        std::conditional_t<Gm::KEYS, RowsAt, Row<E, D>> k;
        Row<E, D> v;
        v.load((const E*)a.v + krow * D, live, h);
        if constexpr (Gm::KEYS) {
            const Loader<E, D, kRows> lk((uint32_t)(a.Hk * D * (int)sizeof(E)), wave, lane);
            lk.load((const E*)a.k + ((size_t)b * a.Tk * a.Hk + kh) * D, k0, end, lds_of(sh.keys), wave);
            k.p = sh.keys + R::row(w0 - k0);
        } else {
            k.load((const E*)a.k + krow * D, live, h);
        }
        auto walk = [&](auto careful) {
            constexpr bool CAREFUL = decltype(careful)::value;
            into = 0, next_t = t0 + i0 % nt, next_h = kh * G + i0 / nt;
            int at = 0, tile = next_t;
            for (int i = 0; i < min(NB - 1, n); ++i) issue();
            for (int i = 0; i < n; ++i) {
                wait_tile<NB, 2 * Loader<E, D, TT>::N + 1>(i, n);
                if (i + NB - 1 < n) issue();
                const unsigned char *Q = sh.tile[at], *G_ = Q + BYTES;
                const float* rows = &sh.row[at][0][0];
                const int pt = past + tile * TT;
                at = at + 1 < NB ? at + 1 : 0;
                tile = tile + 1 < t0 + nt ? tile + 1 : t0;
#pragma unroll 1
                for (int u = 0; u < TT / 32; ++u) {
                    const int pp = pt + 32 * u;   // the rows' first position
                    if (!works || (seg && (pp / 32 & 1) != wave % 2) || pp + 31 < max(w0, plo) || pp > phi ||
                        (pp - a.W >= w0 + 31 && w0 >= a.sinks))
                        continue;
                    const bool masked = pp < w0 + 31 || pp + 31 - a.W >= w0 || pp < plo || pp + 31 > phi;
                    f32x16 s, ds;
                    rows_dot_two<D>(Q, G_, 32 * u, k, v, s, ds, l32, h);
                    const float* sr = rows + 32 * u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f32x4 m = *reinterpret_cast<const f32x4*>(sr + 8 * j + 4 * h);
                        const f32x4 li = *reinterpret_cast<const f32x4*>(sr + TT + 8 * j + 4 * h);
                        const f32x4 Dq = *reinterpret_cast<const f32x4*>(sr + 2 * TT + 8 * j + 4 * h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[4 * j + e] = exp2_hw(fmaf(s[4 * j + e], a.c, -m[e])) * li[e];
                            // rows without a score, whose q or dy may be infinite, take no part
                            if constexpr (CAREFUL) s[4 * j + e] = li[e] == 0.f ? __uint_as_float(kMasked) : s[4 * j + e];
                            ds[4 * j + e] -= Dq[e];
                        }
                    }
                    if (masked) {
                        const int d = pp + 4 * h - tok;
                        if (w0 < a.sinks || pp < plo || pp + 31 > phi) {
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const int p = pp + 8 * (r / 4) + 4 * h + r % 4;
                                s[r] = (visible(a, tok, p) & (p >= plo) & (p <= phi)) ? s[r] : __uint_as_float(kMasked);
                            }
                        } else {
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                s[r] = (uint32_t)(d + 8 * (r / 4) + r % 4) < (uint32_t)a.W ? s[r] : __uint_as_float(kMasked);
                        }
                    }
                    add_cols<CAREFUL, TWO, E, D>(ov, G_, 32 * u, s, sh.scratch[wave], l32, h);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        if constexpr (CAREFUL)
                            ds[r] = __float_as_uint(s[r]) == kMasked ? s[r] : seen(s[r] * ds[r]);
                        else
                            ds[r] *= s[r];
                    }
                    add_cols<CAREFUL, TWO, E, D>(ok, Q, 32 * u, ds, sh.scratch[wave], l32, h);
                }
            }
        };
        walk(std::false_type{});
        if (any_of(live && !(finite(ok) && finite(ov)), &sh.flag)) {
#pragma unroll
            for (int t = 0; t < DT; ++t) ok[t] = ov[t] = zero16();
            walk(std::true_type{});
        }
    }
    if (a.nseg > 0 && (seg || (a.ksplit == 1 && k0 == 0)) && w0 < a.sinks) {   // the first tokens' sums: slot 0 the window's, 1 + 2 s + (0, 1) a segment's
        const int slot = seg ? 1 + 2 * (job - nk) + wave % 2 : 0;
        if (tok < a.sinks) {
            float* p = a.part + (((size_t)bk * (1 + 2 * a.nseg) + slot) * 2 * a.sinks + tok) * D;
            store_row<float, D>(p, ok, a.scale, h);
            store_row<float, D>(p + (size_t)a.sinks * D, ov, 1.f, h);
        }
        if (tok < a.sinks) return;
    }
    if (seg || tok >= a.Tk) return;
    if (a.ksplit > 1) {
        float* p = a.kpart + ((((size_t)bk * a.ksplit + split) * 2) * a.Tk + tok) * D;
        store_row<float, D>(p, ok, a.scale, h);
        store_row<float, D>(p + (size_t)a.Tk * D, ov, 1.f, h);
        return;
    }
    const size_t krow = ((size_t)b * a.Tk + tok) * a.Hk + kh;
    E *dk = (E*)a.dk + krow * D, *dv = (E*)a.dv + krow * D;
    if (live) {
        store_row<E, D>(dk, ok, a.scale, h);
        store_row<E, D>(dv, ov, 1.f, h);
    } else {
        store_zero<E, D>(dk, h);
        store_zero<E, D>(dv, h);
    }
}

template <typename E, int D>
__global__ __launch_bounds__(256, (Geo<E, D, kDkv>::WAVES)) void win_dkv_kernel(WinArgs a) {
    __shared__ Shared<E, D, kDkv> sh;
    const int id = block_of(a.blocks);
    if (id >= a.blocks) return;
    const int nk = (a.Tk + kRows - 1) / kRows, per = nk * a.ksplit + a.nseg;
    const int at = id % per, bk = id / per, kh = bk % a.Hk, b = bk / a.Hk;
    const int job = at < nk * a.ksplit ? at / a.ksplit : at - nk * (a.ksplit - 1), split = at % a.ksplit;
    // the first rows' queries are those of the first 128 tokens' workgroup
    if (sizeof(E) == 2 && (a.few || (job == 0 && a.Tk - a.T < kRows)))
        win_dkv<E, D, sizeof(E) == 2>(a, sh, job, split, nk, bk, kh, b);
    else
        win_dkv<E, D, false>(a, sh, job, split, nk, bk, kh, b);
}

// dk, dv from their parts, added up in order, four columns a thread: of the first n tokens, or of all where the
// queries were dealt to several workgroups.
template <typename E, int D>
__global__ __launch_bounds__(256) void win_sum_kernel(WinArgs a, int n) {
    const int slots = 1 + 2 * a.nseg;
    const size_t total = (size_t)a.B * a.Hk * 2 * n * (D / 4);
    for (size_t x = (size_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (size_t)gridDim.x * 256) {
        const int col = (int)(x % (D / 4)) * 4, tok = (int)(x / (D / 4) % n), of = (int)(x / (D / 4) / n % 2);
        const int bk = (int)(x / (D / 4) / n / 2), kh = bk % a.Hk, b = bk / a.Hk;
        f32x4 s = zero4();
        if (a.ksplit > 1)
#pragma unroll 4
            for (int i = 0; i < a.ksplit; ++i)
                s += *reinterpret_cast<const f32x4*>(a.kpart + ((((size_t)bk * a.ksplit + i) * 2 + of) * a.Tk + tok) * D + col);
        if (a.nseg > 0 && tok < a.sinks)
#pragma unroll 4
            for (int i = a.ksplit > 1 ? 1 : 0; i < slots; ++i)
                s += *reinterpret_cast<const f32x4*>(a.part + ((((size_t)bk * slots + i) * 2 + of) * a.sinks + tok) * D + col);
        const float f[4] = {s[0], s[1], s[2], s[3]};
        store4((E*)(of ? a.dv : a.dk) + (((size_t)b * a.Tk + tok) * a.Hk + kh) * D + col, f, nullptr);
    }
}

// ---------------------------------------------------------------- one token for S sequences

struct StepArgs {
    const void *q, *k, *v;
    void *ck, *cv, *y;
    const int* pos;
    float* part;
    float2* pstat;
    int S, H, Hk, W, sinks, blocks, nsplit, groups;
    float c;
};

// Workgroup (s, kh, 16 query heads, split): its waves take chunks of 32 (fp32: 16) slots in turn and join at the
// end.  K goes from memory straight into operands, V through LDS of the wave's own, to be read across.
// S^T = K Q^T (slots x heads) in 16 x 16 tiles, O^T += V^T P^T.  bf16 rounds P, and the sum takes what it rounds to;
// in two parts registers were stored and loaded again (512 sequences 223 us, 191 this way).  HBM bounds it: the next chunk's keys and values are
// asked for as soon as the registers of this one's are free, and three waves a SIMD (168 registers) keep enough on
// their way.  With two chunks in registers instead they were stored and loaded again: 318 us for 512 sequences over
// 1028 slots of 4 heads of 128, 191 this way.
template <typename E, int D>
struct StepCfg {
    static constexpr int CH = sizeof(E) == 2 ? 32 : 16, DT = D / 16;
    static constexpr int NC = D * (int)sizeof(E) / 16;                       // pieces a row
    static constexpr int NK = sizeof(E) == 2 ? (D + 31) / 32 : D / 16;       // pieces of a lane's row of K
    static constexpr int NL = (CH * NC + 63) / 64;                           // loads of a chunk of V
    static constexpr int VB = CH * NC * 16 > D * 64 ? CH * NC * 16 : D * 64;  // V's chunk, later O [D][16]
};

template <typename E, int D>
__global__ __launch_bounds__(256, sizeof(E) == 4 && D == 128 ? 2 : 3) void win_step_kernel(StepArgs a) {
    using C = StepCfg<E, D>;
    __shared__ __align__(16) unsigned char sv[4][C::VB];
    __shared__ float2 sst[4][16];
    int id = block_of(a.blocks);
    if (id >= a.blocks) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, l16 = lane % 16, g4 = lane / 16;
    const int split = id % a.nsplit;
    id /= a.nsplit;
    const int hg = id % a.groups, kh = id / a.groups % a.Hk, s = id / a.groups / a.Hk;
    const int G = a.H / a.Hk, slots = a.sinks + a.W, pos = a.pos[s];
    const int held = pos < 0 ? 0 : min(pos, slots - 1) + 1;
    const int now = pos < a.sinks ? pos : a.sinks + (pos - a.sinks) % a.W;   // the new token's slot
    const int nch = (held + C::CH - 1) / C::CH, per = (nch + a.nsplit - 1) / a.nsplit;
    const int c0 = split * per, c1 = min(c0 + per, nch);
    const int hq = hg * 16 + l16;   // the lane's query head of those that share kh
    const size_t qrow = (size_t)s * a.H + kh * G + min(hq, G - 1);
    const size_t first = ((size_t)s * slots * a.Hk + kh) * D, rowlen = (size_t)a.Hk * D;
    const E *nk = (const E*)a.k + ((size_t)s * a.Hk + kh) * D, *nv = (const E*)a.v + ((size_t)s * a.Hk + kh) * D;
    E *ck = (E*)a.ck + first, *cv = (E*)a.cv + first;
    unsigned char* V = sv[wave];
    auto key = [](int r) { return C::NC >= 8 ? ((r & 3) << 1) | ((r >> 2) & 1) : C::NC >= 4 ? (r & 2) | ((r >> 2) & 1) : 0; };

    uint4 qf[C::NK];
#pragma unroll
    for (int k = 0; k < C::NK; ++k)
        qf[k] = hq < G && 4 * k + g4 < C::NC ? reinterpret_cast<const uint4*>((const E*)a.q + qrow * D)[4 * k + g4] : uint4{0, 0, 0, 0};
    f32x4 o[C::DT];
#pragma unroll
    for (int t = 0; t < C::DT; ++t) o[t] = zero4();
    float mx = -INFINITY, mc = -INFINITY, l = 0.f;

    constexpr int RT = C::CH / 16;
    uint4 kf[RT][C::NK], vf[C::NL];   // a chunk's keys and values, on their way while the last one is worked on
    auto load_k = [&](int c) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int j = c * C::CH + 16 * t + l16;
            const E* p = j == now || j >= held ? nk : ck + j * rowlen;
#pragma unroll
            for (int k = 0; k < C::NK; ++k)
                kf[t][k] = 4 * k + g4 < C::NC ? reinterpret_cast<const uint4*>(p)[4 * k + g4] : uint4{0, 0, 0, 0};
        }
    };
    auto load_v = [&](int c) {
#pragma unroll
        for (int i = 0; i < C::NL; ++i) {
            const int x = i * 64 + lane, j = c * C::CH + x / C::NC;
            const E* p = j == now || j >= held ? nv : cv + j * rowlen;
            vf[i] = reinterpret_cast<const uint4*>(p)[x % C::NC];
        }
    };
    int c = c0 + wave;
    if (c < c1) {
        load_k(c);
        load_v(c);
    }
    for (; c < c1; c += 4) {
        const int j0 = c * C::CH;
        // the new token into the caches, by the one workgroup that has its slot
        if (hg == 0 && now >= j0 && now < j0 + C::CH) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
                if (j0 + 16 * t + l16 == now) {
#pragma unroll
                    for (int k = 0; k < C::NK; ++k)
                        if (4 * k + g4 < C::NC) reinterpret_cast<uint4*>(ck + now * rowlen)[4 * k + g4] = kf[t][k];
                }
#pragma unroll
            for (int i = 0; i < C::NL; ++i) {
                const int x = i * 64 + lane;
                if (j0 + x / C::NC == now) reinterpret_cast<uint4*>(cv + now * rowlen)[x % C::NC] = vf[i];
            }
        }
        f32x4 sc[RT];
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            f32x4 x = zero4();
#pragma unroll
            for (int k = 0; k < C::NK; ++k) {
                if constexpr (sizeof(E) == 2) {
                    x = mfma_bf16(__builtin_bit_cast(bf16x8, kf[t][k]), __builtin_bit_cast(bf16x8, qf[k]), x);
                } else {
                    const f32x4 p = __builtin_bit_cast(f32x4, kf[t][k]), q = __builtin_bit_cast(f32x4, qf[k]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(p[e], q[e], x, 0, 0, 0);
                }
            }
            sc[t] = x;
        }
        if (c + 4 < c1) load_k(c + 4);
        // V into LDS, zero where no token is
#pragma unroll
        for (int i = 0; i < C::NL; ++i) {
            const int x = i * 64 + lane, r = x / C::NC, p = x % C::NC;
            *reinterpret_cast<uint4*>(V + (r * C::NC + (p ^ key(r))) * 16) = j0 + r < held ? vf[i] : uint4{0, 0, 0, 0};
        }
        if (c + 4 < c1) load_v(c + 4);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                sc[t][r] = j0 + 16 * t + 4 * g4 + r >= held ? -INFINITY : sc[t][r];
                top = fmaxf(top, sc[t][r]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > mx)) {
            mx = fmaxf(mx, top);
            const float next = mx == -INFINITY ? -INFINITY : mx * a.c;
            const float f = next == -INFINITY ? 0.f : exp2_hw(mc - next);
            mc = next;
            l *= f;
#pragma unroll
            for (int t = 0; t < C::DT; ++t) o[t] *= f;
        }
        const float base = mc == -INFINITY ? 0.f : mc;
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                sc[t][r] = exp2_hw(fmaf(sc[t][r], a.c, -base));
                if constexpr (sizeof(E) == 4) l += sc[t][r];
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if constexpr (sizeof(E) == 2) {
            const bf16x8 w = __builtin_bit_cast(bf16x8, uint4{cvt_pk_bf16(sc[0][0], sc[0][1]), cvt_pk_bf16(sc[0][2], sc[0][3]),
                                                              cvt_pk_bf16(sc[1][0], sc[1][1]), cvt_pk_bf16(sc[1][2], sc[1][3])});
            l = pairs_sum(w, l);
#pragma unroll
            for (int t = 0; t < C::DT; ++t) {
                const int r = 4 * g4 + (l16 >> 2), col = 16 * t + 4 * (l16 & 3);
                auto at = [&](int r) { return V + (r * C::NC + ((col / 8) ^ key(r))) * 16 + (col % 8) * 2; };
                const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)at(r));
                const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)at(r + 16));
                o[t] = mfma_bf16(__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7), w, o[t]);
            }
        } else {
#pragma unroll
            for (int t = 0; t < C::DT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 4 * g4 + r, col = 16 * t + l16;
                    const float x = *reinterpret_cast<const float*>(V + (row * C::NC + ((col / 4) ^ key(row))) * 16 + (col % 4) * 4);
                    o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, sc[0][r], o[t], 0, 0, 0);
                }
        }
        __builtin_amdgcn_wave_barrier();
    }
    // the waves' maxima and sums, and their O about the common maximum
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    l = sum_of(l, mc);
    if (g4 == 0) sst[wave][l16] = float2{mc, l};
    __syncthreads();
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, sst[w][l16].x);
    const float f = mc == -INFINITY ? 0.f : exp2_hw(mc - m);
    float* O = reinterpret_cast<float*>(V);   // [D][16]
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) O[(16 * t + 4 * g4 + r) * 16 + l16] = mc == -INFINITY ? 0.f : o[t][r] * f;
    __syncthreads();
    const int nh = min(16, G - hg * 16);
    for (int x = threadIdx.x; x < nh * D; x += 256) {
        const int hh = x / D, d = x % D;
        float sum = 0.f, tot = 0.f, mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            sum += reinterpret_cast<const float*>(sv[w])[d * 16 + hh];
            mm = fmaxf(mm, sst[w][hh].x);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 st = sst[w][hh];
            if (st.y != 0.f) tot = fmaf(exp2_hw(st.x - mm), st.y, tot);
        }
        const size_t row = (size_t)s * a.H + kh * G + hg * 16 + hh;
        if (a.nsplit > 1) {
            const size_t at = (size_t)split * a.S * a.H + row;
            a.part[at * D + d] = sum;
            if (d == 0) a.pstat[at] = float2{mm, tot};
        } else {
            const float r = tot == 0.f ? 0.f : sum / tot;
            if constexpr (sizeof(E) == 2)
                ((uint16_t*)a.y)[row * D + d] = f32_to_bf16(r);
            else
                ((float*)a.y)[row * D + d] = r;
        }
    }
}

// ---------------------------------------------------------------- launches

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// Whether every row sees few tokens.  Else those at the first kRows positions are taken as such.
bool sees_few(const WinShape& s) {
    return ((int64_t)s.window + s.sinks < s.Tk ? (int64_t)s.window + s.sinks : s.Tk) < kFew;
}

WinArgs args_of(const WinShape& s, const void* q, const void* k, const void* v, const int* len) {
    WinArgs a{};
    a.q = q, a.k = k, a.v = v, a.len = len;
    a.B = s.B, a.T = s.T, a.Tk = s.Tk, a.H = s.H, a.Hk = s.Hk;
    a.W = s.window < s.Tk ? s.window : (s.Tk > 0 ? s.Tk : 1);
    a.sinks = s.sinks, a.scale = s.scale, a.c = s.scale * 1.4426950408889634f;
    a.nsplit = a.ksplit = 1, a.few = sees_few(s);
    a.T64 = (s.T + 63) / 64 * 64;
    return a;
}

// The saved context: stat, then the rest of y.
void with_saved(const WinShape& s, WinArgs& a, void* saved) {
    a.stat = static_cast<float2*>(saved);
    if (s.bf16) a.rest = static_cast<int8_t*>(saved) + align256((size_t)s.B * s.T * s.H * sizeof(float2));
}

template <typename E, int D>
void join(size_t rows, int nsplit, const float* part, const float2* pstat, void* y, float2* stat, int8_t* rest, hipStream_t st) {
    // a thread for every four columns fills the chip (a prompt in four parts, d32, us by threads and by a workgroup a row:
    // 16384 threads 18.6 and 18.8, 65536 22.2 and 23.5, 131072 29.5 and 33.5; one row of 32 parts 12.9 and 3.4, the join alone)
    if (rows * (D / 4) >= 256 * 256)
        hipLaunchKernelGGL((win_join_rows_kernel<E, D>), dim3((unsigned)((rows * (D / 4) + 255) / 256)), dim3(256), 0, st, rows,
                           nsplit, part, pstat, (E*)y, stat, rest);
    else
        hipLaunchKernelGGL((win_join_kernel<E, D>), dim3((unsigned)rows), dim3(2 * D), 0, st, rows, nsplit, part, pstat, (E*)y,
                           stat, rest);
}

unsigned grid_of(int64_t blocks) { return (unsigned)((blocks + 7) / 8 * 8); }

// Keys are dealt to several workgroups where those of the queries are fewer than CUs, at least 256 keys to each.  bf16: only
// where a row's keys are many tiles, and the more the more queries, since the join reads each row's parts (us, all keys
// visible, d64, one workgroup a row and dealt out: B4 T512 H8 11 and 15, after 1500 tokens 31 and 27; B2 T512 H8 11 and
// 13, after 512 tokens 17.6 and 16.2; B1 T1024 H4 17.7 and 12.6; B8 T512 H8, 256 workgroups, 12 and 22, after 3500 tokens
// 58 and 54).  An fp32 tile takes some times as long (B4 T512 H8 44 and 32; B8 T512 H8 45 and 49).
int splits(const WinShape& s) {
    const int64_t blocks = (int64_t)s.B * s.H * ((s.T + kRows - 1) / kRows);
    const int64_t reach = (int64_t)s.window + kRows < s.Tk ? (int64_t)s.window + kRows : s.Tk;
    const int64_t tiles = (reach + 63) / 64 + (s.sinks > 0);
    if (blocks == 0 || blocks >= 256 || (s.bf16 && (tiles < 16 || 4 * tiles < blocks))) return 1;
    int64_t n = 512 / blocks;
    if (n > tiles / 4) n = tiles / 4;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

// The queries that see 128 tokens are dealt to several workgroups where tokens are too few for a workgroup a CU, at
// least 128 (of all heads that share the tokens) to each: B3 T777 H6 Hk2 d64 window 100, 42 workgroups of which left
// most of the chip idle, took 71 us for its backward, dealt to five each 43.
int key_splits(const WinShape& s) {
    const int64_t blocks = (int64_t)s.B * s.Hk * (((int64_t)s.Tk + kRows - 1) / kRows);
    const int64_t W = s.window < s.Tk ? s.window : s.Tk, reach = W + kRows < s.T ? W + kRows : s.T;
    if (blocks == 0 || blocks >= 256) return 1;
    int64_t n = 512 / blocks;
    if (n > reach * (s.H / s.Hk) / 128) n = reach * (s.H / s.Hk) / 128;
    return (int)(n < 1 ? 1 : n > 16 ? 16 : n);
}

// Queries a segment of the first tokens' sums: twice as many as a workgroup of 128 tokens walks (each of its waves takes
// every second 32), and at most 512, so that no segment outlasts the rest (B8 T2048 H16 d128 window 512: 387 us for the
// backward, with 1024 424).
int segment(const WinShape& s) {
    const int64_t W = s.window < s.Tk ? s.window : s.Tk, n = 2 * (W + kRows) < 512 ? 2 * (W + kRows) : 512;
    return (int)(n / key_splits(s) < 64 ? 64 : n / key_splits(s) / 64 * 64);
}

int segments(const WinShape& s) {
    if (s.sinks == 0) return 0;
    const int64_t W = s.window < s.Tk ? s.window : s.Tk, past = s.Tk - s.T;
    const int64_t behind = past > kRows - 1 + W ? past : kRows - 1 + W, n = s.Tk - behind;
    return n > 0 ? (int)((n + segment(s) - 1) / segment(s)) : 0;
}

template <typename E, int D>
hipError_t fwd(const WinShape& s, WinArgs a, void* ck, void* cv, hipStream_t st) {
    if (a.T > 0) {
        hipLaunchKernelGGL((win_fwd_kernel<E, D>), dim3(grid_of(a.blocks)), dim3(256), 0, st, a);
        if (a.nsplit > 1) {
            const size_t rows = (size_t)a.B * a.T * a.H;
            join<E, D>(rows, a.nsplit, a.part, a.pstat, a.o, a.stat, a.rest, st);
        }
    }
    if (ck) {
        WinArgs c = a;
        c.W = s.window;
        const size_t n = (size_t)s.B * (s.sinks + (size_t)s.window) * s.Hk * D * sizeof(E) / 16;
        hipLaunchKernelGGL((win_cache_kernel<E, D>), dim3((unsigned)(n / 256 + 1 < 8192 ? n / 256 + 1 : 8192)), dim3(256), 0, st, c,
                           (uint4*)ck, (uint4*)cv);
    }
    return hipGetLastError();
}

template <typename E, int D>
hipError_t bwd(WinArgs a, hipStream_t st) {
    const int nq = (a.T + kRows - 1) / kRows, nk = (a.Tk + kRows - 1) / kRows;
    if (nk == 0) return hipSuccess;
    a.blocks = a.B * a.H * nq;
    if (a.blocks > 0) hipLaunchKernelGGL((win_dq_kernel<E, D>), dim3(grid_of(a.blocks)), dim3(256), 0, st, a);
    a.blocks = a.B * a.Hk * (nk * a.ksplit + a.nseg);
    hipLaunchKernelGGL((win_dkv_kernel<E, D>), dim3(grid_of(a.blocks)), dim3(256), 0, st, a);
    if (a.nseg > 0 || a.ksplit > 1) {
        const int n = a.ksplit > 1 || a.sinks > a.Tk ? a.Tk : a.sinks;
        const size_t threads = (size_t)a.B * a.Hk * 2 * n * (D / 4);
        const size_t blocks = (threads + 255) / 256;   // a launch's threads are 32-bit
        hipLaunchKernelGGL((win_sum_kernel<E, D>), dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), 0, st, a, n);
    }
    return hipGetLastError();
}

template <typename F>
hipError_t by_type(bool bf16, int d, F&& f) {
    switch (d) {
        case 16: return bf16 ? f(uint16_t{}, std::integral_constant<int, 16>{}) : f(float{}, std::integral_constant<int, 16>{});
        case 32: return bf16 ? f(uint16_t{}, std::integral_constant<int, 32>{}) : f(float{}, std::integral_constant<int, 32>{});
        case 64: return bf16 ? f(uint16_t{}, std::integral_constant<int, 64>{}) : f(float{}, std::integral_constant<int, 64>{});
        case 128: return bf16 ? f(uint16_t{}, std::integral_constant<int, 128>{}) : f(float{}, std::integral_constant<int, 128>{});
    }
    return hipErrorInvalidValue;
}

int step_groups(const StepShape& s) { return (s.H / s.Hk + 15) / 16; }

// Slots are dealt to several workgroups where sequences and heads are too few for four workgroups a CU, at least a
// chunk to a wave; not where 16 chunks do not pay the join's launch, nor at 192 to 256 workgroups, a CU's each, nor at more
// of fewer than 128 chunks (us, one workgroup and by the rule above: bf16 d128, one sequence over 256 slots 6.6 and 8.2,
// 1024 slots 14.4 and 8.3, 4096 44 and 9.5; 128 workgroups over 1024 slots 17 and 18, 4096 54 and 47; 256 over 1024 slots
// 23 and 27, 4096 100 and 103; 512 over 1024 slots 44 and 47; 384 over 4096 165 and 153; fp32 d64, seven sequences of 3
// heads over 128 slots 5.4 and 7.4, 256 slots 7.4 and 7.4, 512 slots 11.6 and 7.5).
int step_splits(const StepShape& s) {
    const int64_t blocks = (int64_t)s.S * s.Hk * step_groups(s);
    const int64_t chunks = ((int64_t)s.window + s.sinks + (s.bf16 ? 31 : 15)) / (s.bf16 ? 32 : 16);
    if (chunks < 16 || (blocks >= 192 && (blocks <= 256 || chunks < 128))) return 1;
    int64_t n = 1024 / blocks;
    if (n > chunks / 4) n = chunks / 4;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

}  // namespace

int64_t window_blocks(const WinShape& s) {
    const int64_t nq = ((int64_t)s.T + kRows - 1) / kRows, nk = ((int64_t)s.Tk + kRows - 1) / kRows;
    const int64_t fwd = (int64_t)s.B * s.H * nq, dkv = (int64_t)s.B * s.Hk * (nk * key_splits(s) + segments(s));
    return fwd > dkv ? fwd : dkv;
}

size_t window_saved(const WinShape& s) {
    const size_t rows = (size_t)s.B * s.T * s.H;
    return align256(rows * sizeof(float2)) + (s.bf16 ? rows * s.d : 0);
}

size_t window_workspace(const WinShape& s, bool backward) {
    const size_t rows = (size_t)s.B * s.T * s.H;
    if (!backward) {
        const int n = splits(s);
        return n > 1 ? align256(n * rows * s.d * sizeof(float)) + n * rows * sizeof(float2) : 0;
    }
    const size_t t64 = (size_t)(s.T + 63) / 64 * 64, rest = (size_t)s.B * s.Hk * 2 * s.d * sizeof(float);
    const int nseg = segments(s), n = key_splits(s);
    return align256(3 * s.B * s.H * t64 * sizeof(float)) + align256(nseg > 0 ? rest * (1 + 2 * (size_t)nseg) * s.sinks : 0) +
           (n > 1 ? rest * n * s.Tk : 0);
}

hipError_t launch_window_fwd(const WinShape& s, const void* q, const void* k, const void* v, const int* len, void* y,
                             void* saved, void* ck, void* cv, void* ws, hipStream_t st) {
    WinArgs a = args_of(s, q, k, v, len);
    a.o = y;
    if (saved) with_saved(s, a, saved);
    a.nsplit = splits(s);
    const size_t rows = (size_t)s.B * s.T * s.H;
    if (a.nsplit > 1) {
        a.part = static_cast<float*>(ws);
        a.pstat = reinterpret_cast<float2*>(static_cast<char*>(ws) + align256(a.nsplit * rows * s.d * sizeof(float)));
    }
    a.sums = saved || a.nsplit > 1;
    a.blocks = s.B * s.H * ((s.T + kRows - 1) / kRows) * a.nsplit;
    return by_type(s.bf16, s.d, [&](auto e, auto d) { return fwd<decltype(e), decltype(d)::value>(s, a, ck, cv, st); });
}

hipError_t launch_window_bwd(const WinShape& s, const void* q, const void* k, const void* v, const int* len, const void* y,
                             const void* saved, const void* dy, void* dq, void* dk, void* dv, void* ws, hipStream_t st) {
    WinArgs a = args_of(s, q, k, v, len);
    a.y = y, a.dy = dy, a.dq = dq, a.dk = dk, a.dv = dv;
    with_saved(s, a, const_cast<void*>(saved));
    a.rows = static_cast<float*>(ws);
    a.nseg = segments(s), a.seg = segment(s), a.ksplit = key_splits(s);
    a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + align256(3 * (size_t)s.B * s.H * a.T64 * sizeof(float)));
    a.kpart = a.part + align256(a.nseg > 0 ? (size_t)s.B * s.Hk * 2 * s.d * sizeof(float) * (1 + 2 * (size_t)a.nseg) * s.sinks : 0) / 4;
    return by_type(s.bf16, s.d, [&](auto e, auto d) { return bwd<decltype(e), decltype(d)::value>(a, st); });
}

size_t window_step_workspace(const StepShape& s) {
    const int n = step_splits(s);
    const size_t rows = (size_t)s.S * s.H;
    return n > 1 ? align256(n * rows * s.d * sizeof(float)) + n * rows * sizeof(float2) : 0;
}

hipError_t launch_window_step(const StepShape& s, const void* q, const void* k, const void* v, const int* pos, void* ck,
                              void* cv, void* y, void* ws, hipStream_t st) {
    StepArgs a{};
    a.q = q, a.k = k, a.v = v, a.pos = pos, a.ck = ck, a.cv = cv, a.y = y;
    a.S = s.S, a.H = s.H, a.Hk = s.Hk, a.W = s.window, a.sinks = s.sinks;
    a.nsplit = step_splits(s), a.groups = step_groups(s), a.c = s.scale * 1.4426950408889634f;
    a.blocks = s.S * s.Hk * a.groups * a.nsplit;
    const size_t rows = (size_t)s.S * s.H;
    if (a.nsplit > 1) {
        a.part = static_cast<float*>(ws);
        a.pstat = reinterpret_cast<float2*>(static_cast<char*>(ws) + align256(a.nsplit * rows * s.d * sizeof(float)));
    }
    return by_type(s.bf16, s.d, [&](auto e, auto dd) {
        using E = decltype(e);
        constexpr int D = decltype(dd)::value;
        hipLaunchKernelGGL((win_step_kernel<E, D>), dim3(grid_of(a.blocks)), dim3(256), 0, st, a);
        if (a.nsplit > 1)
            join<E, D>(rows, a.nsplit, a.part, a.pstat, a.y, nullptr, nullptr, st);
        return hipGetLastError();
    });
}

}  // namespace kla
