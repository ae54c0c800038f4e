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
// start state.  All exponents are at least 0, so no factor exceeds 1 for g <= 0; e^{-inf * 0} is 1.
//
// A wave owns CW value columns of one sequence (or segment of one) and their state, in registers;
// the waves of a workgroup share the chunk's Q, K and V in LDS, double buffered.  Operands: the
// contraction index of a 32-deep product is {4g .. 4g+3} u {16+4g .. 16+4g+3} for lane group g in
// every product, so that Q's fragments serve Q K^T and Q R, V's fragments (Q K^T) V and K^T V, and
// accumulators are operands as they stand.  Rows are stored in 16-byte pieces, piece p of row r at
// p ^ f(r), which spreads both the reads along rows and those across rows over the LDS banks.
//
// bf16: v_mfma_f32_16x16x32_bf16.  q, k, v are exact operands; fp32 factors are split into bf16
// parts: the masked scores and the state (whose products are rounded to bf16 at the end) into two,
// 16 bits, the decayed values that are added to the fp32 state into three, its 24 bits.
// fp32: v_mfma_f32_16x16x4_f32.
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
    __device__ static int at(int r, int col) {
        constexpr int PER = 16 / (int)sizeof(E);
        return piece(r, col / PER) + (col % PER) * (int)sizeof(E);
    }
};

// Operands of a 32-deep product: eight values per lane.
template <typename E>
struct Op;

template <>
struct Op<uint16_t> {
    bf16x8 x;
    template <int W>
    __device__ static Op row(const unsigned char* t, int r, int col, int g4) {   // along row r, from column col
        using TL = Tile<uint16_t, W>;
        const uint2 a = *reinterpret_cast<const uint2*>(t + TL::at(r, col + 4 * g4));
        uint2 b = {0u, 0u};
        if constexpr (W > 16) b = *reinterpret_cast<const uint2*>(t + TL::at(r, col + 16 + 4 * g4));
        return {__builtin_bit_cast(bf16x8, uint4{a.x, a.y, b.x, b.y})};
    }
    template <int W>
    __device__ static Op col(const unsigned char* t, int col0, int g4, int l16) {   // down column col0 + l16
        using TL = Tile<uint16_t, W>;
        const int r = 4 * g4 + (l16 >> 2), c = col0 + 4 * (l16 & 3);
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)(t + TL::at(r, c)));
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)(t + TL::at(r + 16, c)));
        return {__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
    }
};

template <>
struct Op<float> {
    float x[8];
    template <int W>
    __device__ static Op row(const unsigned char* t, int r, int col, int g4) {
        using TL = Tile<float, W>;
        const float4 a = *reinterpret_cast<const float4*>(t + TL::at(r, col + 4 * g4));
        float4 b = {0.f, 0.f, 0.f, 0.f};
        if constexpr (W > 16) b = *reinterpret_cast<const float4*>(t + TL::at(r, col + 16 + 4 * g4));
        return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
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

// Accumulators (rows 4 g4 + rr of two 16-row tiles) as operands.
template <typename E>
struct Acc;
template <>
struct Acc<uint16_t> {
    bf16x8 h, l;   // 16 bits
    __device__ Acc(const f32x4& a, const f32x4& b) { split8(a, b, h, l); }
};
template <>
struct Acc<float> {
    float x[8];
    __device__ Acc(const f32x4& a, const f32x4& b) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = a[e];
            x[4 + e] = b[e];
        }
    }
};

// v scaled by w, as an operand of the state's update.
template <typename E>
struct Scaled;
template <>
struct Scaled<uint16_t> {
    bf16x8 p[3];   // 24 bits
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
    return mfma2b(a.x, b.h, b.l, c);
}
template <int STEPS = 8>
__device__ __forceinline__ f32x4 mma(const Acc<uint16_t>& a, const Op<uint16_t>& b, f32x4 c) {
    return mfma2a(a.h, a.l, b.x, c);
}
template <int STEPS = 8>
__device__ __forceinline__ f32x4 mma(const Op<uint16_t>& a, const Scaled<uint16_t>& b, f32x4 c) {
    c = mfma_bf16(a.x, b.p[2], c);
    c = mfma_bf16(a.x, b.p[1], c);
    return mfma_bf16(a.x, b.p[0], c);
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
template <int STEPS = 8>
__device__ __forceinline__ f32x4 mma(const Acc<float>& a, const Op<float>& b, f32x4 c) {
    return mma_f32<STEPS>(a.x, b.x, c);
}
template <int STEPS = 8>
__device__ __forceinline__ f32x4 mma(const Op<float>& a, const Scaled<float>& b, f32x4 c) {
    return mma_f32<STEPS>(a.x, b.x, c);
}

// Four output values of one token.
__device__ __forceinline__ void store4(uint16_t, const f32x4& y, rsrc_t r, uint32_t voff) {
    buf_st64(uint2{cvt_pk_bf16(y[0], y[1]), cvt_pk_bf16(y[2], y[3])}, r, voff);
}
__device__ __forceinline__ void store4(float, const f32x4& y, rsrc_t r, uint32_t voff) {
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, y), r, voff, 0, 0);
}

// e^{g n}, 1 for n = 0 whatever g is; formed in fp64 because g n may be large where g has few digits left
__device__ __forceinline__ float decay_pow(float g, int n) { return n == 0 ? 1.f : (float)exp((double)g * n); }

__device__ __forceinline__ float lds_val(uint16_t, const unsigned char* p) {
    return bf16_to_f32(*reinterpret_cast<const uint16_t*>(p));
}
__device__ __forceinline__ float lds_val(float, const unsigned char* p) { return *reinterpret_cast<const float*>(p); }

// (Q K^T o D) V of a chunk again, where a product was not finite: a matrix instruction multiplies later
// tokens' values by zero scores, and a value that is not finite must not reach the tokens before it.
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

struct LinArgs {
    const void *q, *k, *v;   // Q, K [B, T, H, N], V [B, T, H, D]
    const float* g;          // [H]
    const int* len;          // [B] or none
    const float* start;      // start states, or none (0): by sequence, or with ns > 1 by sequence and segment
    void* y;                 // [B, T, H, D]
    float* end;              // final states, or none; NOY: the segments' own, by sequence and segment
    int B, T, H;
    int ns, lc, run;         // segments per sequence, chunks in one, segments run
    int flip;                // bit 0: the start states, bit 1: the final ones are stored [D][N] instead of [N][D]
};

// Tokens of sequence b.
__device__ __forceinline__ int seq_len(const LinArgs& a, int b) {
    return a.len ? min(max(a.len[b], 0), a.T) : a.T;
}

template <typename E, int N, int NW, int CW>
constexpr int kLinLds = 2 * (2 * Tile<E, N>::BYTES + Tile<E, NW * CW>::BYTES) + 2 * kLC * (int)sizeof(float);

template <typename E, int N, int D, int NW, int CW, bool REV, bool NOY>
__global__ __launch_bounds__(NW * 64) void linattn_kernel(LinArgs a) {
    constexpr int DT = NW * CW, NTILE = D / DT, NDT = CW / 16, NRT = N / 16, KS = (N + 31) / 32;
    constexpr int O = REV ? 0 : 1, ES = (int)sizeof(E);
    using TQ = Tile<E, N>;
    using TV = Tile<E, DT>;
    constexpr int UQ = NOY ? 0 : TQ::UNITS, UK = TQ::UNITS, UNITS = UQ + UK + TV::UNITS;
    constexpr int NL = (UNITS + NW - 1) / NW;   // a wave's loads per chunk
    constexpr int BUF = 2 * TQ::BYTES + TV::BYTES;
    extern __shared__ __align__(16) unsigned char smem[];
    float* pw = reinterpret_cast<float*>(smem + 2 * BUF);   // e^{g n}

    int vi, tile;   // the tiles of one sequence on one XCD: they read the same Q and K
    {
        const int i = blockIdx.x, nv = a.B * a.H * a.run;
        if (nv % 8 == 0) {
            const int slot = i / 8;
            tile = slot % NTILE;
            vi = (slot / NTILE) * 8 + i % 8;
        } else {
            tile = i % NTILE;
            vi = i / NTILE;
        }
    }
    const int bh = vi / a.run, seg = vi % a.run, b = bh / a.H, h = bh % a.H, H = a.H;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g4 = lane >> 4;
    const float g = a.g[h];
    const int Tb = seq_len(a, b);
    const int u0 = seg * a.lc * kLC, nu = min(max(Tb - u0, 0), a.lc * kLC);   // this segment's tokens, in walk order
    const int nchunk = (nu + kLC - 1) / kLC;
    const int dm0 = tile * DT + wave * CW, dl0 = wave * CW;

    if (threadIdx.x < 2 * kLC) pw[threadIdx.x] = decay_pow(g, threadIdx.x);

    // chunk c: its tokens n, and the first of them in memory
    auto chunk_n = [&](int c) { return min(max(nu - c * kLC, 0), kLC); };
    auto chunk_t0 = [&](int c, int n) {
        const int u = u0 + c * kLC;
        return REV ? Tb - u - n : u;
    };
    auto row_off = [&](int r, int n, uint32_t stride) {   // rows past the chunk's tokens fall outside the buffer
        return REV ? (r < n ? (uint32_t)(n - 1 - r) * stride : 0x80000000u) : (uint32_t)r * stride;
    };
    auto rsrc_of = [&](const void* p, int w, int col, int t0, int n, int cols) {
        const char* base = static_cast<const char*>(p) + (((size_t)b * a.T + t0) * H + h) * (size_t)(w * ES) + col * ES;
        return make_rsrc(n > 0 ? base : p, n > 0 ? (uint32_t)(((n - 1) * H * w + cols) * ES) : 0u);
    };

    uint4 stage[NL];
    auto load = [&](int c) {
        const int n = chunk_n(c), t0 = n > 0 ? chunk_t0(c, n) : 0;
        const rsrc_t rq = rsrc_of(a.q, N, 0, t0, NOY ? 0 : n, N), rk = rsrc_of(a.k, N, 0, t0, n, N);
        const rsrc_t rv = rsrc_of(a.v, D, tile * DT, t0, n, DT);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int u = i * NW + wave;
            if (u < UQ + UK) {
                const int x = (u < UQ ? u : u - UQ) * 64 + lane;
                const uint32_t off = row_off(x / TQ::NC, n, (uint32_t)(H * N * ES)) + (uint32_t)(x % TQ::NC) * 16;
                stage[i] = buf_ld128(u < UQ ? rq : rk, off, 0);
            } else if (u < UNITS) {
                const int x = (u - UQ - UK) * 64 + lane;
                const uint32_t off = row_off(x / TV::NC, n, (uint32_t)(H * D * ES)) + (uint32_t)(x % TV::NC) * 16;
                stage[i] = buf_ld128(rv, off, 0);
            }
        }
    };
    auto put = [&](int c) {
        unsigned char* buf = smem + (c & 1) * BUF;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int u = i * NW + wave;
            if (u < UQ + UK) {
                const int x = (u < UQ ? u : u - UQ) * 64 + lane;
                *reinterpret_cast<uint4*>(buf + (u < UQ ? 0 : TQ::BYTES) + TQ::piece(x / TQ::NC, x % TQ::NC)) = stage[i];
            } else if (u < UNITS) {
                const int x = (u - UQ - UK) * 64 + lane;
                *reinterpret_cast<uint4*>(buf + 2 * TQ::BYTES + TV::piece(x / TV::NC, x % TV::NC)) = stage[i];
            }
        }
    };

    // state R[n, d], n = 16 rt + 4 g4 + rr, d = dm0 + 16 dt + l16
    const size_t srow = (size_t)bh * a.ns + seg;
    f32x4 R[NRT][NDT];
    auto state_at = [&](int rt, int dt, int rr, bool flip) {
        const int n = 16 * rt + 4 * g4 + rr, d = dm0 + 16 * dt + l16;
        return flip ? d * N + n : n * D + d;
    };
    if (nchunk > 0) load(0);
    {
        const float* s0 = NOY || !a.start ? nullptr : a.start + srow * (size_t)(N * D);
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) R[rt][dt][rr] = s0 ? s0[state_at(rt, dt, rr, a.flip & 1)] : 0.f;
    }
    __syncthreads();   // pw
    float dia[4], off[4], rd[2], kw[8];
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
        const int lag = l16 - 4 * g4 - rr;
        dia[rr] = lag >= 0 ? pw[max(lag, 0)] : 0.f;
        off[rr] = pw[16 + lag];
    }
    rd[0] = pw[l16 + O];
    rd[1] = pw[16 + l16 + O];
    auto weights = [&](int n) {   // of the state's update; values past the chunk's tokens are zero
#pragma unroll
        for (int e = 0; e < 8; ++e) kw[e] = pw[max(n - O - (4 * g4 + (e & 3) + (e & 4) * 4), 0)];
    };
    weights(kLC);
    float gn = pw[kLC];
    if (nchunk > 0) put(0);
    if (nchunk > 1) load(1);
    __syncthreads();

    for (int c = 0; c < nchunk; ++c) {
        const int n = chunk_n(c);
        const unsigned char* buf = smem + (c & 1) * BUF;
        const unsigned char *sQ = buf, *sK = buf + TQ::BYTES, *sV = buf + 2 * TQ::BYTES;
        if (n < kLC) {
            weights(n);
            gn = pw[n];
        }
        Op<E> vf[NDT];
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) vf[dt] = Op<E>::template col<DT>(sV, dl0 + 16 * dt, g4, l16);

        if constexpr (!NOY) {
            // S^T[j, i] = K_j . Q_i, tiles (jt, it) = (0,0), (0,1), (1,1); Y^T[d, i] from the state
            f32x4 s00 = zero4(), s01 = zero4(), s11 = zero4(), y[NDT][2];
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) y[dt][0] = y[dt][1] = zero4();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                constexpr int ST = N == 16 ? 4 : 8;
                const Op<E> q0 = Op<E>::template row<N>(sQ, l16, 32 * ks, g4), q1 = Op<E>::template row<N>(sQ, 16 + l16, 32 * ks, g4);
                const Op<E> k0 = Op<E>::template row<N>(sK, l16, 32 * ks, g4), k1 = Op<E>::template row<N>(sK, 16 + l16, 32 * ks, g4);
                s00 = mma<ST>(k0, q0, s00);
                s01 = mma<ST>(k0, q1, s01);
                s11 = mma<ST>(k1, q1, s11);
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) {
                    const Acc<E> r(R[2 * ks][dt], N == 16 ? zero4() : R[N == 16 ? 0 : 2 * ks + 1][dt]);
                    y[dt][0] = mma<ST>(r, q0, y[dt][0]);
                    y[dt][1] = mma<ST>(r, q1, y[dt][1]);
                }
            }
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {   // scores of later tokens are no factor, whatever they are
                s00[rr] = l16 >= 4 * g4 + rr ? s00[rr] * dia[rr] : 0.f;
                s01[rr] *= off[rr];
                s11[rr] = l16 >= 4 * g4 + rr ? s11[rr] * dia[rr] : 0.f;
            }
            const Acc<E> p0(s00, zero4()), p1(s01, s11);
            const int t0 = chunk_t0(c, n);
            const rsrc_t ry = rsrc_of(a.y, D, dm0, t0, n, CW);
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                f32x4 in[2] = {mma<4>(vf[dt], p0, zero4()), mma<8>(vf[dt], p1, zero4())};
                float fin = 0.f;
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) fin += 0.f * in[0][rr] + 0.f * in[1][rr];
                if (__any(fin != 0.f))
#pragma unroll
                    for (int it = 0; it < 2; ++it)
                        in[it] = masked_sums<E, N, DT>(sQ, sK, sV, pw, dl0 + 16 * dt, 16 * it + l16, g4);
#pragma unroll
                for (int it = 0; it < 2; ++it) {
#pragma unroll
                    for (int rr = 0; rr < 4; ++rr) y[dt][it][rr] = y[dt][it][rr] * rd[it] + in[it][rr];
                    store4(E(), y[dt][it], ry,
                           row_off(16 * it + l16, n, (uint32_t)(H * D * ES)) + (uint32_t)((16 * dt + 4 * g4) * ES));
                }
            }
        }

        // R <- e^{g n} R + K^T (w V)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
            const Scaled<E> vs(vf[dt], kw);
#pragma unroll
            for (int rt = 0; rt < NRT; ++rt) {
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) R[rt][dt][rr] *= gn;
                R[rt][dt] = mma<8>(Op<E>::template col<N>(sK, 16 * rt, g4, l16), vs, R[rt][dt]);
            }
        }
        if (c + 1 < nchunk) put(c + 1);
        if (c + 2 < nchunk) load(c + 2);
        __syncthreads();
    }

    if (a.end && (NOY || seg == a.ns - 1)) {
        float* o = a.end + (NOY ? srow : (size_t)bh) * (size_t)(N * D);
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) o[state_at(rt, dt, rr, !NOY && (a.flip & 2))] = R[rt][dt][rr];
    }
    if constexpr (!NOY) {   // rows past the sequence's length are zero
        const int z1 = min(a.T, u0 + a.lc * kLC);
        constexpr int PV = DT * ES / 16;
        char* y0 = static_cast<char*>(a.y);
        for (size_t x = (size_t)max(Tb, u0) * PV + threadIdx.x; x < (size_t)z1 * PV; x += NW * 64)
            *reinterpret_cast<uint4*>(y0 + ((((size_t)b * a.T + x / PV) * H + h) * D + tile * DT) * ES + (x % PV) * 16) =
                uint4{0u, 0u, 0u, 0u};
    }
}

// Start states of the segments from their own end states, in place: a workgroup takes 256 elements of
// one sequence's state through its segments.
__global__ __launch_bounds__(256) void linattn_join_kernel(LinArgs a, int N, int D, const float* __restrict__ s0,
                                                           float* __restrict__ ends) {
    const int per = N * D / 256, bh = blockIdx.x / per, x = (blockIdx.x % per) * 256 + threadIdx.x;
    const int Tb = seq_len(a, bh / a.H), L = a.lc * kLC;
    const float g = a.g[bh % a.H];
    float* e = ends + (size_t)bh * a.ns * N * D + x;
    const int sx = a.flip & 1 ? (x % D) * N + x / D : x;
    float R = s0 ? s0[(size_t)bh * N * D + sx] : 0.f;
    const float whole = decay_pow(g, L);
    for (int s = 0; s < a.ns; ++s) {
        const float own = s < a.ns - 1 ? e[(size_t)s * N * D] : 0.f;
        e[(size_t)s * N * D] = R;
        const int n = min(max(Tb - s * L, 0), L);
        R = (n == L ? whole : decay_pow(g, n)) * R + own;
    }
}

template <typename E, int N, int D, int NW, int CW, bool REV, bool NOY>
hipError_t launch(const LinArgs& a, hipStream_t st) {
    auto kern = linattn_kernel<E, N, D, NW, CW, REV, NOY>;
    constexpr int LDS = kLinLds<E, N, NW, CW>;
    // more than 64 KiB of LDS must be opted into once per kernel (thread-safe static init)
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (attr != hipSuccess) return attr;
    const unsigned grid = (unsigned)((size_t)a.B * a.H * a.run * (D / (NW * CW)));
    hipLaunchKernelGGL(kern, dim3(grid), dim3(NW * 64), LDS, st, a);
    return hipGetLastError();
}

template <typename E, int N, int D, bool REV>
hipError_t run_pass(LinArgs a, const float* s0, float* ws, hipStream_t st) {
    constexpr int CW = 16, NW = D >= 64 ? 4 : D / 16;
    a.run = a.ns;
    a.start = s0;
    if (a.ns > 1) {   // the segments' own end states, their start states from those, then the segments
        LinArgs p = a;
        p.run = a.ns - 1;
        p.end = ws;
        hipError_t e = launch<E, N, D, NW, CW, REV, true>(p, st);
        if (e != hipSuccess) return e;
        linattn_join_kernel<<<dim3((unsigned)((size_t)a.B * a.H * (N * D / 256))), dim3(256), 0, st>>>(a, N, D, s0, ws);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.start = ws;
        a.flip &= 2;
    }
    return launch<E, N, D, NW, CW, REV, false>(a, st);
}

template <typename E, int N, int D>
hipError_t run_dir(const LinArgs& a, bool rev, const float* s0, float* ws, hipStream_t st) {
    return rev ? run_pass<E, N, D, true>(a, s0, ws, st) : run_pass<E, N, D, false>(a, s0, ws, st);
}

template <typename E>
hipError_t run(const LinArgs& a, int N, int D, bool rev, const float* s0, float* ws, hipStream_t st) {
#define KLA_LIN(N_, D_) \
    if (N == N_ && D == D_) return run_dir<E, N_, D_>(a, rev, s0, ws, st);
#define KLA_LIN_ROW(N_) KLA_LIN(N_, 16) KLA_LIN(N_, 32) KLA_LIN(N_, 64) KLA_LIN(N_, 128)
    KLA_LIN_ROW(16) KLA_LIN_ROW(32) KLA_LIN_ROW(64) KLA_LIN_ROW(128)
#undef KLA_LIN_ROW
#undef KLA_LIN
    return hipErrorInvalidValue;
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
    if (s.dv == 128) KLA_STEP(128);
    else if (s.dv == 64) KLA_STEP(64);
    else if (s.dv == 32) KLA_STEP(32);
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

// Segments of a pass whose values are D wide, and chunks in one.
void segments(const Shape& s, int D, int& ns, int& lc) {
    const int nc = (s.T + kLC - 1) / kLC;
    const long groups = (long)s.B * s.H * (D >= 64 ? D / 64 : 1);
    ns = 1;
    while (groups * ns < 512 && nc / (2 * ns) >= 8) ns *= 2;
    lc = (nc + ns - 1) / ns;
    ns = lc > 0 ? (nc + lc - 1) / lc : 1;
    if (ns < 1) ns = 1;
}

}  // namespace

size_t linattn_workspace(const Shape& s, bool backward) {
    size_t most = 0;
    for (int D : {s.dv, backward ? s.dk : s.dv}) {
        int ns, lc;
        segments(s, D, ns, lc);
        const size_t n = ns > 1 ? (size_t)s.B * s.H * ns * s.dk * s.dv * sizeof(float) : 0;
        most = n > most ? n : most;
    }
    return most;
}

hipError_t launch_linattn(const Shape& s, const LinPass& p, const float* g, const int* len, void* ws, hipStream_t st) {
    LinArgs a{};
    a.q = p.q;
    a.k = p.k;
    a.v = p.v;
    a.g = g;
    a.len = len;
    a.y = p.y;
    a.end = p.end;
    a.B = s.B;
    a.T = s.T;
    a.H = s.H;
    a.flip = (p.flip_start ? 1 : 0) | (p.flip_end ? 2 : 0);
    segments(s, p.D, a.ns, a.lc);
    return s.bf16 ? run<uint16_t>(a, p.N, p.D, p.rev, p.start, static_cast<float*>(ws), st)
                  : run<float>(a, p.N, p.D, p.rev, p.start, static_cast<float*>(ws), st);
}

hipError_t launch_linattn_step(const Shape& s, const void* q, const void* k, const void* v, const float* g, float* state,
                               void* y, hipStream_t st) {
    return s.bf16 ? step<uint16_t>(s, q, k, v, g, state, y, st) : step<float>(s, q, k, v, g, state, y, st);
}

}  // namespace kla
