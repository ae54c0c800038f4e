// Norms of queries and keys for each head and the position rotation, in one pass.
//
//   u = x r w,  r = 1 / sqrt(mean(x^2) + eps)                       over the n elements of one head of one token
//   (u_a, u_b) -> (u_a cos - u_b sin, u_b cos + u_a sin)            over the pairs, angle position * freq
//
// The pairs are elements i and i + P of the first 2 P (half-split) or 2i and 2i + 1 (interleaved); the other
// elements are not rotated.  The backward turns dout back by the same angles and differentiates the norm,
// with r formed again from the row it reads anyway: nothing is saved.
//
// HBM bounds both passes (two accesses an element forward, three backward): 16384 tokens of 32 heads of 128, bf16, take
// 57 us forward (4.7 TB/s) and 79 backward (5.1, a large copy's rate).  A thread takes two 16-byte pieces
// (8 bf16 elements each; 2 x 16 bytes for fp32) of a row that hold both elements of its pairs, so the rotation
// needs no exchange, and n / 16 lanes a row add up its squares by butterflies.  A workgroup takes the rows of
// all heads, of q and of k, of a few tokens: an angle costs an fp64 product, its reduction and an accurate
// sine and cosine (some 80 instructions), so each is formed once per token, by one thread, and read from LDS
// by all heads.  Angles are reduced in fp64 turns: positions up to 2^31 leave 2^-22 of a turn at worst.
#include "kla_buf.hpp"
#include "kla_internal.hpp"
#include "kla_mfma.hpp"

namespace kla {
namespace {

constexpr int kAngles = 512;   // angles of a workgroup's tokens in LDS

struct RopeArgs {
    const void* x[2];      // q, k
    const void* dout[2];
    void* out[2];          // outputs; in the backward the inputs' gradients
    const float* w[2];     // NULL: ones
    const double* freq;
    const int* pos;        // NULL: the index within the sequence
    float* part;           // backward: [blocks][2][n]
    int64_t tokens;
    int T, H[2], pairs, tile;
    float eps;
};

template <typename S>
struct Piece;
template <>
struct Piece<bf16_t> {   // 8 elements
    uint4 u;
    __device__ void load(const void* p, size_t i) { u = *reinterpret_cast<const uint4*>((const uint16_t*)p + i); }
    __device__ void get(float* f) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = __uint_as_float(w[e] << 16);
            f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
    __device__ static void put(void* p, size_t i, const float* f) {
        *reinterpret_cast<uint4*>((uint16_t*)p + i) =
            uint4{cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]), cvt_pk_bf16(f[4], f[5]), cvt_pk_bf16(f[6], f[7])};
    }
};
template <>
struct Piece<f32_t> {
    float4 a, b;
    __device__ void load(const void* p, size_t i) {
        a = *reinterpret_cast<const float4*>((const float*)p + i);
        b = *reinterpret_cast<const float4*>((const float*)p + i + 4);
    }
    __device__ void get(float* f) const {
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    }
    __device__ static void put(void* p, size_t i, const float* f) {
        *reinterpret_cast<float4*>((float*)p + i) = float4{f[0], f[1], f[2], f[3]};
        *reinterpret_cast<float4*>((float*)p + i + 4) = float4{f[4], f[5], f[6], f[7]};
    }
};

template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int m = G / 2; m >= 1; m /= 2) v += __shfl_xor(v, m, G);
    return v;
}

// The two pieces of lane t of a row: those of pairs 8t .. 8t+7 (half-split), or neighbours.
__device__ __forceinline__ void pieces(int t, int pairs, bool inter, int& a, int& b) {
    if (!inter && 8 * t < pairs) {
        a = t;
        b = t + pairs / 8;
    } else {
        a = 2 * t;
        b = 2 * t + 1;
    }
}

// f[0..7] piece a, f[8..15] piece b; sign -1 turns back.
template <bool INTER>
__device__ __forceinline__ void rotate(float (&f)[16], const float2* cs, int a, int b, int pairs, float sign) {
    if constexpr (INTER) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = (e < 4 ? 4 * a + e : 4 * b + e - 4);
            if (i >= pairs) continue;
            const float2 c = cs[i];
            const float s = sign * c.y, x = f[2 * e], y = f[2 * e + 1];
            f[2 * e] = x * c.x - y * s;
            f[2 * e + 1] = y * c.x + x * s;
        }
    } else if (8 * a < pairs) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 c = cs[8 * a + e];
            const float s = sign * c.y, x = f[e], y = f[8 + e];
            f[e] = x * c.x - y * s;
            f[8 + e] = y * c.x + x * s;
        }
    }
}

// (cos, sin) of the tile's tokens times the frequencies
__device__ __forceinline__ void angles(const RopeArgs& p, int64_t tok0, int ntok, float2* cs) {
    for (int i = threadIdx.x; i < ntok * p.pairs; i += blockDim.x) {
        const int64_t tok = tok0 + i / p.pairs;
        const double at = p.pos ? (double)p.pos[tok] : (double)(tok % p.T);
        double turn = at * p.freq[i % p.pairs] * 0.15915494309189533577;   // 1 / (2 pi)
        turn -= rint(turn);
        float s, c;
        sincospif(2.f * (float)turn, &s, &c);
        cs[i] = float2{c, s};
    }
}

template <typename S, int N, bool INTER, bool BWD>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs p) {
    constexpr int L = N / 16, RP = 256 / L;   // lanes a row, rows a pass
    __shared__ float2 cs[kAngles];
    __shared__ float sums[BWD ? 256 * 16 : 1];
    const int t = threadIdx.x % L, r0 = threadIdx.x / L;
    int a, b;
    pieces(t, p.pairs, INTER, a, b);
    float w[2][16], acc[2][16];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            w[m][e] = p.w[m] ? p.w[m][8 * (e < 8 ? a : b) + e % 8] : 1.f;
            acc[m][e] = 0.f;
        }
    const int64_t tiles = (p.tokens + p.tile - 1) / p.tile;
    for (int64_t tl = blockIdx.x; tl < tiles; tl += gridDim.x) {
        const int64_t tok0 = tl * p.tile;
        const int ntok = (int)(p.tokens - tok0 < p.tile ? p.tokens - tok0 : p.tile);
        if (p.pairs > 0) {
            angles(p, tok0, ntok, cs);
            __syncthreads();
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int H = p.H[m], rows = ntok * H;
            const size_t base = (size_t)tok0 * H * N;
            for (int r = r0; r < rows; r += RP) {
                const size_t at = base + (size_t)r * N;
                Piece<S> xa, xb, ga, gb;
                xa.load(p.x[m], at + 8 * a);
                xb.load(p.x[m], at + 8 * b);
                if constexpr (BWD) {
                    ga.load(p.dout[m], at + 8 * a);
                    gb.load(p.dout[m], at + 8 * b);
                }
                float f[16];
                xa.get(f);
                xb.get(f + 8);
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) ss = fmaf(f[e], f[e], ss);
                const float rs = __builtin_amdgcn_rsqf(lanes_sum<L>(ss) * (1.f / N) + p.eps);
                const float2* c = cs + (r / H) * p.pairs;
                if constexpr (!BWD) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) f[e] = f[e] * rs * w[m][e];
                    rotate<INTER>(f, c, a, b, p.pairs, 1.f);
                    Piece<S>::put(p.out[m], at + 8 * a, f);
                    Piece<S>::put(p.out[m], at + 8 * b, f + 8);
                } else {
                    float g[16];
                    ga.get(g);
                    gb.get(g + 8);
                    rotate<INTER>(g, c, a, b, p.pairs, -1.f);
                    float dot = 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        f[e] *= rs;
                        acc[m][e] = fmaf(g[e], f[e], acc[m][e]);
                        g[e] *= w[m][e];
                        dot = fmaf(f[e], g[e], dot);
                    }
                    const float mean = lanes_sum<L>(dot) * (1.f / N);
#pragma unroll
                    for (int e = 0; e < 16; ++e) g[e] = rs * fmaf(-f[e], mean, g[e]);
                    Piece<S>::put(p.out[m], at + 8 * a, g);
                    Piece<S>::put(p.out[m], at + 8 * b, g + 8);
                }
            }
        }
        if (p.pairs > 0) __syncthreads();
    }
    if constexpr (BWD) {   // one part a workgroup: its rows added in a fixed order
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[r0 * N + 8 * (e < 8 ? a : b) + e % 8] = acc[m][e];
            __syncthreads();
            if (threadIdx.x < N) {
                float s = 0.f;
                for (int r = 0; r < RP; ++r) s += sums[r * N + threadIdx.x];
                p.part[((size_t)blockIdx.x * 2 + m) * N + threadIdx.x] = s;
            }
            __syncthreads();
        }
    }
}

// dw[m][i] = sum of the parts, a workgroup for each: 256 strided sums, then a tree
__global__ __launch_bounds__(256) void rope_wgrad_kernel(int parts, int N, const float* __restrict__ part, float* dwq,
                                                         float* dwk) {
    __shared__ float s[256];
    const int col = blockIdx.x;
    float v = 0.f;
    for (int i = threadIdx.x; i < parts; i += 256) v += part[(size_t)i * 2 * N + col];
    s[threadIdx.x] = v;
    __syncthreads();
    for (int h = 128; h >= 1; h /= 2) {
        if ((int)threadIdx.x < h) s[threadIdx.x] += s[threadIdx.x + h];
        __syncthreads();
    }
    float* dw = col < N ? dwq : dwk;
    if (threadIdx.x == 0 && dw) dw[col % N] = s[0];
}

constexpr int kRopeParts = 1024;   // workgroups of the backward at most

// Tokens a workgroup: about four passes over its rows, so that the angles are formed behind other
// workgroups' loads, but one token where there are too few for every CU.
int tile_of(const RopeShape& s) {
    const int64_t tokens = (int64_t)s.B * s.T;
    const int64_t lanes = (int64_t)(s.H + s.Hk) * s.n / 16;
    int64_t tile = (1024 + lanes - 1) / lanes;
    if (s.pairs > 0 && tile > kAngles / s.pairs) tile = kAngles / s.pairs;
    if (tile > tokens / 512) tile = tokens / 512;
    return (int)(tile < 1 ? 1 : tile);
}

template <typename S, int N, bool BWD>
hipError_t launch(const RopeShape& s, const RopeArgs& p, int64_t blocks, hipStream_t st) {
    if (s.interleaved)
        hipLaunchKernelGGL((rope_kernel<S, N, true, BWD>), dim3((unsigned)blocks), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((rope_kernel<S, N, false, BWD>), dim3((unsigned)blocks), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <typename S, bool BWD>
hipError_t launch_n(const RopeShape& s, const RopeArgs& p, int64_t blocks, hipStream_t st) {
    switch (s.n) {
        case 16: return launch<S, 16, BWD>(s, p, blocks, st);
        case 32: return launch<S, 32, BWD>(s, p, blocks, st);
        case 64: return launch<S, 64, BWD>(s, p, blocks, st);
        case 128: return launch<S, 128, BWD>(s, p, blocks, st);
    }
    return hipErrorInvalidValue;
}

RopeArgs args_of(const RopeShape& s, const void* q, const void* k, const float* wq, const float* wk, const double* freq,
                 const int* pos) {
    RopeArgs p{};
    p.x[0] = q, p.x[1] = k;
    p.w[0] = wq, p.w[1] = wk;
    p.freq = freq, p.pos = pos;
    p.tokens = (int64_t)s.B * s.T;
    p.T = s.T, p.H[0] = s.H, p.H[1] = s.Hk, p.pairs = s.pairs, p.tile = tile_of(s), p.eps = s.eps;
    return p;
}

}  // namespace

size_t rope_parts_bytes(int n) { return (size_t)kRopeParts * 2 * n * sizeof(float); }

hipError_t launch_rope_fwd(const RopeShape& s, const void* q, const void* k, const float* wq, const float* wk,
                           const double* freq, const int* pos, void* oq, void* ok, hipStream_t st) {
    RopeArgs p = args_of(s, q, k, wq, wk, freq, pos);
    if (p.tokens == 0) return hipSuccess;
    p.out[0] = oq, p.out[1] = ok;
    int64_t blocks = (p.tokens + p.tile - 1) / p.tile;
    if (blocks > 1 << 20) blocks = 1 << 20;
    return s.bf16 ? launch_n<bf16_t, false>(s, p, blocks, st) : launch_n<f32_t, false>(s, p, blocks, st);
}

hipError_t launch_rope_bwd(const RopeShape& s, const void* q, const void* k, const float* wq, const float* wk,
                           const double* freq, const int* pos, const void* doq, const void* dok, void* dq, void* dk,
                           float* dwq, float* dwk, float* part, hipStream_t st) {
    RopeArgs p = args_of(s, q, k, wq, wk, freq, pos);
    p.dout[0] = doq, p.dout[1] = dok, p.out[0] = dq, p.out[1] = dk, p.part = part;
    int64_t blocks = (p.tokens + p.tile - 1) / p.tile;
    if (blocks > kRopeParts) blocks = kRopeParts;
    if (blocks > 0) {
        const hipError_t e = s.bf16 ? launch_n<bf16_t, true>(s, p, blocks, st) : launch_n<f32_t, true>(s, p, blocks, st);
        if (e != hipSuccess) return e;
    }
    if (!dwq && !dwk) return hipSuccess;
    hipLaunchKernelGGL(rope_wgrad_kernel, dim3(2 * s.n), dim3(256), 0, st, (int)blocks, s.n, part, dwq, dwk);
    return hipGetLastError();
}

}  // namespace kla
