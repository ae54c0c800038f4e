// Layer norm over rows of n elements, forward and backward.
//
//   out = (x - mean) rstd w + bias,  mean = sum x / n,  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps)
//   xh = (x - mean) rstd,  d = dout w
//   dx = rstd (d - sum d / n - xh sum (d xh) / n),   dw = sum_rows dout xh,   dbias = sum_rows dout
//
// Bound by HBM: x is read and out written once, x and dout read and dx written once.  A group of TPR
// lanes holds a row in registers (EPT elements a lane, in vectors of VEC), so the sum of squares is
// taken about the mean in a second pass over registers, which also corrects the mean, and the sums are
// fp32.  A lane's columns are the same in every row: w and bias are loaded once, and the backward adds
// its rows' dw and dbias up in registers, joins a workgroup's groups in LDS and leaves one part per
// workgroup, which a second kernel adds in a fixed order: results are bitwise reproducible.
#include "kla_buf.hpp"
#include "kla_device.hpp"
#include "kla_internal.hpp"

namespace kla {
namespace {

template <typename E, int VEC>
__device__ __forceinline__ void load_vec(const E* p, float* f) {
    if constexpr (sizeof(E) == 4) {
        if constexpr (VEC == 4) {
            const float4 v = *reinterpret_cast<const float4*>(p);
            f[0] = v.x;
            f[1] = v.y;
            f[2] = v.z;
            f[3] = v.w;
        } else {
            f[0] = p[0];
        }
    } else if constexpr (VEC == 1) {
        f[0] = bf16_to_f32(p[0]);
    } else {
        uint32_t w[VEC / 2];
        if constexpr (VEC == 8) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            w[0] = u.x;
            w[1] = u.y;
            w[2] = u.z;
            w[3] = u.w;
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        }
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) {
            f[2 * e] = __uint_as_float(w[e] << 16);
            f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
}

template <typename E, int VEC>
__device__ __forceinline__ void store_vec(E* p, const float* f) {
    if constexpr (sizeof(E) == 4) {
        if constexpr (VEC == 4)
            *reinterpret_cast<float4*>(p) = float4{f[0], f[1], f[2], f[3]};
        else
            p[0] = f[0];
    } else if constexpr (VEC == 8) {
        *reinterpret_cast<uint4*>(p) =
            uint4{cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]), cvt_pk_bf16(f[4], f[5]), cvt_pk_bf16(f[6], f[7])};
    } else if constexpr (VEC == 2) {
        *reinterpret_cast<uint32_t*>(p) = cvt_pk_bf16(f[0], f[1]);
    } else {
        p[0] = f32_to_bf16(f[0]);
    }
}

// VEC fp32 values of a weight, zero where there is none (none are read past a row's end: VEC divides n).
template <int VEC>
__device__ __forceinline__ void load_w(const float* w, int c, int n, float* f) {
    if (w && c < n) {
        if constexpr (VEC % 4 == 0) {
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                const float4 v = *reinterpret_cast<const float4*>(w + c + e);
                f[e] = v.x;
                f[e + 1] = v.y;
                f[e + 2] = v.z;
                f[e + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = w[c + e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = 0.f;
    }
}

// Sums of M values over the TPR lanes of a row, in every lane.  buf: LDS for groups of several waves, two
// slots of 2 x TPR / 64 floats taken in turn, so that one barrier per call is enough.
template <int TPR, int M>
__device__ __forceinline__ void group_sum(float (&a)[M], float* buf, int& turn) {
    if constexpr (TPR < 64) {
#pragma unroll
        for (int m = 1; m < TPR; m *= 2)
#pragma unroll
            for (int i = 0; i < M; ++i) a[i] += __shfl_xor(a[i], m);
    } else {
#pragma unroll
        for (int i = 0; i < M; ++i) a[i] = wave_sum(a[i]);
        if constexpr (TPR > 64) {
            constexpr int NW = TPR / 64;
            const int group = threadIdx.x / TPR, wave = (threadIdx.x % TPR) / 64;
            const int groups = blockDim.x / TPR;
            float* s = buf + (turn * groups + group) * 2 * NW;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < M; ++i) s[M * wave + i] = a[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < M; ++i) a[i] = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int i = 0; i < M; ++i) a[i] += s[M * w + i];
        }
    }
}

// Workgroup sizes: forward 256 threads, more for rows of more lanes; backward 1024, one workgroup a CU, so that
// there are few parts (16384 x 2048 bf16: 46 us; 50 with 512 threads, 54 with two such workgroups a CU;
// 65536 x 256: 28, 37, 27).
template <int TPR>
constexpr int kFwdThreads = TPR > 256 ? TPR : 256;
constexpr int kBwdThreads = 1024;

template <typename E, int VEC, int EPT, int TPR>
__global__ __launch_bounds__(kFwdThreads<TPR>) void layernorm_fwd_kernel(size_t rows, int n, const E* __restrict__ x,
                                                                       const float* __restrict__ w,
                                                                       const float* __restrict__ bias, float eps,
                                                                       E* __restrict__ out, float* __restrict__ mean,
                                                                       float* __restrict__ rstd) {
    constexpr int HB = EPT / VEC, RPB = kFwdThreads<TPR> / TPR;
    __shared__ float buf[TPR > 64 ? 2 * RPB * 2 * (TPR / 64) : 1];
    const int tl = threadIdx.x % TPR;
    const float inv = 1.f / (float)n;
    float wr[EPT], br[EPT];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        load_w<VEC>(w, (i * TPR + tl) * VEC, n, wr + i * VEC);
        load_w<VEC>(bias, (i * TPR + tl) * VEC, n, br + i * VEC);
    }
    int turn = 0;
    // every group of the workgroup takes part in each round: the sums hold barriers
    for (size_t r0 = (size_t)blockIdx.x * RPB; r0 < rows; r0 += (size_t)gridDim.x * RPB) {
        const size_t r = r0 + threadIdx.x / TPR;
        const bool live = r < rows;
        float v[EPT], s[1] = {0.f}, t[2] = {0.f, 0.f};   // t: of squares and of what the mean leaves
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int c = (i * TPR + tl) * VEC;
            if (live && c < n) {
                load_vec<E, VEC>(x + r * n + c, v + i * VEC);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i * VEC + e] = 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < EPT; ++e) s[0] += v[e];
        group_sum<TPR>(s, buf, turn);
        // The sum's roundings are up to 2^-20 of |x|, which rstd may raise 300 times: the mean of what it leaves
        // corrects it, at the barrier that the squares need.  x - mu is exact near a mu that is rounded: kept from
        // being contracted with the product.
        float mu = s[0] * inv;
        asm("" : "+v"(mu));
#pragma unroll
        for (int i = 0; i < HB; ++i)
            if ((i * TPR + tl) * VEC < n)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[i * VEC + e] -= mu;
                    t[0] += v[i * VEC + e] * v[i * VEC + e];
                    t[1] += v[i * VEC + e];
                }
        group_sum<TPR>(t, buf, turn);
        const float c = t[1] * inv, var = t[0] * inv - c * c, rs = 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);
        mu += c;
        if (!live) continue;
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int at = (i * TPR + tl) * VEC;
            if (at < n) {
                float o[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = fmaf(v[i * VEC + e], rs, -c * rs) * wr[i * VEC + e] + br[i * VEC + e];
                store_vec<E, VEC>(out + r * n + at, o);
            }
        }
        if (tl == 0) {
            if (mean) mean[r] = mu;
            if (rstd) rstd[r] = rs;
        }
    }
}

// part: [gridDim.x][2][n], the workgroups' sums of dw and dbias.
template <typename E, int VEC, int EPT, int TPR>
__global__ __launch_bounds__(kBwdThreads) void layernorm_bwd_kernel(size_t rows, int n, const E* __restrict__ x,
                                                                       const float* __restrict__ w,
                                                                       const float* __restrict__ mean,
                                                                       const float* __restrict__ rstd,
                                                                       const E* __restrict__ dout, E* __restrict__ dx,
                                                                       float* __restrict__ part) {
    constexpr int HB = EPT / VEC, RPB = kBwdThreads / TPR;
    __shared__ float buf[TPR > 64 ? 2 * RPB * 2 * (TPR / 64) : 1];
    constexpr int JG = kBwdThreads / (TPR < 64 ? 64 : TPR);   // groups that join: of a wave at least
    __shared__ float join[JG > 1 ? 2 * EPT * TPR : 1];
    const int tl = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const float inv = 1.f / (float)n;
    float wr[EPT], sw[EPT], sb[EPT];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        load_w<VEC>(w, (i * TPR + tl) * VEC, n, wr + i * VEC);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sw[i * VEC + e] = sb[i * VEC + e] = 0.f;
    }
    int turn = 0;
    for (size_t r0 = (size_t)blockIdx.x * RPB; r0 < rows; r0 += (size_t)gridDim.x * RPB) {
        const size_t r = r0 + group;
        const bool live = r < rows;
        float v[EPT], d[EPT];
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int c = (i * TPR + tl) * VEC;
            if (live && c < n) {
                load_vec<E, VEC>(x + r * n + c, v + i * VEC);
                load_vec<E, VEC>(dout + r * n + c, d + i * VEC);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i * VEC + e] = d[i * VEC + e] = 0.f;
            }
        }
        const float mu = live ? mean[r] : 0.f, rs = live ? rstd[r] : 0.f;
        float t[2] = {0.f, 0.f};   // sums of d and of d xh
#pragma unroll
        for (int i = 0; i < HB; ++i)
            if ((i * TPR + tl) * VEC < n)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int j = i * VEC + e;
                    v[j] = (v[j] - mu) * rs;
                    sw[j] += d[j] * v[j];
                    sb[j] += d[j];
                    d[j] *= wr[j];
                    t[0] += d[j];
                    t[1] += d[j] * v[j];
                }
        group_sum<TPR>(t, buf, turn);
        const float c1 = t[0] * inv, c2 = t[1] * inv;
        if (!live) continue;
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int c = (i * TPR + tl) * VEC;
            if (c < n) {
                float o[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = rs * (d[i * VEC + e] - c1 - v[i * VEC + e] * c2);
                store_vec<E, VEC>(dx + r * n + c, o);
            }
        }
    }
    if constexpr (TPR < 64) {   // a wave's groups
#pragma unroll
        for (int m = TPR; m < 64; m *= 2)
#pragma unroll
            for (int j = 0; j < EPT; ++j) {
                sw[j] += __shfl_xor(sw[j], m);
                sb[j] += __shfl_xor(sb[j], m);
            }
    }
    const int jg = threadIdx.x / (TPR < 64 ? 64 : TPR);
    const bool first = TPR >= 64 || (threadIdx.x & 63) < TPR;   // of its wave's groups
    // the groups' sums one after another into LDS, the last group's into the part
    if constexpr (JG > 1) {
        for (int k = 0; k < JG; ++k) {
            if (jg == k && first) {
#pragma unroll
                for (int j = 0; j < EPT; ++j) {
                    if (k > 0) {
                        sw[j] += join[j * TPR + tl];
                        sb[j] += join[(EPT + j) * TPR + tl];
                    }
                    join[j * TPR + tl] = sw[j];
                    join[(EPT + j) * TPR + tl] = sb[j];
                }
            }
            __syncthreads();
        }
    }
    if (jg == JG - 1 && first) {
        float* p = part + (size_t)blockIdx.x * 2 * n;
#pragma unroll
        for (int i = 0; i < HB; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int c = (i * TPR + tl) * VEC + e;
                if (c < n) {
                    p[c] = sw[i * VEC + e];
                    p[n + c] = sb[i * VEC + e];
                }
            }
    }
}

// dw, dbias: 32 columns of the parts per workgroup, 16 parts side by side.
__global__ __launch_bounds__(512) void layernorm_parts_kernel(int nparts, int n, const float* __restrict__ part,
                                                             float* __restrict__ dw, float* __restrict__ dbias) {
    __shared__ float s[16][33];
    const int col = threadIdx.x % 32, k = threadIdx.x / 32;
    const size_t c = (size_t)blockIdx.x * 32 + col, n2 = 2 * (size_t)n;
    float t = 0.f;
    if (c < n2)
#pragma unroll 8
        for (int p = k; p < nparts; p += 16) t += part[p * n2 + c];
    s[k][col] = t;
    __syncthreads();
    if (k == 0 && c < n2) {
        for (int i = 1; i < 16; ++i) t += s[i][col];
        if (c < (size_t)n)
            dw[c] = t;
        else if (dbias)
            dbias[c - n] = t;
    }
}

constexpr unsigned kParts = 256;   // workgroups of the backward, one per CU

// Calls f<VEC, EPT, TPR> for a row of n elements: the widest vectors that rows of n keep aligned, and the
// fewest lanes that hold a row in 16 registers each (16384 x 2048 bf16, forward: 24 us with 16 elements on
// 128 lanes, 24 with 8 on 256, 27 with 32 on 64; backward, whose lanes hold five such rows: 46, 46, and 168 in
// more registers than its 1024 threads have).
template <typename E, typename F>
hipError_t by_shape(int n, F&& f) {
#define KLA_LN_SHAPES(V_)                                                               \
    if (n <= 128) return f.template run<E, V_, 8, 16>();                       \
    if (n <= 512) return f.template run<E, V_, 8, 64>();                                  \
    if (n <= 1024) return f.template run<E, V_, 16, 64>();                                \
    if (n <= 2048) return f.template run<E, V_, 16, 128>();                                \
    if (n <= 4096) return f.template run<E, V_, 16, 256>();                               \
    if (n <= 8192) return f.template run<E, V_, 16, 512>();                               \
    return f.template run<E, V_, 16, 1024>();
    if constexpr (sizeof(E) == 2) {
        if (n % 8 == 0) {
            KLA_LN_SHAPES(8)
        }
        if (n % 2 == 0) {
            KLA_LN_SHAPES(2)
        }
    } else if (n % 4 == 0) {
        KLA_LN_SHAPES(4)
    }
    KLA_LN_SHAPES(1)
#undef KLA_LN_SHAPES
}

struct Fwd {
    size_t rows;
    int n;
    const void* x;
    const float *w, *bias;
    float eps;
    void* out;
    float *mean, *rstd;
    hipStream_t st;
    template <typename E, int VEC, int EPT, int TPR>
    hipError_t run() {
        constexpr int RPB = kFwdThreads<TPR> / TPR;
        const size_t blocks = (rows + RPB - 1) / RPB;
        const unsigned grid = (unsigned)(blocks < 4096 ? blocks : 4096);
        layernorm_fwd_kernel<E, VEC, EPT, TPR><<<dim3(grid), dim3(kFwdThreads<TPR>), 0, st>>>(
            rows, n, static_cast<const E*>(x), w, bias, eps, static_cast<E*>(out), mean, rstd);
        return hipGetLastError();
    }
};

struct Bwd {
    size_t rows;
    int n;
    const void* x;
    const float *w, *mean, *rstd;
    const void* dout;
    void* dx;
    float *dw, *dbias, *part;
    hipStream_t st;
    template <typename E, int VEC, int EPT, int TPR>
    hipError_t run() {
        constexpr int RPB = kBwdThreads / TPR;
        const size_t blocks = (rows + RPB - 1) / RPB;
        const unsigned grid = (unsigned)(blocks < 1 ? 1 : blocks < kParts ? blocks : kParts);
        layernorm_bwd_kernel<E, VEC, EPT, TPR><<<dim3(grid), dim3(kBwdThreads), 0, st>>>(
            rows, n, static_cast<const E*>(x), w, mean, rstd, static_cast<const E*>(dout), static_cast<E*>(dx), part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        layernorm_parts_kernel<<<dim3((unsigned)((2 * (size_t)n + 31) / 32)), dim3(512), 0, st>>>((int)grid, n, part, dw, dbias);
        return hipGetLastError();
    }
};

}  // namespace

size_t layernorm_parts_bytes(int n) { return (size_t)kParts * 2 * n * sizeof(float); }

hipError_t launch_layernorm_fwd(size_t rows, int n, bool bf16, const void* x, const float* w, const float* bias, float eps,
                                void* out, float* mean, float* rstd, hipStream_t st) {
    if (rows == 0) return hipSuccess;
    Fwd f{rows, n, x, w, bias, eps, out, mean, rstd, st};
    return bf16 ? by_shape<uint16_t>(n, f) : by_shape<float>(n, f);
}

hipError_t launch_layernorm_bwd(size_t rows, int n, bool bf16, const void* x, const float* w, const float* mean,
                                const float* rstd, const void* dout, void* dx, float* dw, float* dbias, float* part,
                                hipStream_t st) {
    Bwd f{rows, n, x, w, mean, rstd, dout, dx, dw, dbias, part, st};
    return bf16 ? by_shape<uint16_t>(n, f) : by_shape<float>(n, f);
}

}  // namespace kla
