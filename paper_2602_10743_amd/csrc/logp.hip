// Log probabilities of tokens from logits, with the entropy and the top alternatives, and the
// gradient of the logits.
//
//   m = max_v x_v,  s = sum_v e^{x_v - m},  u = sum_v e^{x_v - m} (x_v - m)
//   logp = x_target - m - log s,   entropy = log s - u / s
//   dx_v = dlogp ([v = target] - p_v) - dent p_v (log p_v + entropy),   p_v = e^{x_v - m} / s
//
// Bound by HBM: the forward reads the logits once, a thread keeping the running maximum of its
// elements and the two sums about it, rescaled when the maximum rises; the backward reads and writes
// them once.  m and s are kept for the backward rather than log(sum e^x), whose rounding would be that
// of the largest logit.  A row is cut over several workgroups where there are few rows, and a second
// kernel joins the parts in a fixed order.
//
// The top alternatives come from a threshold: the K-th largest of 64 lanes' maxima is at most the
// K-th largest element.  It is taken after each thread's first blocks; the elements from it on are
// collected as the rest is read, and from the first blocks again.  They are ranked by a key that is
// larger for a larger value and, among equals, for the lower index; keys are unique, so the order in
// which they were collected does not matter.  Where there are more than there is room for, the row is
// read again with the threshold of all its elements, and where that does not help either (rows of
// equal elements) or too few lie above it (fewer than K above -inf), K readings take one each.
//
// Rows may start anywhere: threads read the aligned 16-byte blocks that lie inside the row whole, and
// the elements of the two at its ends one by one.
#include <type_traits>

#include "kla_device.hpp"
#include "kla_internal.hpp"

namespace kla {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTop = 32;
constexpr int kRoom = 1024;     // collected elements
constexpr int kMaxParts = 64;   // of a row
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eLo = (float)(1.4426950408889634 - (double)kLog2e);

template <typename E>
constexpr int kVec = 16 / (int)sizeof(E);

__device__ __forceinline__ void unpack(const uint4& u, float* f, uint16_t) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(w[e] << 16);
        f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& u, float* f, float) {
    f[0] = __uint_as_float(u.x);
    f[1] = __uint_as_float(u.y);
    f[2] = __uint_as_float(u.z);
    f[3] = __uint_as_float(u.w);
}

// The blocks of row r, [a, a + V) in elements, that part `part` of `parts` takes.
template <typename E>
struct Span {
    size_t a, b;      // the row's elements
    size_t lo, hi;    // its aligned blocks, those of this part
    __device__ Span(size_t r, int V, int part, int parts) {
        constexpr int N = kVec<E>;
        a = r * V;
        b = a + V;
        const size_t first = a / N, n = (b + N - 1) / N - first, per = (n + parts - 1) / parts;
        lo = first + (size_t)part * per;
        hi = lo + per < first + n ? lo + per : first + n;
    }
    __device__ bool whole(size_t blk) const { return blk * kVec<E> >= a && (blk + 1) * kVec<E> <= b; }
};

// f(x, v) for the elements x of a block that are the row's (v: its index in the row).
template <typename E, typename F>
__device__ __forceinline__ void one_block(const E* x, const Span<E>& s, size_t blk, F&& f) {
    constexpr int N = kVec<E>;
    if (s.whole(blk)) {
        float v[N];
        unpack(reinterpret_cast<const uint4*>(x)[blk], v, E());
#pragma unroll
        for (int e = 0; e < N; ++e) f(v[e], (uint32_t)(blk * N + e - s.a));
    } else {
        for (size_t i = blk * N > s.a ? blk * N : s.a; i < (blk + 1) * N && i < s.b; ++i) f(ld(x, i), (uint32_t)(i - s.a));
    }
}

// The same for the blocks of this part before `hi` that a thread takes.
template <typename E, typename F>
__device__ __forceinline__ void each(const E* x, const Span<E>& s, size_t hi, F&& f) {
    for (size_t blk = s.lo + threadIdx.x; blk < hi; blk += kThreads) one_block<E>(x, s, blk, f);
}

// Running maximum m (finite) and the sums about it.
struct Sums {
    float m, s, u;
};

// e^d of d <= 0 as 2^x of a rounded x: off by 2^-24 |x| of itself and the instruction's 2^-23.  For the sums, where
// |d| e^d is under 1/2 of the largest term, and for outputs of 8 bits.
__device__ __forceinline__ float exp2_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// The same with what x loses, for the fp32 gradients of unlikely tokens (d = -80: 2e-7 instead of 3e-6).  0 from
// d = -150 on, and for NaN.
__device__ __forceinline__ float exp_of(float d) {
    d = fmaxf(d, -150.f);
    const float x = d * kLog2e, lo = fmaf(d, kLog2eLo, fmaf(d, kLog2e, -x)), e = __builtin_amdgcn_exp2f(x);
    return fmaf(e, lo * 0.693147181f, e);
}

__device__ __forceinline__ void rise(Sums& t, float m) {   // m >= t.m
    const float d = fmaxf(t.m - m, kLowest), r = exp2_of(d);
    t.u = t.u * r + t.s * (d * r);   // d r is 0 where r is, however far the maximum rose
    t.s *= r;
    t.m = m;
}

template <bool ENT>
__device__ __forceinline__ void add(Sums& t, float x) {   // x <= t.m, or NaN
    const float d = x - t.m, e = exp2_of(d);
    t.s += e;
    if constexpr (ENT) t.u += e * fmaxf(d, kLowest);      // 0 for x = -inf
}

__device__ __forceinline__ Sums joined(const Sums& a, const Sums& b) {
    const float m = fmaxf(a.m, b.m);
    Sums p = a, q = b;
    rise(p, m);
    rise(q, m);
    return {m, p.s + q.s, p.u + q.u};
}

__device__ __forceinline__ Sums wave_join(Sums t) {
#pragma unroll
    for (int k = 1; k < 64; k *= 2) t = joined(t, Sums{__shfl_xor(t.m, k), __shfl_xor(t.s, k), __shfl_xor(t.u, k)});
    return t;
}

// Over the workgroup's threads, in every thread.
__device__ __forceinline__ Sums block_join(Sums t, Sums* buf) {
    t = wave_join(t);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x / 64] = t;
    __syncthreads();
    t = buf[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) t = joined(t, buf[w]);
    return t;
}

// Orders by value, the lower index first among equals; 0 for NaN, which is no alternative.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);   // -0 as 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t v) {
    return x == x ? (uint64_t)order_of(x) << 32 | (0xffffffffu - v) : 0;
}

struct TopScratch {
    uint64_t keys[kRoom];
    float lane[kThreads];
    uint64_t best[kThreads / 64];
    uint32_t count;
    float least;
};

// A bound at or below the K-th largest of the elements seen so far, m their maximum in this thread; the
// list is emptied.
__device__ __forceinline__ void set_least(int K, float m, TopScratch& t) {
    t.lane[threadIdx.x] = m;
    if (threadIdx.x == 0) t.count = 0;
    __syncthreads();
    if (threadIdx.x < 64) {
        float v = t.lane[threadIdx.x];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) v = fmaxf(v, t.lane[threadIdx.x + 64 * w]);
        // the K-th largest of the 64, to its upper 16 bits: bit by bit the largest prefix that K reach
        const uint32_t o = order_of(v);
        uint32_t pre = 0;
#pragma unroll
        for (int bit = 31; bit >= 16; --bit) {
            const uint32_t tryit = pre | 1u << bit;
            if (__popcll(__ballot(o >= tryit)) >= K) pre = tryit;
        }
        if (threadIdx.x == 0) t.least = value_of(pre);
    }
    __syncthreads();
}

__device__ __forceinline__ void collect(TopScratch& t, float least, float v, uint32_t i) {
    if (v >= least) {
        const uint32_t at = atomicAdd(&t.count, 1u);
        if (at < kRoom) t.keys[at] = key_of(v, i);
    }
}

// The K largest keys of this part's elements, in order, into out (0 where there are fewer), from those
// collected with a bound of the first blocks.  m: the maximum of the thread's own elements.
template <typename E>
__device__ void top_keys(const E* x, const Span<E>& sp, int K, float m, TopScratch& t, uint64_t* out) {
    __syncthreads();
    if (t.count > kRoom) {
        __syncthreads();   // every thread has read the count
        set_least(K, m, t);
        const float least = t.least;
        each<E>(x, sp, sp.hi, [&](float v, uint32_t i) { collect(t, least, v, i); });
        __syncthreads();
    }
    const int n = (int)t.count;
    if (n >= K && n <= kRoom) {
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const uint64_t mine = t.keys[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += t.keys[j] > mine;
            if (rank < K) out[rank] = mine;
        }
        return;
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < K; ++k) {
        uint64_t best = 0;
        each<E>(x, sp, sp.hi, [&](float v, uint32_t i) {
            const uint64_t key = key_of(v, i);
            if (key < last && key > best) best = key;
        });
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint64_t o = (uint64_t)__shfl_xor((int)(best >> 32), d) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)best, d);
            best = o > best ? o : best;
        }
        __syncthreads();   // the round before has read t.best
        if ((threadIdx.x & 63) == 0) t.best[threadIdx.x / 64] = best;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) best = t.best[w] > best ? t.best[w] : best;
        if (threadIdx.x == 0) out[k] = best;
        last = best;   // 0: no more elements
    }
}

struct LogpArgs {
    size_t rows, n;           // rows = S n
    int V, top, parts;
    const void* logits;
    const int64_t* target;    // [n]
    float *logp, *entropy, *stat, *top_logp;
    int64_t* top_index;
    Sums* sums;               // [rows][parts]
    uint64_t* keys;           // [rows][parts][top]
};

// A row's target and its logit; rows are less than 2^31.
struct Hot {
    int64_t at;
    float x;
};
__device__ __forceinline__ int64_t target_of(const LogpArgs& a, size_t r) { return a.target[(uint32_t)r % (uint32_t)a.n]; }
template <typename E>
__device__ __forceinline__ Hot hot_of(const LogpArgs& a, size_t r) {
    const int64_t tg = target_of(a, r);
    return {tg, tg >= 0 && tg < a.V ? ld(static_cast<const E*>(a.logits), r * a.V + (size_t)tg) : 0.f};
}

// What is written of a row: t in every thread, the row's keys in LDS, h in thread 0.
__device__ __forceinline__ void finish(const LogpArgs& a, size_t r, const Sums& t, const Hot& h, const uint64_t* best) {
    const float ls = logf(t.s);   // -inf for a row of -inf
    if (threadIdx.x == 0) {
        float lp = 0.f;           // no target
        if (h.at >= a.V) lp = __uint_as_float(0x7fc00000u);
        else if (h.at >= 0) lp = t.s == 0.f ? -__builtin_inff() : h.x - t.m - ls;
        a.logp[r] = lp;
        if (a.entropy) a.entropy[r] = t.s == 0.f ? 0.f : ls - t.u / t.s;
        if (a.stat) {
            a.stat[2 * r] = t.m;
            a.stat[2 * r + 1] = t.s;
        }
    }
    if ((int)threadIdx.x < a.top) {
        const uint64_t k = best[threadIdx.x];
        const size_t o = r * a.top + threadIdx.x;
        const float x = value_of((uint32_t)(k >> 32));
        a.top_index[o] = k ? (int64_t)(0xffffffffu - (uint32_t)k) : -1;
        a.top_logp[o] = !k ? __uint_as_float(0x7fc00000u) : t.s == 0.f ? -__builtin_inff() : x - t.m - ls;
    }
}

// One part of one row.
template <typename E, bool ENT, bool TOP>
__global__ __launch_bounds__(kThreads) void logp_fwd_kernel(LogpArgs a) {
    constexpr int N = kVec<E>;
    __shared__ Sums buf[kThreads / 64];
    __shared__ __align__(16) unsigned char scratch[TOP ? sizeof(TopScratch) : 16];
    __shared__ uint64_t best[TOP ? kMaxTop : 1];
    const size_t r = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts;
    const E* x = static_cast<const E*>(a.logits);
    const Span<E> sp(r, a.V, part, a.parts);
    TopScratch& ts = *reinterpret_cast<TopScratch*>(scratch);
    Hot hot{-1, 0.f};   // asked for first: at the end nothing would hide the two reads
    if (threadIdx.x == 0 && a.parts == 1) hot = hot_of<E>(a, r);
    Sums t{kLowest, 0.f, 0.f};
    constexpr int U = 4;   // blocks in flight per thread
    // M blocks of this thread from blk on, kThreads apart
    auto take = [&](size_t blk, auto count, float least) __attribute__((always_inline)) {
        constexpr int M = decltype(count)::value;
        float v[M * N];
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const size_t bi = blk + (size_t)i * kThreads;
            if (sp.whole(bi)) {
                unpack(reinterpret_cast<const uint4*>(x)[bi], v + i * N, E());
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const size_t at = bi * N + e;
                    v[i * N + e] = at >= sp.a && at < sp.b ? ld(x, at) : -__builtin_inff();
                }
            }
        }
        float m = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < M; ++i) {
            float bm = v[i * N];
#pragma unroll
            for (int e = 1; e < N; ++e) bm = fmaxf(bm, v[i * N + e]);
            if constexpr (TOP) {
                if (bm >= least)
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const size_t at = (blk + (size_t)i * kThreads) * N + e;
                        if (at >= sp.a && at < sp.b) collect(ts, least, v[i * N + e], (uint32_t)(at - sp.a));
                    }
            }
            m = fmaxf(m, bm);
        }
        rise(t, fmaxf(t.m, m));
#pragma unroll
        for (int e = 0; e < M * N; ++e) add<ENT>(t, v[e]);
    };
    size_t blk = sp.lo + threadIdx.x;
    auto rest = [&](size_t hi, float least) __attribute__((always_inline)) {
        for (; blk + (U - 1) * kThreads < hi; blk += U * kThreads) take(blk, std::integral_constant<int, U>(), least);
        for (; blk < hi; blk += kThreads) take(blk, std::integral_constant<int, 1>(), least);
    };
    if constexpr (TOP) {
        const size_t first = sp.lo + U * kThreads < sp.hi ? sp.lo + U * kThreads : sp.hi;
        rest(first, __uint_as_float(0x7fc00000u));   // a bound that nothing reaches
        set_least(a.top, t.m, ts);
        const float least = ts.least;
        rest(sp.hi, least);
        each<E>(x, sp, first, [&](float v, uint32_t i) { collect(ts, least, v, i); });
    } else {
        rest(sp.hi, 0.f);
    }
    const float own = t.m;
    t = block_join(t, buf);
    if constexpr (TOP) {
        uint64_t* out = a.parts > 1 ? a.keys + (size_t)blockIdx.x * a.top : best;
        top_keys<E>(x, sp, a.top, own, ts, out);
        __syncthreads();
    }
    if (a.parts > 1) {
        if (threadIdx.x == 0) a.sums[blockIdx.x] = t;
    } else {
        finish(a, r, t, hot, best);
    }
}

// The parts of one row: at most 64, whose lists are in order.  The top-th largest of the parts' first keys is
// at most the top-th largest of all, so only the keys from it on are ranked.
template <typename E>
__global__ __launch_bounds__(kThreads) void logp_join_kernel(LogpArgs a) {
    __shared__ uint64_t best[kMaxTop], keys[kMaxParts * kMaxTop];
    __shared__ uint64_t least;
    __shared__ uint32_t count;
    const size_t r = blockIdx.x;
    Hot hot{-1, 0.f};
    if (threadIdx.x == 0) hot = hot_of<E>(a, r);
    Sums t{kLowest, 0.f, 0.f};   // a part a lane, in every wave
    if ((int)(threadIdx.x & 63) < a.parts) t = a.sums[r * a.parts + (threadIdx.x & 63)];
    t = wave_join(t);
    if (a.top > 0) {
        const int n = a.parts * a.top;
        const uint64_t* in = a.keys + r * n;
        if ((int)threadIdx.x < a.top) best[threadIdx.x] = 0;
        if (threadIdx.x == 0) {
            least = 1;   // 0 is no key
            count = 0;
        }
        __syncthreads();
        if (threadIdx.x < 64 && a.parts >= a.top) {
            const uint64_t first = (int)threadIdx.x < a.parts ? in[threadIdx.x * a.top] : 0;
            int rank = 0;
            for (int p = 0; p < a.parts; ++p)
                rank += ((uint64_t)__builtin_amdgcn_readlane((int)(first >> 32), p) << 32 |
                         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)first, p)) > first;
            if (rank == a.top - 1 && first) least = first;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads)
            if (in[i] >= least) keys[atomicAdd(&count, 1u)] = in[i];
        __syncthreads();
        const int m = (int)count;
        for (int i = threadIdx.x; i < m; i += kThreads) {
            const uint64_t mine = keys[i];
            int rank = 0;
            for (int j = 0; j < m; ++j) rank += keys[j] > mine;
            if (rank < a.top) best[rank] = mine;
        }
        __syncthreads();
    }
    finish(a, r, t, hot, best);
}

// dlogits of one part of one row.
template <typename E>
__global__ __launch_bounds__(kThreads) void logp_bwd_kernel(LogpArgs a, const float* __restrict__ dlogp,
                                                            const float* __restrict__ dent, void* __restrict__ dlogits) {
    constexpr int N = kVec<E>;
    const size_t r = blockIdx.x / a.parts;
    const E* x = static_cast<const E*>(a.logits);
    E* o = static_cast<E*>(dlogits);
    const Span<E> sp(r, a.V, blockIdx.x % a.parts, a.parts);
    const float m = a.stat[2 * r], s = a.stat[2 * r + 1], ls = logf(s), inv = 1.f / s;
    const int64_t tg = target_of(a, r);
    const float dl = tg < 0 || !dlogp ? 0.f : tg < a.V ? dlogp[r] : __uint_as_float(0x7fc00000u);
    const float de = dent ? dent[r] : 0.f;
    // dlogp + dent (log p_v + entropy) = base + dent (x_v - m)
    const float base = dl + (de != 0.f ? de * (a.entropy[r] - ls) : 0.f);
    const size_t hot = tg >= 0 && tg < a.V ? sp.a + (size_t)tg : ~(size_t)0;
    auto grad = [&](float v, size_t at) {
        const float d = v - m, p = (N == 4 ? exp_of(d) : exp2_of(d)) * inv;   // NaN logits are in s
        float y = p == 0.f ? 0.f : -p * (base + de * d);
        if (at == hot) y += dl;
        return s == 0.f ? 0.f : y;
    };
    for (size_t blk = sp.lo + threadIdx.x; blk < sp.hi; blk += kThreads) {
        if (sp.whole(blk)) {
            float v[N];
            unpack(reinterpret_cast<const uint4*>(x)[blk], v, E());
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = grad(v[e], blk * N + e);
            if constexpr (N == 8)
                reinterpret_cast<uint4*>(o)[blk] = uint4{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]),
                                                         cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
            else
                reinterpret_cast<float4*>(o)[blk] = float4{v[0], v[1], v[2], v[3]};
        } else {
            for (size_t i = blk * N > sp.a ? blk * N : sp.a; i < (blk + 1) * N && i < sp.b; ++i) st(o, i, grad(ld(x, i), i));
        }
    }
}

// Parts a row is cut into: three workgroups a CU, none with less than 2048 elements.
int parts_of(size_t rows, int V) {
    int p = 1;
    while (rows * p < 768 && p < kMaxParts && V / (2 * p) >= 2048) p *= 2;
    return p;
}

template <typename E>
hipError_t fwd(const LogpArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)(a.rows * a.parts)), block(kThreads);
    if (a.top > 0) {
        if (a.entropy) logp_fwd_kernel<E, true, true><<<grid, block, 0, st>>>(a);
        else logp_fwd_kernel<E, false, true><<<grid, block, 0, st>>>(a);
    } else {
        if (a.entropy) logp_fwd_kernel<E, true, false><<<grid, block, 0, st>>>(a);
        else logp_fwd_kernel<E, false, false><<<grid, block, 0, st>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1) return e;
    logp_join_kernel<E><<<dim3((unsigned)a.rows), block, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t logp_workspace(size_t rows, int V, int top) {
    const int p = parts_of(rows, V);
    return p > 1 ? rows * p * (size_t)(16 + 8 * top) : 0;
}

hipError_t launch_logp_fwd(int S, size_t n, int V, int top, bool bf16, const void* logits, const int64_t* target,
                           float* logp, float* entropy, float* stat, float* top_logp, int64_t* top_index, void* ws,
                           hipStream_t st) {
    const size_t rows = (size_t)S * n;
    if (rows == 0) return hipSuccess;
    LogpArgs a{};
    a.rows = rows;
    a.n = n;
    a.V = V;
    a.top = top;
    a.parts = parts_of(rows, V);
    a.logits = logits;
    a.target = target;
    a.logp = logp;
    a.entropy = entropy;
    a.stat = stat;
    a.top_logp = top_logp;
    a.top_index = top_index;
    a.keys = static_cast<uint64_t*>(ws);
    a.sums = reinterpret_cast<Sums*>(static_cast<char*>(ws) + rows * a.parts * 8 * (size_t)top);
    return bf16 ? fwd<uint16_t>(a, st) : fwd<float>(a, st);
}

hipError_t launch_logp_bwd(int S, size_t n, int V, bool bf16, const void* logits, const int64_t* target,
                           const float* stat, const float* entropy, const float* dlogp, const float* dentropy,
                           void* dlogits, hipStream_t st) {
    const size_t rows = (size_t)S * n;
    if (rows == 0) return hipSuccess;
    LogpArgs a{};
    a.rows = rows;
    a.n = n;
    a.V = V;
    a.parts = parts_of(rows, V);
    a.logits = logits;
    a.target = target;
    a.stat = const_cast<float*>(stat);
    a.entropy = const_cast<float*>(entropy);
    const dim3 grid((unsigned)(rows * a.parts)), block(kThreads);
    if (bf16) logp_bwd_kernel<uint16_t><<<grid, block, 0, st>>>(a, dlogp, dentropy, dlogits);
    else logp_bwd_kernel<float><<<grid, block, 0, st>>>(a, dlogp, dentropy, dlogits);
    return hipGetLastError();
}

}  // namespace kla
