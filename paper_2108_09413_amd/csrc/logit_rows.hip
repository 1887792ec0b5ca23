// Operators on rows of class logits: log-probabilities of given classes with entropy and top alternatives, distillation from
// a teacher's top logits, and the gradient of both.
//
// Row statistics: m = max x, s = sum exp(scale (x - m)), t = sum exp(.) scale (x - m).  Differences are taken before
// the scale, so rows of the type's lowest value, far offsets and int32 logits (whose differences are exact) lose nothing.
// s is NaN exactly for rows that hold NaN or +infinity, m is -infinity for rows without a possible class.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "logit_rows.h"

namespace isr {

constexpr float NEG_INF = -__builtin_inff();

template <int TYPE> struct Kind;
template <> struct Kind<ISR_F32> {
    using Raw = float; using Val = float; using Grad = float;
    static __device__ __forceinline__ float val(float r) { return r + 0.f; }   // -0 and 0 are one value
    static __device__ __forceinline__ float grad(float g) { return g; }
};
template <> struct Kind<ISR_BF16> {
    using Raw = uint16_t; using Val = float; using Grad = __hip_bfloat16;
    static __device__ __forceinline__ float val(uint16_t r) { return __uint_as_float((uint32_t)r << 16) + 0.f; }
    static __device__ __forceinline__ __hip_bfloat16 grad(float g) { return __float2bfloat16(g); }   // the caller's type: one rounding, to nearest
};
template <> struct Kind<ISR_F16> {
    using Raw = _Float16; using Val = float; using Grad = _Float16;
    static __device__ __forceinline__ float val(_Float16 r) { return (float)r + 0.f; }
    static __device__ __forceinline__ _Float16 grad(float g) { return (_Float16)g; }
};
template <> struct Kind<ISR_I32> {
    using Raw = int32_t; using Val = int32_t; using Grad = float;
    static __device__ __forceinline__ int32_t val(int32_t r) { return r; }
    static __device__ __forceinline__ float grad(float g) { return g; }
};

__device__ __forceinline__ float lowest(float) { return NEG_INF; }
__device__ __forceinline__ int32_t lowest(int32_t) { return INT32_MIN; }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ int32_t larger(int32_t a, int32_t b) { return a > b ? a : b; }
// x - m, m >= x; no possible class at all: x itself, which is -infinity
__device__ __forceinline__ float below(float x, float m) { return x - (m == NEG_INF ? 0.f : m); }
__device__ __forceinline__ float below(int32_t x, int32_t m) { return -(float)((uint32_t)m - (uint32_t)x); }
// the same in 64 bits, of a row that has a possible class: the two ends of fp32 lie further apart than fp32 reaches
template <class Val> __device__ __forceinline__ double below64(Val x, Val m) { return (double)x - (double)m; }
__device__ __forceinline__ bool possible(float x) { return x > NEG_INF; }
__device__ __forceinline__ bool possible(int32_t) { return true; }
__device__ __forceinline__ float bits_of(float m) { return m; }
__device__ __forceinline__ float bits_of(int32_t m) { return __int_as_float(m); }
template <class Val> __device__ __forceinline__ Val of_bits(float b);
template <> __device__ __forceinline__ float of_bits<float>(float b) { return b; }
template <> __device__ __forceinline__ int32_t of_bits<int32_t>(float b) { return __float_as_int(b); }

template <class Val>
struct Stat {
    Val m;
    float s, t;
    __device__ __forceinline__ void clear() { m = lowest(m); s = 0.f; t = 0.f; }
    __device__ __forceinline__ void join(const Stat &o, float scale) {
        const Val top = larger(m, o.m);
        const float d0 = scale * below(m, top), d1 = scale * below(o.m, top);
        const float f0 = s == 0.f ? 0.f : expf(d0), f1 = o.s == 0.f ? 0.f : expf(d1);
        t = f0 * (t + (f0 == 0.f ? 0.f : d0 * s)) + f1 * (o.t + (f1 == 0.f ? 0.f : d1 * o.s));
        s = f0 * s + f1 * o.s;
        m = top;
    }
};

constexpr int THREADS = 256;

template <class Val>
__device__ Stat<Val> block_join(Stat<Val> a, float scale, Stat<Val> *part) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        Stat<Val> o;
        o.m = __shfl_xor(a.m, off, 64); o.s = __shfl_xor(a.s, off, 64); o.t = __shfl_xor(a.t, off, 64);
        a.join(o, scale);
    }
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
    __syncthreads();
    a = part[0];
    for (int w = 1; w < THREADS / 64; ++w) a.join(part[w], scale);
    __syncthreads();
    return a;
}

// Statistics of one row by a workgroup; `skip(j)`: classes that are left out.
template <int TYPE, class Skip>
__device__ Stat<typename Kind<TYPE>::Val> row_stat(const typename Kind<TYPE>::Raw *x, uint32_t classes, float scale, Stat<typename Kind<TYPE>::Val> *part, Skip skip) {
    Stat<typename Kind<TYPE>::Val> a;
    a.clear();
    for (uint32_t j = threadIdx.x; j < classes; j += THREADS) {
        if (skip(j)) continue;
        const auto v = Kind<TYPE>::val(x[j]);
        Stat<typename Kind<TYPE>::Val> one;
        one.m = v; one.s = possible(v) ? 1.f : 0.f; one.t = 0.f;
        if (one.s == 0.f && v != v) one.s = v;
        if ((float)v == -NEG_INF) one.s = __builtin_nanf("");
        a.join(one, scale);
    }
    return block_join(a, scale, part);
}

template <int TYPE>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(const LogprobsParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    __shared__ Stat<Val> part[THREADS / 64];
    __shared__ Val best_v[THREADS / 64];
    __shared__ int best_i[THREADS / 64];
    for (uint64_t r = blockIdx.x; r < p.l.rows; r += gridDim.x) {
        const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
        const Stat<Val> a = row_stat<TYPE>(x, p.l.classes, p.l.scale, part, [](uint32_t) { return false; });
        const bool bad = a.s != a.s, empty = a.s == 0.f;
        const float logs = empty ? 0.f : logf(a.s), nan = __builtin_nanf("");
        if (threadIdx.x == 0) {
            if (p.entropy) p.entropy[r] = bad ? nan : empty ? 0.f : logs - a.t / a.s;
            if (p.stats) { p.stats[2 * r] = bits_of(a.m); p.stats[2 * r + 1] = bad ? nan : empty ? NEG_INF : logs; }
        }
        for (uint32_t g = threadIdx.x; g < p.n_given; g += THREADS) {
            const int32_t c = p.given[r * p.n_given + g];
            float lp = nan;
            if (c < 0) lp = 0.f;
            else if ((uint32_t)c < p.l.classes && !bad) {
                const Val v = K::val(x[c]);
                lp = possible(v) ? p.l.scale * below(v, a.m) - logs : NEG_INF;
            }
            p.logprob[r * p.n_given + g] = lp;
        }
        // the largest of those behind the last one taken
        Val last_v = lowest(Val());
        int last_i = -1;
        for (uint32_t k = 0; k < p.top; ++k) {
            Val bv = lowest(Val());
            int bi = INT32_MAX;
            if (!bad)
                for (uint32_t j = threadIdx.x; j < p.l.classes; j += THREADS) {
                    const Val v = K::val(x[j]);
                    const bool open = possible(v) && (k == 0 || v < last_v || (v == last_v && (int)j > last_i));
                    if (open && (bi == INT32_MAX || v > bv)) { bv = v; bi = (int)j; }
                }
            auto take = [&](Val ov, int oi) { if (oi != INT32_MAX && (bi == INT32_MAX || ov > bv || (ov == bv && oi < bi))) { bv = ov; bi = oi; } };
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) take(__shfl_xor(bv, off, 64), __shfl_xor(bi, off, 64));
            if ((threadIdx.x & 63) == 0) { best_v[threadIdx.x >> 6] = bv; best_i[threadIdx.x >> 6] = bi; }
            __syncthreads();
            for (int w = 0; w < THREADS / 64; ++w) take(best_v[w], best_i[w]);
            __syncthreads();
            if (threadIdx.x == 0) {
                const bool none = bi == INT32_MAX;
                p.top_class[r * p.top + k] = none ? -1 : bi;
                p.top_logprob[r * p.top + k] = bad ? nan : none ? NEG_INF : p.l.scale * below(bv, a.m) - logs;
            }
            if (bi == INT32_MAX) bi = INT32_MAX - 1;   // nothing is behind it
            last_v = bv;
            last_i = bi;
        }
    }
}

template <int TYPE>
__global__ __launch_bounds__(THREADS) void logprobs_grad_kernel(const LogprobsGradParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    for (uint64_t r = blockIdx.x; r < p.l.rows; r += gridDim.x) {
        const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
        auto *out = (typename K::Grad *)p.grad + r * p.grad_stride;
        const Val m = of_bits<Val>(p.stats[2 * r]);
        const float logs = p.stats[2 * r + 1], uh = p.up_entropy ? p.up_entropy[r] : 0.f, h = uh != 0.f ? p.entropy[r] : 0.f;
        float up = 0.f;
        bool any = uh != 0.f;
        for (uint32_t g = 0; g < p.n_given; ++g) {
            const int32_t c = p.given[r * p.n_given + g];
            if (c < 0) continue;
            any = true;
            up += (uint32_t)c < p.l.classes ? p.up_logprob[r * p.n_given + g] : __builtin_nanf("");
        }
        const bool zero = !any || logs == NEG_INF;
        for (uint32_t j = threadIdx.x; j < p.l.classes; j += THREADS) {
            float g = 0.f;
            if (!zero) {
                const float lp = p.l.scale * below(K::val(x[j]), m) - logs, pr = expf(lp);
                g = -pr * up;
                if (uh != 0.f && pr != 0.f) g -= uh * pr * (lp + h);
                for (uint32_t i = 0; i < p.n_given; ++i)
                    if (p.given[r * p.n_given + i] == (int32_t)j) g += p.up_logprob[r * p.n_given + i];
                g *= p.l.scale;
            }
            out[j] = K::grad(g);
        }
    }
}

// Statistics of a row between the loss and its gradient.  zero: neither an entry nor a possible class, the gradient is zero.
struct DistillStat {
    float m, logs;           // of all classes
    float rest_m, rest_logs; // of those that are no entry (rest)
    float value_m, value_logs;   // q = exp(value_scale (value - value_m) - value_logs)
    float total, left;       // sum of q (and q_rest); q_rest
};
static_assert(sizeof(DistillStat) == 32, "eight words a row");

__device__ __forceinline__ float teacher_value(const void *p, int type, uint64_t i) {
    if (type == ISR_F32) return ((const float *)p)[i];
    if (type == ISR_BF16) return Kind<ISR_BF16>::val(((const uint16_t *)p)[i]);
    return (float)((const _Float16 *)p)[i];
}

template <int TYPE>
__global__ __launch_bounds__(THREADS) void distill_kernel(const DistillParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    __shared__ Stat<Val> part[THREADS / 64];
    __shared__ int entry[ISR_MAX_GIVEN];
    const float nan = __builtin_nanf("");
    for (uint64_t r = blockIdx.x; r < p.l.rows; r += gridDim.x) {
        const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
        __syncthreads();
        if (threadIdx.x < p.top) entry[threadIdx.x] = p.entry[r * p.top + threadIdx.x];
        __syncthreads();
        bool any = false, outside = false;
        float vm = NEG_INF;
        for (uint32_t i = 0; i < p.top; ++i) {
            if (entry[i] < 0) continue;
            any = true;
            outside |= (uint32_t)entry[i] >= p.l.classes;
            const float v = teacher_value(p.value, p.value_type, r * p.top + i);
            if (v != v || v == -NEG_INF) outside = true;
            vm = fmaxf(vm, v);
        }
        if (p.rest) vm = 0.f;
        if (!any || vm == NEG_INF) {
            if (threadIdx.x == 0) {
                p.loss[r] = 0.f;
                if (p.stats) *(DistillStat *)(p.stats + 8 * r) = DistillStat{0.f, NEG_INF, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            }
            continue;
        }
        const Stat<Val> a = row_stat<TYPE>(x, p.l.classes, p.l.scale, part, [](uint32_t) { return false; });
        Stat<Val> b = a;
        if (p.rest) b = row_stat<TYPE>(x, p.l.classes, p.l.scale, part, [&](uint32_t j) {
            for (uint32_t i = 0; i < p.top; ++i)
                if (entry[i] == (int)j) return true;
            return false;
        });
        if (threadIdx.x != 0) continue;
        const bool empty = a.s == 0.f;
        const double logs = empty ? 0.0 : log((double)a.s), rest_logs = b.s == 0.f ? NEG_INF : log((double)b.s);
        double z = 0.0;
        for (uint32_t i = 0; i < p.top; ++i)
            if (entry[i] >= 0) z += exp((double)p.value_scale * ((double)teacher_value(p.value, p.value_type, r * p.top + i) - vm));
        const double value_logs = p.rest ? 0.0 : log(z);
        double loss = 0.0, total = 0.0;
        for (uint32_t i = 0; i < p.top; ++i) {
            if (entry[i] < 0 || (uint32_t)entry[i] >= p.l.classes) continue;
            const double logq = (double)p.value_scale * ((double)teacher_value(p.value, p.value_type, r * p.top + i) - vm) - value_logs, q = exp(logq);
            total += q;
            const Val v = K::val(x[entry[i]]);
            const double logp = empty || !possible(v) ? (double)NEG_INF : (double)p.l.scale * below64(v, a.m) - logs;
            if (q > 0.0) loss += q * (logq - logp);
        }
        double left = 0.0;
        if (p.rest) {
            left = 1.0 - total > 0.0 ? 1.0 - total : 0.0;
            total += left;
            const double logr = b.s == 0.f ? (double)NEG_INF : (double)p.l.scale * below64(b.m, a.m) + rest_logs - logs;
            if (left > 0.0) loss += left * (log(left) - logr);
        }
        if (outside || a.s != a.s) loss = total = nan;
        p.loss[r] = (float)loss;
        if (p.stats)
            *(DistillStat *)(p.stats + 8 * r) = DistillStat{bits_of(a.m), empty ? NEG_INF : (float)logs, bits_of(b.m), (float)rest_logs,
                                                             vm, (float)value_logs, (float)total, (float)left};
    }
}

template <int TYPE>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(const DistillParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    __shared__ int entry[ISR_MAX_GIVEN];
    __shared__ float q[ISR_MAX_GIVEN];
    for (uint64_t r = blockIdx.x; r < p.l.rows; r += gridDim.x) {
        const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
        auto *out = (typename K::Grad *)p.grad + r * p.grad_stride;
        const DistillStat st = *(const DistillStat *)(p.stats + 8 * r);
        __syncthreads();
        if (threadIdx.x < p.top) {
            entry[threadIdx.x] = p.entry[r * p.top + threadIdx.x];
            q[threadIdx.x] = expf(p.value_scale * (teacher_value(p.value, p.value_type, r * p.top + threadIdx.x) - st.value_m) - st.value_logs);
        }
        __syncthreads();
        const float w = p.weight ? p.weight[r] : 1.f, f = p.l.scale * w;
        const bool zero = w == 0.f || st.logs == NEG_INF;
        const Val m = of_bits<Val>(st.m), rest_m = of_bits<Val>(st.rest_m);
        const float logr = p.l.scale * below(rest_m, m) + st.rest_logs - st.logs;
        const float rest_c = p.rest ? st.total * expf(logr) - st.left : 0.f;
        for (uint32_t j = threadIdx.x; j < p.l.classes; j += THREADS) {
            float g = 0.f;
            if (!zero) {
                const Val v = K::val(x[j]);
                float sum = 0.f;
                bool is_entry = false;
                for (uint32_t i = 0; i < p.top; ++i)
                    if (entry[i] == (int)j) { is_entry = true; sum += q[i]; }
                if (!p.rest || is_entry) g = st.total * expf(p.l.scale * below(v, m) - st.logs) - sum;
                else g = rest_c * (possible(v) ? expf(p.l.scale * below(v, rest_m) - st.rest_logs) : 0.f);   // NaN in a row of NaN
                g *= f;
            }
            out[j] = K::grad(g);
        }
    }
}

static unsigned row_grid(uint64_t rows) { return (unsigned)(rows < (1u << 20) ? rows : (1u << 20)); }

#define LAUNCH_BY_TYPE(kernel, p, st)                                                                                        \
    const dim3 grid(row_grid((p).l.rows)), block(THREADS);                                                                   \
    switch ((p).l.type) {                                                                                                    \
    case ISR_F32: hipLaunchKernelGGL((kernel<ISR_F32>), grid, block, 0, st, p); break;                                       \
    case ISR_BF16: hipLaunchKernelGGL((kernel<ISR_BF16>), grid, block, 0, st, p); break;                                     \
    case ISR_F16: hipLaunchKernelGGL((kernel<ISR_F16>), grid, block, 0, st, p); break;                                       \
    default: hipLaunchKernelGGL((kernel<ISR_I32>), grid, block, 0, st, p); break;                                            \
    }                                                                                                                        \
    return hipGetLastError()

hipError_t launch_logprobs(const LogprobsParams &p, hipStream_t st) { LAUNCH_BY_TYPE(logprobs_kernel, p, st); }
hipError_t launch_logprobs_grad(const LogprobsGradParams &p, hipStream_t st) { LAUNCH_BY_TYPE(logprobs_grad_kernel, p, st); }
hipError_t launch_distill(const DistillParams &p, hipStream_t st) { LAUNCH_BY_TYPE(distill_kernel, p, st); }
hipError_t launch_distill_grad(const DistillParams &p, hipStream_t st) { LAUNCH_BY_TYPE(distill_grad_kernel, p, st); }

}  // namespace isr
