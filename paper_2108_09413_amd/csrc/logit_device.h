// Device code that the operators on rows of class logits share (logprobs.hip, distill.hip).
//
// Statistics of a set of logits: m = max x, s = sum exp(scale (x - m)), t = sum exp(.) * (scale (x - m) log2 e).  Differences
// are taken before the scale, so rows of the type's lowest value, far offsets and int32 logits (whose differences are exact)
// lose nothing.  s is NaN exactly for rows that hold NaN or +infinity, m is -infinity for rows without a possible class.
#pragma once
#include "logit_rows.h"

namespace isr {

constexpr float NEG_INF = -__builtin_inff();
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NO_SHARE = -200.f;   // 2^-200 is 0 in fp32: finite in place of log2 0, so that 0 * log 0 is 0

// ---- element types -------------------------------------------------------------------

template <int TYPE> struct Kind;
template <> struct Kind<ISR_F32> {
    using Raw = float; using Val = float; using Grad = float;
    static __device__ __forceinline__ float val(float r) { return r; }
    static __device__ __forceinline__ float grad(float g) { return g; }
};
template <> struct Kind<ISR_BF16> {
    using Raw = uint16_t; using Val = float; using Grad = __bf16;
    static __device__ __forceinline__ float val(uint16_t r) { return __uint_as_float((uint32_t)r << 16); }
    static __device__ __forceinline__ __bf16 grad(float g) { return (__bf16)g; }   // the caller's type: one rounding, to nearest
};
template <> struct Kind<ISR_F16> {
    using Raw = _Float16; using Val = float; using Grad = _Float16;
    static __device__ __forceinline__ float val(_Float16 r) { return (float)r; }
    static __device__ __forceinline__ _Float16 grad(float g) { return (_Float16)g; }
};
template <> struct Kind<ISR_I32> {
    using Raw = int32_t; using Val = int32_t; using Grad = float;
    static __device__ __forceinline__ int32_t val(int32_t r) { return r; }
    static __device__ __forceinline__ float grad(float g) { return g; }
};

__device__ __forceinline__ float lowest(float) { return NEG_INF; }
__device__ __forceinline__ int32_t lowest(int32_t) { return INT32_MIN; }
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }   // NaN stays
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

struct __attribute__((packed, aligned(2))) Loose { uint4 v; };   // 16 bytes at any element
template <int TYPE> constexpr int PER_VEC = 16 / sizeof(typename Kind<TYPE>::Raw);

template <int TYPE>
__device__ __forceinline__ void unpack(const uint4 &w, typename Kind<TYPE>::Val (&v)[PER_VEC<TYPE>]) {
    const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (TYPE == ISR_BF16) {
            v[2 * i] = __uint_as_float(q[i] << 16);
            v[2 * i + 1] = __uint_as_float(q[i] & 0xFFFF0000u);
        } else if constexpr (TYPE == ISR_F16) {
            typedef _Float16 h2 __attribute__((ext_vector_type(2)));
            const h2 h = __builtin_bit_cast(h2, q[i]);
            v[2 * i] = (float)h[0];
            v[2 * i + 1] = (float)h[1];
        } else {
            v[i] = __builtin_bit_cast(typename Kind<TYPE>::Val, q[i]);
        }
    }
}

// ---- across 16 lanes, a wave, a workgroup ------------------------------------------------

template <int CTRL> __device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true); }
template <int CTRL, class T> __device__ __forceinline__ T moved(T v) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, dpp<CTRL>(__builtin_bit_cast(int, v)));
    } else {
        const int2 b = __builtin_bit_cast(int2, v);
        return __builtin_bit_cast(T, make_int2(dpp<CTRL>(b.x), dpp<CTRL>(b.y)));
    }
}
template <class T> __device__ __forceinline__ T lane_value(T v, int lane) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        const int2 b = __builtin_bit_cast(int2, v);
        return __builtin_bit_cast(T, make_int2(__builtin_amdgcn_readlane(b.x, lane), __builtin_amdgcn_readlane(b.y, lane)));
    }
}
template <class T, class Op>
__device__ __forceinline__ T fold16(T v, Op op) {   // of the 16 lanes of a DPP row, in every one
    v = op(v, moved<0xB1>(v));    // lane ^ 1
    v = op(v, moved<0x4E>(v));    // lane ^ 2
    v = op(v, moved<0x141>(v));   // the other half of eight
    return op(v, moved<0x140>(v));   // the other half of sixteen
}
template <class T, class Op>
__device__ __forceinline__ T wave_fold(T v, Op op) {
    v = fold16(v, op);
    return op(op(lane_value(v, 0), lane_value(v, 16)), op(lane_value(v, 32), lane_value(v, 48)));
}
template <class T> __device__ __forceinline__ T wave_sum(T v) { return wave_fold(v, [](T a, T b) { return a + b; }); }
template <class T> __device__ __forceinline__ T wave_max(T v) { return wave_fold(v, [](T a, T b) { return larger(a, b); }); }
template <class T> __device__ __forceinline__ T sum16(T v) { return fold16(v, [](T a, T b) { return a + b; }); }
template <class T> __device__ __forceinline__ T max16(T v) { return fold16(v, [](T a, T b) { return larger(a, b); }); }
__device__ __forceinline__ bool lane_of(uint64_t bits) { return bits >> (threadIdx.x & 63) & 1; }
// what the wave has stored in LDS is what it reads from here on
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
}

template <class Val>
struct Stat {
    Val m;
    float s, t;
};

template <int T>
struct SharedStat {
    uint32_t m[T / 64];   // Val
    float s[T / 64], t[T / 64];
};

// A thread's or lane's share of a set's statistics, referred to the set's maximum.
template <class Val>
__device__ __forceinline__ void refer(Stat<Val> &a, Val m, float c) {
    const float d = c * below(a.m, m), f = __builtin_amdgcn_exp2f(d);
    a.t = a.s == 0.f ? 0.f : f * (a.t + fmaxf(d, NO_SHARE) * a.s);
    a.s = a.s == 0.f ? 0.f : f * a.s;
    a.m = m;
}

// The workgroup's statistics from those of its T threads.  Two barriers; `between` may store what is read behind the first.
template <int T, bool ENT, class Val, class Between>
__device__ __forceinline__ Stat<Val> block_stat(Stat<Val> a, float c, SharedStat<T> &sh, Between between) {
    const int wave = threadIdx.x >> 6;
    const Val wm = wave_max(a.m);
    if ((threadIdx.x & 63) == 0) sh.m[wave] = __builtin_bit_cast(uint32_t, wm);
    between();
    __syncthreads();
    Val m = __builtin_bit_cast(Val, sh.m[0]);
#pragma unroll
    for (int w = 1; w < T / 64; ++w) m = larger(m, __builtin_bit_cast(Val, sh.m[w]));
    refer(a, m, c);
    const float ws = wave_sum(a.s), wt = ENT ? wave_sum(a.t) : 0.f;
    if ((threadIdx.x & 63) == 0) {
        sh.s[wave] = ws;
        if (ENT) sh.t[wave] = wt;
    }
    __syncthreads();
    a = {m, sh.s[0], ENT ? sh.t[0] : 0.f};
#pragma unroll
    for (int w = 1; w < T / 64; ++w) {
        a.s += sh.s[w];
        if (ENT) a.t += sh.t[w];
    }
    return a;
}

// ---- chunks of a row -----------------------------------------------------------------------

// The part of a row that a workgroup of T threads holds: NV vectors a thread, and in the row's last chunk the elements beside the
// vectors, one a thread of the first PV: those behind the last vector and, where a row of 16-bit logits starts between two
// words, its first one.  Vectors at any word cost nothing, between words they took a fifth of the rate (4096 x 65537
// bf16, 52 us where 65536 took 43).
template <int TYPE, int T, int NV>
struct Chunk {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    static constexpr int PV = PER_VEC<TYPE>;
    const typename K::Raw *x;
    uint32_t head, first, n, end;   // classes in front of the row's vectors; first class of the chunk's, their number; end of the row's
    uint32_t beside;             // the thread's class beside the vectors
    bool last, edge_valid;
    uint4 raw[NV];
    typename K::Raw edge;

    __device__ __forceinline__ Chunk(const LogitRows &l, uint64_t r, uint32_t chunk, uint32_t chunks, uint32_t chunk_vecs)
        : x((const typename K::Raw *)l.x + r * l.stride) {
        head = sizeof(typename K::Raw) == 2 ? (uint32_t)((uintptr_t)x >> 1 & 1) : 0;
        const uint32_t vecs = (l.classes - head) / PV, v0 = chunk * chunk_vecs;   // at least one: rows of 16 classes and more
        n = min(chunk_vecs, vecs - min(vecs, v0));
        first = head + v0 * PV;
        end = head + vecs * PV;
        last = chunk == chunks - 1;
        const bool front = threadIdx.x == PV - 1;   // free: fewer than PV lie behind the vectors
        beside = front ? 0 : end + threadIdx.x;
        edge_valid = last && (front ? head == 1 : beside < l.classes && threadIdx.x < PV);
        const uint32_t final_vec = min(v0 + max(n, 1u), vecs) - 1;
        // none of these in a branch, behind whose end the compiler would wait for all that is in flight
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i] = ((const Loose *)(x + head + (size_t)min(v0 + i * T + threadIdx.x, final_vec) * PV))->v;
        edge = x[last ? min(beside, l.classes - 1) : head + min(v0, vecs - 1) * PV];   // of use where edge_valid
    }
    __device__ __forceinline__ bool owns(uint32_t j) const { return j - first < n * PV || (last && (j < head || j >= end)); }   // j below the number of classes
    __device__ __forceinline__ bool has(int i) const { return i * T + threadIdx.x < n; }
    __device__ __forceinline__ uint32_t at(int i) const { return first + (i * T + threadIdx.x) * PV; }
    // Between two passes over the vectors: what one has unpacked is not held in registers for the next.
    __device__ __forceinline__ void keep_packed() {
#pragma unroll
        for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(raw[i].x), "+v"(raw[i].y), "+v"(raw[i].z), "+v"(raw[i].w));
    }
    // f(i, first class, values) for the thread's vectors
    template <class F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!has(i)) continue;
            Val v[PV];
            unpack<TYPE>(raw[i], v);
            f(i, at(i), v);
        }
    }
};

// What a chunk leaves for the join.
struct Part {
    uint32_t m;
    float s, t;
    uint32_t listed;
};

// The chunks of a row together, by one wave.
template <class Val>
__device__ __forceinline__ Stat<Val> join_parts(const Part *parts, uint32_t chunks, float c) {
    const uint32_t lane = threadIdx.x & 63;
    Stat<Val> a{lowest(Val()), 0.f, 0.f};
    for (uint32_t i = lane; i < chunks; i += 64) {
        const Part q = parts[i];
        Stat<Val> b{__builtin_bit_cast(Val, q.m), q.s, q.t};
        const Val m = larger(a.m, b.m);
        refer(a, m, c);
        refer(b, m, c);
        a.s += b.s;
        a.t += b.t;
    }
    refer(a, wave_max(a.m), c);
    return {a.m, wave_sum(a.s), wave_sum(a.t)};
}

// Up to 128 named classes of a row, two a lane: of index lane and lane + 64.
struct Named {
    int32_t c[2];   // negative: none
    __device__ __forceinline__ void load(const int32_t *p, uint32_t n) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t i = (threadIdx.x & 63) + 64 * h;
            c[h] = i < n ? p[i] : -1;
        }
    }
    // f(j, class) in ascending order for the indexes whose bit is set in `of`
    template <class F>
    __device__ __forceinline__ void visit(const uint64_t (&of)[2], F f) const {
        for (uint64_t left = of[0]; left; left &= left - 1) {
            const int j = __builtin_ctzll(left);
            f(j, __builtin_amdgcn_readlane(c[0], j));
        }
        for (uint64_t left = of[1]; left; left &= left - 1) {
            const int j = __builtin_ctzll(left);
            f(j + 64, __builtin_amdgcn_readlane(c[1], j));
        }
    }
    // of the indexes in `of`, those whose class an earlier one of them has
    __device__ __forceinline__ void repeated(const uint64_t (&of)[2], uint64_t (&again)[2]) const {
        again[0] = again[1] = 0;
        visit(of, [&](int j, int cls) {
            const uint64_t same0 = __ballot(c[0] == cls), same1 = __ballot(c[1] == cls);
            if (j < 64) {
                again[0] |= same0 & (~1ull << j);
                again[1] |= same1;
            } else {
                again[1] |= same1 & (~1ull << (j - 64));
            }
        });
    }
    // sum[h] += value of every index in `of` that has the lane's class, in ascending order
    __device__ __forceinline__ void add_same(const uint64_t (&of)[2], const float (&value)[2], float (&sum)[2]) const {
        visit(of, [&](int j, int cls) {
            const float v = lane_value(j < 64 ? value[0] : value[1], j & 63);
#pragma unroll
            for (int h = 0; h < 2; ++h) sum[h] += c[h] == cls ? v : 0.f;
        });
    }
};

// ---- gradients -------------------------------------------------------------------------------

// With d = c (x - m) - l2 the log2 of a probability, an element's gradient is 2^d (a0 + a1 d).
template <class Val, bool LINEAR>
struct Slope {
    Val m;
    float c, l2, a0, a1;
    bool zero;   // the row's gradient is zero
    __device__ __forceinline__ float operator()(Val x) const {
        const float d = c * below(x, m) - l2, e = __builtin_amdgcn_exp2f(d);
        return LINEAR ? e * (a0 + a1 * fmaxf(d, NO_SHARE)) : e * a0;
    }
};

template <int TYPE, int T, int NV, class F>
__device__ __forceinline__ void store_slopes(const Chunk<TYPE, T, NV> &k, typename Kind<TYPE>::Grad *out, const F &f) {
    using K = Kind<TYPE>;
    constexpr int PV = PER_VEC<TYPE>;
    typedef typename K::Grad Vec __attribute__((ext_vector_type(PV)));
    k.each([&](int, uint32_t j, const typename K::Val (&v)[PV]) {
        Vec g = 0;
        if (!f.zero) {
#pragma unroll
            for (int e = 0; e < PV; ++e) g[e] = K::grad(f(v[e]));
        }
        ((Loose *)(out + j))->v = __builtin_bit_cast(uint4, g);
    });
    if (k.edge_valid) out[k.beside] = K::grad(f.zero ? 0.f : f(K::val(k.edge)));
}

// A chunk of a gradient's row: every element by its slope, the named classes as `special` says from their logit and the sum of
// `part(h)` over the names of one class.  Wave 0 stores theirs behind a barrier; where the gradient goes over the logits it reads
// them in front of another.
template <int TYPE, int T, int NV, class F, class Add, class Special>
__device__ __forceinline__ void store_gradient(const Chunk<TYPE, T, NV> &k, uint32_t classes, typename Kind<TYPE>::Grad *out, bool over, const F &f,
                                               const Named &named, Add part, Special special) {
    using K = Kind<TYPE>;
    uint64_t here[2];   // the names in this chunk, the same in every wave
#pragma unroll
    for (int h = 0; h < 2; ++h) here[h] = f.zero ? 0 : __ballot((uint32_t)named.c[h] < classes && k.owns((uint32_t)named.c[h]));
    const bool some = (here[0] | here[1]) != 0;
    float own[2] = {};
    bool mine[2] = {};
    auto named_values = [&] {
        uint64_t again[2];
        named.repeated(here, again);
        float add[2], sum[2] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) add[h] = lane_of(here[h]) ? part(h) : 0.f;
        named.add_same(here, add, sum);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            mine[h] = lane_of(here[h] & ~again[h]);
            if (mine[h]) own[h] = special(K::val(k.x[named.c[h]]), sum[h]);
        }
    };
    if (some && over) {
        if (threadIdx.x < 64) named_values();
        __syncthreads();
    }
    store_slopes(k, out, f);
    if (some) {
        if (!over && threadIdx.x < 64) named_values();
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (mine[h]) out[named.c[h]] = K::grad(own[h]);
    }
}

// ---- launches ----------------------------------------------------------------------------------

constexpr int THREADS = 256;

// launch(rows) for the runs of rows that a launch takes
template <class Params, class Launch>
hipError_t by_runs(Params &p, uint32_t rows_of_launch, Launch launch) {
    for (p.row0 = 0; p.row0 < p.l.rows; p.row0 += rows_of_launch) {
        const uint64_t left = p.l.rows - p.row0;
        launch((uint32_t)(left < rows_of_launch ? left : rows_of_launch));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

#define ISR_BY_TYPE(type, CALL)                      \
    switch (type) {                                  \
    case ISR_F32: CALL(ISR_F32); break;              \
    case ISR_BF16: CALL(ISR_BF16); break;            \
    case ISR_F16: CALL(ISR_F16); break;              \
    default: CALL(ISR_I32); break;                   \
    }

}  // namespace isr
