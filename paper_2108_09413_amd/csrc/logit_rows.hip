// Operators on rows of class logits: log-probabilities of given classes with entropy and top alternatives, distillation from
// a teacher's top logits, and the gradient of both.
//
// Statistics of a set of logits: m = max x, s = sum exp(scale (x - m)), t = sum exp(.) * (scale (x - m) log2 e).  Differences
// are taken before the scale, so rows of the type's lowest value, far offsets and int32 logits (whose differences are exact)
// lose nothing.  s is NaN exactly for rows that hold NaN or +infinity, m is -infinity for rows without a possible class.
//
// Forward: a row is cut into chunks of up to 256 * NV vectors of 16 bytes, one workgroup each, which holds its chunk in
// registers: one pass over memory, then maximum, exponentials and candidates of the top alternatives from registers.  The
// chunks' results meet in a second launch (join), or in the same one where a row is one chunk.
// Gradient: element by element from the row's statistics; the few classes that are named (given, or entries of the teacher)
// are overwritten behind a barrier by one thread each.
#include <algorithm>

#include "logit_rows.h"

namespace isr {

constexpr float NEG_INF = -__builtin_inff();

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


constexpr int THREADS = 256;
constexpr int LIST = 512;                 // candidates of the top alternatives in LDS
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NO_SHARE = -200.f;        // 2^-200 is 0 in fp32: finite in place of log2 0, so that 0 * log 0 is 0

// ---- across a wave, across a workgroup ------------------------------------------

template <int CTRL> __device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true); }
template <class T, class Op>
__device__ __forceinline__ T wave_fold(T v, Op op) {   // of all 64 lanes, in every lane
    auto as = [](int b) { return __builtin_bit_cast(T, b); };
    auto bits = [](T x) { return __builtin_bit_cast(int, x); };
    v = op(v, as(dpp<0xB1>(bits(v))));    // lane ^ 1
    v = op(v, as(dpp<0x4E>(bits(v))));    // lane ^ 2
    v = op(v, as(dpp<0x141>(bits(v))));   // the other half of eight
    v = op(v, as(dpp<0x140>(bits(v))));   // the other half of sixteen
    auto at = [&](int lane) { return as(__builtin_amdgcn_readlane(bits(v), lane)); };
    return op(op(at(0), at(16)), op(at(32), at(48)));
}
__device__ __forceinline__ float wave_sum(float v) { return wave_fold(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ int wave_sum(int v) { return wave_fold(v, [](int a, int b) { return a + b; }); }
template <class T> __device__ __forceinline__ T wave_max(T v) { return wave_fold(v, [](T a, T b) { return larger(a, b); }); }
__device__ __forceinline__ double wave_sum(double v) {
    auto add = [&](auto of) {
        const int2 b = __builtin_bit_cast(int2, v);
        v += __builtin_bit_cast(double, make_int2(of(b.x), of(b.y)));
    };
    add([](int b) { return dpp<0xB1>(b); });
    add([](int b) { return dpp<0x4E>(b); });
    add([](int b) { return dpp<0x141>(b); });
    add([](int b) { return dpp<0x140>(b); });
    const int2 b = __builtin_bit_cast(int2, v);
    auto at = [&](int lane) { return __builtin_bit_cast(double, make_int2(__builtin_amdgcn_readlane(b.x, lane), __builtin_amdgcn_readlane(b.y, lane))); };
    return (at(0) + at(16)) + (at(32) + at(48));
}

template <class Val>
struct Stat {
    Val m;
    float s, t;
};

struct SharedStat {
    uint32_t m[THREADS / 64];   // Val
    float s[THREADS / 64], t[THREADS / 64];
};
struct Shared : SharedStat {
    uint32_t listed;
    int count[THREADS / 64];
    alignas(16) uint32_t key[THREADS];   // largest key of each thread
    alignas(16) uint2 list[LIST + 2];    // candidates: (key, ~class), so that the larger 64-bit number comes first
};

// The workgroup's statistics from those of its threads.  Two barriers; `with_keys` has something stored before the first.
template <class Val, class Between>
__device__ __forceinline__ Stat<Val> block_stat(Stat<Val> a, float c, SharedStat &sh, Between with_keys) {
    const int wave = threadIdx.x >> 6;
    const Val wm = wave_max(a.m);
    if ((threadIdx.x & 63) == 0) sh.m[wave] = __builtin_bit_cast(uint32_t, wm);
    with_keys();
    __syncthreads();
    Val m = __builtin_bit_cast(Val, sh.m[0]);
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) m = larger(m, __builtin_bit_cast(Val, sh.m[w]));
    const float d = c * below(a.m, m), f = __builtin_amdgcn_exp2f(d);
    const float s = a.s == 0.f ? 0.f : f * a.s, t = a.s == 0.f ? 0.f : f * (a.t + fmaxf(d, NO_SHARE) * a.s);
    const float ws = wave_sum(s), wt = wave_sum(t);
    if ((threadIdx.x & 63) == 0) { sh.s[wave] = ws; sh.t[wave] = wt; }
    __syncthreads();
    return {m, (sh.s[0] + sh.s[1]) + (sh.s[2] + sh.s[3]), (sh.t[0] + sh.t[1]) + (sh.t[2] + sh.t[3])};
}

// ---- top alternatives ---------------------------------------------------------------
// Logits as unsigned keys in the same order (-0 as 0).  The k-th largest of the threads' own maxima, cut to its leading bits,
// is a bound that k elements at least reach and few more: those are listed, and each finds its place by counting
// the listed ones in front of it.  Where more are listed than there is room (rows with many equal logits), the exact bound
// by (key, class) is searched bit by bit and exactly k are listed.

__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint32_t key_of(int32_t x) { return (uint32_t)x ^ 0x80000000u; }
template <class Val> __device__ __forceinline__ Val of_key(uint32_t k);
template <> __device__ __forceinline__ float of_key<float>(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k); }
template <> __device__ __forceinline__ int32_t of_key<int32_t>(uint32_t k) { return (int32_t)(k ^ 0x80000000u); }
template <class Val> __device__ __forceinline__ uint32_t least_key();   // of a possible class
template <> __device__ __forceinline__ uint32_t least_key<float>() { return 0x00800000u; }
template <> __device__ __forceinline__ uint32_t least_key<int32_t>() { return 0; }
template <class Val> constexpr int LOW_BITS = 16;                // fp32 keys: a relative step of 2^-7
template <> constexpr int LOW_BITS<int32_t> = 0;

// Every wave for itself: the largest bound of leading bits that k of the threads' keys reach, 0 if fewer threads have any.
// Up to 32 alternatives the threads go by fours.
template <int LOW>
__device__ __forceinline__ uint32_t key_bound(const Shared &sh, uint32_t k) {
    const uint4 q = ((const uint4 *)sh.key)[threadIdx.x & 63];
    uint32_t bound = 0;
    if (k <= 32) {
        const uint32_t top = max(max(q.x, q.y), max(q.z, q.w));
        for (int b = 31; b >= LOW; --b) {
            const uint32_t next = bound | (1u << b);
            if ((uint32_t)__popcll(__ballot(top >= next)) >= k) bound = next;
        }
    } else {
        for (int b = 31; b >= LOW; --b) {
            const uint32_t next = bound | (1u << b);
            const int n = __popcll(__ballot(q.x >= next)) + __popcll(__ballot(q.y >= next)) + __popcll(__ballot(q.z >= next)) + __popcll(__ballot(q.w >= next));
            if ((uint32_t)n >= k) bound = next;
        }
    }
    return bound;
}

__device__ __forceinline__ int block_count(int n, Shared &sh) {
    n = wave_sum(n);
    if ((threadIdx.x & 63) == 0) sh.count[threadIdx.x >> 6] = n;
    __syncthreads();
    n = (sh.count[0] + sh.count[1]) + (sh.count[2] + sh.count[3]);
    __syncthreads();
    return n;
}

// each(f): f(key, class) for the thread's own possible elements, of which all threads together have more than k.  Lists
// exactly k.  Returns with the list complete for all threads.
template <class Each>
__device__ void list_exactly(Each each, uint32_t k, Shared &sh) {
    uint32_t hi = 0, lo = 0;
    bool done = false;
    for (int b = 31; b >= 0 && !done; --b) {
        const uint32_t next = hi | (1u << b);
        int n = 0;
        each([&](uint32_t key, uint32_t) { n += key >= next; });
        n = block_count(n, sh);
        if ((uint32_t)n >= k) { hi = next; done = (uint32_t)n == k; }
    }
    if (!done) lo = 0xFF000000u;   // classes are below 2^24
    for (int b = 23; b >= 0 && !done; --b) {
        const uint32_t next = lo | (1u << b);
        int n = 0;
        each([&](uint32_t key, uint32_t cls) { n += key > hi || (key == hi && ~cls >= next); });
        n = block_count(n, sh);
        if ((uint32_t)n >= k) { lo = next; done = (uint32_t)n == k; }
    }
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    each([&](uint32_t key, uint32_t cls) {
        if (key > hi || (key == hi && ~cls >= lo)) {
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < LIST) sh.list[at] = make_uint2(key, ~cls);
        }
    });
    __syncthreads();
}

// ---- rows and their chunks -------------------------------------------------------------

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

// What a chunk leaves for the join.
struct Part {
    uint32_t m;
    float s, t;
    uint32_t listed;
};

// Results of a row of logits, by its workgroup.
template <class Val>
struct Logp {
    float scale, logs;
    Val m;
    bool bad, empty;
    __device__ __forceinline__ Logp(const LogitRows &l, const Stat<Val> &a) : scale(l.scale), logs(a.s == 0.f ? 0.f : logf(a.s)), m(a.m), bad(a.s != a.s), empty(a.s == 0.f) {}
    __device__ __forceinline__ float operator()(Val v) const { return bad ? __builtin_nanf("") : possible(v) ? scale * below(v, m) - logs : NEG_INF; }
};

// The given classes, one a thread of the first 64 or 128, read ahead of what their results wait for.
template <int TYPE>
struct Given {
    int32_t c[2];
    typename Kind<TYPE>::Val at[2];
    __device__ __forceinline__ void load(const LogprobsParams &p, uint64_t r) {
        const auto *x = (const typename Kind<TYPE>::Raw *)p.l.x + r * p.l.stride;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t g = threadIdx.x + h * blockDim.x;
            c[h] = g < p.n_given ? p.given[r * p.n_given + g] : -1;
            at[h] = (uint32_t)c[h] < p.l.classes ? Kind<TYPE>::val(x[c[h]]) : lowest(typename Kind<TYPE>::Val());
        }
    }
};

template <int TYPE>
__device__ __forceinline__ void finish_values(const LogprobsParams &p, uint64_t r, const Stat<typename Kind<TYPE>::Val> &a, const Given<TYPE> &given) {
    const Logp<typename Kind<TYPE>::Val> logp(p.l, a);
    const float nan = __builtin_nanf("");
    if (threadIdx.x == 0) {
        if (p.entropy) p.entropy[r] = logp.bad ? nan : logp.empty ? 0.f : logp.logs - LN2 * (a.t / a.s);
        if (p.stats) { p.stats[2 * r] = bits_of(a.m); p.stats[2 * r + 1] = logp.bad ? nan : logp.empty ? NEG_INF : logp.logs; }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t g = threadIdx.x + h * blockDim.x;
        if (g < p.n_given) p.logprob[r * p.n_given + g] = given.c[h] < 0 ? 0.f : (uint32_t)given.c[h] < p.l.classes ? logp(given.at[h]) : nan;
    }
}

// The list is complete.
template <int TYPE>
__device__ __forceinline__ void finish_top(const LogprobsParams &p, uint64_t r, const Stat<typename Kind<TYPE>::Val> &a, Shared &sh) {
    using Val = typename Kind<TYPE>::Val;
    const Logp<Val> logp(p.l, a);
    const uint32_t n = logp.bad ? 0 : min(sh.listed, (uint32_t)LIST);
    for (uint32_t i = threadIdx.x; i < n; i += THREADS) {
        const uint2 mine = sh.list[i];
        const uint64_t own = (uint64_t)mine.x << 32 | mine.y;
        uint32_t place = 0;
        for (uint32_t j = 0; j < n; j += 2) {
            const uint4 two = *(const uint4 *)&sh.list[j];
            place += ((uint64_t)two.x << 32 | two.y) > own;
            place += j + 1 < n && ((uint64_t)two.z << 32 | two.w) > own;
        }
        if (place < p.top) {
            p.top_class[r * p.top + place] = (int32_t)~mine.y;
            p.top_logprob[r * p.top + place] = logp(of_key<Val>(mine.x));
        }
    }
    for (uint32_t k = n + threadIdx.x; k < p.top; k += THREADS) {
        p.top_class[r * p.top + k] = -1;
        p.top_logprob[r * p.top + k] = logp.bad ? __builtin_nanf("") : NEG_INF;
    }
}

// A chunk of a row: NV vectors a thread in registers, and what is left behind the row's last vector, an element a thread.
template <int TYPE, int NV, bool TOP, bool ENT>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(const LogprobsParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    constexpr int PV = PER_VEC<TYPE>;
    __shared__ __attribute__((aligned(16))) Shared sh;
    const uint32_t tid = threadIdx.x, row = blockIdx.x / p.chunks, chunk = blockIdx.x - row * p.chunks;
    const uint64_t r = p.row0 + row;
    const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
    const uint32_t vecs = p.l.classes / PV, v0 = chunk * p.chunk_vecs, n = min(p.chunk_vecs, vecs - min(vecs, v0));
    const uint32_t rest = vecs * PV + tid;
    const bool tail = chunk == p.chunks - 1 && rest < p.l.classes;   // fewer than PV threads
    uint4 raw[NV];
    if (n) {
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i] = ((const Loose *)(x + (size_t)(v0 + min(i * THREADS + tid, n - 1)) * PV))->v;
    }
    const Val edge = tail ? K::val(x[rest]) : lowest(Val());
    Given<TYPE> given;
    if (p.chunks == 1) given.load(p, r);
    Stat<Val> a{edge, 0.f, 0.f};
    if (TOP && tid == 0) sh.listed = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * THREADS + tid >= n) continue;
        Val v[PV];
        unpack<TYPE>(raw[i], v);
#pragma unroll
        for (int e = 0; e < PV; ++e) a.m = larger(a.m, v[e]);
    }
    const float c = p.l.scale * LOG2E;
    auto add = [&](Val v) {
        const float d = c * below(v, a.m), e = __builtin_amdgcn_exp2f(d);
        a.s += e;
        if (ENT) a.t += e * fmaxf(d, NO_SHARE);
    };
    if (tail) add(edge);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * THREADS + tid >= n) continue;
        Val v[PV];
        unpack<TYPE>(raw[i], v);
#pragma unroll
        for (int e = 0; e < PV; ++e) add(v[e]);
    }
    const Stat<Val> all = block_stat(a, c, sh, [&] { if (TOP) sh.key[tid] = key_of(a.m); });
    if constexpr (TOP) {
        const uint32_t bound = key_bound<LOW_BITS<Val>>(sh, p.top);
        const Val from = of_key<Val>(max(bound, least_key<Val>()));
        auto take = [&](Val v, uint32_t cls) {
            if (v >= from) {
                const uint32_t at = atomicAdd(&sh.listed, 1u);
                if (at < LIST) sh.list[at] = make_uint2(key_of(v), ~cls);
            }
        };
        if (a.m >= from) {
            if (tail) take(edge, rest);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i * THREADS + tid >= n) continue;
                Val v[PV];
                unpack<TYPE>(raw[i], v);
#pragma unroll
                for (int e = 0; e < PV; ++e) take(v[e], (v0 + i * THREADS + tid) * PV + e);
            }
        }
        __syncthreads();
        if (sh.listed > p.list_cap) {   // uniform; from memory again, an element at a time
            const uint32_t first = min(v0, vecs) * PV, last = chunk == p.chunks - 1 ? p.l.classes : first + n * PV;
            __syncthreads();
            list_exactly([&](auto f) {
                for (uint32_t j = first + tid; j < last; j += THREADS) {
                    const Val v = K::val(x[j]);
                    if (possible(v)) f(key_of(v), j);
                }
            }, p.top, sh);
        }
    }
    if (p.chunks == 1) {
        finish_values<TYPE>(p, r, all, given);
        if constexpr (TOP) finish_top<TYPE>(p, r, all, sh);
        return;
    }
    const size_t at = (size_t)row * p.chunks + chunk;
    if (tid == 0) p.parts[at] = Part{__builtin_bit_cast(uint32_t, all.m), all.s, all.t, TOP ? sh.listed : 0};
    if constexpr (TOP)
        for (uint32_t i = tid; i < sh.listed; i += THREADS) p.lists[at * p.list_cap + i] = sh.list[i];
}

// The chunks of a row together, by one wave.
template <class Val>
__device__ __forceinline__ Stat<Val> join_parts(const Part *parts, uint32_t chunks, float c) {
    const uint32_t lane = threadIdx.x & 63;
    Stat<Val> a{lowest(Val()), 0.f, 0.f};
    for (uint32_t i = lane; i < chunks; i += 64) {
        const Part q = parts[i];
        const Val qm = __builtin_bit_cast(Val, q.m), m = larger(a.m, qm);
        const float d0 = c * below(a.m, m), d1 = c * below(qm, m), f0 = __builtin_amdgcn_exp2f(d0), f1 = __builtin_amdgcn_exp2f(d1);
        const float s0 = a.s == 0.f ? 0.f : f0 * a.s, t0 = a.s == 0.f ? 0.f : f0 * (a.t + fmaxf(d0, NO_SHARE) * a.s);
        const float s1 = q.s == 0.f ? 0.f : f1 * q.s, t1 = q.s == 0.f ? 0.f : f1 * (q.t + fmaxf(d1, NO_SHARE) * q.s);
        a = {m, s0 + s1, t0 + t1};
    }
    const Val m = wave_max(a.m);
    const float d = c * below(a.m, m), f = __builtin_amdgcn_exp2f(d);
    return {m, wave_sum(a.s == 0.f ? 0.f : f * a.s), wave_sum(a.s == 0.f ? 0.f : f * (a.t + fmaxf(d, NO_SHARE) * a.s))};
}

// Without top alternatives a wave a row, with them a workgroup.
template <int TYPE>
__global__ __launch_bounds__(64) void logprobs_join_kernel(const LogprobsParams p) {
    using Val = typename Kind<TYPE>::Val;
    Given<TYPE> given;
    given.load(p, p.row0 + blockIdx.x);
    const Stat<Val> all = join_parts<Val>(p.parts + (size_t)blockIdx.x * p.chunks, p.chunks, p.l.scale * LOG2E);
    finish_values<TYPE>(p, p.row0 + blockIdx.x, all, given);
}

// FEW: at most 16 lists of at most 128: everything is read at once, the lists as far as they have room, and kept.
template <int TYPE, bool FEW>
__global__ __launch_bounds__(THREADS) void logprobs_top_join_kernel(const LogprobsParams p) {
    using Val = typename Kind<TYPE>::Val;
    __shared__ __attribute__((aligned(16))) Shared sh;
    const uint32_t tid = threadIdx.x, row = blockIdx.x, lane = tid & 63, wave = tid >> 6;
    const Part *parts = p.parts + (size_t)row * p.chunks;
    const uint2 *lists = p.lists + (size_t)row * p.chunks * p.list_cap;
    Given<TYPE> given;
    given.load(p, p.row0 + row);
    uint2 kept[FEW ? 8 : 1];
    if constexpr (FEW) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t q = wave + 4 * (i >> 1), at = lane + 64 * (i & 1);
            kept[i] = q < p.chunks && at < p.list_cap ? lists[(size_t)q * p.list_cap + at] : make_uint2(0, 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t q = wave + 4 * (i >> 1), at = lane + 64 * (i & 1);
            if (q >= p.chunks || at >= parts[q].listed) kept[i] = make_uint2(0, 0);   // less than any key of a possible class
        }
    }
    auto each = [&](auto f) {   // a wave a list
        if constexpr (FEW) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (kept[i].y) f(kept[i].x, ~kept[i].y);
        } else {
            for (uint32_t q = wave; q < p.chunks; q += THREADS / 64) {
                const uint32_t n = parts[q].listed;
                for (uint32_t i = lane; i < n; i += 64) {
                    const uint2 w = lists[(size_t)q * p.list_cap + i];
                    f(w.x, ~w.y);
                }
            }
        }
    };
    uint32_t best = 0;
    each([&](uint32_t key, uint32_t) { best = max(best, key); });
    sh.key[tid] = best;
    if (tid == 0) sh.listed = 0;
    const Stat<Val> all = join_parts<Val>(parts, p.chunks, p.l.scale * LOG2E);   // every wave for itself
    __syncthreads();
    const uint32_t bound = key_bound<LOW_BITS<Val>>(sh, p.top);
    each([&](uint32_t key, uint32_t cls) {
        if (key >= bound) {
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < LIST) sh.list[at] = make_uint2(key, ~cls);
        }
    });
    __syncthreads();
    if (sh.listed > LIST) {
        __syncthreads();
        list_exactly(each, p.top, sh);
    }
    finish_values<TYPE>(p, p.row0 + row, all, given);
    finish_top<TYPE>(p, p.row0 + row, all, sh);
}

// ---- distillation -----------------------------------------------------------------------

// Statistics of a row between the loss and its gradient.  logs == -infinity: the gradient is zero.
struct DistillStat {
    float m, logs;               // of all classes; m: Val
    float rest_m, rest_logs;     // of those that are no entry (rest), else as m and logs
    float value_m, value_logs;   // q = exp(value_scale (value - value_m) - value_logs)
    float total, left;           // sum of q and q_rest; q_rest
};
static_assert(sizeof(DistillStat) == 32, "eight words a row");

__device__ __forceinline__ float teacher_value(const void *p, int type, uint64_t i) {
    if (type == ISR_F32) return ((const float *)p)[i];
    if (type == ISR_BF16) return Kind<ISR_BF16>::val(((const uint16_t *)p)[i]);
    return Kind<ISR_F16>::val(((const _Float16 *)p)[i]);
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
    // visit(j, class) in ascending order for the indexes whose bit is set in `of`
    template <class Visit>
    __device__ __forceinline__ void visit(const uint64_t (&of)[2], Visit f) const {
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
};
constexpr int SLOTS = 2048;
__device__ __forceinline__ bool lane_of(uint64_t bits) { return bits >> (threadIdx.x & 63) & 1; }

// Loss and statistics of a row, by one wave, from the statistics of all classes or (rest) of those that are no entry.  The sums
// over the entries are in 64 bits: q_rest is next to 0 where the entries hold nearly all, and the loss of a student close to its
// teacher is a sum that cancels.
template <int TYPE>
struct Entries : Named {
    float v[2];                      // the teacher's
    typename Kind<TYPE>::Val at[2];  // the student's
    __device__ __forceinline__ void load(const DistillParams &p, uint64_t r) {
        const auto *x = (const typename Kind<TYPE>::Raw *)p.l.x + r * p.l.stride;
        Named::load(p.entry + r * p.top, p.top);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v[h] = c[h] >= 0 ? teacher_value(p.value, p.value_type, r * p.top + (threadIdx.x & 63) + 64 * h) : NEG_INF;
            at[h] = (uint32_t)c[h] < p.l.classes ? Kind<TYPE>::val(x[c[h]]) : lowest(typename Kind<TYPE>::Val());   // not negative either
        }
    }
};

// Which of a row's entries are the first of their class, by one wave.  The lowest index of those that fall on one slot of a table
// knows about itself and all of its class; only entries that find another class there (2 of 64 on average) are gone through in
// turn.  All in turn took 3 us a row of 64.
__device__ __forceinline__ void first_entries(const Named &e, uint32_t *table, bool (&is)[2]) {
    const uint32_t lane = threadIdx.x & 63;
    auto ordered = [] {   // within the wave
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        __builtin_amdgcn_wave_barrier();
    };
#pragma unroll
    for (int i = 0; i < SLOTS / 256; ++i) ((uint4 *)table)[i * 64 + lane] = make_uint4(~0u, ~0u, ~0u, ~0u);
    ordered();
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (e.c[h] >= 0) atomicMin(&table[e.c[h] % SLOTS], lane + 64 * h);
    ordered();
    bool other[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t j = e.c[h] >= 0 ? table[e.c[h] % SLOTS] : lane + 64 * h;
        const int c0 = __shfl(e.c[0], j & 63, 64), c1 = __shfl(e.c[1], j & 63, 64);
        other[h] = e.c[h] >= 0 && (j < 64 ? c0 : c1) != e.c[h];
        is[h] = e.c[h] >= 0 && j == lane + 64 * h;
    }
    const uint64_t of[2] = {__ballot(other[0]), __ballot(other[1])};
    uint64_t again[2];
    e.repeated(of, again);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (other[h]) is[h] = !lane_of(again[h]);
}

template <int TYPE>
__device__ DistillStat finish_distill(const DistillParams &p, uint64_t r, const Stat<typename Kind<TYPE>::Val> &a, const Entries<TYPE> &e, uint32_t *table) {
    using Val = typename Kind<TYPE>::Val;
    const Val (&at)[2] = e.at;
    bool bad = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) bad |= e.c[h] >= 0 && ((uint32_t)e.c[h] >= p.l.classes || e.v[h] != e.v[h] || e.v[h] == -NEG_INF);
    bad = __any(bad);
    const float vm = p.rest ? 0.f : wave_max(larger(e.v[0], e.v[1])), c = p.l.scale * LOG2E;
    if (!__any(e.c[0] >= 0 || e.c[1] >= 0) || vm == NEG_INF) {
        if ((threadIdx.x & 63) == 0) p.loss[r] = 0.f;
        return DistillStat{0.f, NEG_INF, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    }
    double lq[2], q[2], total, left = 0.0;
    float value_logs = 0.f;
    Stat<Val> all = a;
#pragma unroll
    for (int h = 0; h < 2; ++h) lq[h] = (double)p.value_scale * ((double)e.v[h] - vm);
    if (p.rest) {
#pragma unroll
        for (int h = 0; h < 2; ++h) q[h] = e.c[h] >= 0 ? exp(lq[h]) : 0.0;
        total = wave_sum(q[0] + q[1]);
        left = fmax(1.0 - total, 0.0);
        bool is[2];
        first_entries(e, table, is);
        all.m = larger(a.m, wave_max(larger(is[0] ? at[0] : lowest(Val()), is[1] ? at[1] : lowest(Val()))));
        float s = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (is[h]) s += __builtin_amdgcn_exp2f(c * below(at[h], all.m));
        all.s = wave_sum(s) + (a.s == 0.f ? 0.f : a.s * __builtin_amdgcn_exp2f(c * below(a.m, all.m)));
    } else {
        float z = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) z += e.c[h] >= 0 ? expf((float)lq[h]) : 0.f;
        value_logs = logf(wave_sum(z));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            lq[h] -= value_logs;
            q[h] = e.c[h] >= 0 ? expf((float)lq[h]) : 0.f;
        }
        total = wave_sum(q[0] + q[1]);
    }
    const bool empty = all.s == 0.f;
    const float logs = empty ? 0.f : logf(all.s), rest_logs = a.s == 0.f ? NEG_INF : logf(a.s);
    double loss = 0.0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const double lp = empty || !possible(at[h]) ? (double)NEG_INF : (double)p.l.scale * below64(at[h], all.m) - logs;
        if (q[h] > 0.0) loss += q[h] * (lq[h] - lp);
    }
    loss = wave_sum(loss);
    if (left > 0.0) {
        const double lr = a.s == 0.f ? (double)NEG_INF : (double)p.l.scale * below64(a.m, all.m) + ((double)rest_logs - logs);
        loss += left * (logf((float)left) - lr);
    }
    total += left;
    if (bad || all.s != all.s) loss = total = __builtin_nan("");
    if ((threadIdx.x & 63) == 0) p.loss[r] = (float)loss;
    return DistillStat{bits_of(all.m), empty ? NEG_INF : logs, bits_of(a.m), rest_logs, vm, value_logs, (float)total, (float)left};
}

__device__ __forceinline__ void store_stat(const DistillParams &p, uint64_t r, const DistillStat &st) {
    if (p.stats && (threadIdx.x & 63) == 0) *(DistillStat *)(p.stats + 8 * r) = st;
}

// The chunk of a row as in logprobs_kernel.  REST: without the entries, which a byte of bits for each vector in LDS tells: a
// thread's NV bytes are one read, and vectors without an entry (nearly all) go the same way as in the other case.
template <int TYPE, int NV, bool REST>
__global__ __launch_bounds__(THREADS) void distill_kernel(const DistillParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    constexpr int PV = PER_VEC<TYPE>;
    __shared__ SharedStat sh;
    __shared__ __attribute__((aligned(8))) uint32_t mask[REST ? NV * THREADS / 4 : 1];
    __shared__ __attribute__((aligned(16))) uint32_t table[REST ? SLOTS : 4];
    __shared__ uint32_t tail_mask;
    const uint32_t tid = threadIdx.x, row = blockIdx.x / p.chunks, chunk = blockIdx.x - row * p.chunks;
    const uint64_t r = p.row0 + row;
    const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
    const uint32_t vecs = p.l.classes / PV, v0 = chunk * p.chunk_vecs, n = min(p.chunk_vecs, vecs - min(vecs, v0));
    const uint32_t rest = vecs * PV + tid;
    bool tail = chunk == p.chunks - 1 && rest < p.l.classes;
    // in front of the row's loads, which would have to arrive first otherwise
    const int32_t e = REST && tid < p.top ? p.entry[r * p.top + tid] : -1;
    uint4 raw[NV];
    if (n) {
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i] = ((const Loose *)(x + (size_t)(v0 + min(i * THREADS + tid, n - 1)) * PV))->v;
    }
    const Val edge = tail ? K::val(x[rest]) : lowest(Val());
    uint32_t out[NV / 4 ? NV / 4 : 1] = {};   // bits of the entries among this thread's vectors, a byte each
    if constexpr (REST) {
        for (int i = tid; i < NV * THREADS / 4; i += THREADS) mask[i] = 0;
        if (tid == 0) tail_mask = 0;
        __syncthreads();
        const uint32_t j = (uint32_t)e - v0 * PV;
        if (e >= 0 && (uint32_t)e >= v0 * PV && j < n * PV) {
            const uint32_t vec = j / PV, byte = vec % THREADS * NV + vec / THREADS;
            atomicOr(&mask[byte >> 2], 1u << (8 * (byte & 3) + j % PV));
        } else if (e >= 0 && (uint32_t)e >= vecs * PV && (uint32_t)e < p.l.classes) {
            atomicOr(&tail_mask, 1u << ((uint32_t)e - vecs * PV));
        }
        __syncthreads();
        if constexpr (NV == 8) {
            const uint2 w = *(const uint2 *)&mask[tid * 2];
            out[0] = w.x;
            out[1] = w.y;
        } else {
            static_assert(NV == 2);
            out[0] = ((const uint16_t *)mask)[tid];
        }
        tail = tail && !(tail_mask >> tid & 1);
    }
    auto bits = [&](int i) { return out[i / 4] >> (8 * (i & 3)) & 0xFF; };
    Stat<Val> a{tail ? edge : lowest(Val()), 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * THREADS + tid >= n) continue;
        Val v[PV];
        unpack<TYPE>(raw[i], v);
        if (REST && bits(i)) {
#pragma unroll
            for (int e = 0; e < PV; ++e) v[e] = bits(i) >> e & 1 ? lowest(Val()) : v[e];
        }
#pragma unroll
        for (int e = 0; e < PV; ++e) a.m = larger(a.m, v[e]);
    }
    const float c = p.l.scale * LOG2E;
    auto share = [&](Val v) { return __builtin_amdgcn_exp2f(c * below(v, a.m)); };
    if (tail) a.s = share(edge);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * THREADS + tid >= n) continue;
        Val v[PV];
        unpack<TYPE>(raw[i], v);
        if (REST && bits(i)) {
#pragma unroll
            for (int e = 0; e < PV; ++e) a.s += bits(i) >> e & 1 ? 0.f : share(v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < PV; ++e) a.s += share(v[e]);
        }
    }
    const Stat<Val> all = block_stat(a, c, sh, [] {});
    if (p.chunks == 1) {
        if (tid < 64) {
            Entries<TYPE> named;
            named.load(p, r);
            store_stat(p, r, finish_distill<TYPE>(p, r, all, named, table));
        }
        return;
    }
    if (tid == 0) p.parts[(size_t)row * p.chunks + chunk] = Part{__builtin_bit_cast(uint32_t, all.m), all.s, 0.f, 0};
}

template <int TYPE>
__global__ __launch_bounds__(64) void distill_join_kernel(const DistillParams p) {
    using Val = typename Kind<TYPE>::Val;
    __shared__ __attribute__((aligned(16))) uint32_t table[SLOTS];
    const uint64_t r = p.row0 + blockIdx.x;
    Entries<TYPE> named;
    named.load(p, r);
    const Stat<Val> all = join_parts<Val>(p.parts + (size_t)blockIdx.x * p.chunks, p.chunks, p.l.scale * LOG2E);
    store_stat(p, r, finish_distill<TYPE>(p, r, all, named, table));
}

// ---- gradients --------------------------------------------------------------------------

// A chunk of a gradient's row: with d = c (x - m) - l2 the log2 of a probability, every element gets 2^d (a0 + a1 d), and the
// named classes what `special` says of them, from their logit and the sum of `part(h)` over the names of one class.
// Wave 0 stores theirs behind a barrier; where the gradient goes over the logits it reads them in front of another.
template <class Val>
struct Slope {
    Val m;
    float l2, a0, a1;
    bool zero;   // the row's gradient is zero
};

template <int TYPE, int NV, bool LINEAR, class Params, class Part, class Special>
__device__ __forceinline__ void store_gradient(const Params &p, uint64_t r, uint32_t chunk, const Slope<typename Kind<TYPE>::Val> &f, const Named &named,
                                               const uint4 (&raw)[NV], Part part, Special special) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    constexpr int PV = PER_VEC<TYPE>;
    const uint32_t tid = threadIdx.x;
    const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
    auto *out = (typename K::Grad *)p.grad + r * p.grad_stride;
    const uint32_t vecs = p.l.classes / PV, v0 = chunk * p.chunk_vecs, n = min(p.chunk_vecs, vecs - min(vecs, v0));
    const uint32_t rest = vecs * PV + tid, lo = min(v0, vecs) * PV, hi = chunk == p.chunks - 1 ? p.l.classes : lo + n * PV;
    const bool tail = chunk == p.chunks - 1 && rest < p.l.classes;
    const float c = p.l.scale * LOG2E;
    auto value = [&](Val v) {
        const float d = c * below(v, f.m) - f.l2, e = __builtin_amdgcn_exp2f(d);
        return LINEAR ? e * (f.a0 + f.a1 * fmaxf(d, NO_SHARE)) : e * f.a0;
    };
    uint64_t here[2];   // the names in this chunk, the same in every wave
#pragma unroll
    for (int h = 0; h < 2; ++h) here[h] = f.zero ? 0 : __ballot(named.c[h] >= 0 && (uint32_t)named.c[h] >= lo && (uint32_t)named.c[h] < hi);
    const bool some = (here[0] | here[1]) != 0, over = p.grad == p.l.x;
    const Val edge = tail && !f.zero ? K::val(x[rest]) : lowest(Val());
    float own[2] = {};
    bool mine[2] = {};
    auto named_values = [&] {
        uint64_t again[2];
        named.repeated(here, again);
        float add[2], sum[2] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) add[h] = lane_of(here[h]) ? part(h) : 0.f;
        named.visit(here, [&](int j, int cls) {
            const float aj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(j < 64 ? add[0] : add[1]), j & 63));
#pragma unroll
            for (int h = 0; h < 2; ++h) sum[h] += named.c[h] == cls ? aj : 0.f;
        });
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            mine[h] = lane_of(here[h] & ~again[h]);
            if (mine[h]) own[h] = special(K::val(x[named.c[h]]), sum[h], value);
        }
    };
    if (some && over) {
        if (tid < 64) named_values();
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * THREADS + tid >= n) continue;
        typedef typename K::Grad Vec __attribute__((ext_vector_type(PV)));
        Vec g = 0;
        if (!f.zero) {
            Val v[PV];
            unpack<TYPE>(raw[i], v);
#pragma unroll
            for (int e = 0; e < PV; ++e) g[e] = K::grad(value(v[e]));
        }
        ((Loose *)(out + (size_t)(v0 + i * THREADS + tid) * PV))->v = __builtin_bit_cast(uint4, g);
    }
    if (tail) out[rest] = K::grad(f.zero ? 0.f : value(edge));
    if (some) {
        if (!over && tid < 64) named_values();
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (mine[h]) out[named.c[h]] = K::grad(own[h]);
    }
}

template <int TYPE, int NV, class Params>
__device__ __forceinline__ void load_chunk(const Params &p, uint64_t r, uint32_t chunk, uint4 (&raw)[NV]) {
    constexpr int PV = PER_VEC<TYPE>;
    const auto *x = (const typename Kind<TYPE>::Raw *)p.l.x + r * p.l.stride;
    const uint32_t vecs = p.l.classes / PV, v0 = chunk * p.chunk_vecs, n = min(p.chunk_vecs, vecs - min(vecs, v0));
    if (n) {
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i] = ((const Loose *)(x + (size_t)(v0 + min(i * THREADS + threadIdx.x, n - 1)) * PV))->v;
    }
}

// scale (sum_g u_g ([j = c_g] - p_j) - u_H p_j (log p_j + H))
template <int TYPE, int NV, bool ENT>
__global__ __launch_bounds__(THREADS) void logprobs_grad_kernel(const LogprobsGradParams p) {
    using Val = typename Kind<TYPE>::Val;
    const uint32_t row = blockIdx.x / p.chunks, chunk = blockIdx.x - row * p.chunks, lane = threadIdx.x & 63;
    const uint64_t r = p.row0 + row;
    uint4 raw[NV];
    load_chunk<TYPE, NV>(p, r, chunk, raw);
    Named named;
    named.load(p.given + r * p.n_given, p.n_given);
    float u[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t c = (uint32_t)named.c[h];
        u[h] = named.c[h] < 0 ? 0.f : c < p.l.classes ? p.up_logprob[r * p.n_given + lane + 64 * h] : __builtin_nanf("");
    }
    const float up = p.n_given == 1 ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(u[0]), 0)) : wave_sum(u[0] + u[1]);
    const float uh = ENT ? p.up_entropy[r] : 0.f, logs = p.stats[2 * r + 1];
    Slope<Val> f;
    f.m = of_bits<Val>(p.stats[2 * r]);
    f.l2 = logs * LOG2E;
    f.a0 = -p.l.scale * (up + (uh != 0.f ? uh * p.entropy[r] : 0.f));
    f.a1 = -p.l.scale * uh * LN2;
    f.zero = !(__any(named.c[0] >= 0 || named.c[1] >= 0) || uh != 0.f) || logs == NEG_INF;
    store_gradient<TYPE, NV, ENT>(p, r, chunk, f, named, raw, [&](int h) { return u[h]; },
                                  [&](Val v, float sum, auto value) { return value(v) + p.l.scale * sum; });
}

// w scale (Q p_j - sum of the q of j), and with the rest class for those that are no entry w scale (p_j / p_rest) (Q p_rest - q_rest)
template <int TYPE, int NV>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(const DistillParams p) {
    using Val = typename Kind<TYPE>::Val;
    const uint32_t row = blockIdx.x / p.chunks, chunk = blockIdx.x - row * p.chunks, lane = threadIdx.x & 63;
    const uint64_t r = p.row0 + row;
    uint4 raw[NV];
    load_chunk<TYPE, NV>(p, r, chunk, raw);
    const DistillStat st = *(const DistillStat *)(p.stats + 8 * r);
    const float w = p.weight ? p.weight[r] : 1.f, c = p.l.scale * LOG2E;
    Named named;
    named.load(p.entry + r * p.top, p.top);
    const Val m = of_bits<Val>(st.m), rest_m = of_bits<Val>(st.rest_m);
    Slope<Val> f;
    f.zero = w == 0.f || st.logs == NEG_INF;
    f.a0 = p.l.scale * w * st.total;
    f.a1 = 0.f;
    f.m = m;
    f.l2 = st.logs * LOG2E;
    if (p.rest) {
        const bool none = st.rest_logs == NEG_INF;   // no possible class outside the entries: their gradient is 0 by 2^d alone
        f.a0 = p.l.scale * w * (none ? -st.left : st.total * expf(p.l.scale * below(rest_m, m) + st.rest_logs - st.logs) - st.left);
        f.m = rest_m;
        f.l2 = none ? 0.f : st.rest_logs * LOG2E;
        if (st.total != st.total) f.a0 = st.total;
    }
    store_gradient<TYPE, NV, false>(p, r, chunk, f, named, raw, [&](int h) {
        return expf(p.value_scale * (teacher_value(p.value, p.value_type, r * p.top + lane + 64 * h) - st.value_m) - st.value_logs);
    }, [&](Val v, float sum, auto) { return p.l.scale * w * (st.total * __builtin_amdgcn_exp2f(c * below(v, m) - st.logs * LOG2E) - sum); });
}

// ---- launches ------------------------------------------------------------------------

template <int TYPE, int NV>
static void launch_chunks(const LogprobsParams &p, uint32_t rows, hipStream_t st) {
    const dim3 grid(rows * p.chunks), block(THREADS);
    if (p.top && p.entropy) hipLaunchKernelGGL((logprobs_kernel<TYPE, NV, true, true>), grid, block, 0, st, p);
    else if (p.top) hipLaunchKernelGGL((logprobs_kernel<TYPE, NV, true, false>), grid, block, 0, st, p);
    else if (p.entropy) hipLaunchKernelGGL((logprobs_kernel<TYPE, NV, false, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((logprobs_kernel<TYPE, NV, false, false>), grid, block, 0, st, p);
}

template <int TYPE>
static void launch_rows(const LogprobsParams &p, uint32_t nv, uint32_t rows, hipStream_t st) {
    if (nv == 2) launch_chunks<TYPE, 2>(p, rows, st);
    else if (nv == 4) launch_chunks<TYPE, 4>(p, rows, st);
    else launch_chunks<TYPE, 8>(p, rows, st);
    if (p.chunks == 1) return;
    if (p.top && p.chunks <= 16 && p.list_cap <= 128) hipLaunchKernelGGL((logprobs_top_join_kernel<TYPE, true>), dim3(rows), dim3(THREADS), 0, st, p);
    else if (p.top) hipLaunchKernelGGL((logprobs_top_join_kernel<TYPE, false>), dim3(rows), dim3(THREADS), 0, st, p);
    else hipLaunchKernelGGL((logprobs_join_kernel<TYPE>), dim3(rows), dim3(64), 0, st, p);
}

RowCut cut_rows(int type, uint32_t classes, uint64_t rows, uint32_t top) {
    RowCut cut;
    const uint32_t per_vec = type == ISR_F32 || type == ISR_I32 ? 4 : 8, vecs = classes / per_vec;
    auto chunks_of = [&](uint32_t nv) { return vecs <= nv * THREADS ? 1 : (vecs + nv * THREADS - 1) / (nv * THREADS); };
    cut.nv = vecs <= 2 * THREADS ? 2 : vecs > 8 * THREADS && rows * chunks_of(8) <= 512 && chunks_of(4) <= 16 && top ? 4 : 8;
    cut.chunks = chunks_of(cut.nv);
    cut.chunk_vecs = vecs ? (vecs + cut.chunks - 1) / cut.chunks : 1;
    cut.list_cap = cut.chunks == 1 ? LIST : 2 * top + 64;
    const uint64_t most = (1u << 22) / cut.chunks;   // workgroups of a launch
    cut.rows = (uint32_t)std::min<uint64_t>(rows, most ? most : 1);
    cut.parts_bytes = cut.chunks == 1 ? 0 : ((size_t)cut.rows * cut.chunks * sizeof(Part) + 255) / 256 * 256;
    cut.lists_bytes = cut.chunks == 1 || !top ? 0 : (size_t)cut.rows * cut.chunks * cut.list_cap * sizeof(uint2);
    return cut;
}

template <class Params>
static void set_cut(Params &p, const RowCut &cut) {
    p.chunks = cut.chunks;
    p.chunk_vecs = cut.chunk_vecs;
}

// launch(rows) for the runs of rows that a launch takes
template <class Params, class Launch>
static hipError_t by_runs(Params &p, const RowCut &cut, Launch launch) {
    for (p.row0 = 0; p.row0 < p.l.rows; p.row0 += cut.rows) {
        launch((uint32_t)std::min<uint64_t>(cut.rows, p.l.rows - p.row0));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

#define BY_TYPE(type, call)                          \
    switch (type) {                                  \
    case ISR_F32: call(ISR_F32); break;              \
    case ISR_BF16: call(ISR_BF16); break;            \
    case ISR_F16: call(ISR_F16); break;              \
    default: call(ISR_I32); break;                   \
    }

hipError_t launch_logprobs(LogprobsParams p, const RowCut &cut, void *workspace, hipStream_t st) {
    set_cut(p, cut);
    p.list_cap = cut.list_cap;
    p.parts = (Part *)workspace;
    p.lists = (uint2 *)((uint8_t *)workspace + cut.parts_bytes);
    return by_runs(p, cut, [&](uint32_t rows) {
#define CALL(T) launch_rows<T>(p, cut.nv, rows, st)
        BY_TYPE(p.l.type, CALL)
#undef CALL
    });
}

template <int TYPE>
static void launch_distill_rows(const DistillParams &p, uint32_t nv, uint32_t rows, hipStream_t st) {
    const dim3 grid(rows * p.chunks), block(THREADS);
    if (p.rest && nv == 2) hipLaunchKernelGGL((distill_kernel<TYPE, 2, true>), grid, block, 0, st, p);
    else if (p.rest) hipLaunchKernelGGL((distill_kernel<TYPE, 8, true>), grid, block, 0, st, p);
    else if (nv == 2) hipLaunchKernelGGL((distill_kernel<TYPE, 2, false>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((distill_kernel<TYPE, 8, false>), grid, block, 0, st, p);
    if (p.chunks > 1) hipLaunchKernelGGL((distill_join_kernel<TYPE>), dim3(rows), dim3(64), 0, st, p);
}

// Gradients keep less of a row in registers: nothing is exchanged between threads but the named classes.
static RowCut cut_gradient(const LogitRows &l) {
    RowCut cut{};
    const uint32_t per_vec = l.type == ISR_F32 || l.type == ISR_I32 ? 4 : 8, vecs = l.classes / per_vec;
    cut.nv = 4;
    cut.chunks = vecs <= 4 * THREADS ? 1 : (vecs + 4 * THREADS - 1) / (4 * THREADS);
    cut.chunk_vecs = vecs ? (vecs + cut.chunks - 1) / cut.chunks : 1;
    const uint64_t most = (1u << 22) / cut.chunks;
    cut.rows = (uint32_t)std::min<uint64_t>(l.rows, most ? most : 1);
    return cut;
}

hipError_t launch_logprobs_grad(LogprobsGradParams p, hipStream_t st) {
    const RowCut cut = cut_gradient(p.l);
    set_cut(p, cut);
    return by_runs(p, cut, [&](uint32_t rows) {
        const dim3 grid(rows * p.chunks), block(THREADS);
#define CALL(T)                                                                                             \
    if (p.up_entropy) hipLaunchKernelGGL((logprobs_grad_kernel<T, 4, true>), grid, block, 0, st, p);        \
    else hipLaunchKernelGGL((logprobs_grad_kernel<T, 4, false>), grid, block, 0, st, p)
        BY_TYPE(p.l.type, CALL)
#undef CALL
    });
}

static void launch_distill_grad_rows(const DistillParams &p, uint32_t rows, hipStream_t st) {
#define CALL(T) hipLaunchKernelGGL((distill_grad_kernel<T, 4>), dim3(rows * p.chunks), dim3(THREADS), 0, st, p)
    BY_TYPE(p.l.type, CALL)
#undef CALL
}

hipError_t launch_distill(DistillParams p, RowCut cut, void *workspace, hipStream_t st) {
    p.parts = (Part *)workspace;
    const RowCut gradient = cut_gradient(p.l);
    return by_runs(p, cut, [&](uint32_t rows) {
        set_cut(p, cut);
#define CALL(T) launch_distill_rows<T>(p, cut.nv, rows, st)
        BY_TYPE(p.l.type, CALL)
#undef CALL
        if (!p.grad) return;
        set_cut(p, gradient);
        launch_distill_grad_rows(p, rows, st);
    });
}

hipError_t launch_distill_grad(DistillParams p, hipStream_t st) {
    const RowCut cut = cut_gradient(p.l);
    set_cut(p, cut);
    return by_runs(p, cut, [&](uint32_t rows) { launch_distill_grad_rows(p, rows, st); });
}

}  // namespace isr
