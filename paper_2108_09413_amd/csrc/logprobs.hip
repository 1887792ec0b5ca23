// Log-probabilities of given classes with entropy and top alternatives, and their gradient.
//
// Forward: a row is cut into chunks of up to 256 * NV vectors of 16 bytes, one workgroup each, which holds its chunk in
// registers: one pass over memory, then maximum, exponentials and candidates of the top alternatives from registers.  The
// chunks' results meet in a second launch (join), or in the same one where a row is one chunk: up to 2048 vectors, of few rows up
// to 8192 by 1024 threads.  Of many rows with top alternatives a workgroup goes through all chunks of one.  Bound by memory: 4096 rows
// of 131072 bf16 in 182 us, 5.9 TB/s, with 20 alternatives in 197.  Few rows are bound by latency: one row of 32000 bf16 with 20
// alternatives and entropy takes 8.2 us, one of 131072 11.8 in two launches.
// Gradient: element by element from the row's statistics, bound by memory too: 2048 x 65537 bf16 with entropy in 91 us, 5.9 TB/s (97 a
// call in a row of calls); the few named classes are stored behind the others.
// Rows of up to 256 classes go by 16 lanes each, 100000 x 256 bf16 with entropy in 13 us (4.0 TB/s); of up to 1024 by a wave
// each, 100000 x 1000 bf16 in 48 (4.2 TB/s).
#include <algorithm>

#include "logit_device.h"

namespace isr {

constexpr int LIST = 512;   // candidates of the top alternatives in LDS
constexpr int KEYS = 256;
struct Shared {
    uint32_t listed;
    int count[16];   // of each wave
    alignas(16) uint32_t key[KEYS];   // largest key of each thread, or of neighbours together
    alignas(16) uint2 list[LIST + 2];    // candidates: (key, ~class), so that the larger 64-bit number comes first
};

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
template <int TYPE> constexpr int LOW_BITS = TYPE == ISR_BF16 ? 16 : TYPE == ISR_F16 ? 13 : 0;   // of a key, the same in all of them

// Every wave for itself: the largest bound of leading bits that k of the threads' keys reach, 0 if fewer threads have any.  Up to
// 32 alternatives the threads go by fours, up to 64 by twos: fewer steps, and few more elements reach the bound.  From the first
// bit in which keys differ; below 16 bits only where that leaves many.
template <int LOW>
__device__ __forceinline__ uint32_t key_bound(const Shared &sh, uint32_t k) {
    const uint4 q = ((const uint4 *)sh.key)[threadIdx.x & 63];
    const uint32_t two[2] = {max(q.x, q.y), max(q.z, q.w)}, four = max(two[0], two[1]);
    auto fold_min = [](uint32_t a, uint32_t b) { return min(a, b); };
    auto fold_max = [](uint32_t a, uint32_t b) { return max(a, b); };
    auto reach = [](uint32_t key, uint32_t next) { return (uint32_t)__popcll(__ballot(key >= next)); };
    const uint32_t low = k <= 32 ? four : k <= 64 ? min(two[0], two[1]) : min(min(q.x, q.y), min(q.z, q.w));
    const uint32_t least = wave_fold(low, fold_min), most = wave_fold(four, fold_max);
    const int top = 31 - __builtin_clz((least ^ most) | 1);   // the highest bit in which two of them differ
    uint32_t bound = (most >> top >> 1) << top << 1, reached = KEYS;
    auto search = [&](int from, int to) {
        for (int b = from; b >= to; --b) {
            const uint32_t next = bound | (1u << b);
            const uint32_t n = k <= 32 ? reach(four, next) : k <= 64 ? reach(two[0], next) + reach(two[1], next)
                                                                     : reach(q.x, next) + reach(q.y, next) + reach(q.z, next) + reach(q.w, next);
            if (n >= k) { bound = next; reached = n; }
        }
    };
    search(top, max(LOW, 16));
    if (LOW < 16 && reached > 2 * k + 16) search(min(top, 15), LOW);   // logits closer to each other than 2^-7 of their size
    return (bound >> LOW) << LOW;
}

template <int T>
__device__ __forceinline__ int block_count(int n, Shared &sh) {
    n = wave_sum(n);
    if ((threadIdx.x & 63) == 0) sh.count[threadIdx.x >> 6] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) n += sh.count[w];
    __syncthreads();
    return n;
}

// each(f): f(key, class) for the thread's own possible elements, of which all threads together have more than k.  Lists
// exactly k: the bound is a number of 56 bits, key and ~class (below 2^24), found bit by bit.  Returns with the list complete for
// all threads.  Rows of equal logits come here, 2048 x 65536 bf16 with 20 alternatives 2.0 ms where other rows take 0.06.
template <int T, class Each>
__device__ void list_exactly(Each each, uint32_t k, Shared &sh) {
    uint64_t bound = 0;
    auto number = [](uint32_t key, uint32_t cls) { return (uint64_t)key << 24 | (~cls & 0xFFFFFF); };
    for (int b = 55; b >= 0; --b) {
        const uint64_t next = bound | (1ull << b);
        int n = 0;
        each([&](uint32_t key, uint32_t cls) { n += number(key, cls) >= next; });
        n = block_count<T>(n, sh);
        if ((uint32_t)n >= k) bound = next;
        if ((uint32_t)n == k) break;
    }
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    each([&](uint32_t key, uint32_t cls) {
        if (number(key, cls) >= bound) {
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < LIST) sh.list[at] = make_uint2(key, ~cls);
        }
    });
    __syncthreads();
}

// Results of a row of logits, by its workgroup.
template <class Val>
struct Logp {
    float scale, logs;
    Val m;
    bool bad, empty;
    __device__ __forceinline__ Logp(const LogitRows &l, const Stat<Val> &a) : scale(l.scale), logs(a.s == 0.f ? 0.f : logf(a.s)), m(a.m), bad(a.s != a.s), empty(a.s == 0.f) {}
    __device__ __forceinline__ float operator()(Val v) const {
        if (bad) return __builtin_nanf("");
        if (!possible(v)) return NEG_INF;
        const float d = below(v, m);
        return d == NEG_INF ? (float)(scale * below64(v, m) - logs) : scale * d - logs;   // a difference beyond fp32, which the scale may bring back
    }
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
template <int TYPE, int T>
__device__ __forceinline__ void finish_top(const LogprobsParams &p, uint64_t r, const Stat<typename Kind<TYPE>::Val> &a, const Shared &sh) {
    using Val = typename Kind<TYPE>::Val;
    const Logp<Val> logp(p.l, a);
    const uint32_t n = logp.bad ? 0 : min(sh.listed, (uint32_t)LIST);
    for (uint32_t i = threadIdx.x; i < n; i += T) {
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
    for (uint32_t k = n + threadIdx.x; k < p.top; k += T) {
        p.top_class[r * p.top + k] = -1;
        p.top_logprob[r * p.top + k] = logp.bad ? __builtin_nanf("") : NEG_INF;
    }
}

// Places in a list for the lanes that want one, by one atomic a wave: an atomic a candidate, each waited for, took longer than
// anything else behind the loads (top 64 of 2048 x 32771 f32, 65 -> 58 us).
__device__ __forceinline__ uint32_t places(uint32_t n, uint32_t *listed) {   // of n, the same in the wave
    uint32_t base = 0;
    if ((threadIdx.x & 63) == 0) base = atomicAdd(listed, n);
    return __builtin_amdgcn_readfirstlane(base);
}
__device__ __forceinline__ uint32_t lanes_before(uint64_t of) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(of >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)of, 0)); }

// The elements that reach the bound, of those that the wave's lanes have; by all its lanes.
template <class Val>
__device__ __forceinline__ void list_element(bool valid, Val v, uint32_t cls, Val from, Shared &sh) {
    const uint64_t of = __ballot(valid && v >= from);
    if (!of) return;
    const uint32_t at = places(__popcll(of), &sh.listed) + lanes_before(of);
    if (lane_of(of) && at < LIST) sh.list[at] = make_uint2(key_of(v), ~cls);
}

// Vectors that hold candidates, with their first class.
constexpr int VECS = 512;
struct SharedVecs {
    uint4 raw[VECS];
    uint32_t first[VECS], listed;
};
struct Nothing {};

// The chunk's vectors that reach the bound (few; NaN does, all results of its row are NaN).
template <int TYPE, int T, int NV>
__device__ __forceinline__ void list_vectors(const Chunk<TYPE, T, NV> &k, const typename Kind<TYPE>::Val (&most)[NV], typename Kind<TYPE>::Val from, SharedVecs &vecs) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) n += __popcll(__ballot(k.has(i) && !(most[i] < from)));
    if (n == 0) return;
    uint32_t at = places(n, &vecs.listed);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint64_t of = __ballot(k.has(i) && !(most[i] < from));
        const uint32_t mine = at + lanes_before(of);
        if (lane_of(of) && mine < VECS) {
            vecs.raw[mine] = k.raw[i];
            vecs.first[mine] = k.at(i);
        }
        at += __popcll(of);
    }
}

// Their elements to the list, a thread each.  Between two barriers of the caller.
template <int TYPE, int T>
__device__ __forceinline__ void list_elements(const SharedVecs &vecs, typename Kind<TYPE>::Val from, Shared &sh) {
    using K = Kind<TYPE>;
    constexpr int PV = PER_VEC<TYPE>;
    const uint32_t n = min(vecs.listed, (uint32_t)VECS) * PV;
    for (uint32_t i0 = 0; i0 < n; i0 += T) {
        const uint32_t i = i0 + threadIdx.x, j = min(i, n - 1);
        list_element(i < n, K::val(((const typename K::Raw *)vecs.raw)[j]), vecs.first[j / PV] + j % PV, from, sh);
    }
}

// A chunk of a row.
template <int TYPE, int T, int NV, bool TOP, bool ENT>
__global__ __launch_bounds__(T) void logprobs_kernel(const LogprobsParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    constexpr int PV = PER_VEC<TYPE>;
    __shared__ SharedStat<T> sums;
    __shared__ __attribute__((aligned(16))) std::conditional_t<TOP, Shared, Nothing> sh;
    __shared__ __attribute__((aligned(16))) std::conditional_t<TOP, SharedVecs, Nothing> vecs;
    const uint32_t tid = threadIdx.x, row = blockIdx.x / p.chunks, chunk = blockIdx.x - row * p.chunks;
    const uint64_t r = p.row0 + row;
    Chunk<TYPE, T, NV> k(p.l, r, chunk, p.chunks, p.chunk_vecs);
    Given<TYPE> given;
    if (p.chunks == 1) given.load(p, r);
    const Val edge = K::val(k.edge);
    Stat<Val> a{k.edge_valid ? edge : lowest(Val()), 0.f, 0.f};
    if constexpr (TOP) {
        if (tid == 0) sh.listed = vecs.listed = 0;
    }
    Val most[NV];   // TOP: of each vector
    k.each([&](int i, uint32_t, const Val (&v)[PV]) {
        if constexpr (TOP) {
            most[i] = v[0];
#pragma unroll
            for (int e = 1; e < PV; ++e) most[i] = larger(most[i], v[e]);
            a.m = larger(a.m, most[i]);
        } else {
#pragma unroll
            for (int e = 0; e < PV; ++e) a.m = larger(a.m, v[e]);
        }
    });
    k.keep_packed();
    const float c = p.l.scale * LOG2E;
    auto add = [&](Val v) {
        const float d = c * below(v, a.m), e = __builtin_amdgcn_exp2f(d);
        a.s += e;
        if (ENT) a.t += e * fmaxf(d, NO_SHARE);
    };
    if (k.edge_valid) add(edge);
    k.each([&](int, uint32_t, const Val (&v)[PV]) {
#pragma unroll
        for (int e = 0; e < PV; ++e) add(v[e]);
    });
    const Stat<Val> all = block_stat<T, ENT>(a, c, sums, [&] {
        if constexpr (TOP) {
            uint32_t key = key_of(a.m);
            if (T > KEYS) {
                key = max(key, moved<0xB1>(key));
                key = max(key, moved<0x4E>(key));
            }
            if (tid % (T / KEYS) == 0) sh.key[tid / (T / KEYS)] = key;
        }
    });
    if constexpr (TOP) {
        const uint32_t bound = key_bound<LOW_BITS<TYPE>>(sh, p.top);
        const Val from = of_key<Val>(max(bound, least_key<Val>()));
        k.keep_packed();
        // the few vectors that reach the bound, then their elements
        if (p.chunks == 1 || chunk == p.chunks - 1) list_element(k.edge_valid, edge, k.beside, from, sh);
        list_vectors(k, most, from, vecs);
        __syncthreads();
        list_elements<TYPE, T>(vecs, from, sh);
        if (vecs.listed > VECS && tid == 0) atomicMax(&sh.listed, LIST + 1u);   // some are missing: more than fit
        __syncthreads();
        const uint32_t listed = all.s == all.s ? sh.listed : 0;   // uniform; of a row with NaN nothing is asked for
        if (listed > p.list_cap && listed <= LIST) {   // neighbours that reach the bound together: of the listed, two a thread
            const uint2 mine[2] = {tid < listed ? sh.list[tid] : make_uint2(0, 0), T < LIST && tid + T < listed ? sh.list[tid + T] : make_uint2(0, 0)};
            __syncthreads();
            list_exactly<T>([&](auto f) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (mine[h].y) f(mine[h].x, ~mine[h].y);   // ~class is never 0
            }, p.top, sh);
        } else if (listed > LIST) {   // from memory again
            __syncthreads();
            list_exactly<T>([&](auto f) {
                for (uint32_t j = k.first + tid * PV; j < k.first + k.n * PV; j += T * PV) {
                    Val v[PV];
                    unpack<TYPE>(((const Loose *)(k.x + j))->v, v);
#pragma unroll
                    for (int e = 0; e < PV; ++e)
                        if (possible(v[e])) f(key_of(v[e]), j + e);
                }
                if (k.edge_valid && possible(edge)) f(key_of(edge), k.beside);
            }, p.top, sh);
        }
    }
    if (p.chunks == 1) {
        finish_values<TYPE>(p, r, all, given);
        if constexpr (TOP) finish_top<TYPE, T>(p, r, all, sh);
        return;
    }
    const size_t at = (size_t)row * p.chunks + chunk;
    uint32_t n = 0;
    if constexpr (TOP) n = all.s == all.s ? sh.listed : 0;   // at most list_cap by now
    if (tid == 0) p.parts[at] = Part{__builtin_bit_cast(uint32_t, all.m), all.s, all.t, n};
    if constexpr (TOP)
        for (uint32_t i = tid; i < n; i += T) p.lists[at * p.list_cap + i] = sh.list[i];
}

// 2^d, d <= 0.  A row that rises chunk by chunk multiplies its sum by one after the other, so next to 0 the difference from 1 is
// right to a few half steps of itself: expm1's series, whose end is 2e-8 of it at -1/2.
__device__ __forceinline__ double exp2_near_1(float d) {
    const float x = d * LN2;
    const float near = x + x * x * (0.5f + x * (1.f / 6 + x * (1.f / 24 + x * (1.f / 120 + x * (1.f / 720 + x * (1.f / 5040))))));
    return d < -0.5f ? (double)__builtin_amdgcn_exp2f(d) : 1.0 + near;
}

// Many rows with top alternatives: a workgroup goes through its row chunk by chunk, and no join is needed.  The bound of the
// first chunk serves until the listed vectors may want room; then, and at the end, it is raised to what `top` of the listed
// reach, and those below are dropped.  A chunk with more than there is room for (a row that ascends) raises it to its own; rows with
// more candidates all the same (of many equal logits) are searched in memory.
// us of a call with 20 / 64 / 128 alternatives, by chunks and join -> this way: 2048 x 32000 bf16 38 / 49 / 89 -> 33 / 38 / 46,
// 2048 x 32771 f32 56 / 61 / 74 -> 48 / 53 / 59, 4096 x 131072 bf16 210 / 222 / 244 -> 197 / 235 / 247.  So: enough rows for four
// workgroups a CU, and few alternatives or few chunks.
constexpr uint64_t WHOLE_ROWS = 1024;
constexpr uint32_t WHOLE_TOP = 32, WHOLE_CHUNKS = 5;
template <int TYPE, int NV, bool ENT>
__global__ __launch_bounds__(THREADS) void logprobs_row_top_kernel(const LogprobsParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    constexpr int PV = PER_VEC<TYPE>, OWN = VECS / THREADS;
    __shared__ SharedStat<THREADS> sums;
    __shared__ __attribute__((aligned(16))) Shared sh;
    __shared__ __attribute__((aligned(16))) SharedVecs vecs;
    const uint32_t tid = threadIdx.x;
    const uint64_t r = p.row0 + blockIdx.x;
    const float c = p.l.scale * LOG2E;
    // A thread adds up its part of a chunk (at most 64 terms) in fp32 and the chunks in 64 bits: one by one into a sum next to 1, the
    // terms of a long flat tail are lost (262144 bf16 of which one is 17 above the others: log-probabilities off by 5e-5, 4194304: 4e-4).
    Val m_all = lowest(Val());
    __shared__ double sum[THREADS], weighted[ENT ? THREADS : 1];   // of each thread; in registers they cost a sixth of the waves
    sum[tid] = 0.0;
    if (ENT) weighted[tid] = 0.0;
    Val from = of_key<Val>(least_key<Val>());
    bool lost = false;     // candidates that found no room; this and the next are the same for all threads
    uint32_t listed = 0, added = 0;
    if (tid == 0) sh.listed = vecs.listed = 0;
    auto most_of = [](const Val (&v)[PV]) __attribute__((always_inline)) {
        Val m = v[0];
#pragma unroll
        for (int e = 1; e < PV; ++e) m = larger(m, v[e]);
        return m;
    };
    auto raise = [&](uint32_t key) __attribute__((always_inline)) {   // to what `top` of the threads' keys reach; a barrier
        sh.key[tid] = key;
        __syncthreads();
        from = larger(from, of_key<Val>(max(key_bound<LOW_BITS<TYPE>>(sh, p.top), least_key<Val>())));
    };
    auto raise_by_listed = [&](Val (&most)[OWN]) __attribute__((always_inline)) {
        uint32_t key = 0;
#pragma unroll
        for (int h = 0; h < OWN; ++h) {
            Val v[PV];
            unpack<TYPE>(vecs.raw[tid + h * THREADS], v);
            most[h] = most_of(v);
            if (tid + h * THREADS < listed) key = max(key, key_of(most[h]));
        }
        raise(key);
    };
    Val edge = lowest(Val());
    uint32_t edge_class = 0;
    bool edge_valid = false;
    for (uint32_t chunk = 0; chunk < p.chunks; ++chunk) {
        if (listed + added + added / 2 + 40 > VECS && !lost) {   // if the next chunk adds what the last one did, and many deviations more
            Val most[OWN];
            typedef uint32_t Words __attribute__((ext_vector_type(4)));
            Words raw[OWN];
            uint32_t first[OWN];
            raise_by_listed(most);
#pragma unroll
            for (int h = 0; h < OWN; ++h) {
                raw[h] = ((const Words *)vecs.raw)[tid + h * THREADS];
                first[h] = vecs.first[tid + h * THREADS];
            }
            if (tid == 0) vecs.listed = 0;
            __syncthreads();
#pragma unroll
            for (int h = 0; h < OWN; ++h) {
                const bool stays = tid + h * THREADS < listed && !(most[h] < from);
                const uint64_t of = __ballot(stays);
                const uint32_t at = places(__popcll(of), &vecs.listed) + lanes_before(of);
                if (stays) { ((Words *)vecs.raw)[at] = raw[h]; vecs.first[at] = first[h]; }
            }
            __syncthreads();
            listed = vecs.listed;
        }
        Chunk<TYPE, THREADS, NV> k(p.l, r, chunk, p.chunks, p.chunk_vecs);
        Val most[NV], m = lowest(Val());
        k.each([&](int i, uint32_t, const Val (&v)[PV]) {
            most[i] = most_of(v);
            m = larger(m, most[i]);
        });
        k.keep_packed();
        edge = K::val(k.edge);
        edge_class = k.beside;
        edge_valid = k.edge_valid;
        Stat<Val> a{larger(m_all, edge_valid ? larger(m, edge) : m), 0.f, 0.f};
        const float d = c * below(m_all, a.m);   // what there is so far is referred to the new maximum
        m_all = a.m;
        auto add = [&](Val v) {
            const float d = c * below(v, a.m), e = __builtin_amdgcn_exp2f(d);
            a.s += e;
            if (ENT) a.t += e * fmaxf(d, NO_SHARE);
        };
        if (edge_valid) add(edge);
        k.each([&](int, uint32_t, const Val (&v)[PV]) {
#pragma unroll
            for (int e = 0; e < PV; ++e) add(v[e]);
        });
        const double f = exp2_near_1(d), s = sum[tid];
        if (ENT) weighted[tid] = f * (weighted[tid] + fmaxf(d, NO_SHARE) * s) + a.t;
        sum[tid] = f * s + a.s;
        k.keep_packed();
        if (chunk == 0) raise(key_of(m));
        else __syncthreads();   // all have read the count
        for (bool again = false;; again = true) {
            list_vectors(k, most, from, vecs);
            __syncthreads();
            const uint32_t n = vecs.listed;
            if (n <= VECS || again || lost) {
                lost = lost || n > VECS;
                added = min(n, (uint32_t)VECS) - listed;
                listed += added;
                break;
            }
            raise(key_of(m));
            if (tid == 0) vecs.listed = listed;
            __syncthreads();
        }
    }
    Given<TYPE> given;
    given.load(p, r);
    const Stat<Val> all = block_stat<THREADS, ENT>(Stat<Val>{m_all, (float)sum[tid], ENT ? (float)weighted[tid] : 0.f}, c, sums, [] {});
    Val most[OWN];
    raise_by_listed(most);
    list_element(edge_valid, edge, edge_class, from, sh);
    list_elements<TYPE, THREADS>(vecs, from, sh);
    __syncthreads();
    if ((lost || sh.listed > LIST) && all.s == all.s) {   // of a row with NaN nothing is asked for
        __syncthreads();
        const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
        const uint32_t whole = p.l.classes / PV * PV;
        list_exactly<THREADS>([&](auto f) {
            for (uint32_t j = tid * PV; j < whole; j += THREADS * PV) {
                Val v[PV];
                unpack<TYPE>(((const Loose *)(x + j))->v, v);
#pragma unroll
                for (int e = 0; e < PV; ++e)
                    if (possible(v[e])) f(key_of(v[e]), j + e);
            }
            if (whole + tid < p.l.classes) {
                const Val v = K::val(x[whole + tid]);
                if (possible(v)) f(key_of(v), whole + tid);
            }
        }, p.top, sh);
    }
    finish_values<TYPE>(p, r, all, given);
    finish_top<TYPE, THREADS>(p, r, all, sh);
}

// The chunks of a row together: without top alternatives by a wave, with them by a workgroup.
template <int TYPE>
__global__ __launch_bounds__(64) void logprobs_join_kernel(const LogprobsParams p) {
    using Val = typename Kind<TYPE>::Val;
    Given<TYPE> given;
    given.load(p, p.row0 + blockIdx.x);
    const Stat<Val> all = join_parts<Val>(p.parts + (size_t)blockIdx.x * p.chunks, p.chunks, p.l.scale * LOG2E);
    finish_values<TYPE>(p, p.row0 + blockIdx.x, all, given);
}

// DEEP > 0: lists of at most 64 * DEEP, 8 / DEEP a wave at most: everything is read at once, the lists as far as they have room, and
// kept.  One row of 131072 with 20 alternatives 10 -> 6 us.
template <int TYPE, int DEEP>
__global__ __launch_bounds__(THREADS) void logprobs_top_join_kernel(const LogprobsParams p) {
    using Val = typename Kind<TYPE>::Val;
    constexpr int KEPT = 8;
    __shared__ __attribute__((aligned(16))) Shared sh;
    const uint32_t tid = threadIdx.x, row = blockIdx.x, lane = tid & 63, wave = tid >> 6;
    const Part *parts = p.parts + (size_t)row * p.chunks;
    const uint2 *lists = p.lists + (size_t)row * p.chunks * p.list_cap;
    Given<TYPE> given;
    given.load(p, p.row0 + row);
    uint2 kept[KEPT];
    if constexpr (DEEP != 0) {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) {
            const uint32_t q = wave + 4 * (i / DEEP), at = lane + 64 * (i % DEEP);
            kept[i] = q < p.chunks && at < p.list_cap ? lists[(size_t)q * p.list_cap + at] : make_uint2(0, 0);
        }
#pragma unroll
        for (int i = 0; i < KEPT; ++i) {
            const uint32_t q = wave + 4 * (i / DEEP), at = lane + 64 * (i % DEEP);
            if (q >= p.chunks || at >= parts[q].listed) kept[i] = make_uint2(0, 0);   // ~class is never 0
        }
    }
    auto each = [&](auto f) {   // a wave a list
        if constexpr (DEEP != 0) {
#pragma unroll
            for (int i = 0; i < KEPT; ++i)
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
    const uint32_t bound = key_bound<LOW_BITS<TYPE>>(sh, p.top);
    each([&](uint32_t key, uint32_t cls) {
        if (key >= bound) {
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < LIST) sh.list[at] = make_uint2(key, ~cls);
        }
    });
    __syncthreads();
    if (sh.listed > LIST) {
        __syncthreads();
        list_exactly<THREADS>(each, p.top, sh);
    }
    finish_values<TYPE>(p, p.row0 + row, all, given);
    finish_top<TYPE, THREADS>(p, p.row0 + row, all, sh);
}

// scale (sum_g u_g ([j = c_g] - p_j) - u_H p_j (log p_j + H))
template <class Val, bool ENT>
__device__ __forceinline__ Slope<Val, ENT> row_slope(const LogprobsGradParams &p, uint64_t r, float up, bool counted) {
    const float uh = ENT ? p.up_entropy[r] : 0.f, logs = p.stats[2 * r + 1];
    return {of_bits<Val>(p.stats[2 * r]), p.l.scale * LOG2E, logs * LOG2E, -p.l.scale * (up + (uh != 0.f ? uh * p.entropy[r] : 0.f)),
            -p.l.scale * uh * LN2, !(counted || uh != 0.f) || logs == NEG_INF};
}

template <int TYPE, int T, int NV, bool ENT>
__global__ __launch_bounds__(T) void logprobs_grad_kernel(const LogprobsGradParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    const uint32_t row = blockIdx.x / p.chunks, chunk = blockIdx.x - row * p.chunks, lane = threadIdx.x & 63;
    const uint64_t r = p.row0 + row;
    const Chunk<TYPE, T, NV> k(p.l, r, chunk, p.chunks, p.chunk_vecs);
    Named named;
    named.load(p.given + r * p.n_given, p.n_given);
    float u[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
        u[h] = named.c[h] < 0 ? 0.f : (uint32_t)named.c[h] < p.l.classes ? p.up_logprob[r * p.n_given + lane + 64 * h] : __builtin_nanf("");
    const float up = p.n_given == 1 ? lane_value(u[0], 0) : wave_sum(u[0] + u[1]);
    const Slope<Val, ENT> f = row_slope<Val, ENT>(p, r, up, __any(named.c[0] >= 0 || named.c[1] >= 0));
    store_gradient(k, p.l.classes, (typename K::Grad *)p.grad + r * p.grad_stride, p.grad == p.l.x, f, named, [&](int h) { return u[h]; },
                   [&](Val v, float sum) { return f(v) + p.l.scale * sum; });
}

// ---- rows of few classes: 16 lanes a row, E elements a lane ---------------------------------

template <int TYPE, int E, bool ENT>
__global__ __launch_bounds__(THREADS) void logprobs_small_kernel(const LogprobsParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    const uint32_t lane = threadIdx.x & 15, row = blockIdx.x * (THREADS / 16) + (threadIdx.x >> 4), n = p.l.classes;
    const uint64_t r = p.row0 + min(row, p.run - 1);   // lanes without a row go along with the last one's
    const bool store = row < p.run;
    const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
    typename K::Raw raw[E];
#pragma unroll
    for (int i = 0; i < E; ++i) raw[i] = x[min(lane + 16 * i, n - 1)];
    Stat<Val> a{lowest(Val()), 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (lane + 16 * i < n) a.m = larger(a.m, K::val(raw[i]));
    a.m = max16(a.m);
    const float c = p.l.scale * LOG2E;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if (lane + 16 * i >= n) continue;
        const float d = c * below(K::val(raw[i]), a.m), e = __builtin_amdgcn_exp2f(d);
        a.s += e;
        if (ENT) a.t += e * fmaxf(d, NO_SHARE);
    }
    a.s = sum16(a.s);
    if (ENT) a.t = sum16(a.t);
    const Logp<Val> logp(p.l, a);
    const float nan = __builtin_nanf("");
    if (store && lane == 0) {
        if (ENT) p.entropy[r] = logp.bad ? nan : logp.empty ? 0.f : logp.logs - LN2 * (a.t / a.s);
        if (p.stats) { p.stats[2 * r] = bits_of(a.m); p.stats[2 * r + 1] = logp.bad ? nan : logp.empty ? NEG_INF : logp.logs; }
    }
    for (uint32_t g = lane; g < p.n_given && store; g += 16) {
        const int32_t cls = p.given[r * p.n_given + g];
        p.logprob[r * p.n_given + g] = cls < 0 ? 0.f : (uint32_t)cls < n ? logp(K::val(x[cls])) : nan;
    }
    if (p.top == 0) return;
    // one alternative after the other: the largest (key, ~class) of those left
    uint32_t key[E], left = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const Val v = K::val(raw[i]);
        key[i] = key_of(v);
        left |= (uint32_t)(lane + 16 * i < n && possible(v) && !logp.bad) << i;
    }
    for (uint32_t t = 0; t < p.top; ++t) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const uint64_t own = (uint64_t)key[i] << 32 | ~(lane + 16 * i);
            if ((left >> i & 1) && own > best) best = own;
        }
        best = fold16(best, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
        const uint32_t cls = ~(uint32_t)best;
        if (best && (cls & 15) == lane) left &= ~(1u << (cls >> 4));
        if (store && lane == 0) {
            p.top_class[r * p.top + t] = best ? (int32_t)cls : -1;
            p.top_logprob[r * p.top + t] = best ? logp(of_key<Val>((uint32_t)(best >> 32))) : logp.bad ? nan : NEG_INF;
        }
    }
}

template <int TYPE, int E, bool ENT>
__global__ __launch_bounds__(THREADS) void logprobs_grad_small_kernel(const LogprobsGradParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    const uint32_t lane = threadIdx.x & 15, row = blockIdx.x * (THREADS / 16) + (threadIdx.x >> 4), n = p.l.classes;
    if (row >= p.run) return;
    const uint64_t r = p.row0 + row;
    const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
    auto *out = (typename K::Grad *)p.grad + r * p.grad_stride;
    typename K::Raw raw[E];
#pragma unroll
    for (int i = 0; i < E; ++i) raw[i] = x[min(lane + 16 * i, n - 1)];
    float up = 0.f, named[E] = {};
    bool counted = false;
    for (uint32_t g = 0; g < p.n_given; ++g) {   // every lane all of them
        const int32_t cls = p.given[r * p.n_given + g];
        if (cls < 0) continue;
        const float u = (uint32_t)cls < n ? p.up_logprob[r * p.n_given + g] : __builtin_nanf("");
        counted = true;
        up += u;
#pragma unroll
        for (int i = 0; i < E; ++i) named[i] += (uint32_t)cls == lane + 16 * i ? u : 0.f;
    }
    const Slope<Val, ENT> f = row_slope<Val, ENT>(p, r, up, counted);
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (lane + 16 * i < n) out[lane + 16 * i] = K::grad(f.zero ? 0.f : f(K::val(raw[i])) + p.l.scale * named[i]);
}

// ---- rows of up to 1024 classes: a wave a row, E elements a lane ----------------------------

// A bound that k of the lanes' largest reach lets few elements more through.  Where it lets too many, and for many alternatives, the
// bound is searched among all elements: exactly k reach it, or those equal to it are taken by ascending class.
template <int TYPE, int E, bool TOP, bool ENT>
__global__ __launch_bounds__(THREADS) void logprobs_wave_kernel(const LogprobsParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    __shared__ __attribute__((aligned(16))) uint2 lists[TOP ? THREADS / 64 : 1][ISR_MAX_TOP];
    const uint32_t lane = threadIdx.x & 63, row = blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6), n = p.l.classes;
    if (row >= p.run) return;   // the whole wave
    const uint64_t r = p.row0 + row;
    const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
    typename K::Raw raw[E];
#pragma unroll
    for (int i = 0; i < E; ++i) raw[i] = x[min(lane + 64 * i, n - 1)];
    auto has = [&](int i) { return lane + 64 * i < n; };
    int32_t c[2];
    Val at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t g = lane + 64 * h;
        c[h] = g < p.n_given ? p.given[r * p.n_given + g] : -1;
        at[h] = (uint32_t)c[h] < n ? K::val(x[c[h]]) : lowest(Val());
    }
    Stat<Val> a{lowest(Val()), 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (has(i)) a.m = larger(a.m, K::val(raw[i]));
    a.m = wave_max(a.m);
    const float scale = p.l.scale * LOG2E;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if (!has(i)) continue;
        const float d = scale * below(K::val(raw[i]), a.m), e = __builtin_amdgcn_exp2f(d);
        a.s += e;
        if (ENT) a.t += e * fmaxf(d, NO_SHARE);
    }
    a.s = wave_sum(a.s);
    if (ENT) a.t = wave_sum(a.t);
    const Logp<Val> logp(p.l, a);
    const float nan = __builtin_nanf("");
    if (lane == 0) {
        if (ENT) p.entropy[r] = logp.bad ? nan : logp.empty ? 0.f : logp.logs - LN2 * (a.t / a.s);
        if (p.stats) { p.stats[2 * r] = bits_of(a.m); p.stats[2 * r + 1] = logp.bad ? nan : logp.empty ? NEG_INF : logp.logs; }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t g = lane + 64 * h;
        if (g < p.n_given) p.logprob[r * p.n_given + g] = c[h] < 0 ? 0.f : (uint32_t)c[h] < n ? logp(at[h]) : nan;
    }
    if constexpr (TOP) {
        uint32_t key[E], valid = 0, least = ~0u;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const Val v = K::val(raw[i]);
            const bool is = has(i) && possible(v) && !logp.bad;
            key[i] = is ? key_of(v) : 0;
            valid |= (uint32_t)is << i;
            least = min(least, is ? key[i] : ~0u);
        }
        const uint32_t most = key_of(a.m);
        least = min(wave_fold(least, [](uint32_t u, uint32_t v) { return min(u, v); }), most);
        auto count = [&](auto test) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < E; ++i) m += __popcll(__ballot((valid >> i & 1) && test(key[i])));
            return m;
        };
        const uint32_t all = count([](uint32_t) { return true; }), k = min(p.top, all);
        // listed are `more` elements above the bound, and as many that are equal to it, by class, as make `total`
        uint32_t bound = 0, more = k, total = k;
        // us of 100000 rows by the lanes' bound / exactly: 256 classes f32 with 48 147 / 156, 56: 172 / 157; 1000 classes 220 / 282, 273 / 286
        bool exactly = k > 48 && all > k;
        if (all > k) {
            uint32_t own = 0;
#pragma unroll
            for (int i = 0; i < E; ++i) own = max(own, key[i]);
            const int top = 31 - __builtin_clz((least ^ most) | 1);
            const uint32_t prefix = (most >> top >> 1) << top << 1;
            if (!exactly) {
                bound = prefix;
                uint32_t reached = 64;
                for (int b = top; b >= LOW_BITS<TYPE> && reached != k; --b) {
                    const uint32_t next = bound | (1u << b), m = (uint32_t)__popcll(__ballot(own >= next));
                    if (m >= k) { bound = next; reached = m; }
                }
                more = total = count([&](uint32_t u) { return u >= bound; });
                bound -= 1;   // from 0 on all reach it
                exactly = total > ISR_MAX_TOP;
            }
            if (exactly) {
                bound = prefix;
                total = k;
                uint32_t reached = all;
                for (int b = top; b >= LOW_BITS<TYPE> && reached != k; --b) {
                    const uint32_t next = bound | (1u << b), m = count([&](uint32_t u) { return u >= next; });
                    if (m >= k) { bound = next; reached = m; }
                }
                if (reached == k) {
                    more = k;
                    bound -= 1;
                } else {
                    if (LOW_BITS<TYPE>) bound |= bound >> 31 ? 0 : (1u << LOW_BITS<TYPE>) - 1;   // the bits that all 16-bit logits have there
                    more = count([&](uint32_t u) { return u > bound; });
                }
            }
        }
        const bool whole = total == all;
        uint2 *const list = lists[threadIdx.x >> 6];
        uint32_t above = 0, equal = more;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const bool is = valid >> i & 1, up = is && (whole || key[i] > bound), even = is && !up && key[i] == bound;
            const uint64_t ups = __ballot(up), evens = __ballot(even);
            const uint32_t place = up ? above + lanes_before(ups) : equal + lanes_before(evens);
            if ((up || even) && place < total) list[place] = make_uint2(key[i], ~(lane + 64 * i));
            above += __popcll(ups);
            equal += __popcll(evens);
        }
        wave_order();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t i = lane + 64 * h;
            if (i < total) {
                const uint2 mine = list[i];
                const uint64_t own = (uint64_t)mine.x << 32 | mine.y;
                uint32_t place = 0;
                for (uint32_t j = 0; j < total; ++j) place += ((uint64_t)list[j].x << 32 | list[j].y) > own;
                if (place < k) {
                    p.top_class[r * p.top + place] = (int32_t)~mine.y;
                    p.top_logprob[r * p.top + place] = logp(of_key<Val>(mine.x));
                }
            }
            if (i >= k && i < p.top) {
                p.top_class[r * p.top + i] = -1;
                p.top_logprob[r * p.top + i] = logp.bad ? nan : NEG_INF;
            }
        }
    }
}

// ---- launches --------------------------------------------------------------------------------

// 16 lanes a row, of up to 16 elements each, where what they do one after the other (`serial` steps, each over a lane's elements) stays
// below `most`; always below 16 classes, where a vector of 16 bytes may not fit.  100000 rows of f32, us by 16 lanes / by a wave:
// 256 classes with entropy 17 / 29, with 10 alternatives 71 / 87, 16: 103 / 90; 64 classes with 40: 95 / 96, 48: 112 / 100; loss of
// 256 classes and 16 entries 72 / 92, 64 and 64: 72 / 94, 17 and 128: 128 / 107.
constexpr uint32_t SMALL = 256;   // classes
static bool sixteen_lanes(uint32_t classes, uint32_t serial, uint32_t most) {
    return classes < 16 || (classes <= SMALL && serial * ((classes + 15) / 16) <= most);
}

static uint32_t vecs_of(int type, uint32_t classes) { return classes / (type == ISR_F32 || type == ISR_I32 ? 4 : 8); }
static uint32_t chunks_of(uint32_t vecs, uint32_t nv) { return (vecs + nv * THREADS - 1) / (nv * THREADS); }
constexpr uint32_t MOST_GROUPS = 1u << 22;   // of a launch
constexpr uint32_t FEW_CHUNKS = 512;         // of a launch, that leave CUs idle

// Rows whose workgroup (or its share) does them in one go, `groups` rows a workgroup.
static RowCut whole_rows(Way way, int type, uint32_t classes, uint64_t rows, uint32_t groups) {
    RowCut cut{};
    cut.way = way;
    cut.chunks = 1;
    cut.chunk_vecs = vecs_of(type, classes);
    cut.rows = (uint32_t)std::min<uint64_t>(rows, (uint64_t)MOST_GROUPS * groups);
    return cut;
}

// By chunks; up to `alone` rows of a size that many threads hold at once by a workgroup each, without a join.
static RowCut cut_rows(int type, uint32_t classes, uint64_t rows, uint32_t top, uint64_t alone) {
    RowCut cut{};
    const uint32_t vecs = vecs_of(type, classes);
    if (vecs > 8 * THREADS && vecs <= 8 * ALONE && rows <= alone) {
        cut = whole_rows(Way::alone, type, classes, rows, 1);
        cut.nv = vecs <= 4 * ALONE ? 4 : 8;
        cut.list_cap = LIST;
        return cut;
    }
    cut.way = Way::chunks;
    // Few rows: smaller chunks on more CUs, as long as the join still reads their lists at once
    cut.nv = vecs <= 2 * THREADS ? 2 : vecs > 8 * THREADS && rows * chunks_of(vecs, 8) <= FEW_CHUNKS && chunks_of(vecs, 4) <= 16 && top ? 4 : 8;
    cut.chunks = chunks_of(vecs, cut.nv);
    cut.chunk_vecs = (vecs + cut.chunks - 1) / cut.chunks;
    cut.chunks = (vecs + cut.chunk_vecs - 1) / cut.chunk_vecs;   // none of them empty
    if (top && cut.chunks > 1 && rows >= WHOLE_ROWS && (top <= WHOLE_TOP || cut.chunks <= WHOLE_CHUNKS)) cut.way = Way::row;
    cut.list_cap = cut.chunks == 1 ? LIST : std::max(128u, 2 * top + 64);
    cut.rows = (uint32_t)std::min<uint64_t>(rows, std::max<uint32_t>(1, MOST_GROUPS / cut.chunks));
    if (cut.way == Way::row || cut.chunks == 1) return cut;
    cut.parts_bytes = ((size_t)cut.rows * cut.chunks * sizeof(Part) + 255) / 256 * 256;
    cut.lists_bytes = top ? (size_t)cut.rows * cut.chunks * cut.list_cap * sizeof(uint2) : 0;
    return cut;
}

RowCut cut_gradient(const LogitRows &l) {
    // 100000 rows of f32 by 16 lanes / by a wave, us: 256 classes with 1 named 33 / 40, 32: 75 / 111, 128: 305 / 340, 17 with 128: 162 / 336
    if (l.classes <= SMALL) return whole_rows(Way::sixteen, l.type, l.classes, l.rows, THREADS / 16);
    const uint32_t vecs = vecs_of(l.type, l.classes);
    // 100000 rows, four waves a row / one, us: 257 f32 127 / 44, 1000 f32 202 / 153, 1000 bf16 187 / 79
    if (vecs <= WAVE_VECS) return whole_rows(Way::wave, l.type, l.classes, l.rows, 1);
    RowCut cut{};
    cut.way = Way::chunks;
    cut.nv = 4;   // nothing is exchanged between threads but the named classes: smaller chunks, more of them
    cut.chunks = (vecs + 4 * THREADS - 1) / (4 * THREADS);
    cut.chunk_vecs = (vecs + cut.chunks - 1) / cut.chunks;
    cut.chunks = (vecs + cut.chunk_vecs - 1) / cut.chunk_vecs;
    cut.rows = (uint32_t)std::min<uint64_t>(l.rows, std::max<uint32_t>(1, MOST_GROUPS / cut.chunks));
    return cut;
}

RowCut cut_logprobs(int type, uint32_t classes, uint64_t rows, uint32_t top) {
    if (sixteen_lanes(classes, top, 176)) return whole_rows(Way::sixteen, type, classes, rows, THREADS / 16);
    // 16 elements a lane at most.  100000 rows by a workgroup / by a wave, us: 257 f32 with entropy 98 / 30, with 5 alternatives
    // 267 / 85; 1024 f32 125 / 71, 273 / 148; 1024 bf16 111 / 49, 271 / 146
    if (classes <= 1024) return whole_rows(Way::wave, type, classes, rows, THREADS / 64);
    // us by chunks and join / by a workgroup a row: 16 x 32000 bf16 with entropy and 20 alternatives 11.4 / 8.7, without 6.4 / 5.3; 512 rows
    // 18.6 / 16.6, 11.0 / 8.8; 1000 rows 26.3 / 31.2, 16.7 / 16.2; 512 x 50001 with them 23.5 / 23.7, 256: 15.9 / 11.2.  In
    // registers of 16 vectors a thread it lost: 1 x 131072 with them 11.8 / 16.7.
    return cut_rows(type, classes, rows, top, top == 0 ? 1023 : vecs_of(type, classes) <= 4 * ALONE ? 512 : 256);
}

// What the call with most need of 1 to `rows` rows takes.  It grows with the rows but where another way begins, behind FEW_CHUNKS and at
// WHOLE_ROWS, where there may be none from there on.
size_t logprobs_workspace(int type, uint32_t classes, uint64_t rows, uint32_t top) {
    size_t most = 0;
    for (const uint64_t ends : {rows, WHOLE_ROWS - 1, (uint64_t)FEW_CHUNKS / std::max(1u, chunks_of(vecs_of(type, classes), 8))}) {
        const RowCut cut = cut_logprobs(type, classes, std::max<uint64_t>(1, std::min(rows, ends)), top);
        most = std::max(most, cut.parts_bytes + cut.lists_bytes);
    }
    return most;
}

RowCut cut_distill(int type, uint32_t classes, uint64_t rows, uint32_t top, bool rest) {
    if (sixteen_lanes(classes, top, 256)) return whole_rows(Way::sixteen, type, classes, rows, THREADS / 16);
    // 100000 rows by four waves / by one, loss / with gradient, us: 257 f32 140, 193 / 90, 100; 1000 bf16 172, 254 / 114, 152
    if (vecs_of(type, classes) <= WAVE_VECS) return whole_rows(Way::wave, type, classes, rows, 1);
    // us by chunks and join / by a workgroup a row, 64 entries, rest / none: 64 x 32000 bf16 8.8 / 7.8, 7.3 / 5.1; 512: 14.5 / 12.5, 11.7 / 7.9;
    // 1000: 21.4 / 22.0, 17.5 / 14.7
    return cut_rows(type, classes, rows, 0, rest ? 512 : 1023);
}

template <int TYPE, int T, int NV, bool TOP>
static void launch_chunks_of(const LogprobsParams &p, hipStream_t st) {
    const dim3 grid(p.run * p.chunks), block(T);
    if (p.entropy) hipLaunchKernelGGL((logprobs_kernel<TYPE, T, NV, TOP, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((logprobs_kernel<TYPE, T, NV, TOP, false>), grid, block, 0, st, p);
}
template <int TYPE, int T, int NV>
static void launch_chunks(const LogprobsParams &p, hipStream_t st) {
    if (p.top) launch_chunks_of<TYPE, T, NV, true>(p, st);
    else launch_chunks_of<TYPE, T, NV, false>(p, st);
}

template <int TYPE, int E>
static void launch_small(const LogprobsParams &p, hipStream_t st) {
    const dim3 grid((p.run + THREADS / 16 - 1) / (THREADS / 16)), block(THREADS);
    if (p.entropy) hipLaunchKernelGGL((logprobs_small_kernel<TYPE, E, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((logprobs_small_kernel<TYPE, E, false>), grid, block, 0, st, p);
}
template <int TYPE, int E>
static void launch_small(const LogprobsGradParams &p, hipStream_t st) {
    const dim3 grid((p.run + THREADS / 16 - 1) / (THREADS / 16)), block(THREADS);
    if (p.up_entropy) hipLaunchKernelGGL((logprobs_grad_small_kernel<TYPE, E, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((logprobs_grad_small_kernel<TYPE, E, false>), grid, block, 0, st, p);
}
template <int TYPE, class Params>
static void launch_small(const Params &p, hipStream_t st) {
    if (p.l.classes <= 16) launch_small<TYPE, 1>(p, st);
    else if (p.l.classes <= 64) launch_small<TYPE, 4>(p, st);
    else if (p.l.classes <= 128) launch_small<TYPE, 8>(p, st);
    else launch_small<TYPE, 16>(p, st);
}

template <int TYPE, int E>
static void launch_wave(const LogprobsParams &p, hipStream_t st) {
    const dim3 grid((p.run + THREADS / 64 - 1) / (THREADS / 64)), block(THREADS);
    if (p.top && p.entropy) hipLaunchKernelGGL((logprobs_wave_kernel<TYPE, E, true, true>), grid, block, 0, st, p);
    else if (p.top) hipLaunchKernelGGL((logprobs_wave_kernel<TYPE, E, true, false>), grid, block, 0, st, p);
    else if (p.entropy) hipLaunchKernelGGL((logprobs_wave_kernel<TYPE, E, false, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((logprobs_wave_kernel<TYPE, E, false, false>), grid, block, 0, st, p);
}

template <int TYPE>
static void launch_rows(const LogprobsParams &p, Way way, uint32_t nv, hipStream_t st) {
    if (way == Way::sixteen) return launch_small<TYPE>(p, st);
    if (way == Way::wave) return p.l.classes <= 512 ? launch_wave<TYPE, 8>(p, st) : launch_wave<TYPE, 16>(p, st);
    const dim3 grid(p.run), block(THREADS);
    if (way == Way::row) {
        if (p.entropy) hipLaunchKernelGGL((logprobs_row_top_kernel<TYPE, 8, true>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((logprobs_row_top_kernel<TYPE, 8, false>), grid, block, 0, st, p);
        return;
    }
    if (way == Way::alone) {
        if (nv == 4) launch_chunks<TYPE, ALONE, 4>(p, st);
        else launch_chunks<TYPE, ALONE, 8>(p, st);
        return;
    }
    if (nv == 2) launch_chunks<TYPE, THREADS, 2>(p, st);
    else if (nv == 4) launch_chunks_of<TYPE, THREADS, 4, true>(p, st);   // cut_rows() takes it with alternatives only
    else launch_chunks<TYPE, THREADS, 8>(p, st);
    if (p.chunks == 1) return;
    if (!p.top) hipLaunchKernelGGL((logprobs_join_kernel<TYPE>), grid, dim3(64), 0, st, p);
    else if (p.chunks <= 16 && p.list_cap <= 128) hipLaunchKernelGGL((logprobs_top_join_kernel<TYPE, 2>), grid, block, 0, st, p);
    else if (p.chunks <= 8 && p.list_cap <= 256) hipLaunchKernelGGL((logprobs_top_join_kernel<TYPE, 4>), grid, block, 0, st, p);
    else if (p.chunks <= 4 && p.list_cap <= 512) hipLaunchKernelGGL((logprobs_top_join_kernel<TYPE, 8>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((logprobs_top_join_kernel<TYPE, 0>), grid, block, 0, st, p);
}

hipError_t launch_logprobs(LogprobsParams p, const RowCut &cut, void *workspace, hipStream_t st) {
    p.chunks = cut.chunks;
    p.chunk_vecs = cut.chunk_vecs;
    p.list_cap = cut.list_cap;
    p.parts = (Part *)workspace;
    p.lists = (uint2 *)((uint8_t *)workspace + cut.parts_bytes);
    return by_runs(p, cut.rows, [&](uint32_t rows) {
        p.run = rows;
#define CALL(T) launch_rows<T>(p, cut.way, cut.nv, st)
        ISR_BY_TYPE(p.l.type, CALL)
#undef CALL
    });
}

template <int TYPE, int T>
static void launch_grad_chunks(const LogprobsGradParams &p, hipStream_t st) {
    const dim3 grid(p.run * p.chunks), block(T);
    if (p.up_entropy) hipLaunchKernelGGL((logprobs_grad_kernel<TYPE, T, 4, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((logprobs_grad_kernel<TYPE, T, 4, false>), grid, block, 0, st, p);
}
template <int TYPE>
static void launch_grad_rows(const LogprobsGradParams &p, Way way, hipStream_t st) {
    if (way == Way::sixteen) launch_small<TYPE>(p, st);
    else if (way == Way::wave) launch_grad_chunks<TYPE, 64>(p, st);
    else launch_grad_chunks<TYPE, THREADS>(p, st);
}

hipError_t launch_logprobs_grad(LogprobsGradParams p, hipStream_t st) {
    const RowCut cut = cut_gradient(p.l);
    p.chunks = cut.chunks;
    p.chunk_vecs = cut.chunk_vecs;
    return by_runs(p, cut.rows, [&](uint32_t rows) {
        p.run = rows;
#define CALL(T) launch_grad_rows<T>(p, cut.way, st)
        ISR_BY_TYPE(p.l.type, CALL)
#undef CALL
    });
}

}  // namespace isr
