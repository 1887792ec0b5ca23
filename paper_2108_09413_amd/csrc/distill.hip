// Distillation from a teacher's top logits: the loss of each row and its gradient.
//
// Loss alone: chunks of a row in registers, one workgroup each, and a join, as for the log-probabilities; with a rest class the
// entries are left out of the chunks' sums; of few rows 1024 threads hold up to 8192 vectors, and no join follows.  Gradient alone: by elements from the row's statistics.
// Both at once, rows that fit the registers of a workgroup (up to 16384 vectors of 16 bytes): the row is read once, held, and
// its gradient stored from there, 4096 x 131072 bf16 with 64 entries and rest in 458 us a call (4.7 TB/s, of 5.9 that the
// gradient alone reaches), 8192 x 32000 in 206 (5.1).  Longer rows take the two ways one after the other, with three movements of the row.
// Rows of up to 256 classes go by 16 lanes each unless they have many entries; rows of up to 256 vectors by a single wave.
#include <algorithm>

#include "logit_device.h"

namespace isr {

__device__ __forceinline__ float teacher_value(const void *p, int type, uint64_t i) {
    if (type == ISR_F32) return ((const float *)p)[i];
    if (type == ISR_BF16) return Kind<ISR_BF16>::val(((const uint16_t *)p)[i]);
    return Kind<ISR_F16>::val(((const _Float16 *)p)[i]);
}

// log q and q of an entry of value v: the loss and the gradient from the statistics have the same bits.  With the rest class q is the
// exponential in 64 bits, where 1 - sum q is next to 0; otherwise its exponent is rounded to fp32, off by |log q| half steps of q.
__device__ __forceinline__ double log_share(const DistillParams &p, float v, float value_m, float value_logs) {
    return (double)p.value_scale * ((double)v - value_m) - value_logs;
}
__device__ __forceinline__ float share_of(const DistillParams &p, float v, float value_m, float value_logs) {
    const double lq = log_share(p, v, value_m, value_logs);
    return p.rest ? (float)exp(lq) : expf((float)lq);
}

// Where the entries hold all of the teacher's probability, 1 - sum q is what rounding leaves of it, as often above 0 as below.  A student
// whose other classes are impossible (or that has none) would be infinitely far off for that, one that masks them by a low number 1e-8 of
// that number.  So q_rest is 0 where p_rest is 0 in fp32 too and 1 - sum q can be rounding alone: that of the values as they are stored,
// and of their making in fp32, a sum of up to `top` exponentials, a logarithm and a difference.  e = -sum q_i log q_i.
constexpr double NO_REST = -104.0;   // below log 2^-150
__device__ __forceinline__ bool no_rest(const DistillParams &p, double left, double log_p, double e) {
    const double half = p.value_type == ISR_F32 ? 0x1p-24 : p.value_type == ISR_BF16 ? 0x1p-8 : 0x1p-11;   // a step's, relative; below 2^-14 f16's stay
    return log_p < NO_REST && left <= half * (e + p.value_scale * 0x1p-14) + 0x1p-24 * (p.top + 16 + 4 * e);
}

// ---- the entries of a row, by one wave, two a lane ------------------------------------------

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

// Which of them are the first of their class.  The lowest index of those that fall on one slot of a table knows about itself and
// all of its class; only entries that find another class there (2 of 64 on average) are gone through in turn.  All in
// turn took 3 us a row of 64.
constexpr int SLOTS = 2048;
__device__ __forceinline__ void first_entries(const Named &e, uint32_t *table, bool (&is)[2]) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < SLOTS / 256; ++i) ((uint4 *)table)[i * 64 + lane] = make_uint4(~0u, ~0u, ~0u, ~0u);
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (e.c[h] >= 0) atomicMin(&table[e.c[h] % SLOTS], lane + 64 * h);
    wave_order();
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

// What the teacher says, before anything is known of the student.  The sum that leads to q_rest is in 64 bits: it is next to 0
// where the entries hold nearly all.  The same for all lanes but q and is.
struct Taught {
    float q[2];
    double total, left;   // sum of q and q_rest; q_rest
    float value_m, value_logs;
    bool is[2];           // first of its class
    bool none, bad;       // no teacher; no result
    __device__ __forceinline__ double logq(const DistillParams &p, float v) const { return log_share(p, v, value_m, value_logs); }
};
template <int TYPE>
__device__ __forceinline__ Taught taught(const DistillParams &p, const Entries<TYPE> &e, uint32_t *table) {
    Taught t;
    bool bad = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) bad |= e.c[h] >= 0 && ((uint32_t)e.c[h] >= p.l.classes || e.v[h] != e.v[h] || e.v[h] == -NEG_INF);
    t.bad = __any(bad);
    t.value_m = p.rest ? 0.f : wave_max(larger(e.v[0], e.v[1]));
    t.none = !__any(e.c[0] >= 0 || e.c[1] >= 0) || t.value_m == NEG_INF;
    if (t.none) t.value_m = 0.f;
    t.value_logs = 0.f;
    t.left = 0.0;
    first_entries(e, table, t.is);
    if (p.rest) {
        double sum = 0.0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const double q = e.c[h] >= 0 ? exp(t.logq(p, e.v[h])) : 0.0;
            sum += q;
            t.q[h] = (float)q;
        }
        sum = wave_sum(sum);
        t.left = fmax(1.0 - sum, 0.0);
        t.total = sum + t.left;
    } else {
        float z = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) z += e.c[h] >= 0 ? share_of(p, e.v[h], t.value_m, 0.f) : 0.f;
        t.value_logs = logf(wave_sum(z));
#pragma unroll
        for (int h = 0; h < 2; ++h) t.q[h] = e.c[h] >= 0 ? share_of(p, e.v[h], t.value_m, t.value_logs) : 0.f;
        t.total = wave_sum((double)t.q[0] + t.q[1]);
    }
    return t;
}

// Loss (stored) and statistics of a row, from the statistics of all classes or (rest) of those that are no entry.  The loss of a
// student close to its teacher is a sum that cancels, so its terms and their sum are in 64 bits; log Z and log q_rest in them are fp32's, off
// by their rounding.
template <int TYPE>
__device__ __forceinline__ DistillStat conclude(const DistillParams &p, uint64_t r, const Stat<typename Kind<TYPE>::Val> &a, const Entries<TYPE> &e, const Taught &t) {
    using Val = typename Kind<TYPE>::Val;
    const bool writes = (threadIdx.x & 63) == 0;
    if (t.none) {
        if (writes) p.loss[r] = 0.f;
        return DistillStat{0.f, NEG_INF, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    }
    const float c = p.l.scale * LOG2E;
    Stat<Val> all = a;
    if (p.rest) {
        Val m = lowest(Val());
#pragma unroll
        for (int h = 0; h < 2; ++h) m = larger(m, t.is[h] ? e.at[h] : lowest(Val()));
        m = larger(a.m, wave_max(m));
        float s = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (t.is[h]) s += __builtin_amdgcn_exp2f(c * below(e.at[h], m));
        refer(all, m, c);
        all.s += wave_sum(s);
    }
    const bool empty = all.s == 0.f;
    const float logs = empty ? 0.f : logf(all.s), rest_logs = a.s == 0.f ? NEG_INF : logf(a.s);
    double loss = 0.0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const double lp = empty || !possible(e.at[h]) ? (double)NEG_INF : (double)p.l.scale * below64(e.at[h], all.m) - logs;
        if (t.q[h] > 0.f) loss += (double)t.q[h] * (t.logq(p, e.v[h]) - lp);
    }
    loss = wave_sum(loss);
    if (!p.rest) loss /= t.total;   // the q are rounded to 24 bits, and a sum of theirs above 1 would take a loss near the largest number to infinity
    double total = t.total, left = t.left;
    if (left > 0.0) {
        const double lr = a.s == 0.f ? (double)NEG_INF : (double)p.l.scale * below64(a.m, all.m) + ((double)rest_logs - logs);
        double e_share = 0.0;
        if (lr < NO_REST) {   // the same for all lanes
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (t.q[h] > 0.f) e_share -= (double)t.q[h] * t.logq(p, e.v[h]);
            e_share = wave_sum(e_share);
        }
        if (no_rest(p, left, lr, e_share)) {
            total -= left;
            left = 0.0;
        } else {
            loss += left * (logf((float)left) - lr);
        }
    }
    const bool bad = t.bad || all.s != all.s;
    if (writes) p.loss[r] = bad ? __builtin_nanf("") : (float)loss;
    return DistillStat{bits_of(all.m), empty && !bad ? NEG_INF : logs, bits_of(a.m), rest_logs, t.value_m, t.value_logs, bad ? __builtin_nanf("") : (float)total, (float)left};
}

// ---- gradient ---------------------------------------------------------------------------------

// f = w scale.  Classes that are no entry: f Q p_j, with the rest class f (p_j / p_rest) (Q p_rest - q_rest).
template <class Val>
__device__ __forceinline__ Slope<Val, false> row_slope(const DistillParams &p, const DistillStat &st, float w) {
    const Val m = of_bits<Val>(st.m), rest_m = of_bits<Val>(st.rest_m);
    const float c = p.l.scale * LOG2E, f = p.l.scale * w;
    const bool zero = w == 0.f || st.logs == NEG_INF;
    if (!p.rest) return {m, c, st.logs * LOG2E, f * st.total, 0.f, zero};
    const bool none = st.rest_logs == NEG_INF;   // no possible class outside the entries: 2^d alone makes their gradient 0
    const float share = none ? 0.f : expf(p.l.scale * below(rest_m, m) + st.rest_logs - st.logs);
    return {rest_m, c, none ? 0.f : st.rest_logs * LOG2E, f * (st.total * share - st.left), 0.f, zero};
}
// An entry's class: f (Q p_j - sum of its q).
template <class Val>
__device__ __forceinline__ float entry_slope(const DistillParams &p, const DistillStat &st, float w, Val x, float q) {
    return p.l.scale * w * (st.total * __builtin_amdgcn_exp2f(p.l.scale * LOG2E * below(x, of_bits<Val>(st.m)) - st.logs * LOG2E) - q);
}

template <int TYPE, int T, int NV>
__global__ __launch_bounds__(T) void distill_grad_kernel(const DistillParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    const uint32_t row = blockIdx.x / p.chunks, chunk = blockIdx.x - row * p.chunks, lane = threadIdx.x & 63;
    const uint64_t r = p.row0 + row;
    const Chunk<TYPE, T, NV> k(p.l, r, chunk, p.chunks, p.chunk_vecs);
    const DistillStat st = p.stats[r];
    const float w = p.weight ? p.weight[r] : 1.f;
    Named named;
    named.load(p.entry + r * p.top, p.top);
    store_gradient(k, p.l.classes, (typename K::Grad *)p.grad + r * p.grad_stride, p.grad == p.l.x, row_slope<Val>(p, st, w), named, [&](int h) {
        return share_of(p, teacher_value(p.value, p.value_type, r * p.top + lane + 64 * h), st.value_m, st.value_logs);
    }, [&](Val v, float sum) { return entry_slope(p, st, w, v, sum); });
}

// ---- loss ---------------------------------------------------------------------------------------

// Statistics of the thread's share of a chunk.  REST: without the entries, which a byte of bits for each vector in LDS tells; a
// thread's NV bytes lie together, and vectors without an entry (nearly all) go the same way as in the other case.
template <bool REST, int T, int NV> struct SharedMask { uint32_t bits[NV * T / 4], tail; };
template <int T, int NV> struct SharedMask<false, T, NV> {};

template <int T>
struct RowEntries {   // of the row, one a thread, two of a single wave
    int32_t c[T == 64 ? 2 : 1];
    __device__ __forceinline__ RowEntries(const DistillParams &p, uint64_t r) {
#pragma unroll
        for (uint32_t h = 0; h < sizeof(c) / 4; ++h) c[h] = threadIdx.x + h * T < p.top ? p.entry[r * p.top + threadIdx.x + h * T] : -1;
    }
};

template <bool REST, int TYPE, int T, int NV>
__device__ __forceinline__ Stat<typename Kind<TYPE>::Val> chunk_stat(Chunk<TYPE, T, NV> &k, uint32_t classes, float c, const RowEntries<T> &entries, SharedMask<REST, T, NV> &sh) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    constexpr int PV = PER_VEC<TYPE>, WORDS = (NV + 3) / 4;
    const uint32_t tid = threadIdx.x;
    bool edge_valid = k.edge_valid;
    uint32_t out[WORDS] = {};   // bits of the entries among the thread's vectors, a byte each
    if constexpr (REST) {
#pragma unroll
        for (int i = 0; i < (NV * T / 4 + T - 1) / T; ++i)
            if (i * T + tid < NV * T / 4) sh.bits[i * T + tid] = 0;
        if (tid == 0) sh.tail = 0;
        __syncthreads();
#pragma unroll
        for (const int32_t entry : entries.c) {
            if ((uint32_t)entry >= classes || !k.owns((uint32_t)entry)) continue;   // or negative
            const uint32_t j = (uint32_t)entry - k.first;
            if (j < k.n * PV) {
                const uint32_t vec = j / PV, byte = vec % T * NV + vec / T;
                atomicOr(&sh.bits[byte >> 2], 1u << (8 * (byte & 3) + j % PV));
            } else {
                atomicOr(&sh.tail, 1u << ((uint32_t)entry < k.head ? PV - 1 : (uint32_t)entry - k.end));
            }
        }
        __syncthreads();
        if constexpr (NV == 2) {
            out[0] = ((const uint16_t *)sh.bits)[tid];
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) out[i] = sh.bits[tid * WORDS + i];
        }
        edge_valid = edge_valid && !(sh.tail >> (tid & 31) & 1);
    }
    auto bits = [&](int i) { return out[i / 4] >> (8 * (i & 3)) & 0xFF; };
    const Val edge = K::val(k.edge);
    Stat<Val> a{edge_valid ? edge : lowest(Val()), 0.f, 0.f};
    k.each([&](int i, uint32_t, Val (&v)[PV]) {
        if (REST && bits(i)) {
#pragma unroll
            for (int e = 0; e < PV; ++e) v[e] = bits(i) >> e & 1 ? lowest(Val()) : v[e];
        }
#pragma unroll
        for (int e = 0; e < PV; ++e) a.m = larger(a.m, v[e]);
    });
    k.keep_packed();
    auto share = [&](Val v) { return __builtin_amdgcn_exp2f(c * below(v, a.m)); };
    if (edge_valid) a.s = share(edge);
    k.each([&](int i, uint32_t, const Val (&v)[PV]) {
        if (REST && bits(i)) {
#pragma unroll
            for (int e = 0; e < PV; ++e) a.s += bits(i) >> e & 1 ? 0.f : share(v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < PV; ++e) a.s += share(v[e]);
        }
    });
    return a;
}

// A chunk of a row, or (p.chunks == 1) a whole one.
template <int TYPE, int T, int NV, bool REST>
__global__ __launch_bounds__(T) void distill_kernel(const DistillParams p) {
    using Val = typename Kind<TYPE>::Val;
    __shared__ SharedStat<T> sh;
    __shared__ SharedMask<REST, T, NV> mask;
    __shared__ __attribute__((aligned(16))) uint32_t table[SLOTS];
    const uint32_t tid = threadIdx.x, row = blockIdx.x / p.chunks, chunk = blockIdx.x - row * p.chunks;
    const uint64_t r = p.row0 + row;
    // in front of the row's loads, behind which it would have to wait for them
    const RowEntries<T> entries(p, r);
    const bool whole = p.chunks == 1;
    Entries<TYPE> e;
    if (whole && tid < 64) e.load(p, r);
    Chunk<TYPE, T, NV> k(p.l, r, chunk, p.chunks, p.chunk_vecs);
    Taught t;
    if (whole && tid < 64) t = taught<TYPE>(p, e, table);   // while the row arrives
    const float c = p.l.scale * LOG2E;
    const Stat<Val> all = block_stat<T, false>(chunk_stat<REST>(k, p.l.classes, c, entries, mask), c, sh, [] {});
    if (!whole) {
        if (tid == 0) p.parts[(size_t)row * p.chunks + chunk] = Part{__builtin_bit_cast(uint32_t, all.m), all.s, 0.f, 0};
        return;
    }
    if (tid >= 64) return;
    const DistillStat st = conclude<TYPE>(p, r, all, e, t);
    if (p.stats && tid == 0) p.stats[r] = st;
}

template <int TYPE>
__global__ __launch_bounds__(64) void distill_join_kernel(const DistillParams p) {
    using Val = typename Kind<TYPE>::Val;
    __shared__ __attribute__((aligned(16))) uint32_t table[SLOTS];
    const uint64_t r = p.row0 + blockIdx.x;
    Entries<TYPE> e;
    e.load(p, r);
    const Stat<Val> all = join_parts<Val>(p.parts + (size_t)blockIdx.x * p.chunks, p.chunks, p.l.scale * LOG2E);
    const DistillStat st = conclude<TYPE>(p, r, all, e, taught<TYPE>(p, e, table));
    if (p.stats && threadIdx.x == 0) p.stats[r] = st;
}

// Loss and gradient of a row from registers.
template <int TYPE, int T, int NV, bool REST>
__global__ __launch_bounds__(T) void distill_row_kernel(const DistillParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    __shared__ SharedStat<T> sh;
    __shared__ SharedMask<REST, T, NV> mask;
    __shared__ __attribute__((aligned(16))) uint32_t table[SLOTS];
    __shared__ DistillStat stat;
    const uint32_t tid = threadIdx.x;
    const uint64_t r = p.row0 + blockIdx.x;
    const RowEntries<T> entries(p, r);
    Entries<TYPE> e;
    if (tid < 64) e.load(p, r);
    const float w = p.weight ? p.weight[r] : 1.f;
    Chunk<TYPE, T, NV> k(p.l, r, 0, 1, p.chunk_vecs);
    Taught t;
    if (tid < 64) t = taught<TYPE>(p, e, table);   // while the row arrives
    const float c = p.l.scale * LOG2E;
    const Stat<Val> all = block_stat<T, false>(chunk_stat<REST>(k, p.l.classes, c, entries, mask), c, sh, [] {});
    if (tid < 64) {
        const DistillStat st = conclude<TYPE>(p, r, all, e, t);
        if (tid == 0) {
            stat = st;
            if (p.stats) p.stats[r] = st;
        }
    }
    __syncthreads();
    const DistillStat st = stat;
    const Slope<Val, false> f = row_slope<Val>(p, st, w);
    auto *out = (typename K::Grad *)p.grad + r * p.grad_stride;
    store_slopes(k, out, f);
    __syncthreads();
    if (tid >= 64 || f.zero) return;
    float sum[2] = {t.q[0], t.q[1]};
    const uint64_t again[2] = {__ballot(e.c[0] >= 0 && !t.is[0]), __ballot(e.c[1] >= 0 && !t.is[1])};
    e.add_same(again, t.q, sum);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (t.is[h] && (uint32_t)e.c[h] < p.l.classes) out[e.c[h]] = K::grad(entry_slope(p, st, w, e.at[h], sum[h]));
}

// ---- rows of few classes: 16 lanes a row, E elements a lane ---------------------------------

// FORWARD: loss and statistics, and the gradient if there is a place for it; otherwise the gradient from the statistics.
template <int TYPE, int E, bool FORWARD>
__global__ __launch_bounds__(THREADS) void distill_small_kernel(const DistillParams p) {
    using K = Kind<TYPE>;
    using Val = typename K::Val;
    const uint32_t lane = threadIdx.x & 15, row = blockIdx.x * (THREADS / 16) + (threadIdx.x >> 4), n = p.l.classes;
    const uint64_t r = p.row0 + min(row, p.run - 1);   // lanes without a row go along with the last one's
    const bool store = row < p.run;
    const auto *x = (const typename K::Raw *)p.l.x + r * p.l.stride;
    Val v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = K::val(x[min(lane + 16 * i, n - 1)]);
    const float w = p.weight ? p.weight[r] : 1.f, c = p.l.scale * LOG2E;
    // the entries: each lane every sixteenth, then in LDS for all of the row's
    __shared__ int32_t entries[THREADS / 16][ISR_MAX_GIVEN];
    __shared__ float shares[THREADS / 16][ISR_MAX_GIVEN];
    int32_t *const ec = entries[threadIdx.x >> 4];
    float *const eq = shares[threadIdx.x >> 4];   // the teacher's value, then q
    float value_m = NEG_INF;
    int any = 0, bad = 0;
    for (uint32_t i = lane; i < p.top; i += 16) {
        const int32_t cls = p.entry[r * p.top + i];
        const float value = cls >= 0 ? teacher_value(p.value, p.value_type, r * p.top + i) : NEG_INF;
        ec[i] = cls;
        eq[i] = value;
        any |= cls >= 0;
        bad |= cls >= 0 && ((uint32_t)cls >= n || value != value || value == -NEG_INF);
        value_m = larger(value_m, value);
    }
    DistillStat st;
    if constexpr (!FORWARD) st = p.stats[r];
    float value_logs = 0.f;
    double left = 0.0, total = 0.0, entropy = 0.0;   // q_rest, sum of q, sum of q log q
    bool none = false;
    if constexpr (FORWARD) {
        any = fold16(any, [](int a, int b) { return a | b; });
        bad = fold16(bad, [](int a, int b) { return a | b; });
        value_m = p.rest ? 0.f : max16(value_m);
        none = !any || value_m == NEG_INF;
        if (none) value_m = 0.f;
        if (!p.rest) {
            float z = 0.f;
            for (uint32_t i = lane; i < p.top; i += 16) z += ec[i] >= 0 ? share_of(p, eq[i], value_m, 0.f) : 0.f;
            value_logs = logf(sum16(z));
        }
    } else {
        value_m = st.value_m;
        value_logs = st.value_logs;
    }
    for (uint32_t i = lane; i < p.top; i += 16) {
        float share = 0.f;
        if (ec[i] >= 0) {
            const double lq = log_share(p, eq[i], value_m, value_logs);
            if (p.rest) {   // the sum that leads to q_rest in 64 bits
                const double full = exp(lq);
                share = (float)full;   // as share_of()
                if (FORWARD) total += full;
            } else {
                share = expf((float)lq);
                if (FORWARD) total += share;
            }
            if (FORWARD && share > 0.f) entropy += (double)share * lq;
        }
        eq[i] = share;
    }
    wave_order();
    // sum of q by class: every lane sees all entries in turn and keeps those of its elements
    float q[E] = {};
    uint32_t member = 0;
    for (uint32_t i = 0; i < p.top; ++i) {
        const int32_t cls = ec[i];
        const float share = eq[i];
        const int own = cls >= 0 && (cls & 15) == (int)lane ? cls >> 4 : -1;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            q[e] += own == e ? share : 0.f;
            member |= (uint32_t)(own == e) << e;
        }
    }
    if constexpr (FORWARD) {
        total = sum16(total);
        entropy = sum16(entropy);
        if (p.rest) left = fmax(1.0 - total, 0.0);
        total += left;
        // of the classes that are no entry (rest), and of all
        Stat<Val> a{lowest(Val()), 0.f, 0.f}, all;
        all.m = a.m;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (lane + 16 * i >= n) continue;
            all.m = larger(all.m, v[i]);
            if (!(member >> i & 1)) a.m = larger(a.m, v[i]);
        }
        all.m = max16(all.m);
        a.m = max16(a.m);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (lane + 16 * i >= n) continue;
            if (!(member >> i & 1)) a.s += __builtin_amdgcn_exp2f(c * below(v[i], a.m));
            s += __builtin_amdgcn_exp2f(c * below(v[i], all.m));
        }
        all.s = sum16(s);
        a.s = sum16(a.s);
        if (!p.rest) a = all;
        const bool empty = all.s == 0.f;
        const float logs = empty ? 0.f : logf(all.s), rest_logs = a.s == 0.f ? NEG_INF : logf(a.s);
        double cross = 0.0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (lane + 16 * i >= n || !(q[i] > 0.f)) continue;
            cross += (double)q[i] * (empty || !possible(v[i]) ? (double)NEG_INF : (double)p.l.scale * below64(v[i], all.m) - logs);
        }
        double loss = entropy - sum16(cross);
        if (!p.rest) loss /= total;   // as in conclude()
        if (left > 0.0) {
            const double lr = a.s == 0.f ? (double)NEG_INF : (double)p.l.scale * below64(a.m, all.m) + ((double)rest_logs - logs);
            if (no_rest(p, left, lr, -entropy)) {
                total -= left;
                left = 0.0;
            } else {
                loss += left * (logf((float)left) - lr);
            }
        }
        const bool nan = bad || all.s != all.s;
        st = DistillStat{bits_of(all.m), empty && !nan ? NEG_INF : logs, bits_of(a.m), rest_logs, value_m, value_logs,
                         nan ? __builtin_nanf("") : (float)total, (float)left};
        if (none) st = DistillStat{0.f, NEG_INF, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (store && lane == 0) {
            p.loss[r] = none ? 0.f : nan ? __builtin_nanf("") : (float)loss;
            if (p.stats) p.stats[r] = st;
        }
        if (!p.grad) return;
    }
    const Slope<Val, false> f = row_slope<Val>(p, st, w);
    auto *out = (typename K::Grad *)p.grad + r * p.grad_stride;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if (!store || lane + 16 * i >= n) continue;
        const float g = f.zero ? 0.f : member >> i & 1 ? entry_slope(p, st, w, v[i], q[i]) : f(v[i]);
        out[lane + 16 * i] = K::grad(g);
    }
}

// ---- launches --------------------------------------------------------------------------------

static uint32_t vecs_of(int type, uint32_t classes) { return classes / (type == ISR_F32 || type == ISR_I32 ? 4 : 8); }

bool distill_in_one(int type, uint32_t classes) { return vecs_of(type, classes) <= 16 * 1024; }

template <int TYPE, int T, int NV>
static void launch_row_kernel(const DistillParams &p, hipStream_t st) {
    if (p.rest) hipLaunchKernelGGL((distill_row_kernel<TYPE, T, NV, true>), dim3(p.run), dim3(T), 0, st, p);
    else hipLaunchKernelGGL((distill_row_kernel<TYPE, T, NV, false>), dim3(p.run), dim3(T), 0, st, p);
}

template <int TYPE, bool FORWARD>
static void launch_small(const DistillParams &p, hipStream_t st) {
    const dim3 grid((p.run + THREADS / 16 - 1) / (THREADS / 16)), block(THREADS);
    if (p.l.classes <= 16) hipLaunchKernelGGL((distill_small_kernel<TYPE, 1, FORWARD>), grid, block, 0, st, p);
    else if (p.l.classes <= 64) hipLaunchKernelGGL((distill_small_kernel<TYPE, 4, FORWARD>), grid, block, 0, st, p);
    else if (p.l.classes <= 128) hipLaunchKernelGGL((distill_small_kernel<TYPE, 8, FORWARD>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((distill_small_kernel<TYPE, 16, FORWARD>), grid, block, 0, st, p);
}

template <int TYPE, int T, int NV>
static void launch_chunks(const DistillParams &p, hipStream_t st) {
    const dim3 grid(p.run * p.chunks), block(T);
    if (p.rest) hipLaunchKernelGGL((distill_kernel<TYPE, T, NV, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((distill_kernel<TYPE, T, NV, false>), grid, block, 0, st, p);
}
template <int TYPE>
static void launch_loss(const DistillParams &p, Way way, uint32_t nv, hipStream_t st) {
    if (way == Way::wave) launch_chunks<TYPE, 64, 4>(p, st);
    else if (way == Way::alone && nv == 4) launch_chunks<TYPE, ALONE, 4>(p, st);
    else if (way == Way::alone) launch_chunks<TYPE, ALONE, 8>(p, st);
    else if (nv == 2) launch_chunks<TYPE, THREADS, 2>(p, st);
    else launch_chunks<TYPE, THREADS, 8>(p, st);
    if (p.chunks > 1) hipLaunchKernelGGL((distill_join_kernel<TYPE>), dim3(p.run), dim3(64), 0, st, p);
}

// 16 vectors a thread and as few threads as that takes: several workgroups share a CU, and what one sums another's loads cover.  us with
// 256 threads of 16 / 1024 of 8: 8192 x 24000 bf16 148 / 231, 8192 x 32000 199 / 263, with 512 of 16: 4096 x 64000 195 / 227.
template <int TYPE>
static void launch_in_one(DistillParams &p, hipStream_t st) {
    const uint32_t vecs = vecs_of(TYPE, p.l.classes);
    p.chunks = 1;
    p.chunk_vecs = vecs;
    if (vecs <= WAVE_VECS) launch_row_kernel<TYPE, 64, 4>(p, st);
    else if (vecs <= 2 * THREADS) launch_row_kernel<TYPE, THREADS, 2>(p, st);
    else if (vecs <= 8 * THREADS) launch_row_kernel<TYPE, THREADS, 8>(p, st);
    else if (vecs <= 16 * THREADS) launch_row_kernel<TYPE, THREADS, 16>(p, st);
    else if (vecs <= 16 * 512) launch_row_kernel<TYPE, 512, 16>(p, st);
    else launch_row_kernel<TYPE, 1024, 16>(p, st);
}

template <int TYPE>
static void launch_gradient(const DistillParams &p, Way way, hipStream_t st) {
    const dim3 grid(p.run * p.chunks);
    if (way == Way::sixteen) launch_small<TYPE, false>(p, st);
    else if (way == Way::wave) hipLaunchKernelGGL((distill_grad_kernel<TYPE, 64, 4>), grid, dim3(64), 0, st, p);
    else hipLaunchKernelGGL((distill_grad_kernel<TYPE, THREADS, 4>), grid, dim3(THREADS), 0, st, p);
}

hipError_t launch_distill(DistillParams p, const RowCut &cut, void *workspace, hipStream_t st) {
    const bool in_one = p.grad && distill_in_one(p.l.type, p.l.classes);
    const RowCut gradient = cut_gradient(p.l);
    p.parts = (Part *)workspace;
    return by_runs(p, cut.rows, [&](uint32_t rows) {
        p.run = rows;
        p.chunks = cut.chunks;
        p.chunk_vecs = cut.chunk_vecs;
#define CALL(T)                                                                          \
    if (cut.way == Way::sixteen) launch_small<T, true>(p, st);                           \
    else if (in_one) launch_in_one<T>(p, st);                                            \
    else launch_loss<T>(p, cut.way, cut.nv, st)
        ISR_BY_TYPE(p.l.type, CALL)
#undef CALL
        if (!p.grad || in_one) return;
        p.chunks = gradient.chunks;
        p.chunk_vecs = gradient.chunk_vecs;
#define CALL(T) launch_gradient<T>(p, gradient.way, st)
        ISR_BY_TYPE(p.l.type, CALL)
#undef CALL
    });
}

hipError_t launch_distill_grad(DistillParams p, hipStream_t st) {
    const RowCut cut = cut_gradient(p.l);
    p.chunks = cut.chunks;
    p.chunk_vecs = cut.chunk_vecs;
    return by_runs(p, cut.rows, [&](uint32_t rows) {
        p.run = rows;
#define CALL(T) launch_gradient<T>(p, cut.way, st)
        ISR_BY_TYPE(p.l.type, CALL)
#undef CALL
    });
}

}  // namespace isr
