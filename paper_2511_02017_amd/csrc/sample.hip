// Tokens drawn under a temperature and filters, and the filtered logits.
//
//   d_j = (x_j - max) / T,  w_j = e^(d_j);  order: larger x first, equal ones by index
//   top-k: the first k;  top-p: the shortest run from the start whose mass reaches p of the top-k's;  min-p: w_j >= min_p
//   token: smallest j whose sum of kept weights up to and with j exceeds u Z;  log q = d_token - ln Z
//
// All three filters keep a run from the start of the order, so what a row keeps is said by its last element: a key (the logit's bits, mapped to
// integers that order alike) and the index up to which elements of that key are kept.  The row is not sorted: a histogram over the distance from
// the maximum names the bin in which the run ends, and the few elements of that bin are ranked among each other (a bin with many is cut again, by
// keys, down to a single key).
//
// Weights are summed as whole numbers of 2^-S of the largest, S = 62 - log2 V (45 at V = 128256): sums of them do not depend on their order, so
// any division of the work gives the same bits, and each is off by half a unit, so that a sum is off by about 1e-12 of the largest weight, far
// less than the gaps between neighbouring sums that a decision could fall into.
#include "exp_device.h"

namespace tapout {
namespace {

constexpr int kThreads = 1024, kBins = 2048, kList = 1024, kLoads = 4;
constexpr float kTopKBins = 256.f;             // bins of a unit of logits where elements are counted

__device__ __forceinline__ uint32_t key_of(float x)             // -0 and 0 are one value
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu)); }
constexpr uint32_t kMasked = 0x007fffffu;      // the key of -infinity: only larger ones are ever kept

// Last element of a run: keys above, and equal ones up to the index, are in it.
struct Bound {
    uint32_t key; int32_t index;
    __device__ __forceinline__ bool holds(uint32_t k, int32_t j) const { return k > key || (k == key && j <= index); }
};
__device__ __forceinline__ Bound shorter(Bound a, Bound b) { return a.key > b.key || (a.key == b.key && a.index < b.index) ? a : b; }

struct Shared {
    double table[256];                         // 2^(k / 256)
    uint64_t bins[kBins];
    uint64_t list_w[kList];
    uint32_t list_key[kList];
    int32_t list_index[kList];
    uint64_t waves[kThreads / kWave];
    float waves_f[kThreads / kWave];
    uint32_t lo, hi;
    int32_t count, found, nan;
    uint64_t sum;
    Bound bound;
};

// A row's weights.
struct Weight {
    double max, c; int shift;                  // c = 256 / (T ln 2);  shift: log2 of the units of the largest weight
    // (x - max) / T in units of ln2 / 256, from 0 down to where weights are no unit any more
    __device__ __forceinline__ double steps(float x) const { return fmax(((double)x - max) * c, -256.0 * 64.0); }
    __device__ __forceinline__ uint64_t units(double t, int &ni, const double *table) const
    {
        const double tm = t + kMagic;
        ni = __double2loint(tm);
        const double r = t - (tm - kMagic), tk = table[ni & 255];
        const double q = r * fma(r, fma(r, fma(r, kExpC1 * kExpC1 * kExpC1 * kExpC1 / 24.0, kExpC3), kExpC2), kExpC1);
        const double e = ldexp(fma(tk, q, tk), (ni >> 8) + shift);
        return (uint64_t)(__double_as_longlong(e + 4503599627370496.0) & 0xfffffffffffffll);          // to nearest: e is at most 2^50
    }
    __device__ __forceinline__ uint64_t of(float x, const double *table) const { int ni; return units(steps(x), ni, table); }
};

// Sixteen bytes of a row, as values; what lies outside it is -infinity.
template <int DT> struct RowReader {
    static constexpr int n = Elem<DT>::vec;
    const char *base;                          // the row's start rounded down to 16 bytes
    int before, V, vecs;                       // elements of the first vector that lie before the row
    __device__ __forceinline__ RowReader(const void *row, int V_) : V(V_)
    {
        before = (int)((uintptr_t)row & 15) / Elem<DT>::size;
        base = (const char *)row - before * Elem<DT>::size;
        vecs = (V + before + n - 1) / n;
    }
    __device__ __forceinline__ int first(int v) const { return v * n - before; }        // index of a vector's first element
    __device__ __forceinline__ bool whole(int v) const { return first(v) >= 0 && first(v) + n <= V; }
    __device__ __forceinline__ void load(int v, float (&x)[n]) const
    {
        if (v < vecs && whole(v)) {
            unpack<DT>(*(const u32x4 *)(base + (int64_t)v * 16), x);
        } else {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const int j = first(v) + e;
                x[e] = j >= 0 && j < V ? load_elem<DT>(base, (int64_t)v * n + e) : -INFINITY;
            }
        }
    }
};

// f(vector, values) for the row's vectors, a turn of kThreads at a time, several turns' loads under way.  Every thread takes part in every turn: behind
// the row it has values of -infinity.
template <int DT, class F>
__device__ __forceinline__ void each_vector(const RowReader<DT> &row, F f)
{
    constexpr int n = RowReader<DT>::n;
    for (int base = 0; base < row.vecs; base += kThreads * kLoads) {
        if ((base > 0 || row.before == 0) && base + kThreads * kLoads < row.vecs) {
            u32x4 w[kLoads];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) w[u] = *(const u32x4 *)(row.base + (int64_t)(base + u * kThreads + threadIdx.x) * 16);
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                float x[n];
                unpack<DT>(w[u], x);
                f(base + u * kThreads + (int)threadIdx.x, x);
            }
        } else {
            for (int u = 0; u < kLoads && base + u * kThreads < row.vecs; ++u) {
                float x[n];
                row.load(base + u * kThreads + threadIdx.x, x);
                f(base + u * kThreads + (int)threadIdx.x, x);
            }
        }
    }
}

__device__ __forceinline__ uint64_t wave_sum_u(uint64_t v)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v += (uint64_t)__shfl_xor((unsigned long long)v, d);
    return v;
}
// Sum over the workgroup, in every thread.
__device__ __forceinline__ uint64_t block_sum(uint64_t v, Shared &sh)
{
    v = wave_sum_u(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.waves[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int k = 0; k < kThreads / kWave; ++k) v += sh.waves[k];
    return v;
}
// Sum over the threads before this one, and over all.
__device__ __forceinline__ uint64_t block_before(uint64_t v, uint64_t &all, Shared &sh)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t s = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const uint64_t o = (uint64_t)__shfl_up((unsigned long long)s, d);
        if (lane >= d) s += o;
    }
    __syncthreads();
    if (lane == 63) sh.waves[wave] = s;
    __syncthreads();
    uint64_t before = s - v;
    all = 0;
#pragma unroll
    for (int k = 0; k < kThreads / kWave; ++k) {
        if (k < wave) before += sh.waves[k];
        all += sh.waves[k];
    }
    return before;
}

// The first bin with which the bins' sum from `above` on reaches `target`, and the sum before it; -1 if none does.
__device__ __forceinline__ int find_bin(uint64_t target, uint64_t &above, Shared &sh)
{
    constexpr int per = kBins / kThreads;
    uint64_t own = 0, all;
#pragma unroll
    for (int k = 0; k < per; ++k) own += sh.bins[threadIdx.x * per + k];
    uint64_t before = above + block_before(own, all, sh);
    if (threadIdx.x == 0) sh.found = -1;
    __syncthreads();
    if (before < target && before + own >= target) {           // one thread
#pragma unroll
        for (int k = 0; k < per; ++k) {
            const uint64_t next = before + sh.bins[threadIdx.x * per + k];
            if (next >= target) { sh.found = threadIdx.x * per + k; sh.sum = before; break; }
            before = next;
        }
    }
    __syncthreads();
    const int b = sh.found;
    if (b >= 0) above = sh.sum;
    __syncthreads();
    return b;
}

__device__ __forceinline__ void clear_bins(Shared &sh)
{
    __syncthreads();
    for (int k = threadIdx.x; k < kBins; k += kThreads) sh.bins[k] = 0;
    __syncthreads();
}

// The last element of the shortest run of `within` whose measure (a count, or units of weight) reaches `target`; `within` itself if none does.
// first_bin(x): bin from the front for a first division, kBins - 1 for all that lie far behind.  measure(x): of an element.
template <int DT, class Bin, class Measure>
__device__ __forceinline__ Bound reach(const RowReader<DT> &row, Bound within, uint64_t target, Bin first_bin, Measure measure, Shared &sh)
{
    constexpr int n = RowReader<DT>::n;
    clear_bins(sh);
    each_vector<DT>(row, [&](int v, const float (&x)[n]) {
#pragma unroll
        for (int e = 0; e < n; ++e) {
            const uint32_t k = key_of(x[e]);
            if (k > kMasked && within.holds(k, row.first(v) + e)) atomicAdd((unsigned long long *)&sh.bins[first_bin(x[e])], (unsigned long long)measure(x[e]));
        }
    });
    __syncthreads();
    uint64_t above = 0;
    int b = find_bin(target, above, sh);
    if (b < 0) return within;
    uint32_t lo = 0, hi = 0;
    bool by_key = false;
    for (;;) {
        // the elements of this bin
        if (threadIdx.x == 0) { sh.count = 0; sh.lo = 0xffffffffu; sh.hi = 0; }
        __syncthreads();
        uint32_t least = 0xffffffffu, most = 0;
        each_vector<DT>(row, [&](int v, const float (&x)[n]) {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const uint32_t k = key_of(x[e]);
                const int j = row.first(v) + e;
                if (k <= kMasked || (by_key ? k < lo || k > hi : first_bin(x[e]) != b) || !within.holds(k, j)) continue;
                least = min(least, k);
                most = max(most, k);
                const int at = atomicAdd(&sh.count, 1);
                if (at < kList) { sh.list_key[at] = k; sh.list_index[at] = j; }
            }
        });
        if (least <= most) { atomicMin(&sh.lo, least); atomicMax(&sh.hi, most); }
        __syncthreads();
        const int count = sh.count;
        lo = sh.lo; hi = sh.hi;
        __syncthreads();
        if (count <= kList) {
            const int i = threadIdx.x;
            uint32_t k = 0; int j = 0; uint64_t own = 0, before = above;
            if (i < count) {
                k = sh.list_key[i]; j = sh.list_index[i];
                own = measure(value_of(k));
                sh.list_w[i] = own;
            }
            __syncthreads();
            if (i < count) {
                for (int o = 0; o < count; ++o) {
                    const uint32_t ko = sh.list_key[o];
                    if (ko > k || (ko == k && sh.list_index[o] < j)) before += sh.list_w[o];
                }
                if (before < target && before + own >= target) sh.bound = Bound{k, j};          // one thread
            }
            __syncthreads();
            const Bound r = sh.bound;
            __syncthreads();
            return r;
        }
        if (lo == hi) {
            // equal elements: the run ends at the r-th of them by index
            const uint64_t own = measure(value_of(lo)), r = own ? (target - above + own - 1) / own : 1;
            uint64_t seen = 0;
            for (int v0 = 0; v0 < row.vecs; v0 += kThreads) {
                float x[n];
                row.load(v0 + threadIdx.x, x);
                uint32_t equal = 0;
#pragma unroll
                for (int e = 0; e < n; ++e)
                    if (key_of(x[e]) == lo && within.holds(lo, row.first(v0 + threadIdx.x) + e)) equal |= 1u << e;
                uint64_t all;
                uint64_t before = seen + block_before(__popc(equal), all, sh);
                if (before < r && before + __popc(equal) >= r) {
#pragma unroll
                    for (int e = 0; e < n; ++e)
                        if (equal >> e & 1 && ++before == r) sh.bound = Bound{lo, row.first(v0 + threadIdx.x) + e};
                }
                seen += all;
                if (seen >= r) break;
            }
            __syncthreads();
            const Bound q = sh.bound;
            __syncthreads();
            return q;
        }
        // too many: by keys
        const int shift = max(0, 32 - __clz((int)(hi - lo)) - 11);           // (hi - lo) >> shift is below kBins
        clear_bins(sh);
        each_vector<DT>(row, [&](int v, const float (&x)[n]) {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const uint32_t k = key_of(x[e]);
                if (k >= lo && k <= hi && within.holds(k, row.first(v) + e)) atomicAdd((unsigned long long *)&sh.bins[(hi - k) >> shift], (unsigned long long)measure(x[e]));
            }
        });
        __syncthreads();
        b = find_bin(target, above, sh);
        if (b < 0) return within;                                            // not reached: the bin holds what was missing
        by_key = true;
        const uint32_t top = hi - ((uint32_t)b << shift);
        lo = max(lo, top - min(top, (1u << shift) - 1));
        hi = top;
    }
}

// A vector of results at any element-aligned address.
template <class E, int N> __device__ __forceinline__ void store_any(E *to, const float (&y)[N])
{
    struct __attribute__((packed, aligned(sizeof(E)))) Any { u32x4 v; };
    E v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (E)y[e];
#pragma unroll
    for (int k = 0; k < N * (int)sizeof(E) / 16; ++k) ((Any *)to)[k].v = ((const u32x4 *)v)[k];
    if constexpr (N * sizeof(E) == 8) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        struct __attribute__((packed, aligned(sizeof(E)))) Half { u32x2 v; };
        ((Half *)to)->v = *(const u32x2 *)v;
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void filtered_sample_kernel(FilterArgs a)
{
    constexpr int n = RowReader<DT>::n;
    __shared__ Shared sh;
    const int r = blockIdx.x, b = r / a.K, k = r - b * a.K;
    if (a.k_len && k >= a.k_len[b]) return;
    const RowReader<DT> row(row_address(a.base, DT, a.stride_b, a.stride_k, b, k), a.V);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float T = a.temperature ? a.temperature[b] : 1.f, top_p = a.top_p ? a.top_p[b] : 1.f, min_p = a.min_p ? a.min_p[b] : 0.f;
    const int top_k = a.top_k ? a.top_k[b] : 0;
    if (threadIdx.x < 256) sh.table[threadIdx.x] = a.exp_table[threadIdx.x];
    if (threadIdx.x == 0) sh.nan = 0;
    // the maximum
    float m = -INFINITY;
    bool nan = false;
    each_vector<DT>(row, [&](int, const float (&x)[n]) {
#pragma unroll
        for (int e = 0; e < n; ++e) { m = fmaxf(m, x[e]); nan |= x[e] != x[e]; }
    });
    m = lanes_max(m, 0, 6);
    if (lane == 0) sh.waves_f[wave] = m;
    __syncthreads();
    if (nan) sh.nan = 1;
    m = sh.waves_f[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) m = fmaxf(m, sh.waves_f[w]);
    __syncthreads();
    const bool bad = sh.nan || !(fabsf(m) < INFINITY) || T != T, greedy = !(T > 0.f);
    if (a.flags && threadIdx.x == 0) {
        if (a.K == 1) a.flags[b] = bad ? TAPOUT_FLAG_BAD_ROW : 0u;
        else if (bad) atomicOr(&a.flags[b], TAPOUT_FLAG_BAD_ROW);
    }
    // what the row keeps; a bad row nothing
    Bound end{kMasked, -1};                                    // -1: no element of this key
    Weight w{(double)m, greedy || bad ? 0.0 : 256.0 / ((double)T * kLn2), a.shift};
    if (bad) end = Bound{0xffffffffu, -1};
    else {
        if (greedy || (top_k > 0 && top_k < a.V)) {
            const float mf = m;
            end = reach<DT>(row, end, greedy ? 1 : top_k, [=](float x) { return (int)fminf((mf - x) * kTopKBins, (float)(kBins - 1)); }, [](float) { return (uint64_t)1; }, sh);
        }
        if (!greedy && top_p < 1.f) {
            uint64_t mine = 0;
            const Bound within = end;
            each_vector<DT>(row, [&](int v, const float (&x)[n]) {
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    const uint32_t key = key_of(x[e]);
                    if (key > kMasked && within.holds(key, row.first(v) + e)) mine += w.of(x[e], sh.table);
                }
            });
            const uint64_t Z = block_sum(mine, sh);
            const double reached = (double)top_p * (double)Z;
            const uint64_t target = reached > 1.0 ? (uint64_t)ceil(reached) : 1;
            end = reach<DT>(row, within, target, [=](float x) { return min(kBins - 1, (int)(-w.steps(x)) >> 3); }, [&](float x) { return w.of(x, sh.table); }, sh);
        }
        if (!greedy && min_p > 0.f) {
            // the smallest key whose weight is large enough: a 64th of the interval at a time
            const double least = log((double)fminf(min_p, 1.f)), inv = 1.0 / (double)T;
            uint32_t lo = kMasked, hi = key_of(m);                                         // lo: not enough, hi: enough
            while (hi - lo > 1) {
                const uint32_t step = (hi - lo + 63) / 64, at = lo + min((uint32_t)(lane + 1) * step, hi - lo);
                const uint64_t enough = __ballot(((double)value_of(at) - (double)m) * inv >= least);
                const int first = __ffsll((unsigned long long)enough) - 1;                   // the last lane's is hi
                hi = lo + min((uint32_t)(first + 1) * step, hi - lo);
                lo = first ? lo + (uint32_t)first * step : lo;
            }
            end = shorter(end, Bound{hi, 0x7fffffff});
        }
    }
    // what is kept, and its weights by chunks of the row
    const bool draw = a.u != nullptr;
    const int turn = kThreads, turns = (row.vecs + turn - 1) / turn, per = (turns + kBins - 1) / kBins;      // vectors of a turn; turns of a chunk
    const double inv = greedy || bad ? 0.0 : 1.0 / (double)T;
    clear_bins(sh);
    int kept = 0;
    char *out = a.kept ? (char *)row_address(a.kept, a.kept_dtype, a.kept_stride_b, a.kept_stride_k, b, k) : nullptr;
    each_vector<DT>(row, [&](int v, const float (&x)[n]) {
        float y[n];
        uint64_t mine = 0;
        const int j0 = row.first(v);
#pragma unroll
        for (int e = 0; e < n; ++e) {
            const uint32_t key = key_of(x[e]);
            y[e] = -INFINITY;
            if (key > kMasked && end.holds(key, j0 + e)) {
                ++kept;
                y[e] = (float)(((double)x[e] - (double)m) * inv);
                if (draw) mine += w.of(x[e], sh.table);
            }
        }
        if (draw && __any(mine != 0)) {
            mine = wave_sum_u(mine);
            if (lane == 0) atomicAdd((unsigned long long *)&sh.bins[v / turn / per], (unsigned long long)mine);
        }
        if (!out) return;
        if (row.whole(v)) {
            if (a.kept_dtype == TAPOUT_F32) store_any<float, n>((float *)out + j0, y);
            else store_any<__bf16, n>((__bf16 *)out + j0, y);
        } else {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                if (j0 + e < 0 || j0 + e >= a.V) continue;
                if (a.kept_dtype == TAPOUT_F32) ((float *)out)[j0 + e] = y[e];
                else ((__bf16 *)out)[j0 + e] = (__bf16)y[e];
            }
        }
    });
    if (a.n_kept) {
        const uint64_t all = block_sum((uint64_t)kept, sh);
        if (threadIdx.x == 0) a.n_kept[r] = (int32_t)all;
    }
    if (!draw) return;
    if (bad) {
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.logq) a.logq[r] = __uint_as_float(0x7fc00000u);
        }
        return;
    }
    // the token: its chunk, its turn, its thread
    __syncthreads();
    uint64_t own = 0, Z;
#pragma unroll
    for (int q = 0; q < kBins / kThreads; ++q) own += sh.bins[threadIdx.x * (kBins / kThreads) + q];
    (void)block_before(own, Z, sh);
    const float u = a.u[r];
    const double point = (double)u * (double)Z;
    uint64_t target = point >= 0.0 ? (uint64_t)point + 1 : 1;         // the sum has to reach this: whole numbers above u Z
    if (!(u < 1.f) || target > Z) target = Z;
    uint64_t before = 0;
    const int chunk = find_bin(target, before, sh);
    if (threadIdx.x == 0) { sh.found = 0x7fffffff; sh.sum = 0; }
    __syncthreads();
    if (u == 0.f) {
        // the first kept element of any weight at all, units or not
        const double least = -745.13;
        int first = 0x7fffffff;
        each_vector<DT>(row, [&](int v, const float (&x)[n]) {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const uint32_t key = key_of(x[e]);
                if (key > kMasked && end.holds(key, row.first(v) + e) && ((double)x[e] - (double)m) * inv > least) first = min(first, row.first(v) + e);
            }
        });
        atomicMin(&sh.found, first);
    } else {
        for (int t = chunk * per; t < min((chunk + 1) * per, turns); ++t) {
            const int v = t * turn + threadIdx.x;
            float x[n];
            row.load(v, x);
            uint64_t mine = 0, all;
            uint64_t units[n];
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const uint32_t key = key_of(x[e]);
                units[e] = key > kMasked && end.holds(key, row.first(v) + e) ? w.of(x[e], sh.table) : 0;
                mine += units[e];
            }
            uint64_t sum = before + block_before(mine, all, sh);
            if (sum < target && sum + mine >= target) {
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    if (sum < target && sum + units[e] >= target) sh.found = row.first(v) + e;
                    sum += units[e];
                }
            }
            before += all;
            if (before >= target) break;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        const int j = sh.found;
        a.token[r] = j;
        const float x = load_elem<DT>(row.base, (int64_t)j + row.before);
        if (a.logq) a.logq[r] = (float)(((double)x - (double)m) * inv - log(ldexp((double)Z, -a.shift)));
    }
}

__global__ __launch_bounds__(256) void clear_flags_kernel(uint32_t *flags, int B)
{
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b < B) flags[b] = 0;
}

}  // namespace

hipError_t launch_filtered_sample(FilterArgs a, int dtype, hipStream_t st)
{
    int log2_v = 0;
    while ((1ll << log2_v) < a.V) ++log2_v;
    a.shift = 62 - log2_v < 50 ? 62 - log2_v : 50;
    if (a.flags && a.K > 1) {
        clear_flags_kernel<<<(a.B + 255) / 256, 256, 0, st>>>(a.flags, a.B);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const int64_t rows = (int64_t)a.B * a.K;
    if (dtype == TAPOUT_F32) filtered_sample_kernel<TAPOUT_F32><<<rows, kThreads, 0, st>>>(a);
    else filtered_sample_kernel<TAPOUT_BF16><<<rows, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace tapout
