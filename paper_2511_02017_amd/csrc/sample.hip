// Tokens drawn under a temperature and filters, and the filtered logits.
//
//   d_j = (x_j - max) / T,  w_j = e^(d_j);  order: larger x first, equal ones by index
//   top-k: the first k;  top-p: the shortest run from the start whose mass reaches p of the top-k's;  min-p: w_j >= min_p
//   token: smallest j whose sum of kept weights up to and with j exceeds u Z;  log q = d_token - ln Z
//
// All three filters keep a run from the start of the order, so what a row keeps is said by the value of its last element and the index up to
// which elements of that value are kept (Bound).  The row is not sorted.  Its elements are counted by the upper sixteen bits of their values: for
// bfloat16 rows these are the values, so counts times weights are the masses and the counts alone say where every run ends; for binary32 rows they
// name the place in which a run ends, whose few elements are ranked among each other (a place with many is divided again, down to one value).
//
// Weights are summed as whole numbers of 2^-S of the largest, S = 62 - log2 V (45 at V = 128256): sums of them do not depend on their order, so
// any division of the work gives the same bits, and each is off by half a unit, so that a sum is off by about 1e-12 of the largest weight, far
// less than the gaps between neighbouring sums that a decision could fall into.
#include <type_traits>

#include "exp_device.h"

namespace tapout {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave, kLoads = 4;
constexpr int kList = 1024, kBins = 2048;

// ---- values by their upper sixteen bits ----------------------------------------------------------------------
// Entry 2 e + sign: e = 0 magnitudes below 2^-16, e = 1 .. kRegular those up to 2^7, kRegular + 1 beyond.  Places are entries in falling order of
// their values; both signs of e = 0 share one.
constexpr uint32_t kLow = (127 - 16) << 7;
constexpr int kRegular = 23 * 128, kEntries = 2 * (kRegular + 2), kPlaces = kEntries, kTinyPlace = kRegular + 1;
constexpr int kPer = (kPlaces + kThreads - 1) / kThreads;                  // places of a thread
__device__ __forceinline__ int entry_at(int place) { return place <= kTinyPlace ? 2 * (kTinyPlace - place) : 2 * (place - kTinyPlace - 1) + 1; }
__device__ __forceinline__ int entry_of(float x)
{
    const uint32_t u = __float_as_uint(x), m = (u >> 16) & 0x7fffu;
    const int e = min(max((int)m - (int)(kLow - 1), 0), kRegular + 1);
    return 2 * e + (int)(u >> 31);
}
__device__ __forceinline__ int place_of(float x)
{
    const int entry = entry_of(x), e = entry >> 1;
    return (entry & 1) && e ? kTinyPlace + 1 + e : kTinyPlace - e;
}
// The value of a regular place (bfloat16), 0 for the place of the smallest.
__device__ __forceinline__ float value_at(int place)
{
    const int entry = entry_at(place), e = entry >> 1;
    return e ? __uint_as_float(((uint32_t)(entry & 1) << 31) | ((kLow - 1 + (uint32_t)e) << 16)) : 0.f;
}
// Two bfloat16 as they lie in a word to their entries, both at once: six instructions with the addresses.  Of values that are not regular the sign
// is lost: 0 or 1 for small ones, the last two for large ones.
__device__ __forceinline__ u16x2 entries_of(uint32_t w)
{
    const u16x2 v = __builtin_bit_cast(u16x2, w), sign = v >> (u16x2)(unsigned short)15;
    u16x2 d;
    asm("v_pk_mad_u16 %0, %1, 2, %2 op_sel_hi:[1,0,1]" : "=v"(d) : "v"(v), "v"(sign));
    d = __builtin_elementwise_sub_sat(d, (u16x2)(unsigned short)(2 * (kLow - 1)));
    return __builtin_elementwise_min(d, (u16x2)(unsigned short)(kEntries - 1));
}

__device__ __forceinline__ uint32_t key_of(float x)             // ordered like the values; -0 and 0 are one
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu)); }

// Keys of a place's values.  The place behind kTinyPlace, to which the smallest values' other sign would belong, has none: an empty range behind them.
struct Keys { uint32_t lo, hi; };
__device__ __forceinline__ Keys keys_of(int place)
{
    const int entry = entry_at(place), e = entry >> 1;
    const uint32_t least = (kLow - 1 + (uint32_t)e) << 16, most = e == 0 ? (kLow << 16) - 1 : e > kRegular ? 0x7f7fffffu : least | 0xffffu;
    if (place == kTinyPlace + 1) return Keys{~(most | 0x80000000u), ~(most | 0x80000000u) - 1};
    if (e == 0) return Keys{~(most | 0x80000000u), most | 0x80000000u};
    return entry & 1 ? Keys{~(most | 0x80000000u), ~(least | 0x80000000u)} : Keys{least | 0x80000000u, most | 0x80000000u};
}

// Last element of a run: larger values, and equal ones up to the index, are in it.
struct Bound {
    float x; int32_t index;
    __device__ __forceinline__ bool holds(float y, int32_t j) const { return y > x || (y == x && j <= index); }
};
__device__ __forceinline__ float below(float x)                                            // the next smaller value; of 0 a negative one
{
    const uint32_t k = key_of(x) - 1;
    return value_of(k == 0x7fffffffu ? k - 1 : k);              // that key is no value's: it would be -0
}
constexpr int kAll = 0x7fffffff, kNone = (int)0x80000000u;       // of a value's elements (indices before a row are negative)
__device__ __forceinline__ Bound shorter(Bound a, Bound b) { return a.x > b.x || (a.x == b.x && a.index < b.index) ? a : b; }

constexpr int kHalfPlaces = (kPlaces + 1) / 2;

struct Shared {
    double table[256];                         // 2^(k / 256)
    union {                                    // in turn
        uint32_t counts[kEntries];             // bfloat16: of every value
        uint64_t measures[kHalfPlaces];        // of two neighbouring places each
        uint64_t list[2 * kList];              // a place's elements, and their weights
        uint64_t bins[kBins];                  // of a range of keys
    };
    uint64_t waves[2][kWaves];
    uint32_t turn[2][kLoads * kWaves];
    float waves_f[kWaves];
    float tiny[64];                            // values that are not 0 in the place of the smallest
    uint32_t lo, hi;
    int32_t count, found, tinies, bad, irregular;
    uint64_t sum;
    Bound bound;
};

// A row's weights.
struct Weight {
    double max, c; int shift;                  // c = 256 / (T ln 2);  shift: log2 of the units of the largest weight, at most 50
    __device__ __forceinline__ uint64_t of(float x, const double *table) const
    {
        // (x - max) / T in units of ln2 / 256, down to where weights are no unit any more
        const double t = fmax(((double)x - max) * c, -256.0 * 64.0), tm = t + kMagic;
        const int ni = __double2loint(tm);
        const double r = t - (tm - kMagic), tk = table[ni & 255];
        const double q = r * fma(r, fma(r, fma(r, kExpC1 * kExpC1 * kExpC1 * kExpC1 / 24.0, kExpC3), kExpC2), kExpC1);
        const double e = fma(tk, q, tk);       // in [1, 2): scaled through the exponent field
        const double s = __hiloint2double(__double2hiint(e) + ((ni >> 8) + shift) * 0x100000, __double2loint(e)) + 4503599627370496.0;
        return ((uint64_t)(__double2hiint(s) & 0xfffff) << 32) | (uint32_t)__double2loint(s);          // to nearest: below 2^52
    }
};

// What all threads of a workgroup hold alike, in scalar registers: branches on it are the wavefront's own.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform(float v) { return __int_as_float(uniform(__float_as_int(v))); }
__device__ __forceinline__ double uniform(double v) { return __hiloint2double(uniform(__double2hiint(v)), uniform(__double2loint(v))); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) { return ((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)v); }
__device__ __forceinline__ Bound uniform(Bound b) { return Bound{uniform(b.x), uniform(b.index)}; }

// ---- a row's vectors -----------------------------------------------------------------------------------------
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
    // what lies outside the row is -infinity, and is not read
    __device__ __forceinline__ u32x4 load(int v) const
    {
        if (whole(v)) return *(const u32x4 *)(base + (int64_t)v * 16);
        u32x4 w = u32x4{1, 1, 1, 1} * (n == 4 ? 0xff800000u : 0xff80ff80u);
        if (v >= vecs) return w;
#pragma unroll 1
        for (int e = n - 1; e >= 0; --e) {                                              // from the last on, which is shifted to its place
            const int j = first(v) + e;
            const uint32_t u = __float_as_uint(j >= 0 && j < V ? load_elem<DT>(base, (int64_t)j + before) : -INFINITY);
            if constexpr (n == 4) w = u32x4{u, w[0], w[1], w[2]};
            else w = u32x4{__builtin_amdgcn_alignbit(w[0], u, 16), __builtin_amdgcn_alignbit(w[1], w[0], 16), __builtin_amdgcn_alignbit(w[2], w[1], 16),
                           __builtin_amdgcn_alignbit(w[3], w[2], 16)};
        }
        return w;
    }
};

// f(vector, words) for the row's vectors, a turn of kThreads at a time, LOADS turns' loads under way while as many are worked on: where f stores, a wait
// for loads that are younger than its stores would wait for these too.  Every thread takes part in every turn: behind the row it has values of
// -infinity.  A kernel runs through its code once, so code that is not there is what makes it short: the code of f is there LOADS + 1 times, and
// what is done for a few of a row's elements is a loop.
template <int DT, int LOADS, class F>
__device__ __forceinline__ void each_vector(const RowReader<DT> &row, F f, int begin = 0, int end = 0x7fffffff)       // of vectors [begin, end)
{
    constexpr int step = kThreads * LOADS;
    end = min(end, row.vecs);
    u32x4 w[LOADS], next[LOADS];
    auto load = [&](int base, u32x4 (&to)[LOADS]) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) to[u] = *(const u32x4 *)(row.base + (int64_t)(base + u * kThreads + threadIdx.x) * 16);
    };
    auto whole = [&](int base) { return (base > 0 || !row.before) && base + step <= end && base + step < row.vecs; };      // the row's first and last vector may be such in part
    if (whole(begin)) load(begin, w);
#pragma unroll 1
    for (int base = begin; base < end; base += step) {
        if (whole(base + step)) load(base + step, next);
        if (whole(base)) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) f(base + u * kThreads + (int)threadIdx.x, w[u]);
        } else {
            const u32x4 masked = u32x4{1, 1, 1, 1} * (RowReader<DT>::n == 4 ? 0xff800000u : 0xff80ff80u);
#pragma unroll 1
            for (int t = base; t < min(base + step, end); t += kThreads) {
                const int v = t + (int)threadIdx.x;
                f(v, v < end ? row.load(v) : masked);
            }
        }
#pragma unroll
        for (int u = 0; u < LOADS; ++u) w[u] = next[u];
    }
}
// f(value, index) for its elements.
template <int DT, int LOADS, class F>
__device__ __forceinline__ void each_element(const RowReader<DT> &row, F f)
{
    each_vector<DT, LOADS>(row, [&](int v, const u32x4 &w) {
        float x[RowReader<DT>::n];
        unpack<DT>(w, x);
#pragma unroll
        for (int e = 0; e < RowReader<DT>::n; ++e) f(x[e], row.first(v) + e);
    });
}
// f(value, index) for the elements of a vector whose bits are set, a lane's one after the other: as many turns as the lane with the most has.  The words
// are shifted to the element, so that no register is chosen by number.
template <int DT, class F> __device__ __forceinline__ void each_chosen(u32x4 w, uint32_t bits, int first, F f)
{
    const uint64_t front = ((uint64_t)w[1] << 32) | w[0], back = ((uint64_t)w[3] << 32) | w[2];
#pragma unroll 1
    while (bits) {
        const int e = __ffs((int)bits) - 1;
        bits &= bits - 1;
        constexpr int half = Elem<DT>::vec / 2, size = Elem<DT>::size * 8;
        const uint32_t u = (uint32_t)((e < half ? front : back) >> (e % half * size));
        f(__uint_as_float(size == 32 ? u : u << 16), first + e);
    }
}

// ---- sums over the workgroup -----------------------------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ uint64_t dpp_u(uint64_t v)         // lanes without a source: 0
{
    return ((uint64_t)(uint32_t)dpp_mov<CTRL>((int)(v >> 32)) << 32) | (uint32_t)dpp_mov<CTRL>((int)(uint32_t)v);
}
__device__ __forceinline__ uint64_t lane_u(uint64_t v, int lane)
{
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
// Sum over the lanes up to this one; *all: over the wavefront.
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, uint64_t *all)
{
    v += dpp_u<0x111>(v); v += dpp_u<0x112>(v); v += dpp_u<0x114>(v); v += dpp_u<0x118>(v);          // within sixteen lanes
    const uint64_t t0 = lane_u(v, 15), t1 = lane_u(v, 31), t2 = lane_u(v, 47), t3 = lane_u(v, 63);
    const int group = (threadIdx.x & 63) >> 4;
    v += group == 0 ? 0 : group == 1 ? t0 : group == 2 ? t0 + t1 : t0 + t1 + t2;
    *all = t0 + t1 + t2 + t3;
    return v;
}
// Sum over the threads before this one, and over all.  which: 0 and 1 in turn, so that one barrier is enough between two calls.
__device__ __forceinline__ uint64_t block_before(uint64_t v, uint64_t &all, Shared &sh, int which)
{
    uint64_t wave;
    uint64_t before = wave_scan(v, &wave) - v;
    if ((threadIdx.x & 63) == 0) sh.waves[which][threadIdx.x >> 6] = wave;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        const uint64_t q = sh.waves[which][k];
        if (k < (int)(threadIdx.x >> 6)) before += q;
        all += q;
    }
    return before;
}

// ---- the end of a run --------------------------------------------------------------------------------------------
// Index of the r-th element (from 1) that equals x among those of the vectors from `begin` on; r of them are there.
template <int DT>
__device__ __forceinline__ int nth_equal(const RowReader<DT> &row, float x, uint32_t r, Shared &sh, int begin = 0)
{
    constexpr int n = RowReader<DT>::n;
    static_assert(kLoads * kWaves == kWave, "a lane for each wavefront's part of a turn");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t seen = 0;
    int flip = 0;
    for (int base = begin; base < row.vecs; base += kThreads * kLoads, flip ^= 1) {
        uint32_t equal = 0;                                    // a byte for each of the turns
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int v = base + u * kThreads + (int)threadIdx.x;
            float y[n];
            unpack<DT>(row.load(v), y);
            uint32_t of_wave = 0;
#pragma unroll
            for (int e = 0; e < n; ++e) {
                equal |= (y[e] == x ? 1u : 0u) << (u * 8 + e);
                of_wave += (uint32_t)__popcll(__ballot(y[e] == x));
            }
            if (lane == 0) sh.turn[flip][u * kWaves + wave] = of_wave;
        }
        __syncthreads();
        uint64_t batch;
        const uint32_t part = sh.turn[flip][lane], before_part = (uint32_t)wave_scan(part, &batch) - part;
        if (seen + batch >= r) {
#pragma unroll 1
            for (int u = 0; u < kLoads; ++u) {
                uint64_t all;
                const uint32_t bits = equal >> (u * 8) & 0xffu, own = (uint32_t)__popc(bits);
                uint32_t at = seen + (uint32_t)__builtin_amdgcn_readlane((int)before_part, u * kWaves + wave) + (uint32_t)wave_scan(own, &all) - own;
                if (at < r && at + own >= r)
#pragma unroll 1
                    for (int e = 0; e < n; ++e)
                        if ((bits >> e & 1) && ++at == r) sh.found = row.first(base + u * kThreads + (int)threadIdx.x) + e;
            }
            break;
        }
        seen += (uint32_t)batch;
    }
    __syncthreads();
    const int j = uniform(sh.found);
    __syncthreads();
    return j;
}

// The sum of get(p) over this thread's places, and the first place with which the sum over all before it, from `above` on, reaches `target`: in sh.found,
// with the sum before it in sh.sum, behind the next barrier; untouched if none does.  `before`: the sum over the threads before.
template <class Get>
__device__ __forceinline__ uint64_t sum_places(int per, Get get)
{
    uint64_t own = 0;
#pragma unroll 1
    for (int k = 0; k < per; ++k) own += get(threadIdx.x * per + k);
    return own;
}
template <class Get>
__device__ __forceinline__ void mark_place(int per, uint64_t target, uint64_t before, uint64_t own, Get get, Shared &sh)
{
    if (before >= target || before + own < target) return;
#pragma unroll 1
    for (int k = 0; k < per; ++k) {                            // one thread
        const uint64_t v = get(threadIdx.x * per + k);
        if (before < target && before + v >= target) { sh.found = threadIdx.x * per + k; sh.sum = before; }
        before += v;
    }
}
// Both: the place, with the sum before it in `above`; -1 if none does.
template <class Get>
__device__ __forceinline__ int find_place(int per, uint64_t target, uint64_t &above, Get get, Shared &sh)
{
    __syncthreads();
    if (threadIdx.x == 0) sh.found = -1;
    uint64_t all;
    const uint64_t own = sum_places(per, get), before = above + block_before(own, all, sh, 0);
    mark_place(per, target, before, own, get, sh);
    __syncthreads();
    const int place = uniform(sh.found);
    if (place >= 0) above = uniform(sh.sum);
    __syncthreads();
    return place;
}

// What a run is measured in: elements, or units of weight.
struct Measure {
    bool weights; Weight w;
    __device__ __forceinline__ uint64_t of(float x, const double *table) const { return weights ? w.of(x, table) : 1; }
};

// What top-p asks for of a mass: at least a unit.
__device__ __forceinline__ uint64_t share_of(uint64_t all, float top_p)
{
    const double reached = (double)top_p * (double)all;
    return reached > 1.0 ? (uint64_t)ceil(reached) : 1;
}

// The end of the shortest run of `within` whose measure reaches `target`, which ends among the keys of `range`, before which the measure is `above`.
// top_p: `range` holds all of `within`, at most kList elements, and the target is this share of their weights.
template <int DT>
__device__ __forceinline__ Bound end_in(const RowReader<DT> &row, Bound within, uint64_t target, Keys range, uint64_t above, const Measure &m, Shared &sh,
                                        float top_p = -1.f)
{
    constexpr int n = RowReader<DT>::n;
    uint32_t lo = range.lo, hi = range.hi;
    for (;;) {
        __syncthreads();
        if (threadIdx.x == 0) { sh.count = 0; sh.lo = 0xffffffffu; sh.hi = 0; }
        __syncthreads();
        uint32_t least = 0xffffffffu, most = 0;
        each_vector<DT, 4>(row, [&](int v, const u32x4 &w) {
            float x[n];
            unpack<DT>(w, x);
            uint32_t in = 0;
#pragma unroll
            for (int e = 0; e < n; ++e) in |= (key_of(x[e]) - lo <= hi - lo ? 1u : 0u) << e;
            if (__any(in != 0))
                each_chosen<DT>(w, in, row.first(v), [&](float y, int j) {
                    if (!within.holds(y, j)) return;
                    const uint32_t k = key_of(y);
                    least = min(least, k);
                    most = max(most, k);
                    const int at = atomicAdd(&sh.count, 1);
                    if (at < kList) sh.list[at] = ((uint64_t)k << 32) | (0xffffffffu - (uint32_t)j);
                });
        });
        if (least <= most) { atomicMin(&sh.lo, least); atomicMax(&sh.hi, most); }
        __syncthreads();
        const int count = uniform(sh.count);
        lo = (uint32_t)uniform((int)sh.lo); hi = (uint32_t)uniform((int)sh.hi);
        if (count <= kList) {
#pragma unroll 1
            for (int i = threadIdx.x; i < count; i += kThreads) sh.list[kList + i] = m.of(value_of((uint32_t)(sh.list[i] >> 32)), sh.table);
            __syncthreads();
            if (top_p >= 0.f) {
                static_assert(kList <= kThreads, "an element a thread");
                uint64_t all;
                (void)block_before((int)threadIdx.x < count ? sh.list[kList + threadIdx.x] : 0, all, sh, 0);
                target = share_of(all, top_p);
            }
#pragma unroll 1
            for (int i = threadIdx.x; i < count; i += kThreads) {
                const uint64_t me = sh.list[i], own = sh.list[kList + i];
                uint64_t before = above;
#pragma unroll 4
                for (int o = 0; o < count; ++o) before += sh.list[o] > me ? sh.list[kList + o] : 0;
                if (before < target && before + own >= target) sh.bound = Bound{value_of((uint32_t)(me >> 32)), (int)(0xffffffffu - (uint32_t)me)};      // one thread
            }
            __syncthreads();
            const Bound r = uniform(sh.bound);
            __syncthreads();
            return r;
        }
        if (lo == hi) {
            const float x = value_of(lo);
            const uint64_t own = m.of(x, sh.table);                         // not 0: the target is reached here
            return shorter(Bound{x, nth_equal<DT>(row, x, (uint32_t)((target - above + own - 1) / own), sh)}, within);       // `within` may end among the same elements
        }
        // too many: a 2048th of their keys' range each
        const int shift = max(0, 32 - __clz((int)(hi - lo)) - 11);
        __syncthreads();
#pragma unroll 1
        for (int k = threadIdx.x; k < kBins; k += kThreads) sh.bins[k] = 0;
        __syncthreads();
        each_element<DT, 1>(row, [&](float x, int j) {
            const uint32_t k = key_of(x);
            if (k >= lo && k <= hi && within.holds(x, j)) atomicAdd((unsigned long long *)&sh.bins[(hi - k) >> shift], (unsigned long long)m.of(x, sh.table));
        });
        const int b = find_place(kBins / kThreads, target, above, [&](int k) { return sh.bins[k]; }, sh);
        const uint32_t top = hi - ((uint32_t)b << shift);
        lo = max(lo, top - min(top, (1u << shift) - 1));
        hi = top;
    }
}

// The smallest value whose weight is at least min_p, found a 64th of the interval of keys at a time.
__device__ __forceinline__ float least_value(float max, float T, float min_p)
{
    const int lane = threadIdx.x & 63;
    const double least = log((double)fminf(min_p, 1.f)), inv = 1.0 / (double)T;
    uint32_t lo = key_of(-INFINITY), hi = key_of(max);                                     // lo: not enough (or masked), hi: enough
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo + 63) / 64, at = lo + min((uint32_t)(lane + 1) * step, hi - lo);
        const int first = __ffsll((unsigned long long)__ballot(((double)value_of(at) - (double)max) * inv >= least)) - 1;       // the last lane's is hi
        hi = lo + min((uint32_t)(first + 1) * step, hi - lo);
        lo += (uint32_t)first * step;
    }
    return value_of(hi);
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

// What a row asks for.  Temperatures below the smallest normal number are taken as 0.
constexpr float kLeastT = 0x1p-126f;
struct Filters {
    float T, top_p, min_p; int top_k; bool greedy;
};

// Counts of the values of a bfloat16 row's vectors [begin, end).  sh.bad: a NaN or +infinity; sh.irregular: values beyond the table, or too many that
// are smaller than it.
__device__ __forceinline__ void count_values(const RowReader<TAPOUT_BF16> &row, Shared &sh, int begin = 0, int end = 0x7fffffff)
{
#pragma unroll 1
    for (int k = threadIdx.x; k < kEntries; k += kThreads) sh.counts[k] = 0;
    __syncthreads();
    each_vector<TAPOUT_BF16, 4>(row, [&](int, const u32x4 &w) {
        u16x2 d[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            d[q] = entries_of(w[q]);
            atomicAdd(&sh.counts[d[q][0]], 1u);
            atomicAdd(&sh.counts[d[q][1]], 1u);
        }
        const u16x2 top = __builtin_elementwise_max(__builtin_elementwise_max(d[0], d[1]), __builtin_elementwise_max(d[2], d[3]));
        const u16x2 low = __builtin_elementwise_min(__builtin_elementwise_min(d[0], d[1]), __builtin_elementwise_min(d[2], d[3]));
        if (max(top[0], top[1]) >= kEntries - 2 || min(low[0], low[1]) < 2) {
            // what there is beside masked elements and zeros, two at a time: magnitudes less the infinity's bits wrap round below it
            u16x2 large = {0, 0}, nan = {0xffff, 0xffff}, inf = nan, small = nan;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u16x2 m = __builtin_bit_cast(u16x2, w[q] & 0x7fff7fffu), over = m - (u16x2)(unsigned short)0x7f80;
                large = __builtin_elementwise_max(large, over);
                nan = __builtin_elementwise_min(nan, over - (u16x2)(unsigned short)1);
                inf = __builtin_elementwise_min(inf, __builtin_bit_cast(u16x2, w[q] ^ 0x7f807f80u));
                small = __builtin_elementwise_min(small, m - (u16x2)(unsigned short)1);
            }
            if (max(large[0], large[1]) >= (unsigned short)(kLow + kRegular - 0x7f80)) sh.irregular = 1;
            if (min(nan[0], nan[1]) < 0x7f || min(inf[0], inf[1]) == 0) sh.bad = 1;
            if (min(small[0], small[1]) < kLow - 1)
                each_chosen<TAPOUT_BF16>(w, 0xffu, 0, [&](float x, int) {
                    if (x == 0.f || !(fabsf(x) < 0x1p-16f)) return;
                    const int at = atomicAdd(&sh.tinies, 1);
                    if (at < 64) sh.tiny[at] = x;
                    else sh.irregular = 1;
                });
        }
    }, begin, end);
    __syncthreads();
    if (threadIdx.x == 0) { sh.counts[0] += sh.counts[1]; sh.counts[1] = 0; sh.counts[kEntries - 1] = 0; }         // one place; the last are masked
    __syncthreads();
}

}  // namespace

// Where rows are few each is counted in parts, by workgroups of their own, and a part's counts go through memory, in sixteen bits: a part has less than
// 2^16 elements.
struct CountSlice {
    uint16_t counts[kEntries];
    int32_t bad, irregular, tinies, pad;
    float tiny[64];
};
static_assert(sizeof(CountSlice) == kCountSliceBytes, "the context makes room for them");

namespace {

__device__ __host__ __forceinline__ int part_vecs(int vecs, int parts) { return ((vecs + parts - 1) / parts + 63) & ~63; }

__device__ __forceinline__ void load_counts(const CountSlice *parts, int n_parts, Shared &sh)
{
#pragma unroll 1
    for (int k = threadIdx.x; k < kEntries / 2; k += kThreads) {
        uint32_t lo = 0, hi = 0;
#pragma unroll 4
        for (int s = 0; s < n_parts; ++s) {
            const uint32_t both = ((const uint32_t *)parts[s].counts)[k];
            lo += both & 0xffffu;
            hi += both >> 16;
        }
        sh.counts[2 * k] = lo;
        sh.counts[2 * k + 1] = hi;
    }
    if (threadIdx.x < 64) {
        int to = 0, bad = 0, irregular = 0;
#pragma unroll 1
        for (int s = 0; s < n_parts; ++s) {
            const int n = uniform(parts[s].tinies);
            if ((int)threadIdx.x < n && to + (int)threadIdx.x < 64) sh.tiny[to + threadIdx.x] = parts[s].tiny[threadIdx.x];
            to += n;
            bad |= parts[s].bad;
            irregular |= parts[s].irregular;
        }
        if (threadIdx.x == 0) { sh.tinies = to; sh.bad = bad; sh.irregular = irregular | (to > 64 ? 1 : 0); }
    }
    __syncthreads();
}

// A bfloat16 row from its counts: its maximum, where its run ends and how many that keeps.  false: it was not decided here (not regular, without a
// finite value (sh.bad), or a run ends among the small values).
__device__ __forceinline__ bool by_counts(const RowReader<TAPOUT_BF16> &row, const Filters &f, int shift, const CountSlice *parts, int n_parts, float &peak,
                                          Weight &w, Bound &end, int &kept, Shared &sh)
{
    if (n_parts) load_counts(parts, n_parts, sh);
    else count_values(row, sh);
    if (uniform(sh.bad | sh.irregular)) return false;
    const int tinies = uniform(sh.tinies);
    const int p0 = threadIdx.x * kPer;
    uint32_t c[kPer];
    uint64_t all, own = 0, before, units[kPer];
    int first = kPlaces;
#pragma unroll
    for (int k = kPer - 1; k >= 0; --k) {
        c[k] = p0 + k < kPlaces ? sh.counts[entry_at(p0 + k)] : 0;
        own += c[k];
        if (c[k]) first = p0 + k;
    }
    // the first place with an element, and the place of the k-th
    if (threadIdx.x == 0) { sh.found = kPlaces; sh.count = 0; sh.lo = kPlaces; }
    before = block_before(own, all, sh, 0);
    if (uniform((int)(all >> 32) | (int)all) == 0) {
        if (threadIdx.x == 0) sh.bad = 1;
        __syncthreads();
        return false;
    }
    kept = uniform((int)all);
    const uint64_t counted = before, top_k = f.greedy ? 1 : f.top_k > 0 ? f.top_k : 1ull << 40;
    if (own && before == 0) sh.hi = first;                                                 // one thread
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        if (before < top_k && before + c[k] >= top_k) { sh.found = p0 + k; sh.count = (int)(top_k - before); }
        before += c[k];
    }
    __syncthreads();
    int place = uniform(sh.found), n = uniform(sh.count);      // the run: all places before `place`, n elements of it
    first = uniform((int)sh.hi);
    if (first == kTinyPlace && tinies) return false;
    if (place == kTinyPlace && tinies && !f.greedy && f.top_p < 1.f) return false;         // top-p's share is that of the largest of them, which the place does not tell
    peak = value_at(first);
    w = Weight{(double)peak, f.greedy ? 0.0 : 256.0 / ((double)f.T * kLn2), shift};
    // weights by value, masses of what top-k leaves, the first place whose elements are too light; small values one by one
    const double least = !f.greedy && f.min_p > 0.f ? log((double)fminf(f.min_p, 1.f)) * (double)f.T : -INFINITY;          // of x - peak
    bool light = false;
    uint64_t mass[kPer];
    own = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int p = p0 + k;
        mass[k] = units[k] = 0;
        if (!c[k]) continue;
        const float x = value_at(p);
        units[k] = w.of(x, sh.table);
        mass[k] = (uint64_t)(p < place ? c[k] : p == place ? (uint32_t)n : 0u) * units[k];
        if (!light && (double)x - (double)peak < least) {
            atomicMin(&sh.lo, (uint32_t)p);
            light = true;
        }
        if (p == kTinyPlace && tinies) {
            if ((-0x1p-16 - (double)peak < least) != (0x1p-16 - (double)peak < least)) sh.irregular = 1;         // the border among the small values
            if (p < place) {
                mass[k] -= tinies * units[k];
#pragma unroll 1
                for (int q = 0; q < tinies; ++q) mass[k] += w.of(sh.tiny[q], sh.table);
            }
        }
        own += mass[k];
    }
    if (!f.greedy && f.top_p < 1.f) {
        before = block_before(own, all, sh, 1);
        const uint64_t target = share_of(all, f.top_p);
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            if (before < target && before + mass[k] >= target) {                           // one thread
                const uint64_t one = units[k] ? units[k] : 1, need = (target - before + one - 1) / one;
                const uint32_t most = p0 + k == place ? (uint32_t)n : c[k];
                sh.found = p0 + k;
                sh.count = need < most ? (int)need : (int)most;
            }
            before += mass[k];
        }
        __syncthreads();
        place = uniform(sh.found);
        n = uniform(sh.count);
    } else {
        __syncthreads();
    }
    if (uniform(sh.irregular)) return false;
    if (const int lo = uniform((int)sh.lo); place >= lo) { place = lo; n = 0; }
    if (place == kTinyPlace && n && tinies) return false;
    if (place == kPlaces) {
        end = Bound{-INFINITY, kNone};
        return true;
    }
    // how many that keeps
    if (place >= p0 && place < p0 + kPer) {                                                // one thread
        uint64_t ahead = counted;
#pragma unroll
        for (int k = 0; k < kPer; ++k) ahead += p0 + k < place ? c[k] : 0;
        sh.sum = ahead;
    }
    __syncthreads();
    kept = uniform((int)sh.sum) + n;
    const uint32_t here = (uint32_t)uniform((int)sh.counts[entry_at(place)]);
    if (n == 0) end = Bound{place == kTinyPlace ? __uint_as_float((kLow - 1) << 16) : value_at(place), kNone};
    else if ((uint32_t)n >= here) end = Bound{value_at(place), kAll};
    else {
        // among its equals: with the parts' counts the part that the last one lies in
        int begin = 0;
        uint32_t r = (uint32_t)n;
        for (int s = 0; s < n_parts; ++s) {
            const uint32_t of_part = parts[s].counts[entry_at(place)];
            if (of_part >= r) break;
            r -= of_part;
            begin += part_vecs(row.vecs, n_parts);
        }
        end = Bound{value_at(place), nth_equal<TAPOUT_BF16>(row, value_at(place), (uint32_t)uniform((int)r), sh, uniform(begin))};
    }
    return true;
}

// Any row.  A bfloat16 row with a finite value of 128 or more, of either sign, comes here behind its counting, so that rows masked by finite values take
// longer than rows masked by -infinity: 64 rows of 128256 under mixed filters, with their tokens, 119 us for 45, 576 target rows under top-p 333 for 134,
// whether the masked logits are -1e4, -1e9 or the type's lowest value.
template <int DT>
__device__ __forceinline__ void by_places(const RowReader<DT> &row, const Filters &f, int shift, float &peak, Weight &w, Bound &end, Shared &sh)
{
    const bool by_rank = !f.greedy && f.top_k > 0 && f.top_k < row.V;
    __syncthreads();
    if (threadIdx.x == 0) sh.bad = 0;
    if (by_rank) {
#pragma unroll 1
        for (int k = threadIdx.x; k < kPlaces; k += kThreads) sh.counts[k] = 0;
    }
    __syncthreads();
    float m = -INFINITY;
    bool nan = false;
    each_element<DT, DT == TAPOUT_F32 ? 4 : 2>(row, [&](float x, int) {
        m = fmaxf(m, x);
        nan |= x != x;
        if (by_rank && x > -INFINITY) atomicAdd(&sh.counts[place_of(x)], 1u);
    });
    m = lanes_max(m, 0, 6);
    if ((threadIdx.x & 63) == 0) sh.waves_f[threadIdx.x >> 6] = m;
    __syncthreads();
    if (nan) sh.bad = 1;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) m = fmaxf(m, sh.waves_f[k]);
    __syncthreads();
    peak = m;
    end = Bound{-INFINITY, kNone};
    m = uniform(m);
    const bool bad = uniform(sh.bad) || !(fabsf(m) < INFINITY);
    __syncthreads();
    if (bad) {
        if (threadIdx.x == 0) sh.bad = 1;
        __syncthreads();
        return;
    }
    w = Weight{(double)m, f.greedy ? 0.0 : 256.0 / ((double)f.T * kLn2), shift};
    if (f.greedy) {
        end = Bound{m, nth_equal<DT>(row, m, 1, sh)};
        return;
    }
    const bool by_mass = f.top_p < 1.f;
    bool few = false;                                          // the run's elements fit the list
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {                     // top-k, then top-p of what that leaves
        if (!(turn ? by_mass : by_rank)) continue;
        const Measure measure{turn == 1, w};
        const Bound within = end;
        uint64_t target = f.top_k, above = 0;
        Keys range{key_of(within.x), 0xff7fffffu};
        if (turn == 0) {
            const int place = find_place(kPer, target, above, [&](int p) { return p < kPlaces ? (uint64_t)sh.counts[p] : 0; }, sh);
            if (place < 0) continue;
            range = keys_of(place);
            few = f.top_k <= kList;
        } else if (!few) {
            __syncthreads();
#pragma unroll 1
            for (int k = threadIdx.x; k < kHalfPlaces; k += kThreads) sh.measures[k] = 0;
            __syncthreads();
            each_element<DT, 1>(row, [&](float x, int j) {
                if (within.holds(x, j)) atomicAdd((unsigned long long *)&sh.measures[place_of(x) >> 1], (unsigned long long)w.of(x, sh.table));
            });
            __syncthreads();
            constexpr int per = (kHalfPlaces + kThreads - 1) / kThreads;
            auto at = [&](int p) { return p < kHalfPlaces ? sh.measures[p] : 0; };
            uint64_t all;
            (void)block_before(sum_places(per, at), all, sh, 1);
            target = share_of(all, f.top_p);
            const int place = find_place(per, target, above, at, sh);
            if (place < 0) continue;
            range = Keys{keys_of(2 * place + 1).lo, keys_of(2 * place).hi};
        }
        end = end_in<DT>(row, within, target, Keys{(uint32_t)uniform((int)range.lo), (uint32_t)uniform((int)range.hi)}, above, measure, sh,
                         turn && few ? fmaxf(f.top_p, 0.f) : -1.f);
    }
    if (f.min_p > 0.f) end = shorter(end, Bound{least_value(m, f.T, f.min_p), kAll});
}

// ---- kernels -----------------------------------------------------------------------------------------------------
}  // namespace

// What every row keeps.  Elements are kept that are larger than one of two values: up to the index `last` than `from`, behind it than `above`, which
// differ where equal elements are kept in part.
struct FilterRow {
    float max, above, from;
    int32_t last, kept;                        // kept: -1 where it was not counted
    int32_t bad;
    double inv, c;                             // 1 / T, 0 of a greedy row;  see Weight
    // In binary64 and rounded once: in binary32 the difference, the inverse and the product are a rounding each, and a difference beyond it is infinite
    // whatever T is.
    __device__ __forceinline__ float logit(float x) const { return (float)(((double)x - (double)max) * inv); }
};
static_assert(sizeof(FilterRow) == kFilterRowBytes, "the context makes room for it");

namespace {

// A part of a bfloat16 row's values, counted.  Bound by the LDS, which adds one element a lane at a time.
__global__ __launch_bounds__(kThreads, 8) void filter_counts_kernel(FilterArgs a, int parts)
{
    __shared__ Shared sh;
    const int r = blockIdx.x / parts, s = blockIdx.x - r * parts, b = r / a.K, k = r - b * a.K;
    if (a.k_len && k >= a.k_len[b]) return;
    const RowReader<TAPOUT_BF16> row(row_address(a.base, TAPOUT_BF16, a.stride_b, a.stride_k, b, k), a.V);
    if (threadIdx.x == 0) { sh.bad = 0; sh.irregular = 0; sh.tinies = 0; }
    const int per = part_vecs(row.vecs, parts);
    count_values(row, sh, s * per, (s + 1) * per);
    CountSlice &to = a.counts[blockIdx.x];
#pragma unroll 1
    for (int q = threadIdx.x; q < kEntries / 2; q += kThreads) ((uint32_t *)to.counts)[q] = sh.counts[2 * q] | sh.counts[2 * q + 1] << 16;
    if (threadIdx.x < 64) to.tiny[threadIdx.x] = sh.tiny[threadIdx.x];
    if (threadIdx.x == 0) { to.bad = sh.bad; to.irregular = sh.irregular; to.tinies = min(sh.tinies, 64); }
}

// What every row keeps: a workgroup a row.  Bound by latency where rows are few (a pass over a row by one unit, and the barriers between what follows it:
// one row of 32000 binary32 15.0 us, two passes; 120 rows of 50257 47.5 us, up to three passes and a double exponential for each element where top-p
// alone is asked for), and where they are many by what one workgroup of 128 registers a unit has under way (576 rows of 128256 bfloat16 86 us,
// 1.7 TB/s: 2.25 rows a unit, paid as three, LDS 21 % busy; held to 64 registers, two workgroups a unit: 85.5, with spills).
template <int DT>
__global__ __launch_bounds__(kThreads) void filter_rows_kernel(FilterArgs a, int parts)
{
    __shared__ Shared sh;
    const int r = blockIdx.x, b = r / a.K, k = r - b * a.K;
    if (a.k_len && k >= a.k_len[b]) return;
    const RowReader<DT> row(row_address(a.base, DT, a.stride_b, a.stride_k, b, k), a.V);
    Filters f{a.temperature ? a.temperature[b] : 1.f, a.top_p ? a.top_p[b] : 1.f, a.min_p ? a.min_p[b] : 0.f, a.top_k ? a.top_k[b] : 0, false};
    f.greedy = !(f.T >= kLeastT);
    if (threadIdx.x < 256) sh.table[threadIdx.x] = a.exp_table[threadIdx.x];
    if (threadIdx.x == 0) { sh.bad = f.T != f.T; sh.irregular = 0; sh.tinies = 0; sh.found = 0; }
    __syncthreads();
    float max = 0.f;
    Weight w{0.0, 0.0, a.shift};
    Bound end{INFINITY, kNone};
    int kept = -1;
    if (f.T == f.T) {
        bool done = false;
        if constexpr (DT == TAPOUT_BF16) done = by_counts(row, f, a.shift, a.counts + (int64_t)r * parts, parts, max, w, end, kept, sh);
        if (!done && !uniform(sh.bad)) {
            kept = -1;
            by_places<DT>(row, f, a.shift, max, w, end, sh);
        }
    }
    __syncthreads();
    if (threadIdx.x) return;
    const bool bad = sh.bad;
    FilterRow q{max, end.x, end.x, kNone, kept, bad, f.greedy ? 0.0 : 1.0 / (double)f.T, w.c};
    if (bad) q = FilterRow{0.f, INFINITY, INFINITY, kNone, 0, 1, 0.0, 0.0};
    else if (end.index == kAll) q.above = q.from = below(end.x);
    else if (end.index != kNone) { q.from = below(end.x); q.last = end.index; }
    a.rows[r] = q;
}

// The vectors of a slice, and which of their elements are kept.
constexpr int kSliceThreads = 256, kSliceTurns = 2, kSliceVecs = kSliceThreads * kSliceTurns;
template <int N> __device__ __forceinline__ void kept_of(const FilterRow &q, const float (&x)[N], int j0, bool (&in)[N])
{
    const float than = j0 + N - 1 <= q.last ? q.from : q.above;
#pragma unroll
    for (int e = 0; e < N; ++e) in[e] = x[e] > than;
    if (j0 <= q.last && q.last < j0 + N - 1) {                 // one vector of the row
#pragma unroll
        for (int e = 0; e < N; ++e) in[e] = x[e] > (j0 + e <= q.last ? q.from : q.above);
    }
}
__device__ __forceinline__ FilterRow row_record(const FilterArgs &a, int r)
{
    FilterRow q = a.rows[r];
    q.max = uniform(q.max); q.inv = uniform(q.inv); q.above = uniform(q.above); q.from = uniform(q.from);
    q.last = uniform(q.last); q.kept = uniform(q.kept); q.bad = uniform(q.bad); q.c = uniform(q.c);
    return q;
}
// Units of a vector's kept elements: all of its elements in turn where most lanes keep some, else those that are kept (64 rows of 128256 with different
// filters, slices and tokens, us always all / always those kept / by more than 40 lanes: 14.0 + 9.4 / 14.4 + 10.8 / 13.3 + 9.3).
template <int DT> __device__ __forceinline__ uint64_t kept_units(const Weight &w, const u32x4 &words, uint32_t keeps, int j0, const double *table)
{
    uint64_t sum = 0;
    const int lanes = __popcll(__ballot(keeps != 0));
    if (lanes > 40) {
        float x[Elem<DT>::vec];
        unpack<DT>(words, x);
#pragma unroll
        for (int e = 0; e < Elem<DT>::vec; ++e) {
            const uint64_t one = w.of(x[e], table);
            sum += keeps >> e & 1 ? one : 0;
        }
    } else if (lanes) {
        each_chosen<DT>(words, keeps, j0, [&](float x, int) { sum += w.of(x, table); });
    }
    return sum;
}

// The filtered logits, and a slice's kept elements and weights: a workgroup a slice, all of its loads requested first.  Where rows are many bound by
// memory and by the vector unit, which binary64 keeps 79 % busy: 576 rows of 128256 bfloat16, read and written, 49 us, 6.0 TB/s (46 with kept logits in
// binary32, three roundings each).  Measured with those, slices of 256 vectors a turn, us with 1 / 2 / 4 / 8 turns: 66.9 / 46.1 / 49.0 / 50.0, 64 such
// rows with tokens (both kernels) 20.7 / 19.7 / 22.6 / 29.5, one row of 32000 binary32 9.2 / 9.7 / 12.0 / 15.5.
template <int DT>
__global__ __launch_bounds__(kSliceThreads) void filter_slices_kernel(FilterArgs a, int slices)
{
    constexpr int n = RowReader<DT>::n;
    __shared__ double table[256];
    __shared__ uint64_t sums[kSliceThreads / kWave];
    __shared__ int counts[kSliceThreads / kWave];
    const int r = blockIdx.x / slices, s = blockIdx.x - r * slices, b = r / a.K, k = r - b * a.K;
    if (a.k_len && k >= a.k_len[b]) return;
    const RowReader<DT> row(row_address(a.base, DT, a.stride_b, a.stride_k, b, k), a.V);
    const int v0 = s * kSliceVecs;
    if (v0 >= row.vecs) {                                      // a row without a part of a vector before it may have no vector here
        if (threadIdx.x == 0) a.slices[blockIdx.x] = FilterSlice{0, 0, 0};
        return;
    }
    const bool draw = a.u != nullptr;
    if (draw) table[threadIdx.x] = a.exp_table[threadIdx.x];
    u32x4 words[kSliceTurns];
    if ((v0 > 0 || row.before == 0) && v0 + kSliceVecs < row.vecs) {
#pragma unroll
        for (int t = 0; t < kSliceTurns; ++t) words[t] = *(const u32x4 *)(row.base + (int64_t)(v0 + t * kSliceThreads + threadIdx.x) * 16);
    } else {
#pragma unroll
        for (int t = 0; t < kSliceTurns; ++t) words[t] = row.load(v0 + t * kSliceThreads + (int)threadIdx.x);
    }
    const FilterRow q = row_record(a, r);
    const Weight w{(double)q.max, q.c, a.shift};
    char *out = a.kept ? (char *)row_address(a.kept, a.kept_dtype, a.kept_stride_b, a.kept_stride_k, b, k) : nullptr;
    uint64_t mine = 0;
    int count = 0;
    if (draw) __syncthreads();
#pragma unroll
    for (int t = 0; t < kSliceTurns; ++t) {
        const int v = v0 + t * kSliceThreads + (int)threadIdx.x, j0 = row.first(v);
        float x[n], y[n];
        bool in[n];
        unpack<DT>(words[t], x);
        kept_of(q, x, j0, in);
        uint32_t keeps = 0;
#pragma unroll
        for (int e = 0; e < n; ++e) keeps |= (in[e] ? 1u : 0u) << e;
        count += __popc(keeps);
        if (draw) mine += kept_units<DT>(w, words[t], keeps, j0, table);
        if (!out) continue;
#pragma unroll
        for (int e = 0; e < n; ++e) y[e] = in[e] ? q.logit(x[e]) : -INFINITY;
        if (!row.whole(v)) continue;
        if (a.kept_dtype == TAPOUT_F32) store_any<float, n>((float *)out + j0, y);
        else store_any<__bf16, n>((__bf16 *)out + j0, y);
    }
    if (out)
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {                          // the row's first and last vector, where they are vectors in part
            const int v = e ? row.vecs - 1 : 0;
            if (row.whole(v) || (v - v0) % kSliceThreads != (int)threadIdx.x || v < v0 || v >= v0 + kSliceVecs || (e && v == 0)) continue;
            each_chosen<DT>(row.load(v), (1u << n) - 1, row.first(v), [&](float x, int j) {
                if (j < 0 || j >= a.V) return;
                const float z = x > (j <= q.last ? q.from : q.above) ? q.logit(x) : -INFINITY;
                if (a.kept_dtype == TAPOUT_F32) ((float *)out)[j] = z;
                else ((__bf16 *)out)[j] = (__bf16)z;
            });
        }
    uint64_t all;
    (void)wave_scan(mine, &all);
    for (int d = 32; d; d >>= 1) count += __shfl_xor(count, d);
    if ((threadIdx.x & 63) == 0) { sums[threadIdx.x >> 6] = all; counts[threadIdx.x >> 6] = count; }
    __syncthreads();
    if (threadIdx.x == 0) a.slices[blockIdx.x] = FilterSlice{sums[0] + sums[1] + sums[2] + sums[3], counts[0] + counts[1] + counts[2] + counts[3], 0};
}

// How many a row keeps, the flags of its sequence, and its token: the slice that holds it, then the vector, then the element.  A workgroup a row;
// bound by latency, three dependent reads (5 to 8 us).
template <int DT>
__global__ __launch_bounds__(kSliceThreads) void filter_tokens_kernel(FilterArgs a, int slices)
{
    constexpr int n = RowReader<DT>::n, kW = kSliceThreads / kWave;
    __shared__ double table[256];
    __shared__ uint64_t sums[kW], parts[kSliceTurns * kW];
    __shared__ int counts[kW], slice, found;
    __shared__ uint64_t ahead;
    const int r = blockIdx.x, b = r / a.K, k = r - b * a.K, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int live = a.k_len ? min(a.k_len[b], a.K) : a.K;
    if (a.flags && k == 0 && threadIdx.x < kWave) {
        bool bad = false;
        for (int o = lane; o < live; o += kWave) bad |= a.rows[r + o].bad != 0;
        const bool any = __any(bad);
        if (lane == 0) a.flags[b] = any ? TAPOUT_FLAG_BAD_ROW : 0u;
    }
    if (k >= live) return;
    const FilterRow q = row_record(a, r);
    const FilterSlice *p = a.slices + (int64_t)r * slices;
    table[threadIdx.x] = a.exp_table[threadIdx.x];
    const float u = a.u ? a.u[r] : 0.f;
    // every thread a run of slices
    const int per = (slices + kSliceThreads - 1) / kSliceThreads, s0 = threadIdx.x * per, s1 = min(s0 + per, slices);
    uint64_t own = 0, all;
    int count = 0;
    for (int s = s0; s < s1; ++s) { own += p[s].units; count += p[s].kept; }
    uint64_t before = wave_scan(own, &all) - own;
    for (int d = 32; d; d >>= 1) count += __shfl_xor(count, d);
    if (lane == 0) { sums[wave] = all; counts[wave] = count; }
    if (threadIdx.x == 0) { slice = 0; ahead = 0; found = 0x7fffffff; }
    __syncthreads();
    if (a.n_kept && threadIdx.x == 0) a.n_kept[r] = counts[0] + counts[1] + counts[2] + counts[3];
    if (!a.u) return;
    if (q.bad) {
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.logq) a.logq[r] = __uint_as_float(0x7fc00000u);
        }
        return;
    }
    uint64_t Z = 0;
#pragma unroll
    for (int g = 0; g < kW; ++g) { if (g < wave) before += sums[g]; Z += sums[g]; }
    const double point = (double)u * (double)Z;
    uint64_t target = point >= 0.0 ? (uint64_t)point + 1 : 1;                          // whole numbers above u Z reach this
    if (!(u < 1.f) || target > Z) target = Z;
    if (before < target && before + own >= target)                                     // one thread
        for (int s = s0; s < s1; ++s) {
            if (before < target && before + p[s].units >= target) { slice = s; ahead = before; }
            before += p[s].units;
        }
    __syncthreads();
    const RowReader<DT> row(row_address(a.base, DT, a.stride_b, a.stride_k, b, k), a.V);
    const Weight w{(double)q.max, q.c, a.shift};
    if (u == 0.f) {
        // the first kept element that has a weight at all, in units or not
        int first = 0x7fffffff;
#pragma unroll 1
        for (int v = threadIdx.x; v < row.vecs; v += kSliceThreads) {
            const u32x4 words = row.load(v);
            float x[n];
            unpack<DT>(words, x);
#pragma unroll
            for (int e = n - 1; e >= 0; --e) {
                const int j = row.first(v) + e;
                if (x[e] > (j <= q.last ? q.from : q.above) && ((double)x[e] - (double)q.max) * q.inv > -745.13) first = min(first, j);
            }
            if (first < 0x7fffffff) break;
        }
        atomicMin(&found, first);
    } else {
        const int v0 = uniform(slice) * kSliceVecs;
        u32x4 words[kSliceTurns];
        auto keeps_of = [&](const u32x4 &w4, int v) {
            float x[n];
            bool in[n];
            unpack<DT>(w4, x);
            kept_of(q, x, row.first(v), in);
            uint32_t keeps = 0;
#pragma unroll
            for (int e = 0; e < n; ++e) keeps |= (in[e] ? 1u : 0u) << e;
            return keeps;
        };
#pragma unroll
        for (int t = 0; t < kSliceTurns; ++t) words[t] = row.load(v0 + t * kSliceThreads + (int)threadIdx.x);
#pragma unroll
        for (int t = 0; t < kSliceTurns; ++t) {
            uint64_t of_wave;
            const int v = v0 + t * kSliceThreads + (int)threadIdx.x;
            (void)wave_scan(kept_units<DT>(w, words[t], keeps_of(words[t], v), row.first(v), table), &of_wave);
            if (lane == 0) parts[t * kW + wave] = of_wave;
        }
        __syncthreads();
        // the part that holds it, once more: every wavefront does, and the one whose part it is finds it
        static_assert(kSliceTurns * kW <= kWave, "a lane a part");
        uint64_t of_slice;
        const uint64_t part = lane < kSliceTurns * kW ? parts[lane] : 0, upto = ahead + wave_scan(part, &of_slice);
        const int hit = __ffsll((unsigned long long)__ballot(upto >= target && upto - part < target)) - 1;
        if (hit >= 0 && hit % kW == wave) {
            const int v = v0 + hit / kW * kSliceThreads + (int)threadIdx.x;
            const u32x4 w4 = row.load(v);
            uint64_t of_wave;
            const uint32_t keeps = keeps_of(w4, v);
            const uint64_t own = kept_units<DT>(w, w4, keeps, row.first(v), table);
            uint64_t at = lane_u(upto - part, hit) + wave_scan(own, &of_wave) - own;
            if (at < target && at + own >= target)             // one lane
                each_chosen<DT>(w4, keeps, row.first(v), [&](float y, int j) {
                    const uint64_t one = w.of(y, table);
                    if (at < target && at + one >= target) found = j;
                    at += one;
                });
        }
    }
    __syncthreads();
    if (threadIdx.x) return;
    const int j = min(found, a.V - 1);
    a.token[r] = j;
    if (a.logq) {
        const float x = load_elem<DT>(row.base, (int64_t)j + row.before), T = a.temperature ? a.temperature[b] : 1.f;
        a.logq[r] = (float)((T >= kLeastT ? ((double)x - (double)q.max) / (double)T : 0.0) - log(ldexp((double)Z, -a.shift)));
    }
}

}  // namespace

hipError_t launch_filtered_sample(FilterArgs a, int dtype, hipStream_t st)
{
    int log2_v = 0;
    while ((1ll << log2_v) < a.V) ++log2_v;
    a.shift = 62 - log2_v < 50 ? 62 - log2_v : 50;
    const int64_t rows = (int64_t)a.B * a.K;
    const int slices = filter_slices(a.V, dtype);
    const auto launch = [&](auto elem) {
        constexpr int DT = decltype(elem)::value;
        const int parts = DT == TAPOUT_BF16 ? count_parts(rows, a.V) : 0;
        if constexpr (DT == TAPOUT_BF16)
            if (parts) filter_counts_kernel<<<rows * parts, kThreads, 0, st>>>(a, parts);
        filter_rows_kernel<DT><<<rows, kThreads, 0, st>>>(a, parts);
        filter_slices_kernel<DT><<<rows * slices, kSliceThreads, 0, st>>>(a, slices);
        if (a.u || a.n_kept || a.flags) filter_tokens_kernel<DT><<<rows, kSliceThreads, 0, st>>>(a, slices);
    };
    if (dtype == TAPOUT_F32) launch(std::integral_constant<int, TAPOUT_F32>{});
    else launch(std::integral_constant<int, TAPOUT_BF16>{});
    return hipGetLastError();
}

// Parts that a bfloat16 row's counting is divided into, 0: not.  Few rows leave most compute units idle: 64 rows of 128256 take 9.2 us for the counts of 4
// parts each and 17.1 for the rest, 31.4 in one kernel.  Above a row to a compute unit what a second kernel reads again costs more: 576 rows take 39.9
// and 52.8 us with 3 parts, 85.5 without.
int count_parts(int64_t rows, int V)
{
    if (rows > kCountRows) return 0;
    int parts = rows > 128 ? 2 : rows > 32 ? 4 : 8;
    const int most = V / 8192;
    parts = parts < most ? parts : most;
    const int vecs = V / 8 + 2;
    while (parts > 0 && parts <= kCountParts && (int64_t)part_vecs(vecs, parts) * 8 >= 65536) ++parts;
    return parts < 2 || parts > kCountParts ? 0 : parts;
}

// Slices of a row: it may begin anywhere in its first vector.
int filter_slices(int V, int dtype)
{
    const int n = dtype == TAPOUT_F32 ? 4 : 8;
    return (V + n - 1 + kSliceVecs * n - 1) / (kSliceVecs * n);
}

}  // namespace tapout
