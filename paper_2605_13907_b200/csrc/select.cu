// Selection along rows of logits: the K largest entries of a row in order (a teacher's top logits), and one token drawn from a
// row under temperature, top-k, top-p and min-p.
//
// Order of a row: value descending, index ascending.  Every filter keeps a prefix of that order, so a filter is a cut: the last
// entry that is kept, as a 64-bit number (order key of the value above, index below) whose natural order is the row's order.
//  top-k : the k-th number.                       top-p : the first number at which the mass reaches p times the total.
//  min-p : e >= m, a threshold on the value.       The token: the first index at which the kept mass exceeds u times its total.
// with e = exp((x - max) / T).  Nothing is sorted but the few entries around a cut.
//
// A row belongs to a cluster of CTAs (one to eight); each keeps its slice of the row in shared memory, so that HBM is read once.
//  1. slice to shared memory, maximum;   2. histogram of the distance below the maximum (2,048 bins of 1/64 of a unit of
//  log-probability; a bin is a range of the order), and the fp32 sum of exponentials;   3. the bin of the cut: by counts for
//  top-k; for top-p the counts give bounds on the mass above every bin, and only the bins between the bounds get their masses
//  added up;   4. the entries of that bin go to one CTA, which sorts them and finds the cut; a bin of more than 2,048 entries (many
//  equal values, a degenerate temperature) is first divided by the number itself, 2,048 ways at a time.
// A top-k of at most 1,024 takes all entries down to its bin into that list, and the rest happens there.
//
// Precision: which token is drawn and how many are kept are decided by comparing sums over the vocabulary with borders; fp32
// sums (1e-7 relative) would decide one row in a hundred differently.  Masses are 64-bit integers, exponentials in fp64 rounded
// to multiples of 2^-44 (sums of 2^18 terms stay below 2^63): exact to add in any order, so the result does not depend on the
// order of atomics.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ais.h"
#include "host_setup.cuh"
#include "launch.cuh"
#include "select.cuh"

namespace cg = cooperative_groups;

namespace ais {

namespace {

constexpr int kSelThreads = 512;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kBins = 2048;
constexpr int kBinsPerThread = kBins / kSelThreads;
constexpr int kListCap = 2048;           // entries of the list that one CTA sorts
constexpr int kMaxCluster = 8;
constexpr int kSliceBytes = 160 * 1024;  // most of a row that a CTA holds
constexpr float kBinsPerNat = 64.f;
constexpr int kIndexBits = 20;
constexpr double kMassOne = 17592186044416.0;   // 2^44

typedef unsigned long long u64;

struct Published {                       // what a CTA tells the others of its cluster
    float max;
    int bad;
    u64 mass[3];
    u64 lo, hi;
    double full;
    int count;
};

struct alignas(16) SelShared {
    uint32_t hist[kBins];                // of this CTA's slice
    uint32_t tot[kBins];                 // of the row
    u64 mass[kBins];
    union {
        u64 mass_tot[kBins];
        u64 list[kListCap];
    };
    Published pub;
    u64 warp_u64[kSelWarps];
    u64 warp_u64b[kSelWarps];
    double warp_f64[kSelWarps];
    int warp_int[kSelWarps];
    u64 found[4];
    int list_n;
};

struct SelectArgs {
    const void* x;
    int64_t ld;
    int V;
    int cluster;
    int slice;               // elements per CTA, a multiple of 64
    const uint8_t* mask;
    uint32_t* status;
    // sampling
    ais_sampling how;
    const float* u;
    int32_t* tokens;
    float *lp, *lp_full;
    int32_t* n_kept;
    // top logits
    int K;
    float tau;
    int32_t* ids;
    float* values;
    float* lse;
    int64_t ld_out;
};

// 0 (the largest entry) or at least AIS_MIN_TEMPERATURE; not NaN, not infinite.
__host__ __device__ inline bool usable_temperature(float t) { return t == 0.f || (t >= AIS_MIN_TEMPERATURE && t < INFINITY); }

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// The order of a row as one number: larger values first, -0 and 0 alike, then the smaller index.
__device__ __forceinline__ u64 order_of(float x, int index) {
    const uint32_t b = __float_as_uint(x + 0.f);
    const uint32_t up = b ^ ((b >> 31) != 0u ? 0xffffffffu : 0x80000000u);
    return (static_cast<u64>(~up) << kIndexBits) | static_cast<uint32_t>(index);
}
__device__ __forceinline__ float value_of(u64 o) {
    const uint32_t up = ~static_cast<uint32_t>(o >> kIndexBits);
    return __uint_as_float(up ^ ((up >> 31) != 0u ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int index_of(u64 o) { return static_cast<int>(o & ((1u << kIndexBits) - 1u)); }
// the last number of a finite entry
__device__ __forceinline__ u64 last_finite() { return order_of(-INFINITY, 0) - 1; }

struct Scale {
    float top;
    double inv_t;
    float bins;             // bins per unit of x
    float log2_scale;       // log2(e) / T
    __device__ __forceinline__ int bin(float x) const {
        const float y = (top - x) * bins;
        return y < static_cast<float>(kBins - 1) ? static_cast<int>(y) : kBins - 1;
    }
    __device__ __forceinline__ double logw(float x) const { return (static_cast<double>(x) - static_cast<double>(top)) * inv_t; }
    __device__ __forceinline__ u64 mass(float x) const { return __double2ull_rn(exp(logw(x)) * kMassOne); }
};

__device__ __forceinline__ u64 warp_sum(u64 v) {
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double warp_sum(double v) {
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename N>
__device__ __forceinline__ N warp_scan(N v) {          // inclusive
    const int lane = threadIdx.x & 31;
    for (int o = 1; o < 32; o <<= 1) {
        const N up = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += up;
    }
    return v;
}
// Exclusive scan over the block; every thread gets the total, too.
template <typename N>
__device__ __forceinline__ N block_scan(N v, N* scratch, N& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const N inc = warp_scan(v);
    __syncthreads();
    if (lane == 31) scratch[warp] = inc;
    __syncthreads();
    N before = 0, sum = 0;
    for (int w = 0; w < kSelWarps; ++w) {
        const N s = scratch[w];
        if (w < warp) before += s;
        sum += s;
    }
    total = sum;
    return before + inc - v;
}

// What a kernel holds of one row.
template <typename T>
struct Row {
    SelShared& s;
    const T* data;           // this CTA's slice in shared memory
    int begin, n;            // where it starts in the row, its length
    int C, rank;
    Scale sc;

    __device__ __forceinline__ float at(int i) const { return to_f32(data[i]); }
    __device__ void sync() const {
        if (C > 1) cg::this_cluster().sync();
        else __syncthreads();
    }
    template <typename P>
    __device__ P* remote(P* p, int r) const { return C > 1 ? cg::this_cluster().map_shared_rank(p, r) : p; }

    // f(x, i) for the elements of the slice, warp by warp in order of the index: a warp owns consecutive elements
    __device__ __forceinline__ int segment() const { return (n + kSelWarps * 32 - 1) / (kSelWarps * 32) * 32; }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        const int seg = segment(), lane = threadIdx.x & 31, from = (threadIdx.x >> 5) * seg, to = min(from + seg, n);
        for (int i = from + lane; i < to; i += 32) f(at(i), i);
    }
    __device__ void clear_hist(bool with_mass) const {
        for (int b = threadIdx.x; b < kBins; b += kSelThreads) {
            s.hist[b] = 0;
            if (with_mass) s.mass[b] = 0;
        }
        __syncthreads();
    }
    // hist (and mass) of all slices added up in every CTA
    __device__ void merge_hist(bool with_mass) const {
        sync();
        const int share = kBins / C;
        for (int i = threadIdx.x; i < share; i += kSelThreads) {
            const int b = rank * share + i;
            uint32_t c = 0;
            u64 m = 0;
            for (int r = 0; r < C; ++r) {
                c += remote(s.hist, r)[b];
                if (with_mass) m += remote(s.mass, r)[b];
            }
            for (int r = 0; r < C; ++r) {
                remote(s.tot, r)[b] = c;
                if (with_mass) remote(s.mass_tot, r)[b] = m;
            }
        }
        sync();
    }
    // The bin in which the count reaches k (k >= 1, no more than the total): s.found = {bin, entries before it, entries in it}.
    __device__ void find_count(u64 k) const {
        const int b0 = threadIdx.x * kBinsPerThread;
        int c[kBinsPerThread], sum = 0, total;
        for (int j = 0; j < kBinsPerThread; ++j) sum += c[j] = static_cast<int>(s.tot[b0 + j]);
        int before = block_scan(sum, s.warp_int, total);
        for (int j = 0; j < kBinsPerThread; ++j) {
            if (static_cast<u64>(before) < k && static_cast<u64>(before + c[j]) >= k) {
                s.found[0] = b0 + j;
                s.found[1] = before;
                s.found[2] = c[j];
            }
            before += c[j];
        }
        __syncthreads();
    }
    // The bin in which mass0 plus the masses reach p total: s.found = {bin, mass before it, entries in it}; the last bin with an
    // entry where rounding leaves none.
    __device__ void find_mass(u64 mass0, double target) const {
        if (threadIdx.x == 0) s.found[3] = 0;
        const int b0 = threadIdx.x * kBinsPerThread;
        u64 m[kBinsPerThread], sum = 0, total;
        for (int j = 0; j < kBinsPerThread; ++j) sum += m[j] = s.mass_tot[b0 + j];
        u64 before = mass0 + block_scan(sum, s.warp_u64, total);
        for (int j = 0; j < kBinsPerThread; ++j) {
            if (static_cast<double>(before) < target && static_cast<double>(before + m[j]) >= target) {
                s.found[0] = b0 + j;
                s.found[1] = before;
                s.found[2] = s.tot[b0 + j];
                s.found[3] = 1;
            }
            before += m[j];
        }
        __syncthreads();
    }
    // Entries for which keep(x, order) go to the list of rank 0, sorted there.  Every CTA returns after the list is complete;
    // only rank 0 has it.
    template <typename F>
    __device__ int gather_sorted(F keep) const {
        sync();                                    // the list shares its place with mass_tot
        if (threadIdx.x == 0) s.list_n = 0;
        sync();
        int* counter = remote(&s.list_n, 0);
        u64* list = remote(s.list, 0);
        each([&](float x, int i) {
            const u64 o = order_of(x, begin + i);
            if (keep(x, o)) {
                const int at = atomicAdd(counter, 1);
                if (at < kListCap) list[at] = o;
            }
        });
        sync();
        if (rank != 0) return 0;
        const int n_list = min(s.list_n, kListCap);
        int n2 = 2;
        while (n2 < n_list) n2 <<= 1;
        for (int i = n_list + threadIdx.x; i < n2; i += kSelThreads) s.list[i] = ~0ull;
        __syncthreads();
        for (int size = 2; size <= n2; size <<= 1)
            for (int stride = size >> 1; stride > 0; stride >>= 1) {
                for (int t = threadIdx.x; t < n2 / 2; t += kSelThreads) {
                    const int i = 2 * t - (t & (stride - 1)), j = i + stride;
                    const u64 a = s.list[i], b = s.list[j];
                    if ((a > b) == ((i & size) == 0)) {
                        s.list[i] = b;
                        s.list[j] = a;
                    }
                }
                __syncthreads();
            }
        return n_list;
    }
    // Smallest and largest number of the entries that pick(x, order) takes.
    template <typename F>
    __device__ void range_of(F pick, u64& lo, u64& hi) const {
        u64 a = ~0ull, b = 0;
        each([&](float x, int i) {
            const u64 o = order_of(x, begin + i);
            if (pick(x, o)) { a = min(a, o); b = max(b, o); }
        });
        for (int o = 16; o > 0; o >>= 1) {
            a = min(a, __shfl_xor_sync(0xffffffffu, a, o));
            b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
        }
        __syncthreads();
        if ((threadIdx.x & 31) == 0) { s.warp_u64[threadIdx.x >> 5] = a; s.warp_u64b[threadIdx.x >> 5] = b; }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 0; w < kSelWarps; ++w) { a = min(a, s.warp_u64[w]); b = max(b, s.warp_u64b[w]); }
            s.pub.lo = a;
            s.pub.hi = b;
        }
        sync();
        lo = ~0ull;
        hi = 0;
        for (int r = 0; r < C; ++r) {
            lo = min(lo, remote(&s.pub, r)->lo);
            hi = max(hi, remote(&s.pub, r)->hi);
        }
        sync();
    }
    // The cut inside a group of `count` entries, those that pick(x, order) takes: by count, the entry number `want` (from 1) of the
    // group; by mass, the first at which mass0 plus the masses reach `target`.
    template <bool MASS, typename F>
    __device__ u64 cut_in_group(F pick, int count, u64 want, u64 mass0, double target) const {
        if (count > kListCap) {
            u64 lo, hi;
            range_of(pick, lo, hi);
            while (count > kListCap && lo < hi) {
                const int bits = 64 - __clzll(hi - lo);
                const int shift = bits > 11 ? bits - 11 : 0;
                clear_hist(MASS);
                each([&](float x, int i) {
                    const u64 o = order_of(x, begin + i);
                    if (o < lo || o > hi) return;
                    const int b = static_cast<int>((o - lo) >> shift);
                    atomicAdd(&s.hist[b], 1u);
                    if (MASS) atomicAdd(&s.mass[b], sc.mass(x));
                });
                merge_hist(MASS);
                if (MASS) {
                    find_mass(mass0, target);
                    if (s.found[3] == 0) return hi;                  // rounding: the whole group
                    mass0 = s.found[1];
                } else {
                    find_count(want);
                    want -= s.found[1];
                }
                count = static_cast<int>(s.found[2]);
                lo += s.found[0] << shift;
                hi = min(hi, lo + ((1ull << shift) - 1));
            }
            if (lo == hi) return lo;
            return cut_in_list<MASS>([=](float, u64 o) { return o >= lo && o <= hi; }, want, mass0, target);
        }
        return cut_in_list<MASS>(pick, want, mass0, target);
    }
    template <bool MASS, typename F>
    __device__ u64 cut_in_list(F pick, u64 want, u64 mass0, double target) const {
        const int n_list = gather_sorted(pick);
        if (rank == 0) {
            if (MASS) {
                constexpr int kEach = kListCap / kSelThreads;
                u64 m[kEach], sum = 0, total;
                const int i0 = threadIdx.x * kEach;
                for (int j = 0; j < kEach; ++j) sum += m[j] = i0 + j < n_list ? sc.mass(value_of(s.list[i0 + j])) : 0;
                if (threadIdx.x == 0) s.pub.lo = s.list[n_list - 1];
                u64 before = mass0 + block_scan(sum, s.warp_u64, total);
                for (int j = 0; j < kEach; ++j) {
                    if (i0 + j < n_list && static_cast<double>(before) < target && static_cast<double>(before + m[j]) >= target)
                        s.pub.lo = s.list[i0 + j];
                    before += m[j];
                }
            } else if (threadIdx.x == 0) {
                s.pub.lo = s.list[want - 1];
            }
        }
        sync();
        const u64 cut = remote(&s.pub, 0)->lo;
        sync();
        return cut;
    }
    // mass[0..2], count and full of all CTAs; `before` gets the mass[0] of the CTAs ahead of this one
    __device__ void add_up(const u64 (&mine)[3], int count, double full, u64 (&sum)[3], u64& before, int& n_sum, double& f_sum) const {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        u64 m[3];
        for (int j = 0; j < 3; ++j) m[j] = warp_sum(mine[j]);
        const int c = __reduce_add_sync(0xffffffffu, count);
        const double f = warp_sum(full);
        __syncthreads();
        if (lane == 0) {
            s.warp_u64[warp] = m[0];
            s.warp_u64b[warp] = m[1];
            s.warp_f64[warp] = f;
            s.warp_int[warp] = c;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            u64 a = 0, b = 0;
            double t = 0.0;
            int k = 0;
            for (int w = 0; w < kSelWarps; ++w) { a += s.warp_u64[w]; b += s.warp_u64b[w]; t += s.warp_f64[w]; k += s.warp_int[w]; }
            s.pub.mass[0] = a;
            s.pub.mass[1] = b;
            s.pub.full = t;
            s.pub.count = k;
        }
        sync();
        for (int j = 0; j < 3; ++j) sum[j] = 0;
        before = 0;
        n_sum = 0;
        f_sum = 0.0;
        for (int r = 0; r < C; ++r) {
            const Published* p = remote(&s.pub, r);
            if (r < rank) before += p->mass[0];
            sum[0] += p->mass[0];
            sum[1] += p->mass[1];
            n_sum += p->count;
            f_sum += p->full;
        }
        sync();
    }
};

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The slice [begin, begin + n) of a row to shared memory, 16 bytes at a time where they lie inside it; returns its largest value and
// whether it holds a NaN or +inf.  An element keeps its place modulo 16 bytes, so `data` starts up to 15 bytes into the buffer.
template <typename T>
__device__ const T* load_slice(const T* src, int n, unsigned char* buf, float& top, int& bad) {
    constexpr int kEach = 16 / sizeof(T);
    const int mis = static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
    T* data = reinterpret_cast<T*>(buf) + mis;
    const int chunks = (mis + n + kEach - 1) / kEach;
    top = -INFINITY;
    bad = 0;
    auto see = [&](T v) {
        const float x = to_f32(v);
        if (!(x < INFINITY)) bad = 1;
        top = fmaxf(top, x);
    };
    constexpr int kDeep = 4;
    for (int c0 = threadIdx.x; c0 < chunks; c0 += kSelThreads * kDeep) {
        uint4 v[kDeep];
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            const int c = c0 + j * kSelThreads, e = c * kEach - mis;
            if (c < chunks && e >= 0 && e + kEach <= n) v[j] = __ldcs(reinterpret_cast<const uint4*>(src + e));
        }
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            const int c = c0 + j * kSelThreads, e = c * kEach - mis;
            if (c >= chunks) break;
            if (e >= 0 && e + kEach <= n) {
                const T* t = reinterpret_cast<const T*>(&v[j]);
#pragma unroll
                for (int k = 0; k < kEach; ++k) see(t[k]);
                reinterpret_cast<uint4*>(buf)[c] = v[j];
            } else {
                for (int k = 0; k < kEach; ++k)
                    if (e + k >= 0 && e + k < n) {
                        data[e + k] = src[e + k];
                        see(data[e + k]);
                    }
            }
        }
    }
    return data;
}

// Opens a row: slice, maximum, scale.  False where the row has no finite entry or holds a NaN or +inf (`what` says which).
template <typename T>
__device__ bool open_row(Row<T>& r, const SelectArgs& a, int64_t row, unsigned char* buf, float temperature, uint32_t& what) {
    float top;
    int bad;
    r.begin = min(r.rank * a.slice, a.V);
    r.n = min(a.slice, a.V - r.begin);
    r.data = load_slice(static_cast<const T*>(a.x) + row * a.ld + r.begin, r.n, buf, top, bad);
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    bad = __any_sync(0xffffffffu, bad);
    SelShared& s = r.s;
    if ((threadIdx.x & 31) == 0) {
        s.warp_f64[threadIdx.x >> 5] = top;
        s.warp_int[threadIdx.x >> 5] = bad;
    }
    for (int b = threadIdx.x; b < kBins; b += kSelThreads) s.hist[b] = 0;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 0; w < kSelWarps; ++w) {
            top = fmaxf(top, static_cast<float>(s.warp_f64[w]));
            bad |= s.warp_int[w];
        }
        s.pub.max = top;
        s.pub.bad = bad;
    }
    r.sync();
    top = -INFINITY;
    bad = 0;
    for (int k = 0; k < r.C; ++k) {
        const Published* p = r.remote(&s.pub, k);
        top = fmaxf(top, p->max);
        bad |= p->bad;
    }
    r.sync();
    what = bad ? AIS_FLAG_NONFINITE : top == -INFINITY ? AIS_FLAG_EMPTY : 0u;
    r.sc.top = top;
    r.sc.inv_t = 1.0 / static_cast<double>(temperature);
    r.sc.bins = kBinsPerNat / temperature;
    r.sc.log2_scale = static_cast<float>(1.4426950408889634 * r.sc.inv_t);
    return what == 0u;
}

// Histogram of the whole row and the fp32 sum of its exponentials (per thread).
template <typename T>
__device__ float histogram(const Row<T>& r) {
    float full = 0.f;
    r.each([&](float x, int) {
        if (x == -INFINITY) return;
        atomicAdd(&r.s.hist[r.sc.bin(x)], 1u);
        full += ex2_approx((x - r.sc.top) * r.sc.log2_scale);
    });
    return full;
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads, 2) sample_kernel(const __grid_constant__ SelectArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    SelShared& s = *reinterpret_cast<SelShared*>(smem);
    pdl_enter();
    const int64_t row = blockIdx.x / a.cluster;
    Row<T> r{s, nullptr, 0, 0, a.cluster, static_cast<int>(blockIdx.x % a.cluster), Scale()};
    const bool first = r.rank == 0 && threadIdx.x == 0;
    auto neutral = [&](uint32_t flag) {
        if (!first) return;
        a.tokens[row] = -1;
        if (a.lp) a.lp[row] = 0.f;
        if (a.lp_full) a.lp_full[row] = 0.f;
        if (a.n_kept) a.n_kept[row] = 0;
        if (flag && a.status) atomicOr(a.status, flag);
    };
    if (a.mask && a.mask[row] == 0) return neutral(0u);
    float temperature = a.how.temperature_rows ? a.how.temperature_rows[row] : a.how.temperature;
    int64_t k = a.how.top_k_rows ? a.how.top_k_rows[row] : a.how.top_k;
    const float p = a.how.top_p_rows ? a.how.top_p_rows[row] : a.how.top_p;
    const float m = a.how.min_p_rows ? a.how.min_p_rows[row] : a.how.min_p;
    const float u = a.u[row];
    // (each comparison is false for a NaN)
    if (!usable_temperature(temperature) || !(p >= 0.f) || !(m <= 1.f) || !(u >= 0.f && u < 1.f)) return neutral(AIS_FLAG_PARAM);
    if (temperature == 0.f) {
        temperature = 1.f;
        k = 1;
    }
    uint32_t what;
    if (!open_row(r, a, row, smem + sizeof(SelShared), temperature, what)) return neutral(what);
    const Scale sc = r.sc;

    const float full_thread = histogram(r);
    const u64 none[3] = {0, 0, 0};
    u64 sum[3], before;
    int n_fin;
    double full;
    {
        int finite = 0;
        r.each([&](float x, int) { finite += x != -INFINITY; });
        r.add_up(none, finite, static_cast<double>(full_thread), sum, before, n_fin, full);
    }
    if (k <= 0 || k >= n_fin) k = n_fin;
    const bool by_k = k < n_fin, by_p = p < 1.f;
    const double pd = p, md = m;
    auto above_m = [&](float x) { return !(m > 0.f) || x == sc.top || exp(sc.logw(x)) >= md; };
    auto write = [&](u64 o, u64 total, int kept) {
        const double logw = sc.logw(value_of(o));
        a.tokens[row] = index_of(o);
        if (a.lp) a.lp[row] = static_cast<float>(logw - log(static_cast<double>(total) / kMassOne));
        if (a.lp_full) a.lp_full[row] = static_cast<float>(logw - log(full));
        if (a.n_kept) a.n_kept[row] = kept;
    };

    if (by_k || by_p) r.merge_hist(false);
    u64 cut = last_finite();
    if (by_k) {
        r.find_count(k);
        const int bin = static_cast<int>(s.found[0]), ahead = static_cast<int>(s.found[1]), in = static_cast<int>(s.found[2]);
        __syncthreads();
        if (k <= kMaxTopLogits) {
            int n_list;
            if (ahead + in <= kListCap) {
                n_list = r.gather_sorted([&](float x, u64) { return x != -INFINITY && sc.bin(x) <= bin; });
            } else {
                cut = r.template cut_in_group<false>([&](float x, u64) { return x != -INFINITY && sc.bin(x) == bin; }, in, k - ahead, 0, 0.0);
                n_list = r.gather_sorted([&](float, u64 o) { return o <= cut; });
            }
            if (r.rank != 0) return;
            // the first k of the list: masses ahead of every entry give top-p, the value min-p; then the masses by index
            constexpr int kEach = kMaxTopLogits / kSelThreads;
            const int n1 = min(static_cast<int>(k), n_list);
            u64 w[kEach], mine = 0, total;
            const int i0 = threadIdx.x * kEach;
            for (int j = 0; j < kEach; ++j) mine += w[j] = i0 + j < n1 ? sc.mass(value_of(s.list[i0 + j])) : 0;
            u64 cum = block_scan(mine, s.warp_u64, total);
            const double target = pd * static_cast<double>(total);
            int kept = 0;
            for (int j = 0; j < kEach; ++j) {
                const int i = i0 + j;
                if (i < n1 && (i == 0 || ((!by_p || static_cast<double>(cum) < target) && above_m(value_of(s.list[i]))))) ++kept;
                cum += w[j];
            }
            int n_kept;
            block_scan(kept, s.warp_int, n_kept);
            mine = 0;
            for (int j = 0; j < kEach; ++j) {
                s.mass[i0 + j] = w[j];
                if (i0 + j < n_kept) mine += w[j];
            }
            block_scan(mine, s.warp_u64, total);
            const u64 t = __double2ull_rd(static_cast<double>(u) * static_cast<double>(total));
            __syncthreads();
            for (int i = threadIdx.x; i < n_kept; i += kSelThreads) {
                const int v = index_of(s.list[i]);
                u64 c = 0;
                for (int j = 0; j < n_kept; ++j)
                    if (index_of(s.list[j]) < v) c += s.mass[j];
                if (c <= t && t < c + s.mass[i]) write(s.list[i], total, n_kept);
            }
            return;
        }
        cut = r.template cut_in_group<false>([&](float x, u64) { return x != -INFINITY && sc.bin(x) == bin; }, in, k - ahead, 0, 0.0);
    }
    if (by_p) {
        if (by_k) {                                     // the histogram of what top-k has left
            r.clear_hist(false);
            r.each([&](float x, int i) {
                if (order_of(x, r.begin + i) <= cut) atomicAdd(&s.hist[sc.bin(x)], 1u);
            });
            r.merge_hist(false);
        }
        // Bounds on the mass down to every bin from its counts: e^(-b / 64) and e^(-(b + 1) / 64) per entry, a thousandth apart from
        // that for the rounding of the bins.  The cut lies in none of the bins before b1 and none behind b2.
        int b1, b2;
        {
            double hi[kBinsPerThread], lo[kBinsPerThread], hs = 0.0, ls = 0.0, h_total, l_total;
            const int b0 = threadIdx.x * kBinsPerThread;
            for (int j = 0; j < kBinsPerThread; ++j) {
                const double c = s.tot[b0 + j], e = exp(-(b0 + j) / 64.0);
                hs += hi[j] = c * e * 1.001;
                ls += lo[j] = b0 + j == kBins - 1 ? 0.0 : c * e * 0.983;            // e^(-1 / 64) = 0.9845
            }
            double h = block_scan(hs, s.warp_f64, h_total);
            double l = block_scan(ls, s.warp_f64, l_total);
            int n1 = 0, n2 = 0, total;
            for (int j = 0; j < kBinsPerThread; ++j) {
                h += hi[j];
                l += lo[j];
                n1 += h < pd * l_total;
                n2 += l < pd * h_total;
            }
            block_scan(n1, s.warp_int, total);
            b1 = min(total, kBins - 1);
            block_scan(n2, s.warp_int, total);
            b2 = min(total, kBins - 1);
        }
        for (int b = threadIdx.x; b < kBins; b += kSelThreads) s.mass[b] = 0;
        __syncthreads();
        u64 mine[3] = {0, 0, 0};
        r.each([&](float x, int i) {
            if (order_of(x, r.begin + i) > cut) return;
            const u64 w = sc.mass(x);
            const int b = sc.bin(x);
            mine[0] += w;
            if (b < b1) mine[1] += w;
            else if (b <= b2) atomicAdd(&s.mass[b], w);
        });
        int n_none;
        double f_none;
        r.add_up(mine, 0, 0.0, sum, before, n_none, f_none);
        const double target = pd * static_cast<double>(sum[0]);
        r.merge_hist(true);                             // (the counts again: they have not changed)
        r.find_mass(sum[1], target);
        if (s.found[3] != 0) {
            const int bin = static_cast<int>(s.found[0]), in = static_cast<int>(s.found[2]);
            const u64 mass0 = s.found[1], all = cut;
            __syncthreads();
            cut = r.template cut_in_group<true>([&](float x, u64 o) { return o <= all && sc.bin(x) == bin; }, in, 0, mass0, target);
        } else if (target <= 0.0) {
            cut = order_of(sc.top, a.V);                // p = 0: the largest value; its first entry below
        }
    }
    // The kept entries by index.
    u64 mine[3] = {0, 0, 0};
    int kept = 0;
    const bool only_first = by_p && p == 0.f;
    r.each([&](float x, int i) {
        if (order_of(x, r.begin + i) > cut || !above_m(x)) return;
        mine[0] += sc.mass(x);
        ++kept;
    });
    double f_none;
    r.add_up(mine, kept, 0.0, sum, before, kept, f_none);
    u64 t = __double2ull_rd(static_cast<double>(u) * static_cast<double>(sum[0]));
    if (only_first) { t = 0; sum[0] = static_cast<u64>(kMassOne); kept = 1; }
    // (s.warp_u64 still holds the masses of this CTA's warps)
    if (t < before) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int w = 0; w < warp; ++w) before += s.warp_u64[w];
    if (t < before || t >= before + s.warp_u64[warp]) return;
    const int seg = r.segment(), from = warp * seg, to = min(from + seg, r.n);
    for (int i0 = from; i0 < to; i0 += 32) {
        const int i = i0 + lane;
        const float x = i < to ? r.at(i) : -INFINITY;
        const u64 o = order_of(x, r.begin + i);
        const u64 w = i < to && o <= cut && above_m(x) ? sc.mass(x) : 0;
        const u64 inc = before + warp_scan(w);
        const unsigned hit = __ballot_sync(0xffffffffu, inc > t);
        if (hit) {
            if (lane == __ffs(hit) - 1) write(o, sum[0], kept);
            return;
        }
        before = __shfl_sync(0xffffffffu, inc, 31);
    }
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads, 2) top_logits_kernel(const __grid_constant__ SelectArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    SelShared& s = *reinterpret_cast<SelShared*>(smem);
    pdl_enter();
    const int64_t row = blockIdx.x / a.cluster;
    Row<T> r{s, nullptr, 0, 0, a.cluster, static_cast<int>(blockIdx.x % a.cluster), Scale()};
    auto fill = [&](int from) {
        for (int i = from + threadIdx.x; i < a.K; i += kSelThreads) {
            a.ids[row * a.ld_out + i] = -1;
            a.values[row * a.ld_out + i] = -INFINITY;
        }
    };
    auto neutral = [&](uint32_t flag, float lse) {
        if (r.rank != 0) return;
        fill(0);
        if (threadIdx.x != 0) return;
        if (a.lse) a.lse[row] = lse;
        if (flag && a.status) atomicOr(a.status, flag);
    };
    if (a.mask && a.mask[row] == 0) return neutral(0u, 0.f);
    uint32_t what;
    if (!open_row(r, a, row, smem + sizeof(SelShared), a.tau, what)) return neutral(what, what == AIS_FLAG_EMPTY ? -INFINITY : NAN);
    const Scale sc = r.sc;
    const float full_thread = histogram(r);
    const u64 none[3] = {0, 0, 0};
    u64 sum[3], before;
    int n_fin;
    double full;
    int finite = 0;
    r.each([&](float x, int) { finite += x != -INFINITY; });
    r.add_up(none, finite, static_cast<double>(full_thread), sum, before, n_fin, full);
    r.merge_hist(false);
    const int k = min(a.K, n_fin);
    r.find_count(k);
    const int bin = static_cast<int>(s.found[0]), ahead = static_cast<int>(s.found[1]), in = static_cast<int>(s.found[2]);
    __syncthreads();
    int n_list;
    if (ahead + in <= kListCap) {
        n_list = r.gather_sorted([&](float x, u64) { return x != -INFINITY && sc.bin(x) <= bin; });
    } else {
        const u64 cut = r.template cut_in_group<false>([&](float x, u64) { return x != -INFINITY && sc.bin(x) == bin; }, in, k - ahead, 0, 0.0);
        n_list = r.gather_sorted([&](float, u64 o) { return o <= cut; });
    }
    if (r.rank != 0) return;
    for (int i = threadIdx.x; i < min(k, n_list); i += kSelThreads) {
        a.ids[row * a.ld_out + i] = index_of(s.list[i]);
        a.values[row * a.ld_out + i] = value_of(s.list[i]);
    }
    fill(min(k, n_list));
    if (threadIdx.x == 0 && a.lse) a.lse[row] = static_cast<float>(static_cast<double>(sc.top) * sc.inv_t + log(full));
}

template <typename K>
cudaError_t launch_select(K kernel, SelectArgs& a, int64_t rows, int es, cudaStream_t stream) {
    // Slices of 64 KB at most, so that two CTAs share an SM; more CTAs per row while the rows alone do not fill the GPU.
    int c = 1;
    while (c < kMaxCluster && (static_cast<int64_t>(a.V) * es > static_cast<int64_t>(c) * 64 * 1024 || (rows * c < 2 * 148 && a.V > c * 2048))) c *= 2;
    a.cluster = c;
    a.slice = (((a.V + c - 1) / c) + 63) / 64 * 64;
    const size_t smem = sizeof(SelShared) + static_cast<size_t>(a.slice) * es + 32;
    static_assert(sizeof(SelShared) + kSliceBytes + 32 <= 227 * 1024, "shared memory of a CTA");
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * c));
    cfg.blockDim = dim3(kSelThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = c;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<const SelectArgs>(a));
}

int element_size(int dtype) { return dtype == AIS_BF16 || dtype == AIS_F16 ? 2 : dtype == AIS_F32 ? 4 : 0; }

int check_logits(const void* logits, int dtype, int64_t rows, int64_t V, int64_t ld) {
    const int es = element_size(dtype);
    if (es == 0) return AIS_ERR_PARAM;
    if (rows < 0 || V <= 0 || ld < V) return AIS_ERR_SHAPE;
    if (V > AIS_LOGITS_MAX_V || rows > (int64_t(1) << 24)) return AIS_ERR_LIMIT;
    if (rows > 0 && !logits) return AIS_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(logits) % es != 0) return AIS_ERR_ALIGN;
    return AIS_OK;
}

}  // namespace

cudaError_t select_prepare() {
    const void* kernels[] = {reinterpret_cast<const void*>(sample_kernel<__nv_bfloat16>),     reinterpret_cast<const void*>(sample_kernel<__half>),
                             reinterpret_cast<const void*>(sample_kernel<float>),             reinterpret_cast<const void*>(top_logits_kernel<__nv_bfloat16>),
                             reinterpret_cast<const void*>(top_logits_kernel<__half>),        reinterpret_cast<const void*>(top_logits_kernel<float>)};
    for (const void* k : kernels) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace ais

using namespace ais;

extern "C" {

void ais_default_sampling(ais_sampling* how) {
    if (!how) return;
    *how = {1.0f, 0, 1.0f, 0.0f, nullptr, nullptr, nullptr, nullptr};
}

int ais_sample(const void* logits, int dtype, int64_t rows, int64_t V, int64_t ld, const ais_sampling* how, const float* u,
               const uint8_t* mask, int32_t* tokens, float* lp, float* lp_full, int32_t* n_kept, uint32_t* dev_status, void* stream) {
    int st = check_logits(logits, dtype, rows, V, ld);
    if (st != AIS_OK) return st;
    if (!how || (rows > 0 && (!u || !tokens))) return AIS_ERR_NULL;
    if (!how->temperature_rows && !usable_temperature(how->temperature)) return AIS_ERR_PARAM;
    if (!how->top_p_rows && !(how->top_p >= 0.f)) return AIS_ERR_PARAM;
    if (!how->min_p_rows && !(how->min_p <= 1.f)) return AIS_ERR_PARAM;
    st = device_setup(nullptr);
    if (st != AIS_OK) return st;
    if (rows == 0) return AIS_OK;
    SelectArgs a = {};
    a.x = logits;
    a.ld = ld;
    a.V = static_cast<int>(V);
    a.mask = mask;
    a.status = dev_status;
    a.how = *how;
    a.u = u;
    a.tokens = tokens;
    a.lp = lp;
    a.lp_full = lp_full;
    a.n_kept = n_kept;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == AIS_BF16  ? launch_select(sample_kernel<__nv_bfloat16>, a, rows, 2, s)
                          : dtype == AIS_F16 ? launch_select(sample_kernel<__half>, a, rows, 2, s)
                                             : launch_select(sample_kernel<float>, a, rows, 4, s);
    return e == cudaSuccess ? AIS_OK : AIS_ERR_DEVICE;
}

int ais_top_logits(const void* logits, int dtype, int64_t rows, int64_t V, int64_t ld, int32_t K, float temperature, const uint8_t* mask,
                   int32_t* ids, float* values, int64_t ld_out, float* lse, uint32_t* dev_status, void* stream) {
    int st = check_logits(logits, dtype, rows, V, ld);
    if (st != AIS_OK) return st;
    if (K <= 0 || K > V || ld_out < K) return AIS_ERR_SHAPE;
    if (K > AIS_TOP_MAX) return AIS_ERR_LIMIT;
    if (rows > 0 && (!ids || !values)) return AIS_ERR_NULL;
    if (!usable_temperature(temperature) || temperature == 0.f) return AIS_ERR_PARAM;
    st = device_setup(nullptr);
    if (st != AIS_OK) return st;
    if (rows == 0) return AIS_OK;
    SelectArgs a = {};
    a.x = logits;
    a.ld = ld;
    a.V = static_cast<int>(V);
    a.mask = mask;
    a.status = dev_status;
    a.K = K;
    a.tau = temperature;
    a.ids = ids;
    a.values = values;
    a.ld_out = ld_out;
    a.lse = lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == AIS_BF16  ? launch_select(top_logits_kernel<__nv_bfloat16>, a, rows, 2, s)
                          : dtype == AIS_F16 ? launch_select(top_logits_kernel<__half>, a, rows, 2, s)
                                             : launch_select(top_logits_kernel<float>, a, rows, 4, s);
    return e == cudaSuccess ? AIS_OK : AIS_ERR_DEVICE;
}

}  // extern "C"
