// Selection along rows of logits: the K largest entries of a row in order (a teacher's top logits), and one token drawn from a
// row under temperature, top-k, top-p and min-p.
//
// Order of a row: value descending, index ascending.  Every filter keeps a prefix of that order, so a filter is a cut: the last
// entry that is kept, as a 64-bit number (order key of the value above, index below) whose natural order is the row's order.
//  top-k : the k-th number.                       top-p : the first number at which the mass reaches p times the total.
//  min-p : e >= m, a threshold on the value.       The token: the first index at which the kept mass exceeds u times its total.
// with e = exp((x - max) / T).
//
// A row belongs to a cluster of one to eight CTAs, a slice each.  What bounds the kernels is one read of the logits for many rows,
// and the chain of block and cluster barriers for few; so every case reads the row as few times as it can.
//  * The K largest (top_logits, top-k up to 1,024): one pass.  The first tile of a slice gives a threshold (the K-th largest of the
//    maxima of 256 to 1,024 groups of entries: K entries reach it); later 16-byte chunks with an entry above it join a list in shared
//    memory, and each time the list has doubled the threshold rises to the K-th of the list.  The entries of the listed chunks that
//    reach the last threshold are sorted, for all slices together, at the end.
//  * No filter: one pass of fp64 sums per warp, then the one warp's range that holds the token is read again.
//  * Everything else (top-p or min-p over the whole row, longer top-k, lists that overflow, values out of fp32's range): passes over
//    data that is mostly still in L1 or L2.  Maximum; histogram of the distance below it (8,192 bins of 1/256 of a unit of log-
//    probability; a bin is a range of the order).  For top-p the counts bound the mass above every bin, so the cut lies between two
//    bins; one pass of fp64 exponentials gives the total and the mass before the first of them; with these the counts put the cut into
//    one or two bins, whose entries, and those from the first bound on, are listed.  The group around the cut is divided by the
//    entries' numbers, 1,024 ways at a time, until the few entries left are added up one by one.
//
// Precision: which token is drawn and how many are kept are decided by comparing sums over the vocabulary with borders; fp32
// sums (1e-7 relative) would decide one row in a hundred differently.  Exponentials and sums that decide are fp64, summed in an
// order that the sizes fix.  Sums by atomics (masses of parts of a group) are 96-bit integers, exponentials cut to multiples of 2^-76: exact to
// add in any order, so no result depends on the order of atomics, and of 327,680 entries off by 2^-57 at most.  (In 64 bits, multiples of
// 2^-44, entries of one value are all off by the same amount: 300,000 of them at e^-22 by eight entries' mass.)  The 1,024 masses of a list have
// multiples of 2^-53 in 64 bits.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/ais.h"
#include "host_setup.cuh"
#include "launch.cuh"
#include "select.cuh"

namespace cg = cooperative_groups;

namespace ais {

namespace {

constexpr int kSelThreads = 512;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kDeep = 4;                 // 16-byte loads of a thread in flight in the pass for the largest entries
constexpr int kBins = 8192;
constexpr int kListCap = 4096;           // entries of a list
constexpr int kSplit = 1024;             // ways in which a group of entries is divided
constexpr int kChunkCap = 3200;          // chunks in the list of a pass for the largest entries
constexpr int kChunkPrune = 2048;        // which is cut back beyond this
constexpr int kFew = 256;                // entries of a group that are not divided any more
constexpr int kRankSort = 256;           // entries up to which a list is sorted by counting
constexpr int kMaxCluster = 8;
constexpr float kBinsPerNat = 256.f;
constexpr int kIndexBits = 20;
constexpr double kMassOne = 17592186044416.0;       // 2^44: units of a Mass's upper word
constexpr double kListOne = 9007199254740992.0;     // 2^53: units of a list's masses
constexpr int kTableCopies = 16;         // of the table of powers of two

constexpr float kTwo23 = 8388608.f;

typedef unsigned long long u64;

struct Published {                       // what a CTA tells the others of its cluster
    float top;
    int bad;
    double sum[2];
    u64 lo, hi;
    int count;
};

// 72 KB: with two CTAs per SM this leaves 84 KB of L1, which the loads in flight need (at 105 KB the passes took three times as long).
struct alignas(16) SelShared {
    union {
        uint32_t hist[kBins];            // of this CTA's slice; nobody needs it once there is a list
        u64 list[kListCap];
        uint32_t indices[2 * kListCap];  // a list by index alone
    };
    union {
        uint32_t tot[kBins];             // of the row (more than one CTA)
        struct {
            uint32_t mass[3][kSplit];    // dividing a group: masses (lowest word first) and counts of this CTA, of the row (more than one CTA)
            uint32_t mass_tot[3][kSplit];
            uint32_t part[kSplit];
            uint32_t part_tot[kSplit];
        };
        struct {
            u64 few[kFew];               // the last entries of a group
            u64 few_hi[kFew];            // and their masses
            uint32_t few_lo[kFew];
        };
        u64 list_mass[kMaxTopLogits];    // of the entries of a sorted list
        struct {
            uint32_t small_hist[kSelThreads];
            float group_max[2 * kSelThreads];
            u64 chunks[kChunkCap];       // 16-byte chunks with a large entry: that entry above, the chunk below
        };
    };
    double exp2_table[64 * kTableCopies];   // 2^(j / 64)
    double warp_kept[kSelWarps];         // kept mass of every warp's range
    uint32_t warp_listed[3][kSelWarps];  // what the list adds to it
    Published pub[2];                    // in turn, so that one barrier per exchange is enough
    double warp_f64[2][kSelWarps];
    u64 warp_u64[2][kSelWarps];
    int warp_int[kSelWarps];
    double found_mass;
    int found[4];
    int list_n, list_few;
};
// (through the array itself and not through a pointer in a struct: the compiler then knows that it is shared memory)
extern __shared__ __align__(16) unsigned char select_smem[];
__device__ __forceinline__ SelShared& smem() { return *reinterpret_cast<SelShared*>(select_smem); }

struct SelectArgs {
    const void* x;
    int64_t ld;
    int V;
    int cluster;
    int rows_of;             // sampling: kAllRows, or one of the two kinds
    int late;                // nothing of the kernel before is needed: it is waited for at the end only
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

// Rows of one pass (few large entries, or no filter at all), and rows that need several.
enum { kAllRows = 0, kOnePass = 1, kManyPasses = 2 };

// 0 (the largest entry) or at least AIS_MIN_TEMPERATURE; not NaN, not infinite.
__host__ __device__ inline bool usable_temperature(float t) { return t == 0.f || (t >= AIS_MIN_TEMPERATURE && t < INFINITY); }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kEach = 4;
    static constexpr uint32_t kNegInf = 0xff800000u;
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
        x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
    }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kEach = 8;
    static constexpr uint32_t kNegInf = 0xff80ff80u;
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
    }
};
template <> struct Elem<__half> {
    static constexpr int kEach = 8;
    static constexpr uint32_t kNegInf = 0xfc00fc00u;
    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
            x[2 * j] = f.x;
            x[2 * j + 1] = f.y;
        }
    }
};

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

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// An exponential as a multiple of 2^-76, at most 2^76; 2^20 of them add up to 96 bits at most.
struct Mass {
    u64 hi;                  // multiples of 2^-44
    uint32_t lo;
};
// A sum of upper and one of lower words in units of 2^-44.  Rounded, but rising with the exact sum, so that the end of one part and the start
// of the next are the same number.
__device__ __forceinline__ double in_units(u64 hi, u64 lo) {
    return static_cast<double>(hi + (lo >> 32)) + static_cast<double>(static_cast<uint32_t>(lo)) * 0x1p-32;
}
// A 96-bit sum in shared memory (words `stride` apart, the lowest first) by 32-bit atomics, each adding what its word carries: a 64-bit atomic is
// a loop of compare-and-swaps, which takes 300 us for the 2,000 entries of one value that share a sum.
__device__ __forceinline__ void add_mass(uint32_t* sum, int stride, Mass m) {
    const uint32_t old = atomicAdd(sum, m.lo);
    const u64 mid = (m.hi & 0xffffffffull) + (old + m.lo < old ? 1u : 0u);
    const uint32_t mid_lo = static_cast<uint32_t>(mid), old_mid = atomicAdd(sum + stride, mid_lo);
    const uint32_t hi = static_cast<uint32_t>(m.hi >> 32) + static_cast<uint32_t>(mid >> 32) + (old_mid + mid_lo < old_mid ? 1u : 0u);
    if (hi != 0u) atomicAdd(sum + 2 * stride, hi);
}
__device__ __forceinline__ u64 upper_words(const uint32_t* sum, int stride) { return static_cast<u64>(sum[2 * stride]) << 32 | sum[stride]; }

template <typename N>
__device__ __forceinline__ N warp_sum(N v) {
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

// Ascending, n2 a power of two.
template <typename N>
__device__ void block_sort(N* v, int n2) {
    for (int size = 2; size <= n2; size <<= 1)
        for (int stride = size >> 1; stride > 0; stride >>= 1) {
            for (int t = threadIdx.x; t < n2 / 2; t += kSelThreads) {
                const int i = 2 * t - (t & (stride - 1)), j = i + stride;
                const N a = v[i], b = v[j];
                if ((a > b) == ((i & size) == 0)) {
                    v[i] = b;
                    v[j] = a;
                }
            }
            __syncthreads();
        }
}
__device__ __forceinline__ int pow2_from(int n) {
    int n2 = 2;
    while (n2 < n) n2 <<= 1;
    return n2;
}

// e^((x - ref) / T) in fp64 for a fixed T and ref: 2^(k / 64) from a table times a polynomial in the rest, at most ln 2 / 128 (Taylor
// series to the fourth power: 4e-14 relative).  Ten fp64 instructions and a look-up; exp() takes more than twice that.  The table is
// there sixteen times, entry j of copy c at 16 j + c, so that the 16 lanes of a half-warp read 16 different pairs of banks (one
// copy: 5 instead of 2 cycles per look-up).
struct Weight {
    double c64, ref;          // 64 log2(e) / T
    float floor;              // entries below this get no weight (-inf among them); their weight is below 2^-1000
    __device__ __forceinline__ void set(double inv_t, double ref_) {
        c64 = 92.332482616893656877 * inv_t;
        ref = ref_;
        floor = __double2float_ru(fmax(ref - 64000.0 / c64, -3.4028234663852886e38));     // (no more than ref)
    }
    // x >= floor.  (The difference first: with one fused multiply-add for both, ref itself would weigh 1 only to within the rounding of
    // ref / T, and logits of 1e30 anything.)
    __device__ __forceinline__ double of(const double* table, float x) const {
        constexpr double kMagic = 6755399441055744.0;            // 1.5 x 2^52
        constexpr double a1 = 0.010830424696249145, a2 = a1 * a1 / 2, a3 = a2 * a1 / 3, a4 = a3 * a1 / 4;   // ln(2) / 64
        const double y = (static_cast<double>(x) - ref) * c64;
        const double t = y + kMagic;
        const int k = __double2loint(t);
        const double f = y - (t - kMagic);
        const double p = f * fma(f, fma(f, fma(f, a4, a3), a2), a1);
        const double e = table[(k & 63) * kTableCopies + (threadIdx.x & (kTableCopies - 1))];
        const double w = fma(e, p, e);
        return __hiloint2double(__double2hiint(w) + ((k >> 6) << 20), __double2loint(w));
    }
    __device__ __forceinline__ double operator()(const double* table, float x) const {
        const double w = of(table, fmaxf(x, floor));
        return x >= floor ? w : 0.0;
    }
};

__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// What a CTA holds of one row.
template <typename T>
struct Row {
    static constexpr int kEach = Elem<T>::kEach;
    static constexpr int kLight = 16 / kEach;    // chunks in flight in passes of few instructions per entry,
    static constexpr int kHeavy = 8 / kEach;     // and in those with fp64 exponentials (see each())
    const T* x;              // the row
    int V, head;             // its length; elements before the first 16-byte boundary
    int whole;               // 16-byte chunks behind that
    int c0, c1;              // this CTA's
    int C, rank;
    float top;               // largest value (once known)
    float bins;              // histogram bins per unit of x
    double inv_t;
    Weight weight;           // about `top`
    mutable int turn = 0;    // which of the two pub[] the next exchange uses

    __device__ Row(const SelectArgs& a, int64_t row, int rank_) : V(a.V), C(a.cluster), rank(rank_) {
        x = static_cast<const T*>(a.x) + row * a.ld;
        head = min(static_cast<int>((16 - (reinterpret_cast<uintptr_t>(x) & 15)) % 16 / sizeof(T)), V);
        whole = (V - head) / kEach;
        const int per = (whole + C - 1) / C;
        c0 = min(rank * per, whole);
        c1 = min(c0 + per, whole);
    }
    __device__ __forceinline__ int first_index(int c) const { return head + c * kEach; }
    __device__ __forceinline__ uint4 chunk(int c, int end) const {            // -inf from `end` on
        return c < end ? *reinterpret_cast<const uint4*>(x + first_index(c))
                       : make_uint4(Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf);
    }
    // The entries before the first and behind the last whole chunk, fewer than kEach each, belong to the first warp of the first CTA
    // (before its chunks) and to the last warp of the last CTA (behind its chunks).  One of them as a chunk filled up with -inf at its end;
    // false if there is none (for this warp).
    __device__ __forceinline__ bool edge(bool tail, int warp, float (&v)[kEach], int& i) const {
        int n;
        if (tail) {
            i = first_index(whole);
            n = rank == C - 1 && warp == kSelWarps - 1 ? V - i : 0;
        } else {
            i = 0;
            n = rank == 0 && warp == 0 ? head : 0;
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) v[k] = k < n ? to_f32(x[i + k]) : -INFINITY;
        return n > 0;
    }
    // A warp owns consecutive chunks of the slice.
    __device__ __forceinline__ void range(int warp, int& from, int& to) const {
        const int per = ((c1 - c0 + kSelWarps - 1) / kSelWarps + 31) / 32 * 32;
        from = min(c0 + warp * per, c1);
        to = min(from + per, c1);
    }
    // f(values, index of the first, how many are part of the row) for everything this warp owns, a thread at a time, B chunks of it in flight.
    // A chunk's registers are loaded again as soon as it is unpacked: handing them on by moves would wait for the load.  The code of f is
    // there B + 1 times, and fetching it counts, most code here running once per row: four chunks of eight 16-bit entries instead of
    // two took a twelfth longer (256 x 151936 bf16, top-p), four times eight fp64 exponentials twice as long.
    template <int B, typename F>
    __device__ __forceinline__ void each(F f) const {
        int from, to;
        range(threadIdx.x >> 5, from, to);
        const int lane = threadIdx.x & 31;
        uint4 raw[B];
#pragma unroll
        for (int j = 0; j < B; ++j) raw[j] = chunk(from + lane + 32 * j, to);
#pragma unroll 1
        for (int c = from + lane; c < to; c += 32 * B) {
#pragma unroll
            for (int j = 0; j < B; ++j) {
                float v[kEach];
                Elem<T>::unpack(raw[j], v);
                raw[j] = chunk(c + 32 * (B + j), to);
                if (j == 0 || c + 32 * j < to) f(v, first_index(c + 32 * j), kEach);
            }
        }
        // the ends of the row: lane 0 the head, lane 1 the tail
        if (lane < 2) {
            float v[kEach];
            int i;
            if (edge(lane == 1, threadIdx.x >> 5, v, i)) f(v, i, lane == 1 ? V - i : head);
        }
    }

    __device__ void sync() const {
        if (C > 1) cg::this_cluster().sync();
        else __syncthreads();
    }
    template <typename P>
    __device__ P* remote(P* p, int r) const { return C > 1 ? cg::this_cluster().map_shared_rank(p, r) : p; }
    // The histogram bin of a value as a float above 2^23, whose low bits are the bin: the distance below the maximum in bins, rounded.
    __device__ __forceinline__ float bin_f(float v) const { return fminf(fmaf(top - v, bins, kTwo23), kTwo23 + (kBins - 1)); }
    __device__ __forceinline__ int bin(float v) const { return static_cast<int>(__float_as_uint(bin_f(v)) & (kBins - 1)); }
    // The largest value whose bin is `b` or a later one (bin_f falls as its value rises): a comparison with it does for one with the bin.
    __device__ float edge_value(int b) const {
        // a warp tries 32 places at a time of the values in ascending order (see order_of()), from -inf to +inf
        const uint32_t lane = threadIdx.x & 31;
        uint32_t lo = 0x007fffffu, hi = 0xff800000u;
        while (hi - lo > 1u) {
            const uint32_t step = max((hi - lo) / 33u, 1u), at = lo + min((lane + 1u) * step, hi - lo);
            const float v = __uint_as_float(at ^ ((at >> 31) != 0u ? 0x80000000u : 0xffffffffu));
            const unsigned beyond = __ballot_sync(0xffffffffu, at >= hi || v > top || bin_f(v) < kTwo23 + b);
            const uint32_t first = beyond == 0u ? 32u : static_cast<uint32_t>(__ffs(beyond) - 1);     // places before it are not beyond
            const uint32_t from = lo;
            if (first < 32u) hi = min(hi, from + (first + 1u) * step);
            lo = from + first * step;
        }
        return __uint_as_float(lo ^ ((lo >> 31) != 0u ? 0x80000000u : 0xffffffffu));
    }
    __device__ __forceinline__ Mass mass(float v) const {
        const double w = weight(smem().exp2_table, v) * kMassOne;
        Mass m;
        m.hi = __double2ull_rd(w);
        m.lo = __double2uint_rd((w - static_cast<double>(m.hi)) * 0x1p32);
        return m;
    }
    __device__ __forceinline__ const uint32_t* counts() const { return C > 1 ? smem().tot : smem().hist; }
    __device__ __forceinline__ const uint32_t* parts() const { return C > 1 ? smem().part_tot : smem().part; }
    __device__ __forceinline__ const uint32_t* masses() const { return C > 1 ? smem().mass_tot[0] : smem().mass[0]; }

    __device__ void clear_hist() const {
        SelShared& s = smem();
        for (int b = threadIdx.x; b < kBins; b += kSelThreads) s.hist[b] = 0;
        __syncthreads();
    }
    // An array of all slices added up in every CTA (C > 1); barriers around it are the caller's
    template <typename N>
    __device__ void merge(N* mine, N* total, int n) const {
        const int share = n / C;
        for (int i = threadIdx.x; i < share; i += kSelThreads) {
            const int b = rank * share + i;
            N c = 0;
            for (int r = 0; r < C; ++r) c += remote(mine, r)[b];
            for (int r = 0; r < C; ++r) remote(total, r)[b] = c;
        }
    }
    __device__ void merge_masses() const {
        SelShared& s = smem();
        const int share = kSplit / C;
        for (int i = threadIdx.x; i < share; i += kSelThreads) {
            const int b = rank * share + i;
            u64 hi = 0, lo = 0;
            for (int r = 0; r < C; ++r) {
                const uint32_t* m = remote(s.mass[0], r) + b;
                hi += upper_words(m, kSplit);
                lo += m[0];
            }
            hi += lo >> 32;
            for (int r = 0; r < C; ++r) {
                uint32_t* m = remote(s.mass_tot[0], r) + b;
                m[0] = static_cast<uint32_t>(lo);
                m[kSplit] = static_cast<uint32_t>(hi);
                m[2 * kSplit] = static_cast<uint32_t>(hi >> 32);
            }
        }
    }
    __device__ void merge_hist() const {
        SelShared& s = smem();
        sync();
        if (C == 1) return;
        merge(s.hist, s.tot, kBins);
        sync();
    }
    // Two sums, a count and (with MAX) the largest value of all CTAs; `before`: sum[0] of the CTAs ahead of this one.
    struct Totals {
        double sum[2], before;
        float top;
        int count, bad;
    };
    template <bool MAX>
    __device__ Totals add_up(double a, double b, int count, float top_, int bad) const {
        SelShared& s = smem();
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        a = warp_sum(a);
        b = warp_sum(b);
        const int c = __reduce_add_sync(0xffffffffu, count);
        if (MAX) {
            for (int o = 16; o > 0; o >>= 1) top_ = fmaxf(top_, __shfl_xor_sync(0xffffffffu, top_, o));
            bad = __reduce_or_sync(0xffffffffu, bad);
        }
        __syncthreads();
        if (lane == 0) {
            s.warp_f64[0][warp] = a;
            s.warp_f64[1][warp] = b;
            s.warp_int[warp] = c;
            if (MAX) s.warp_u64[0][warp] = (static_cast<u64>(bad) << 32) | __float_as_uint(top_);
        }
        __syncthreads();
        if (warp == 0) {                                          // the warps' parts, a lane each
            const bool some = lane < kSelWarps;
            a = warp_sum(some ? s.warp_f64[0][lane] : 0.0);
            b = warp_sum(some ? s.warp_f64[1][lane] : 0.0);
            const int n = __reduce_add_sync(0xffffffffu, some ? s.warp_int[lane] : 0);
            if (MAX) {
                const u64 of = some ? s.warp_u64[0][lane] : static_cast<u64>(__float_as_uint(-INFINITY));
                top_ = __uint_as_float(static_cast<uint32_t>(of));
                for (int o = 16; o > 0; o >>= 1) top_ = fmaxf(top_, __shfl_xor_sync(0xffffffffu, top_, o));
                bad = __reduce_or_sync(0xffffffffu, static_cast<int>(of >> 32));
            }
            if (lane == 0) {
                s.pub[turn].sum[0] = a;
                s.pub[turn].sum[1] = b;
                s.pub[turn].count = n;
                if (MAX) { s.pub[turn].top = top_; s.pub[turn].bad = bad; }
            }
        }
        sync();
        Totals t = {{0.0, 0.0}, 0.0, -INFINITY, 0, 0};
        for (int r = 0; r < C; ++r) {
            const Published* p = remote(&s.pub[turn], r);
            if (r == rank) t.before = t.sum[0];
            t.sum[0] += p->sum[0];
            t.sum[1] += p->sum[1];
            t.count += p->count;
            if (MAX) { t.top = fmaxf(t.top, p->top); t.bad |= p->bad; }
        }
        turn ^= 1;
        return t;
    }
    // The first of n counts, n a multiple of the threads, at which their sum reaches k (k >= 1, no more than the total): s.found = {which,
    // entries before it, entries in it}.
    template <int N>
    __device__ void find_count(const uint32_t* count, int k) const {
        SelShared& s = smem();
        constexpr int kMine = N / kSelThreads;
        const int b0 = threadIdx.x * kMine;
        int sum = 0, total;
        for (int j = 0; j < kMine; ++j) sum += static_cast<int>(count[b0 + j]);
        int before = block_scan(sum, s.warp_int, total);
        if (before < k && before + sum >= k) {
            for (int j = 0; j < kMine; ++j) {
                const int c = static_cast<int>(count[b0 + j]);
                if (before < k && before + c >= k) {
                    s.found[0] = b0 + j;
                    s.found[1] = before;
                    s.found[2] = c;
                }
                before += c;
            }
        }
        __syncthreads();
    }
    // The part in which mass0 plus the masses reach the target: s.found = {part, -, entries in it, whether there is one}, s.found_mass the
    // mass before it.
    __device__ void find_mass(double mass0, double target) const {
        SelShared& s = smem();
        if (threadIdx.x == 0) s.found[3] = 0;
        constexpr int kMine = kSplit / kSelThreads;
        const int b0 = threadIdx.x * kMine;
        const uint32_t* lo_of = masses();
        u64 hi = 0, lo = 0, total;
        for (int j = 0; j < kMine; ++j) {
            hi += upper_words(lo_of + b0 + j, kSplit);
            lo += lo_of[b0 + j];
        }
        hi = block_scan(hi, s.warp_u64[0], total);
        lo = block_scan(lo, s.warp_u64[1], total);
        for (int j = 0; j < kMine; ++j) {
            const double from = mass0 + in_units(hi, lo);
            hi += upper_words(lo_of + b0 + j, kSplit);
            lo += lo_of[b0 + j];
            if (from < target && mass0 + in_units(hi, lo) >= target) {
                s.found[0] = b0 + j;
                s.found[2] = parts()[b0 + j];
                s.found[3] = 1;
                s.found_mass = from;
            }
        }
        __syncthreads();
    }
    // From the merged counts: the bins b1 .. b2 in which the mass can reach the target.  An entry of bin b weighs between e^(-(b + 1/2) / 256)
    // and e^(-(b - 1/2) / 256), but for the rounding of the bin (4e-6) and of the sums here (6e-6): 2e-5 to either side.
    // Without a total the target is p times the sum, which is bounded alike; with it, bins before b0 weigh `mass0` together.
    // s.found = {entries before b1, entries from b1 to b2, b1, b2}.  (Apart: its registers would be taken from the passes around it.)
    static __device__ __noinline__ void bracket(bool one, double p, double total, double mass0, int from) {
        SelShared& s = smem();
        constexpr int kMine = kBins / kSelThreads;
        const int b0 = threadIdx.x * kMine;
        const float step = -1.4426950408889634f / kBinsPerNat;
        const uint4* count = reinterpret_cast<const uint4*>((one ? s.hist : s.tot) + b0);
        // the exponentials of the bins by steps of e^(-1/256) from the thread's first; a thread's sums in fp32 (3e-6 relative, like the steps).
        // Loops that stay loops: code that runs once is fetched once, and 6 KB of it took 3 us.
        const float down = 0.99610137f, first = ex2_approx((b0 - 0.5f) * step);
        auto walk = [&](auto f) {
            float e = first, hs = 0.f, ls = 0.f;
#pragma unroll 1
            for (int j = 0; j < kMine; j += 4) {
                const uint4 four = count[j / 4];
                const uint32_t c4[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int b = b0 + j + k;
                    const float c = b >= from ? static_cast<float>(c4[k]) : 0.f;
                    hs = fmaf(c * 1.00002f, e, hs);
                    e *= down;
                    ls = fmaf(b < kBins - 1 ? c * 0.99998f : 0.f, e, ls);
                    f(hs, ls, b, c4[k]);
                }
            }
        };
        float hs = 0.f, ls = 0.f;
        walk([&](float h, float l, int, uint32_t) { hs = h; ls = l; });
        double h_total, l_total;
        const double h = mass0 + block_scan(static_cast<double>(hs), s.warp_f64[0], h_total);
        const double l = mass0 + block_scan(static_cast<double>(ls), s.warp_f64[1], l_total);
        const double to_lo = p * (total > 0.0 ? total : l_total), to_hi = p * (total > 0.0 ? total : h_total);
        int n = 0;                                                // bins before b1, and (times 2^16) those before b2 + 1
        walk([&](float hj, float lj, int b, uint32_t) {
            n += (b < from || h + static_cast<double>(hj) < to_lo ? 1 : 0) + (b < from || l + static_cast<double>(lj) < to_hi ? 1 << 16 : 0);
        });
        int sum;
        block_scan(n, s.warp_int, sum);
        const int b1 = min(sum & 0xffff, kBins - 1), b2 = min(sum >> 16, kBins - 1);
        u64 entries = 0;                                          // before b1, and (times 2^32) from b1 to b2
        walk([&](float, float, int b, uint32_t c) { entries += b < b1 ? c : b <= b2 ? static_cast<u64>(c) << 32 : 0; });
        u64 all;
        block_scan(entries, s.warp_u64[0], all);
        if (threadIdx.x == 0) {
            s.found[0] = static_cast<int>(all & 0xffffffffu);
            s.found[1] = static_cast<int>(all >> 32);
            s.found[2] = b1;
            s.found[3] = b2;
        }
        __syncthreads();
    }
    // put(place, value, index) for the entries that keep(value, index) takes; places from *counter on, one atomic for those of a chunk (with
    // one for each entry they queue up: 2,000 took 25 us).
    template <typename F, typename G>
    __device__ __forceinline__ void collect(F keep, int* counter, G put) const {
        each<kLight>([&](const float (&v)[kEach], int i, int) { collect_chunk(v, i, keep, counter, put); });
    }
    template <typename F, typename G>
    static __device__ __forceinline__ int collect_chunk(const float (&v)[kEach], int i, F keep, int* counter, G put) {
        unsigned taken = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) taken |= (keep(v[k], i + k) ? 1u : 0u) << k;
        if (taken == 0u) return 0;
        int at = atomicAdd(counter, __popc(taken));
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (taken >> k & 1u) put(at++, v[k], i + k);
        return at;
    }
    // Entries that keep(value, index) takes, 4,096 at most, go to the list of rank 0; only rank 0 has it (and its length).
    template <typename F>
    __device__ int gather(F keep) const {
        SelShared& s = smem();
        sync();                                    // the list shares its place with the counts
        if (threadIdx.x == 0) s.list_n = 0;
        sync();
        u64* list = remote(s.list, 0);
        collect(keep, remote(&s.list_n, 0), [=](int at, float x, int i) {
            if (at < kListCap) list[at] = order_of(x, i);
        });
        sync();
        return rank == 0 ? min(s.list_n, 4096) : 0;
    }
    // Which warp of the CTA that has it owns the entry with this index (see range() and edge()).
    __device__ __forceinline__ int warp_of(int index) const {
        if (index < head) return 0;
        const int c = (index - head) / kEach;
        if (c >= whole) return kSelWarps - 1;
        return (c - c0) / (((c1 - c0 + kSelWarps - 1) / kSelWarps + 31) / 32 * 32);
    }
    __device__ int sort_list(int n) const {
        SelShared& s = smem();
        const int n2 = pow2_from(n);
        if (n <= kRankSort) {                                     // every entry counts those before it
            const u64 o = threadIdx.x < n ? s.list[threadIdx.x] : 0;
            int at = 0;
            for (int i = 0; threadIdx.x < n && i < n; ++i) at += s.list[i] < o;
            __syncthreads();
            if (threadIdx.x < n) s.list[at] = o;
            __syncthreads();
            return n;
        }
        for (int i = n + threadIdx.x; i < n2; i += kSelThreads) s.list[i] = ~0ull;
        __syncthreads();
        block_sort(s.list, n2);
        return n;
    }
    // A value that at least K of the n values val(i) reach, no more than K / 4 + 8 others if no value is given too often; -inf where
    // fewer than K are finite.  Histograms of 512 bins, each over the bin of the K-th value of the one before.
    template <typename F>
    __device__ float bound(F val, int n, int K, float* largest = nullptr) const {
        SelShared& s = smem();
        float lo = INFINITY, hi = -INFINITY;
        auto extend = [&](float& l, float& h) {                   // over the block
            for (int o = 16; o > 0; o >>= 1) {
                l = fminf(l, __shfl_xor_sync(0xffffffffu, l, o));
                h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, o));
            }
            float2* part = reinterpret_cast<float2*>(s.warp_u64[1]);
            __syncthreads();
            if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = make_float2(l, h);
            __syncthreads();
            for (int w = 0; w < kSelWarps; ++w) {
                l = fminf(l, part[w].x);
                h = fmaxf(h, part[w].y);
            }
        };
        for (int i = threadIdx.x; i < n; i += kSelThreads) {
            const float v = val(i);
            if (v > -INFINITY) { lo = fminf(lo, v); hi = fmaxf(hi, v); }
        }
        extend(lo, hi);
        if (largest) *largest = hi;
        int ahead = 0;
        for (int level = 0; level < 5; ++level) {
            const float scale = hi > lo ? fminf(511.9f / (hi - lo), 1e38f) : 0.f;
            static_assert(kSelThreads == 512, "a thread per bin");
            s.small_hist[threadIdx.x] = 0;
            if (threadIdx.x == 0) s.found[0] = -1;
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += kSelThreads) {
                const float v = val(i);
                if (v >= lo && v <= hi) atomicAdd(&s.small_hist[min(static_cast<int>((hi - v) * scale), 511)], 1u);
            }
            __syncthreads();
            const int c = static_cast<int>(s.small_hist[threadIdx.x]);
            int total;
            const int before = ahead + block_scan(c, s.warp_int, total);
            if (before < K && before + c >= K) {
                s.found[0] = threadIdx.x;
                s.found[1] = before;
                s.found[2] = c;
            }
            __syncthreads();
            const int b = s.found[0], reach = s.found[1] + s.found[2];
            if (b < 0) return -INFINITY;
            ahead = s.found[1];
            float l = INFINITY, h = -INFINITY;
            for (int i = threadIdx.x; i < n; i += kSelThreads) {
                const float v = val(i);
                if (v >= lo && v <= hi && min(static_cast<int>((hi - v) * scale), 511) == b) { l = fminf(l, v); h = fmaxf(h, v); }
            }
            extend(l, h);
            lo = l;
            hi = h;
            if (reach <= K + K / 4 + 8 || lo == hi) break;
        }
        return lo;
    }
    static __device__ __forceinline__ float most_of(u64 chunk) { return __uint_as_float(static_cast<uint32_t>(chunk >> 32)); }
    // The n entries of a list that keep(entry) takes, moved together; their number to *counter.
    template <int CAP, typename F>
    static __device__ void compact(u64* list, int n, int* counter, F keep) {
        constexpr int kMine = (CAP + kSelThreads - 1) / kSelThreads;
        u64 o[kMine];
        unsigned taken = 0;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            const int i = threadIdx.x + j * kSelThreads;
            o[j] = i < n ? list[i] : 0;
            taken |= (i < n && keep(o[j]) ? 1u : 0u) << j;
        }
        __syncthreads();
        if (threadIdx.x == 0) *counter = 0;
        __syncthreads();
        if (taken != 0u) {
            int at = atomicAdd(counter, __popc(taken));
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (taken >> j & 1u) list[at++] = o[j];
        }
        __syncthreads();
    }
    // The K largest of the first n entries of the list, sorted; returns their number.
    __device__ int sort_top(int n, int K) const {
        SelShared& s = smem();
        if (n > kRankSort && n > K + K / 4 + 8) {
            const float thr = bound([&](int i) { return value_of(s.list[i]); }, n, K);
            compact<kListCap>(s.list, n, &s.list_n, [=](u64 o) { return value_of(o) >= thr; });
            n = s.list_n;
            __syncthreads();
        }
        return min(sort_list(n), K);
    }
    // The cut inside a group of `count` entries with numbers from `from` to `to`, those that over(f) calls f(value, number) for, in all CTAs: by count, the entry number `want`
    // (from 1) of the group; by mass, the first at which mass0 plus the masses reach `target` (in units of 2^-44), and the last of the
    // group where rounding leaves none.  The range of numbers is divided 1,024 ways, and again the part with the cut, until no more
    // than 256 entries are left; they go to rank 0, where each adds up those before it.
    template <bool MASS, typename Over>
    __device__ u64 cut_in_group(Over over, u64 from, u64 to, int count, int want, double mass0, double target) const {
        SelShared& s = smem();
        for (bool ends = false; count > kFew; ends = true) {
            // the ends of what is left of the group (equal values leave most of a range empty)
            u64 lo = ends ? ~0ull : from, hi = ends ? 0 : to;
            if (ends)
                over([&](float, u64 o) {
                    if (o >= from && o <= to) { lo = min(lo, o); hi = max(hi, o); }
                });
            if (ends)
                for (int o = 16; o > 0; o >>= 1) {
                    lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
                    hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
                }
            __syncthreads();
            if (ends && (threadIdx.x & 31) == 0) { s.warp_u64[0][threadIdx.x >> 5] = lo; s.warp_u64[1][threadIdx.x >> 5] = hi; }
            for (int b = threadIdx.x; b < kSplit; b += kSelThreads) {
                s.part[b] = 0;
                if (MASS) s.mass[0][b] = s.mass[1][b] = s.mass[2][b] = 0;
            }
            __syncthreads();
            if (ends) {
                if (threadIdx.x == 0) {
                    for (int w = 0; w < kSelWarps; ++w) { lo = min(lo, s.warp_u64[0][w]); hi = max(hi, s.warp_u64[1][w]); }
                    s.pub[turn].lo = lo;
                    s.pub[turn].hi = hi;
                }
                sync();
                for (int r = 0; r < C; ++r) {
                    lo = min(lo, remote(&s.pub[turn], r)->lo);
                    hi = max(hi, remote(&s.pub[turn], r)->hi);
                }
                turn ^= 1;
            }
            const int bits = 64 - __clzll(hi - lo);               // (more than 256 numbers: hi > lo)
            const int shift = bits > 10 ? bits - 10 : 0;
            over([&](float x, u64 o) {
                if (o < lo || o > hi) return;
                const int b = static_cast<int>((o - lo) >> shift);
                atomicAdd(&s.part[b], 1u);
                if (MASS) add_mass(&s.mass[0][b], kSplit, mass(x));
            });
            sync();
            if (C > 1) {
                merge(s.part, s.part_tot, kSplit);
                if (MASS) merge_masses();
                sync();
            }
            if (MASS) {
                find_mass(mass0, target);
                if (s.found[3] == 0) return hi;
                mass0 = s.found_mass;
            } else {
                find_count<kSplit>(parts(), want);
                want -= s.found[1];
            }
            count = s.found[2];
            from = lo + (static_cast<u64>(s.found[0]) << shift);
            to = min(hi, from + ((1ull << shift) - 1));
        }
        sync();                                                   // (nobody reads the parts of rank 0 any more)
        if (threadIdx.x == 0) s.list_few = 0;
        sync();
        int* counter = remote(&s.list_few, 0);
        u64* few = remote(s.few, 0);
        over([&](float, u64 o) {
            if (o < from || o > to) return;
            const int at = atomicAdd(counter, 1);
            if (at < kFew) few[at] = o;
        });
        sync();
        if (rank == 0) {
            const int n = min(s.list_few, kFew);
            const u64 o = threadIdx.x < n ? s.few[threadIdx.x] : 0;
            const Mass m = MASS && threadIdx.x < n ? mass(value_of(o)) : Mass{1, 0};
            if (threadIdx.x < n) {
                s.few_hi[threadIdx.x] = m.hi;
                s.few_lo[threadIdx.x] = m.lo;
            }
            if (threadIdx.x == 0) s.pub[turn].lo = n > 0 ? 0 : last_finite();
            __syncthreads();
            if (threadIdx.x < n) {
                u64 before = 0, before_lo = 0;
                bool is_last = true;
                for (int i = 0; i < n; ++i) {
                    const u64 other = s.few[i];
                    if (other < o) {
                        before += s.few_hi[i];
                        before_lo += s.few_lo[i];
                    } else if (other > o) {
                        is_last = false;
                    }
                }
                const double lo = mass0 + in_units(before, before_lo), hi = mass0 + in_units(before + m.hi, before_lo + m.lo);
                const bool cut = MASS ? (lo < target && hi >= target) || (is_last && hi < target) : before + 1 == static_cast<u64>(want);
                if (cut) s.pub[turn].lo = o;
            }
            __syncthreads();
        }
        sync();
        const u64 cut = remote(&s.pub[turn], 0)->lo;
        turn ^= 1;
        return cut;
    }

    __device__ void set_scale(float top_, double inv_t_) {
        top = top_;
        inv_t = inv_t_;
        bins = static_cast<float>(kBinsPerNat * inv_t_);
        weight.set(inv_t, static_cast<double>(top_));
    }
    // This chunk's part in the row's maximum (NaN if there is one) and in the number of its entries of -inf.
    static __device__ __forceinline__ void see(const float (&v)[kEach], int n, float& most, int& missing) {
        float least = v[0];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            most = max_nan(most, v[k]);
            least = fminf(least, v[k]);
        }
        if (least == -INFINITY) {
#pragma unroll
            for (int k = 0; k < kEach; ++k) missing += k < n && v[k] == -INFINITY;
        }
    }
    // The row's maximum, number of finite entries and whether it holds a NaN or +inf.
    __device__ Totals look() const {
        float most = -INFINITY;
        int missing = 0;
        each<kLight>([&](const float (&v)[kEach], int, int n) { see(v, n, most, missing); });
        return extremes(0.0, most, missing);
    }
    // Totals of a pass that has seen all of this thread's chunks.
    __device__ Totals extremes(double sum, float most, int missing) const {
        Totals t = add_up<true>(sum, 0.0, missing, isnan(most) ? -INFINITY : most, most < INFINITY ? 0 : 1);
        t.count = V - t.count;
        return t;
    }
    // Histogram of the row, merged; with SUM also the fp32 sum of its exponentials about `top` (this thread's part).
    template <bool SUM>
    __device__ double histogram() const {
        SelShared& s = smem();
        const float c = static_cast<float>(1.4426950408889634 * inv_t);
        clear_hist();
        double full = 0.0;
        each<kLight>([&](const float (&v)[kEach], int, int) {
            float f = 0.f;
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                if (v[k] > -INFINITY) atomicAdd(&s.hist[bin(v[k])], 1u);
                if (SUM) f += ex2_approx((v[k] - top) * c);
            }
            if (SUM) full += static_cast<double>(f);
        });
        merge_hist();
        return full;
    }

    // The K largest entries by one pass: rank 0 gets them sorted in s.list and returns their number, and the fp32 sum of exponentials
    // about `ref`, the largest entry of a slice's first tile that has one, in `full` (all threads of all CTAs).  -1: a list overflowed, or the
    // sum says that the row needs a closer look.
    // What the pass lists is chunks, by their largest entry (a tenth of the instructions that listing entries takes; 613 x 151936
    // bf16, K = 64: 94 -> 78 us); the K-th largest of them bounds the K-th entry from below as well.
    // 2,048 x 126464 fp32, K = 128: 248 us, 4.2 TB/s; 512 x 262144 fp16, K = 50: 88 us, 3.1 TB/s, bound by instructions and barriers: 15 instructions
    // per 32 of the 16-bit entries (20 with the entries listed), of which the loop over the tiles has six or so, bounds and sorting the rest.
    __device__ int stream_top(int K, double inv_t_, float& ref, double& full) const {
        SelShared& s = smem();
        constexpr int kTile = kSelThreads * kDeep;
        const float c = static_cast<float>(1.4426950408889634 * inv_t_);
        const int n = c1 - c0;
        if (threadIdx.x == 0) s.list_n = s.list_few = 0;
        __syncthreads();
        uint4 raw[kDeep];
        float thr = -INFINITY;
        ref = -INFINITY;
        full = 0.0;
        bool overflow = false;
        int first = 0;                                            // the first tile with an entry above -inf
#pragma unroll
        for (int j = 0; j < kDeep; ++j) raw[j] = chunk(c0 + j * kSelThreads + threadIdx.x, c1);
        if (n > 0) {
            // Groups: the entries of a thread's first and of its last loads, of a thread, or of two threads.  Tiles of nothing but -inf are
            // passed over: neither a bound nor a reference for the sum comes from them (a NaN stops the search and goes on into the sum).
            float half[2];
#pragma unroll 1
            for (;; first += kTile) {
                half[0] = half[1] = -INFINITY;
#pragma unroll
                for (int j = 0; j < kDeep; ++j) {
                    float v[kEach];
                    Elem<T>::unpack(raw[j], v);
#pragma unroll
                    for (int k = 0; k < kEach; ++k) half[j / (kDeep / 2)] = max_nan(half[j / (kDeep / 2)], v[k]);
                }
                if (__syncthreads_or(max_nan(half[0], half[1]) != -INFINITY) || first + kTile >= n) break;
#pragma unroll
                for (int j = 0; j < kDeep; ++j) raw[j] = chunk(c0 + first + (kDeep + j) * kSelThreads + threadIdx.x, c1);
            }
            float both = fmaxf(half[0], half[1]);
            int groups;
            if (K > kSelThreads / 2) {
                groups = 2 * kSelThreads;
                s.group_max[2 * threadIdx.x] = half[0];
                s.group_max[2 * threadIdx.x + 1] = half[1];
            } else if (K > kSelThreads / 8) {
                groups = kSelThreads;
                s.group_max[threadIdx.x] = both;
            } else {
                groups = kSelThreads / 2;
                both = fmaxf(both, __shfl_xor_sync(0xffffffffu, both, 1));
                if ((threadIdx.x & 1) == 0) s.group_max[threadIdx.x / 2] = both;
            }
            __syncthreads();
            thr = bound([&](int i) { return s.group_max[i]; }, groups, K, &ref);
        }
        if (ref == -INFINITY) {                                   // nothing but the ends of the row, if they
            float v[kEach];
            int i;
            __syncthreads();
            if (threadIdx.x < 2) s.group_max[threadIdx.x] = -INFINITY;
            __syncthreads();
            if ((threadIdx.x & 31) == 0)
                for (int tail = 0; tail < 2; ++tail)
                    if (edge(tail != 0, threadIdx.x >> 5, v, i))
                        for (int k = 0; k < kEach; ++k) s.group_max[tail] = fmaxf(s.group_max[tail], v[k]);
            __syncthreads();
            ref = fmaxf(s.group_max[0], s.group_max[1]);
        }
        const bool some = ref > -INFINITY;                        // of this slice (a tile of NaN alone leaves a reference of 0, and a sum of NaN)
        if (!(fabsf(ref) < INFINITY)) ref = 0.f;
        // a chunk whose largest entry is above `above`: its place in the list
        auto push = [&](float most, int at_chunk) {
            const int at = atomicAdd(&s.list_n, 1);
            if (at < kChunkCap) s.chunks[at] = (static_cast<u64>(__float_as_uint(most)) << 32) | static_cast<uint32_t>(at_chunk);
            return at;
        };
        // 2^(v c + shift) with one multiply-add; the rounding of shift (and that of c, for values near ref) is taken back at the end
        const float shift = -ref * c;
        auto ends = [&](bool tail, float above) {                 // the entries outside the whole chunks: chunk -1, chunk `whole`
            float v[kEach], f = 0.f, m = -INFINITY;
            int i;
            if ((threadIdx.x & 31) != 0 || !edge(tail, threadIdx.x >> 5, v, i)) return;
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                m = fmaxf(m, v[k]);
                f += ex2_approx(fmaf(v[k], c, shift));
            }
            if (m > above) push(m, tail ? whole : -1);
            full += static_cast<double>(f);
        };
        // (>= in the tile whose entries gave the bound; later ones of the same value come after K entries in the order)
        const float first_above = thr > -INFINITY ? nextafterf(thr, -INFINITY) : -INFINITY;
        ends(false, first_above);
        int limit = min(max(512, 4 * K), kChunkPrune);
#pragma unroll 1
        for (int t0 = first; t0 < n; t0 += kTile) {
            int pushed = 0;
            float f = 0.f;
            const float above = t0 == first ? first_above : thr;
#pragma unroll
            for (int j = 0; j < kDeep; ++j) {
                float v[kEach];
                Elem<T>::unpack(raw[j], v);
                raw[j] = chunk(c0 + t0 + (kDeep + j) * kSelThreads + threadIdx.x, c1);
                float m = v[0];
#pragma unroll
                for (int k = 1; k < kEach; ++k) m = fmaxf(m, v[k]);
                if (m > above) pushed = push(m, c0 + t0 + j * kSelThreads + threadIdx.x);
#pragma unroll
                for (int k = 0; k < kEach; ++k) f += ex2_approx(fmaf(v[k], c, shift));
            }
            full += static_cast<double>(f);
            if (t0 + kTile >= n) break;
            // a tighter bound each time the list has doubled
            if (__syncthreads_or(pushed >= limit)) {
                const int have = s.list_n;                        // (nobody adds to it here)
                if (have > kChunkCap) { overflow = true; break; }
                __syncthreads();
                if (have > K) thr = fmaxf(thr, bound([&](int i) { return most_of(s.chunks[i]); }, have, K));
                if (have > kChunkPrune) compact<kChunkCap>(s.chunks, have, &s.list_n, [=](u64 o) { return most_of(o) >= thr; });
                limit = min(2 * s.list_n, kChunkPrune);
                __syncthreads();
            }
        }
        ends(true, thr);
        full *= exp2(-(static_cast<double>(ref) * static_cast<double>(c) + static_cast<double>(shift)));
        __syncthreads();
        const int listed = s.list_n;
        overflow |= listed > kChunkCap;
        if (!overflow) {
            // the entries of the listed chunks that reach the last bound
            if (listed > K) thr = fmaxf(thr, bound([&](int i) { return most_of(s.chunks[i]); }, listed, K));
            for (int q = threadIdx.x; q < listed; q += kSelThreads) {
                const u64 entry = s.chunks[q];
                if (most_of(entry) < thr) continue;
                const int at_chunk = static_cast<int>(static_cast<uint32_t>(entry));
                float v[kEach];
                int i = 0;
                if (at_chunk >= 0 && at_chunk < whole) {
                    Elem<T>::unpack(chunk(at_chunk, whole), v);
                    i = first_index(at_chunk);
                } else {
                    const int m = at_chunk < 0 ? head : V;        // where these entries end
                    if (at_chunk >= 0) i = first_index(whole);
#pragma unroll
                    for (int k = 0; k < kEach; ++k) v[k] = i + k < m ? to_f32(x[i + k]) : -INFINITY;
                }
                collect_chunk(v, i, [=](float value, int) { return value >= thr && value > -INFINITY; }, &s.list_few, [&](int at, float value, int index) {
                    if (at < kListCap) s.list[at] = order_of(value, index);
                });
            }
            __syncthreads();
            overflow = s.list_few > kListCap;
        }
        const int mine = overflow ? -1 : sort_top(s.list_few, K);
        if (C == 1) return mine;
        // the K largest of every slice, sorted together by rank 0
        if (threadIdx.x == 0) { s.pub[turn].count = mine; s.pub[turn].top = some ? ref : -INFINITY; }
        sync();
        int at = 0, all = 0;
        float most = -INFINITY;
        for (int r = 0; r < C; ++r) {
            const int k = remote(&s.pub[turn], r)->count;
            if (k < 0) overflow = true;
            if (r < rank) at += k;
            all += k;
            most = fmaxf(most, remote(&s.pub[turn], r)->top);
        }
        // every CTA's sum about the largest reference (one without an entry has 0, or NaN)
        if (most == -INFINITY) most = 0.f;
        if (some) full *= exp2((static_cast<double>(ref) - static_cast<double>(most)) * static_cast<double>(c));
        ref = most;
        turn ^= 1;
        if (!overflow && rank != 0) {
            u64* list = remote(s.list, 0) + at;
            for (int i = threadIdx.x; i < mine; i += kSelThreads) list[i] = s.list[i];
        }
        sync();
        if (overflow) return -1;
        return rank != 0 ? 0 : sort_top(all, K);
    }
};

// Is a row with these parameters done in one pass (but for what one pass finds to be too much)?
__host__ __device__ inline bool one_pass(int k, float p, float m) { return k > 0 ? k <= kMaxTopLogits : p >= 1.f && !(m > 0.f); }

// The first min(k, n) entries of the sorted list in rank 0: masses ahead of every entry give top-p, the value min-p; then the token by
// the masses in the order of the indices.
template <typename T, typename Write>
__device__ void draw_from_list(Row<T>& r, int n, float p, float m, float u, Write write) {
    SelShared& s = smem();
    constexpr int kMine = kMaxTopLogits / kSelThreads;
    r.set_scale(value_of(s.list[0]), r.inv_t);
    u64* w_of = s.list_mass;
    auto mass = [&](float v) { return __double2ull_rn(r.weight(s.exp2_table, v) * kListOne); };
    u64 w[kMine], mine = 0, total;
    const int i0 = threadIdx.x * kMine;
    for (int j = 0; j < kMine; ++j) mine += w[j] = i0 + j < n ? mass(value_of(s.list[i0 + j])) : 0;
    u64 cum = block_scan(mine, s.warp_u64[0], total);
    const double target = static_cast<double>(p) * static_cast<double>(total), md = m;
    int kept = 0;
    for (int j = 0; j < kMine; ++j) {
        const int i = i0 + j;
        if (i < n && (i == 0 || ((p >= 1.f || static_cast<double>(cum) < target) && (!(m > 0.f) || value_of(s.list[i]) == r.top || r.weight(s.exp2_table, value_of(s.list[i])) >= md)))) ++kept;
        cum += w[j];
    }
    int n_kept;
    block_scan(kept, s.warp_int, n_kept);
    mine = 0;
    for (int j = 0; j < kMine; ++j) {
        w_of[i0 + j] = w[j];
        if (i0 + j < n_kept) mine += w[j];
    }
    block_scan(mine, s.warp_u64[0], total);
    const u64 t = __double2ull_rd(static_cast<double>(u) * static_cast<double>(total));
    __syncthreads();
    for (int i = threadIdx.x; i < n_kept; i += kSelThreads) {
        const int v = index_of(s.list[i]);
        u64 c = 0;
        for (int j = 0; j < n_kept; ++j)
            if (index_of(s.list[j]) < v) c += w_of[j];
        if (c <= t && t < c + w_of[i]) write(s.list[i], log(static_cast<double>(total) / kListOne), n_kept);
    }
}

// The end of a row, by every thread: no CTA leaves while another of its cluster may still read what it has published.
__device__ __forceinline__ void leave_row(int cluster) {
    if (cluster > 1) cg::this_cluster().sync();
}

template <typename T>
__device__ __forceinline__ void sample_row(const SelectArgs& a) {
    SelShared& s = smem();
    const int64_t row = blockIdx.x / a.cluster;
    Row<T> r(a, row, static_cast<int>(blockIdx.x % a.cluster));
    constexpr int kEach = Row<T>::kEach;
    auto neutral = [&](uint32_t flag) {
        if (r.rank != 0 || threadIdx.x != 0) return;
        a.tokens[row] = -1;
        if (a.lp) a.lp[row] = 0.f;
        if (a.lp_full) a.lp_full[row] = 0.f;
        if (a.n_kept) a.n_kept[row] = 0;
        if (flag && a.status) atomicOr(a.status, flag);
    };
    const bool first_kind = a.rows_of != kManyPasses;             // (rows that give nothing are of the first)
    if (a.mask && a.mask[row] == 0) return first_kind ? neutral(0u) : void();
    float temperature = a.how.temperature_rows ? a.how.temperature_rows[row] : a.how.temperature;
    int k = a.how.top_k_rows ? a.how.top_k_rows[row] : a.how.top_k;
    const float p = a.how.top_p_rows ? a.how.top_p_rows[row] : a.how.top_p;
    const float m = a.how.min_p_rows ? a.how.min_p_rows[row] : a.how.min_p;
    const float u = a.u[row];
    // (each comparison is false for a NaN)
    if (!usable_temperature(temperature) || !(p >= 0.f) || !(m <= 1.f) || !(u >= 0.f && u < 1.f)) return first_kind ? neutral(AIS_FLAG_PARAM) : void();
    if (temperature == 0.f) {
        temperature = 1.f;
        k = 1;
    }
    // a top-k of everything is none, unless it makes the whole of a short row the list that the other filters work on
    if (a.V > kMaxTopLogits) {
        if (k >= a.V) k = 0;
    } else if (k > a.V || (k <= 0 && (p < 1.f || m > 0.f))) {
        k = a.V;
    }
    if (a.rows_of != kAllRows && one_pass(k, p, m) != first_kind) return;
    {
        const double e = exp2((threadIdx.x >> 3) / 64.0);
        static_assert(kSelThreads == 64 * 8 && kTableCopies == 16, "eight threads write the copies of an entry");
        s.exp2_table[2 * threadIdx.x] = e;
        s.exp2_table[2 * threadIdx.x + 1] = e;
    }
    __syncthreads();
    r.inv_t = 1.0 / static_cast<double>(temperature);
    const bool by_p = p < 1.f, by_m = m > 0.f;
    const double pd = p, md = m, ud = u;
    // what a row gives: log_full and log_total are relative to `about`
    float about = 0.f;
    double log_full = 0.0;
    auto write = [&](u64 o, double log_total, int kept) {
        const double x = static_cast<double>(value_of(o));
        a.tokens[row] = index_of(o);
        if (a.lp) a.lp[row] = static_cast<float>((x - static_cast<double>(r.top)) * r.inv_t - log_total);
        if (a.lp_full) a.lp_full[row] = static_cast<float>((x - static_cast<double>(about)) * r.inv_t - log_full);
        if (a.n_kept) a.n_kept[row] = kept;
    };

    if (k > 0 && k <= kMaxTopLogits && k * r.C <= 4096) {
        double full;
        const int n = r.stream_top(k, r.inv_t, about, full);
        const double all = r.template add_up<false>(full, 0.0, 0, 0.f, 0).sum[0];
        if (n >= 0 && all > 0.0 && all < INFINITY) {
            if (r.rank != 0) return;
            log_full = log(all);
            return draw_from_list(r, n, p, m, u, write);
        }
    }

    typename Row<T>::Totals t;
    u64 cut = last_finite();
    int kept = 0;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (k <= 0 && !by_p && !by_m) {
        // Everything is kept: the sums about 0, or about the maximum where that leaves the range of fp64.
        double about_d = 0.0;
        for (int again = 0;; ++again) {
            r.weight.set(r.inv_t, about_d);
            double sum = 0.0;
            float most = -INFINITY;
            int missing = 0;
            r.template each<Row<T>::kHeavy>([&](const float (&v)[kEach], int, int n) {
                r.see(v, n, most, missing);
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    const double w = r.weight.of(s.exp2_table, fmaxf(v[j], r.weight.floor));
                    if (v[j] >= r.weight.floor) sum += w;
                }
            });
            const double of_warp = warp_sum(sum);
            if (lane == 0) s.warp_kept[warp] = of_warp;
            t = r.extremes(sum, most, missing);
            if (again || t.bad || t.top == -INFINITY || fabs(t.top * r.inv_t) < 600.0) break;
            about_d = t.top;
        }
        if (t.bad || t.top == -INFINITY) return neutral(t.bad ? AIS_FLAG_NONFINITE : AIS_FLAG_EMPTY);
        about = r.top = static_cast<float>(about_d);
        log_full = log(t.sum[0]);
        kept = t.count;
    } else {
        t = r.look();
        if (t.bad || t.top == -INFINITY) return neutral(t.bad ? AIS_FLAG_NONFINITE : AIS_FLAG_EMPTY);
        r.set_scale(t.top, r.inv_t);
        about = t.top;
        const bool by_k = k > 0 && k < t.count;
        double full = 0.0;                                        // sum of all exponentials (this thread's part)
        if (by_k) full = r.template histogram<true>();
        else if (by_p) r.template histogram<false>();
        // is an entry ahead of the cut, or it
        float cut_value = value_of(cut);
        int cut_index = index_of(cut);
        auto inside = [&](float x, int i) { return x > cut_value || (x == cut_value && i <= cut_index); };
        // the entries of the slice that pick(value, index) takes, as cut_in_group wants them
        auto data = [&](auto pick) {
            return [&r, pick](auto f) {
                r.template each<Row<T>::kLight>([&](const float (&v)[kEach], int i, int) {
                    unsigned taken = 0;
#pragma unroll
                    for (int j = 0; j < kEach; ++j) taken |= (pick(v[j], i + j) ? 1u : 0u) << j;
                    if (taken == 0u) return;
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
                        if (taken >> j & 1u) f(v[j], order_of(v[j], i + j));
                });
            };
        };
        if (by_k) {
            r.template find_count<kBins>(r.counts(), k);
            const int b = s.found[0], ahead = s.found[1], in = s.found[2];
            __syncthreads();
            const bool listed = k <= kMaxTopLogits && ahead + in <= 4096;
            if (!listed) cut = r.template cut_in_group<false>(data([&](float x, int) { return x > -INFINITY && r.bin(x) == b; }), order_of(r.top, 0), last_finite(), in,
                                                                 k - ahead, 0.0, 0.0);
            if (k <= kMaxTopLogits) {
                log_full = log(r.template add_up<false>(full, 0.0, 0, 0.f, 0).sum[0]);
                const int n = r.gather([&](float x, int i) { return listed ? x > -INFINITY && r.bin(x) <= b : order_of(x, i) <= cut; });
                if (r.rank != 0) return;
                return draw_from_list(r, r.sort_top(n, k), p, m, u, write);
            }
            cut_value = value_of(cut);
            cut_index = index_of(cut);
        }
        double above = 0.0;                                       // kept mass (this thread's part)
        bool counted = false;                                     // kept holds the entries that `above` and the lists sum up
        if (threadIdx.x < 3 * kSelWarps) s.warp_listed[0][threadIdx.x] = 0;
        if (by_p) {
            if (by_k) {                                           // the histogram of what top-k has left
                __syncthreads();
                r.clear_hist();
                r.template each<Row<T>::kLight>([&](const float (&v)[kEach], int i, int) {
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
                        if (inside(v[j], i + j)) atomicAdd(&s.hist[r.bin(v[j])], 1u);
                });
                r.merge_hist();
            }
            // the cut lies in none of the bins before b1 and none behind b2
            r.bracket(r.C == 1, pd, 0.0, 0.0, 0);
            const int before = s.found[0], b1 = s.found[2], b2 = s.found[3];
            __syncthreads();
            // one pass for the total and for the mass before b1
            const float from_value = r.edge_value(b1);            // values above it lie in the bins before b1
            double all = 0.0;
            auto add = [&](auto limited) {
                r.template each<Row<T>::kHeavy>([&](const float (&v)[kEach], int i, int) {
#pragma unroll
                    for (int j = 0; j < kEach; ++j) {
                        bool in = v[j] >= r.weight.floor;
                        if constexpr (decltype(limited)::value) in = in && inside(v[j], i + j);
                        const double w = r.weight.of(s.exp2_table, fmaxf(v[j], r.weight.floor));
                        if (in) all += w;
                        if (in && v[j] > from_value) above += w;
                    }
                });
            };
            if (by_k) add(std::true_type());
            else add(std::false_type());
            t = r.template add_up<false>(all, above, 0, 0.f, 0);
            if (!by_k) full = all;                                // (there is no fp32 sum)
            const double target = pd * t.sum[0], mass_b1 = t.sum[1];
            if (target <= 0.0) {
                cut = order_of(r.top, (1 << kIndexBits) - 1);     // p = 0: the largest value
            } else {
                // with the two sums the counts say more: the cut is in none of the bins behind c2
                r.bracket(r.C == 1, pd, t.sum[0], mass_b1, b1);
                const int c2 = s.found[3], between = s.found[0] + s.found[1] - before;
                const float to_value = min(b2, c2) < kBins - 1 ? r.edge_value(min(b2, c2) + 1) : -INFINITY;
                auto open = [&](float x, int i) { return x <= from_value && x > to_value && (!by_k || inside(x, i)); };
                __syncthreads();
                if (between <= 2 * kListCap) {
                    // every CTA lists its entries from b1 on
                    if (threadIdx.x == 0) s.list_n = 0;
                    __syncthreads();
                    r.collect(open, &s.list_n, [&](int at, float, int i) { s.indices[at] = i; });
                    __syncthreads();
                    const int n = s.list_n;
                    auto listed = [&](auto f) {
#pragma unroll 4
                        for (int i = threadIdx.x; i < n; i += kSelThreads) {
                            const int at = s.indices[i];
                            const float x = to_f32(r.x[at]);
                            f(x, order_of(x, at));
                        }
                    };
                    cut = r.template cut_in_group<true>(
                        listed, order_of(from_value, 0), to_value > -INFINITY ? order_of(to_value, 0) - 1 : last_finite(), between, 0, mass_b1 * kMassOne,
                        target * kMassOne);
                    if (!by_m) {
                        counted = true;
                        listed([&](float x, u64 o) {
                            if (o > cut) return;
                            add_mass(&s.warp_listed[0][r.warp_of(index_of(o))], kSelWarps, r.mass(x));
                            ++kept;
                        });
                        if (r.rank == 0 && threadIdx.x == 0) kept += before;
                    }
                } else {
                    cut = r.template cut_in_group<true>(data(open), order_of(from_value, 0), to_value > -INFINITY ? order_of(to_value, 0) - 1 : last_finite(),
                                                        between, 0, mass_b1 * kMassOne, target * kMassOne);
                }
            }
            cut_value = value_of(cut);
            cut_index = index_of(cut);
        }
        if (!counted) {
            above = 0.0;
            const double m_from = by_m ? static_cast<double>(r.top) + log(md) / r.inv_t : 0.0;
            const float m_floor = by_m ? static_cast<float>(m_from - 1e-6 * (fabs(static_cast<double>(r.top)) + fabs(m_from)) - 1e-30) : -INFINITY;
            const float c = static_cast<float>(1.4426950408889634 * r.inv_t);
            const bool sum_full = !by_k && !by_p;
            r.template each<Row<T>::kHeavy>([&](const float (&v)[kEach], int i, int) {
                float f = 0.f;
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    if (sum_full) f += ex2_approx((v[j] - r.top) * c);
                    if (!(v[j] >= m_floor) || !inside(v[j], i + j)) continue;
                    const double w = r.weight(s.exp2_table, v[j]);
                    if (by_m && w < md && v[j] != r.top) continue;
                    above += w;
                    ++kept;
                }
                if (sum_full) full += static_cast<double>(f);
            });
        }
        __syncthreads();
        const double of_warp = warp_sum(above) + in_units(upper_words(&s.warp_listed[0][warp], kSelWarps), s.warp_listed[0][warp]) / kMassOne;
        if (lane == 0) s.warp_kept[warp] = of_warp;
        t = r.template add_up<false>(lane == 0 ? of_warp : 0.0, full, kept, 0.f, 0);
        log_full = log(t.sum[1]);
        kept = t.count;
        if (by_p && p == 0.f) {                                   // ties of the largest value: the first of them alone
            kept = 1;
            t.sum[0] = 1.0;
        }
    }
    // The token: the CTA, the warp's range, a sixteenth of that and the entry at which the kept mass exceeds u times its total.  Sums of
    // the same terms in another order may differ in their last bits, so the last candidate of each step takes what is left.
    const bool first_only = by_p && p == 0.f;
    const double want = first_only ? 0.0 : ud * t.sum[0];
    constexpr double kNone = 1e-290;                              // (entries of -inf may add up to a little less than that)
    auto choose = [&](const double* sums, double left) {          // one warp, a lane per sum
        const double of = lane < kSelWarps && sums[lane] > kNone ? sums[lane] : 0.0, until = warp_scan(of);
        const unsigned some = __ballot_sync(0xffffffffu, of > 0.0), hit = __ballot_sync(0xffffffffu, of > 0.0 && left < until);
        const int chosen = hit != 0u ? __ffs(hit) - 1 : 31 - __clz(some);
        if (lane == 0) s.found[0] = chosen;
        if (lane == chosen) s.found_mass = left - (until - of);
    };
    if (warp == 0) {
        const double mine = s.pub[r.turn ^ 1].sum[0];
        // (t.before of the next CTA is this one's t.before + mine, the same sum: one CTA takes it)
        if (want >= t.before && mine > kNone && want < t.before + mine) choose(s.warp_kept, want - t.before);
        else if (lane == 0) s.found[0] = -1;
    }
    __syncthreads();
    const int owner = s.found[0];
    if (owner < 0) return;
    double left = s.found_mass;
    const float cut_value = value_of(cut), m_top = r.top;
    const int cut_index = index_of(cut);
    int from, to;
    r.range(owner, from, to);
    // the chunks of the range in steps of 32, its head and tail as steps of their own; the weights of a step
    const int steps = (to - from + 31) / 32 + 2, share = (steps + kSelWarps - 1) / kSelWarps;
    auto step = [&](int n, float (&v)[kEach], int& i, double (&w)[kEach]) {
        if (n == 0 || n == steps - 1) {
            r.edge(n != 0, owner, v, i);
            if (lane > 0) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) v[j] = -INFINITY;
            }
        } else {
            const int c = from + (n - 1) * 32 + lane;
            Elem<T>::unpack(r.chunk(c, to), v);
            i = r.first_index(c);
        }
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const bool in = v[j] > cut_value || (v[j] == cut_value && i + j <= cut_index);
            w[j] = in ? r.weight(s.exp2_table, v[j]) : 0.0;
            if (by_m && w[j] < md && v[j] != m_top) w[j] = 0.0;
            sum += w[j];
        }
        return sum;
    };
    const int n0 = warp * share, n1 = min(n0 + share, steps);
    float v[kEach];
    double w[kEach], sum = 0.0;
    int i;
    for (int n = n0; n < n1; ++n) sum += step(n, v, i, w);
    sum = warp_sum(sum);
    __syncthreads();
    if (lane == 0) s.warp_f64[0][warp] = sum;
    __syncthreads();
    if (warp == 0) choose(s.warp_f64[0], left);
    __syncthreads();
    if (s.found[0] != warp) return;
    left = s.found_mass;
    u64 last = ~0ull;                                             // the last entry with a mass (per lane)
    for (int n = n0; n < n1; ++n) {
        sum = step(n, v, i, w);
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (w[j] > 0.0) last = order_of(v[j], i + j);
        const double inc = warp_scan(sum);
        const unsigned hit = __ballot_sync(0xffffffffu, inc > left);
        if (hit) {
            if (lane == __ffs(hit) - 1) {
                double c = inc - sum;
                u64 o = ~0ull;
#pragma unroll
                for (int j = 0; j < kEach; ++j) {                 // the first whose sum exceeds what is left
                    c += w[j];
                    if (o == ~0ull && w[j] > 0.0 && c > left) o = order_of(v[j], i + j);
                }
                write(o == ~0ull ? last : o, log(t.sum[0]), kept);
            }
            return;
        }
        left -= __shfl_sync(0xffffffffu, inc, 31);
    }
    // (rounding: the last entry of all; a later step is a later index, and so is a later lane)
    const int index = last == ~0ull ? -1 : index_of(last);
    if (index == __reduce_max_sync(0xffffffffu, index) && index >= 0) write(last, log(t.sum[0]), kept);
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads, 2) sample_kernel(const __grid_constant__ SelectArgs a) {
    if (!a.late) pdl_wait();
    pdl_trigger();
    sample_row<T>(a);
    leave_row(a.cluster);
    if (a.late) pdl_wait();
}

template <typename T>
__device__ __forceinline__ void top_row(const SelectArgs& a) {
    SelShared& s = smem();
    const int64_t row = blockIdx.x / a.cluster;
    Row<T> r(a, row, static_cast<int>(blockIdx.x % a.cluster));
    auto write = [&](int n, float lse) {                          // n entries of the list, and padding
        for (int i = threadIdx.x; i < a.K; i += kSelThreads) {
            a.ids[row * a.ld_out + i] = i < n ? index_of(s.list[i]) : -1;
            a.values[row * a.ld_out + i] = i < n ? value_of(s.list[i]) : -INFINITY;
        }
        if (threadIdx.x == 0 && a.lse) a.lse[row] = lse;
    };
    auto neutral = [&](uint32_t flag, float lse) {
        if (r.rank != 0) return;
        write(0, lse);
        if (threadIdx.x == 0 && flag && a.status) atomicOr(a.status, flag);
    };
    if (a.mask && a.mask[row] == 0) return neutral(0u, 0.f);
    r.inv_t = 1.0 / static_cast<double>(a.tau);
    if (a.K * r.C <= 4096) {
        float about;
        double full;
        const int n = r.stream_top(a.K, r.inv_t, about, full);
        const double all = r.template add_up<false>(full, 0.0, 0, 0.f, 0).sum[0];
        if (n >= 0 && all > 0.0 && all < INFINITY) {
            if (r.rank == 0) write(n, static_cast<float>(static_cast<double>(about) * r.inv_t + log(all)));
            return;
        }
    }
    const typename Row<T>::Totals t = r.look();
    if (t.bad) return neutral(AIS_FLAG_NONFINITE, NAN);
    if (t.top == -INFINITY) return neutral(AIS_FLAG_EMPTY, -INFINITY);
    r.set_scale(t.top, r.inv_t);
    const double full = r.template add_up<false>(r.template histogram<true>(), 0.0, 0, 0.f, 0).sum[0];
    const int k = min(a.K, t.count);
    r.template find_count<kBins>(r.counts(), k);
    const int b = s.found[0], ahead = s.found[1], in = s.found[2];
    __syncthreads();
    const bool listed = ahead + in <= 4096;
    u64 cut = 0;
    if (!listed)
        cut = r.template cut_in_group<false>(
            [&](auto f) {
                r.template each<Row<T>::kLight>([&](const float (&v)[Row<T>::kEach], int i, int) {
#pragma unroll
                    for (int j = 0; j < Row<T>::kEach; ++j)
                        if (v[j] > -INFINITY && r.bin(v[j]) == b) f(v[j], order_of(v[j], i + j));
                });
            },
            order_of(r.top, 0), last_finite(), in, k - ahead, 0.0, 0.0);
    int n = r.gather([&](float x, int i) { return listed ? x > -INFINITY && r.bin(x) <= b : order_of(x, i) <= cut; });
    if (r.rank == 0) n = r.sort_top(n, k);
    if (r.rank == 0) write(min(n, k), static_cast<float>(static_cast<double>(r.top) * r.inv_t + log(full)));
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads, 2) top_logits_kernel(const __grid_constant__ SelectArgs a) {
    pdl_enter();
    top_row<T>(a);
    leave_row(a.cluster);
}

template <typename K>
cudaError_t launch_select(K kernel, SelectArgs& a, int64_t rows, int es, cudaStream_t stream, int forced /* CTAs per row at least, if the row is long enough */ = 0) {
    // More CTAs per row while all of them still run at once, two per SM, and a slice keeps 16 KB.  Not beyond: each has 20 to 50 us of
    // barriers, merging and instruction fetches of its own (613 rows of 151936 bf16, K = 64: one CTA 78 us, two 104, four 189; 256 rows with
    // top-p 175, 225, 304; unfiltered 66, 71, 80).
    int c = 1;
    while (c < kMaxCluster && rows * c * 2 <= 2 * 148 && static_cast<int64_t>(a.V) * es >= static_cast<int64_t>(c) * 2 * 16384) c *= 2;
    if (forced > 0)
        for (; c < forced && static_cast<int64_t>(a.V) * es >= static_cast<int64_t>(c) * 2 * 16384; c *= 2) {}
    a.cluster = c;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * c));
    cfg.blockDim = dim3(kSelThreads);
    cfg.dynamicSmemBytes = sizeof(SelShared);
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
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(SelShared)));
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
    auto launch = [&](int forced) {
        return dtype == AIS_BF16  ? launch_select(sample_kernel<__nv_bfloat16>, a, rows, 2, s, forced)
               : dtype == AIS_F16 ? launch_select(sample_kernel<__half>, a, rows, 2, s, forced)
                                  : launch_select(sample_kernel<float>, a, rows, 4, s, forced);
    };
    // Rows with filters of their own: those that need several passes get two CTAs each at least, in a launch of their own that the others
    // overlap.  The host does not see how many they are, and the rule is made for few of them.  151936 bf16, top-p 0.95 in an eighth, in half and
    // in all of the rows, two CTAs against one: 256 rows 135, 170, 225 us against 165, 187, 175; 512 rows 202, 314, 401 against 260, 262, 347.  A
    // batch whose rows all take one pass pays 2 to 7 us for the launch that finds nothing to do (64 to 512 rows).
    cudaError_t e = cudaSuccess;
    if (how->top_k_rows || how->top_p_rows || how->min_p_rows) {
        a.rows_of = kManyPasses;
        e = launch(2);
        a.rows_of = kOnePass;
        a.late = 1;
    }
    if (e == cudaSuccess) e = launch(0);
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
