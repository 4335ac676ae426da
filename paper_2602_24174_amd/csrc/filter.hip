// Sampling under top-k, top-p and min-p from given random numbers, and the same filters as masked logits.
//
// A row's tokens in the order of their logits (equal ones by index) are whole numbers of 56 bits, `comp`: the logit's bits, turned so that
// the largest comes first, over the index.  Every filter keeps a prefix of that order, so all of them together come to one last comp, `cut`.
//
// k_filter_parts reads every logit once: the largest, the sum of the weights where it is wanted, and a list of those above a bound that it takes from a
// sample, some 768 of a row.  k_filter_finish, a workgroup a row, puts the lists together, and mostly the cut lies in them: the row is done.  Rows whose
// cut does not (flat distributions: thousands of tokens kept) it lists for three kernels: k_filter_bins counts their logits by 2048 ranges, part by part; in
// k_filter_gather every workgroup finds the few ranges in which the cut lies from bounds on their weights, lists these ranges' tokens of its part and sums what
// is above them; k_filter_close, a workgroup a row, finds the cut in those lists, by exact sums: the ranges are an estimate.  What is left even then (ties of thousands at the
// cut; a top-k beyond the lists together with a top-p; parts whose sample is masked, which have no sum; ranges stretched by masks of large finite numbers) it takes from the row
// itself: 4096 ranges, of which the one with the cut is sorted if it fits, or cut into 4096 again, until one token is left.
// The sample speaks for its part, and the largest of the parts' bounds for the row: of 151936 normal logits 215 to 755 are listed (445 to 534 on average, by the number of rows), of ones that
// fall by 1 a decade of the index 31 to 250, of a row that is masked beyond its first 20000 tokens 37 to 181, or (64 rows) none, since a wave's list overflows.
// Masks: k_filter_apply.  Rows of up to kDirect tokens are their own list and need one launch.  Nothing is waited for between workgroups: a kernel's end orders.
//
// Times here are of one MI355X: 1280 rows of 151936 fp32 logits, 140 of them flat, take 267 us, 155 of them the read (79 % of what a plain read of the bytes
// reaches); one row of 49152, 20 us, all of it latency.
//
// Weights are sums of whole numbers, which no order of the work changes: a bin's of 2^-F of the weight at its middle, so that a bin far from the
// largest is as exact as one next to it, a list's and the draw's of 2^-F of the largest.  Sums over whole rows are fp64 in a fixed order.
#include "numeric.h"
#include <algorithm>
#include <math.h>

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 4096, kWideList = 2048;
constexpr int kListBits = 50;                              // a list's weights: 2^11 of them stay below 2^62
// a workgroup of k_filter_parts, its waves' shares; lists of a row together, and entries that k_filter_finish takes
constexpr int kPartThreads = 256, kPartWaves = kPartThreads / 64, kPer = 16, kStep = 64 * kPer;
constexpr int kPart = 16384, kLeastPart = 4096, kFillParts = 1024, kMostParts = 64, kDirect = 1280, kList = 1536, kCloseList = 6144, kGroups = 64, kWanted = 768;
constexpr int kFinishThreads = 256, kFinishWaves = kFinishThreads / 64, kFinishBins = 512, kFew = 64, kRanges = 2048, kWideGrid = 2048;

// What a part of a row comes to
struct __attribute__((aligned(16))) Part {
    double sum, scale;               // sum of the weights in units of exp(scale), if has_sum
    float top, bound;                // the largest logit; the lists hold all logits from bound on (infinity: they are not whole)
    int32_t live, bad;               // tokens that are not masked; a NaN or an infinity among the logits
    int32_t listed[kPartWaves];
    int32_t has_sum;
    float least;                     // the sample's least logit
    int32_t above;                   // k_filter_gather's: the logits above the range, and their weights
    int32_t pad;
    u64 above_q[kPartWaves];
};
// and a row: kept are the tokens up to `cut`
enum { ROW_DONE = 0, ROW_CUT = 1, ROW_BAD = 2, ROW_WIDE = 3, ROW_SLOW = 4 };     // CUT: what is kept is not in the lists
enum { BY_MASS = 0, BY_COUNT = 1, BY_SHARE = 2 };
struct __attribute__((aligned(16))) RowOut {
    u64 cut;
    int32_t state, type;
    float top, ref;                  // largest logit; the logits below `ref` are not listed (infinity: none is)
    float least;                     // roughly
    int32_t listed;                  // logits from ref on, and their weights in 2^-kListBits
    u64 listed_q;
    float x_lo, x_hi;                // k_filter_gather's: the range that the cut lies in
    double total;                    // sum of all weights, in the largest's
    float x_m;                       // min-p's least logit (-infinity: none)
    int32_t found;                   // k_filter_gather's: what decides on the cut, or -1
    int32_t pad[2];
};

struct FilterArgs {
    const void* logits;
    int64_t row_stride;
    int32_t per, vocab;              // rows of a sequence (they share its parameters)
    const float* temperature;        // nullable [sequences], as all parameters
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;                  // sampling: [rows]
    int32_t* token;
    float* logprob;
    int32_t* kept;
    void* out;                       // filtering
    int64_t out_stride;
    Part* parts;                     // [rows, n_parts]
    u64* lists;                      // [rows, n_parts, kPartWaves, list_len]
    u32* slices;                     // [rows, n_parts, kRanges / 2] counts of ranges, of the rows in `wide`
    RowOut* rows;                    // [rows]
    int32_t* wide;                   // how many rows are listed here, and which
    int32_t n_parts, part_len, list_len;
    int32_t sample_len, sample_rank; // the bound: of 64 groups' largest logits, 16 * sample_len each, the one with so many of them above or at it
    int32_t direct;                  // rows are their own lists
    int32_t in_place, out_aligned;   // out_aligned: rows to write begin at multiples of 16 bytes
};

__device__ __forceinline__ u32 key_of(float x) {           // grows with x; -0 is 0
    const u32 b = __float_as_uint(x + 0.f);
    return b ^ ((u32)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_key(u32 s) { return __uint_as_float(s & 0x80000000u ? s ^ 0x80000000u : ~s); }
__device__ __forceinline__ u64 comp_of(float x, int v) { return (u64)~key_of(x) << 24 | (u32)v; }
__device__ __forceinline__ float logit_of(u64 comp) { return from_key(~(u32)(comp >> 24)); }
__device__ __forceinline__ int token_of(u64 comp) { return (int)(comp & 0xFFFFFF); }

// A row's parameters: the first alone; by count; by mass; by the largest's share
struct Params { double inv; float p, m; int k; bool good, one, by_count, by_mass, by_share; };
__device__ __forceinline__ Params params_of(const FilterArgs& a, int b) {
    const float t = a.temperature ? a.temperature[b] : 1.f;
    Params o;
    o.p = a.top_p ? a.top_p[b] : 1.f;
    o.m = a.min_p ? a.min_p[b] : 0.f;
    o.k = a.top_k ? a.top_k[b] : 0;
    o.good = t >= 0.f && o.p == o.p && o.m == o.m;
    o.inv = t > 0.f ? 1.0 / (double)t : 1.0;
    o.one = t == 0.f || o.p <= 0.f || o.m > 1.f || o.k == 1;
    o.by_count = !o.one && o.k > 0 && o.k < a.vocab;
    o.by_mass = !o.one && o.p < 1.f;
    o.by_share = !o.one && o.m > 0.f;
    return o;
}

template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ u64 dpp_u64(u64 v) { return __builtin_bit_cast(u64, lane64_dpp<CTRL, ROWS>(__builtin_bit_cast(double, v))); }
// Lane l's value; l is the same in all lanes.  Not for a branch that lane l may not be in: what the compiler copies or loads again there is not lane l's.
__device__ __forceinline__ u64 of_lane(u64 v, int l) {
    return (u64)(u32)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 | (u32)__builtin_amdgcn_readlane((int)(u32)v, l);
}
__device__ __forceinline__ int wave_sum_int(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, false);
    return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48);
}
__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
    v += dpp_u64<0xB1>(v);                                  // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
    v += dpp_u64<0x4E>(v);
    v += dpp_u64<0x141>(v);
    v += dpp_u64<0x140>(v);
    return of_lane(v, 0) + of_lane(v, 16) + of_lane(v, 32) + of_lane(v, 48);
}
__device__ __forceinline__ u64 wave_scan_u64(u64 v) {      // inclusive
    v += dpp_u64<0x111>(v);                                 // row_shr 1, 2, 4, 8
    v += dpp_u64<0x112>(v);
    v += dpp_u64<0x114>(v);
    v += dpp_u64<0x118>(v);
    v += dpp_u64<0x142, 0xA>(v);                            // lane 15 of the row before, into rows 1 and 3
    v += dpp_u64<0x143, 0xC>(v);                            // lane 31, into rows 2 and 3
    return v;
}

// The logits of a row, thread by thread: f(x, first index) over SIDE side by side, those behind the vocabulary as masked
template <typename T, bool VEC>
struct RowLoop {
    static constexpr int SIDE = VEC ? 16 / (int)sizeof(T) : 1, AHEAD = 16 / SIDE;
    template <typename F>
    static __device__ __forceinline__ void run(const T* __restrict__ row, int vocab, int tid, F f) {
        for (int v0 = 0; v0 < vocab; v0 += kThreads * SIDE * AHEAD) {
            float x[AHEAD][SIDE];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int v = v0 + (j * kThreads + tid) * SIDE;
                if (VEC && v + SIDE <= vocab) {
                    load_n<SIDE == 1 ? 4 : SIDE>(row + v, x[j]);
                } else {
#pragma unroll
                    for (int e = 0; e < SIDE; ++e) x[j][e] = v + e < vocab ? to_f(row[v + e]) : -__builtin_inff();
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (v0 + j * kThreads * SIDE < vocab) f(x[j], v0 + (j * kThreads + tid) * SIDE);
        }
    }
};

struct __attribute__((aligned(16))) Shared {
    u64 big[kBins];                  // a histogram; lists of kWideList; segments of the draw
    double sum[kWaves];
    u64 whole[kWaves];
    int32_t num[4][kWaves];
    float flt[2][kWaves];
    int32_t count[4];
    u64 found;
    double before;
    u64 whole_found;
};

// What all threads know of a row
struct RowState {
    float top, least;
    int live;                        // tokens that are not masked
    double inv, per_unit, bin_width; // 1 / temperature; bins a logit; (logits over the temperature) a bin
    int bits;                        // F of the bins and of the draw
    u64 cut;                         // kept: comp <= cut
    int kept;                        // -1: not counted yet
    int listed;                      // >= 0: big[0 .. listed) is the sorted list of a prefix that holds all kept ones
};

struct Bin { double f; int at; };    // place relative to the bin's middle, in bins
__device__ __forceinline__ Bin bin_of(const RowState& r, float x) {
    const double t = fmin(((double)r.top - (double)x) * r.per_unit, (double)(kBins - 1)), big = t + 0x1.8p52;
    return Bin{t - (big - 0x1.8p52), (int)(u32)__builtin_bit_cast(u64, big)};
}
// 2^F exp(-f width) to a whole number: |f width| <= 1 / 128, where the series up to the 5th power is within 2^-51 of it
struct BinWeight {
    double a[6];
    __device__ BinWeight(const RowState& r) {
        double p = ldexp(1.0, r.bits);
        a[0] = p + 0x1p52;
        for (int i = 1; i < 6; ++i) a[i] = p *= -r.bin_width / i;
    }
    __device__ __forceinline__ u64 operator()(double f) const {
        double p = a[5];
        for (int i = 4; i >= 0; --i) p = __builtin_fma(p, f, a[i]);
        return __builtin_bit_cast(u64, p) & 0xFFFFFFFFFFFFFull;
    }
};
// 2^bits exp((x - top) / temperature) to a whole number
__device__ __forceinline__ u64 weight_of(const RowState& r, float x, int bits) {
    const double w = exp_neg(((double)x - (double)r.top) * r.inv);
    return __builtin_bit_cast(u64, __builtin_fma(w, __builtin_bit_cast(double, (u64)(bits + 1023) << 52), 0x1p52)) & 0xFFFFFFFFFFFFFull;
}
// The least key for which a condition holds that holds from some key up to the largest logit's: 64 of them at a time
template <typename F>
__device__ __forceinline__ u32 first_key(float top, int lane, F holds) {
    const u32 most = key_of(top), none = key_of(-__builtin_inff());
    u32 base = 0;
    for (int shift = 30; shift >= 0; shift -= 6) {
        const u64 at = (u64)base + ((u64)lane << shift);
        const bool below = at <= 0xFFFFFFFFull && (u32)at < most && ((u32)at <= none || !holds(from_key((u32)at)));
        base += (u32)(__popcll(__ballot(below)) - 1) << shift;
    }
    return base + 1;
}

// The last of 4096 numbers that is not 0 and whose sum of those before it is below `limit`; sums in a fixed order.  limit(total) gives it.
template <typename Of, typename Limit>
__device__ __forceinline__ int last_below(Shared& s, int tid, Of of, Limit limit, double& before) {
    constexpr int PER = kBins / kThreads;
    const int lane = tid & 63, wave = tid >> 6;
    double v[PER], mine = 0.0;
#pragma unroll
    for (int e = 0; e < PER; ++e) mine += v[e] = of(PER * tid + e);
    const double up = wave_scan64_dpp(mine);
    if (lane == 63) s.sum[wave] = up;
    __syncthreads();
    double at = up - mine, total = 0.0;
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) at += total;
        total += s.sum[w];
    }
    const double end = limit(total);
    int last = -1;
    double last_before = 0.0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        if (v[e] > 0.0 && (at < end || PER * tid + e == 0)) {
            last = PER * tid + e;
            last_before = at;
        }
        at += v[e];
    }
    const u64 have = __ballot(last >= 0);
    if (lane == 0) s.num[0][wave] = have ? wave * 64 + 63 - __clzll(have) : -1;      // the thread
    __syncthreads();
    int thread = -1;
    for (int w = 0; w < kWaves; ++w) thread = max(thread, s.num[0][w]);
    if (tid == thread) {
        s.count[0] = last;
        s.before = last_before;
    }
    __syncthreads();
    before = s.before;
    const int found = s.count[0];
    __syncthreads();
    return found;
}

// big[0 .. n) in ascending order
__device__ __forceinline__ void sort_list(u64* list, int n, int tid) {
    int size = 64;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += kThreads) list[i] = ~0ull;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
        for (int step = run / 2; step > 0; step /= 2) {
            if (tid < size / 2) {
                const int i = 2 * tid - (tid & (step - 1)), j = i + step;
                const u64 a = list[i], b = list[j];
                if ((a > b) == ((i & run) == 0)) {
                    list[i] = b;
                    list[j] = a;
                }
            }
            __syncthreads();
        }
}
__device__ __forceinline__ int block_count(Shared& s, int n, int tid) {
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    if ((tid & 63) == 0) s.num[1][tid >> 6] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < kWaves; ++w) n += s.num[1][w];
    __syncthreads();
    return n;
}
// How many of a sorted list's first n have a sum before them, in 2^-kListBits, below `limit(total)`
template <typename Limit>
__device__ __forceinline__ int list_below(Shared& s, const RowState& r, const u64* list, int n, int tid, Limit limit) {
    const int lane = tid & 63, wave = tid >> 6;
    u64 q[2], mine = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) mine += q[e] = 2 * tid + e < n ? weight_of(r, logit_of(list[2 * tid + e]), kListBits) : 0;
    const u64 up = wave_scan_u64(mine);
    if (lane == 63) s.whole[wave] = up;
    __syncthreads();
    u64 at = up - mine, total = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) at += total;
        total += s.whole[w];
    }
    const double end = limit((double)total);
    int kept = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        kept += 2 * tid + e < n && ((double)at < end || 2 * tid + e == 0);
        at += q[e];
    }
    return block_count(s, kept, tid);
}

template <typename T, bool VEC>
struct Row {
    using Loop = RowLoop<T, VEC>;
    static constexpr int SIDE = Loop::SIDE;
    const T* row;
    int vocab, tid, lane, wave;
    Shared& s;
    RowState r;

    __device__ __forceinline__ bool is_kept(float x, int v, float cut_x, int cut_v) const { return x > cut_x || (x == cut_x && v <= cut_v); }

    // largest and least logit, how many there are; false: the row has no distribution
    __device__ bool look() {
        float top = -__builtin_inff(), least = __builtin_inff();
        int live = 0;
        bool nan = false;
        Loop::run(row, vocab, tid, [&](const float* x, int) {
#pragma unroll
            for (int e = 0; e < SIDE; ++e) {
                const bool in = x[e] > -__builtin_inff();
                nan |= x[e] != x[e];
                top = fmaxf(top, x[e]);
                least = fminf(least, in ? x[e] : __builtin_inff());
                live += in;
            }
        });
        top = wave_max_dpp(top);
        least = -wave_max_dpp(-least);
        for (int o = 32; o > 0; o >>= 1) live += __shfl_xor(live, o);
        if (lane == 0) {
            s.flt[0][wave] = top;
            s.flt[1][wave] = least;
            s.num[2][wave] = live;
        }
        if (__any(nan) && lane == 0) s.num[2][wave] = -1;
        __syncthreads();
        r.live = 0;
        bool bad = false;
        for (int w = 0; w < kWaves; ++w) {
            top = fmaxf(top, s.flt[0][w]);
            least = fminf(least, s.flt[1][w]);
            bad |= s.num[2][w] < 0;
            r.live += s.num[2][w];
        }
        __syncthreads();
        r.top = top + 0.f;
        r.least = least;
        return !bad && r.live > 0 && top < __builtin_inff();
    }

    // Cuts the kept ones (comp <= r.cut) to those whose sum before them is below limit(total): of ones each (UNIT) or of their weights
    template <bool UNIT, typename Limit>
    __device__ void select(Limit limit) {
        const float cut_x = logit_of(r.cut);
        const int cut_v = token_of(r.cut);
        for (int i = tid; i < kBins; i += kThreads) s.big[i] = 0;
        __syncthreads();
        const BinWeight weight(r);
        Loop::run(row, vocab, tid, [&](const float* x, int v) {
#pragma unroll
            for (int e = 0; e < SIDE; ++e) {
                if (!is_kept(x[e], v + e, cut_x, cut_v)) continue;
                const Bin b = bin_of(r, x[e]);
                atomicAdd(&s.big[b.at], UNIT ? 1ull : weight(b.f));
            }
        });
        __syncthreads();
        double before, end = 0.0;
        const double unit = ldexp(1.0, -r.bits);
        const int b = last_below(s, tid, [&](int i) { return UNIT ? (double)s.big[i] : (double)s.big[i] * unit * exp_neg(-i * r.bin_width); },
                                 [&](double total) { return end = limit(total); }, before);
        // the bin's tokens, and all up to them
        const u32 lo = first_key(r.top, lane, [&](float x) { return bin_of(r, x).at <= b; });
        const u32 hi = b == 0 ? key_of(__builtin_inff()) : first_key(r.top, lane, [&](float x) { return bin_of(r, x).at < b; });
        const float x_lo = from_key(lo), x_hi = from_key(hi);
        u64 *const all = s.big, *const own = s.big + kWideList;
        if (tid < 2) s.count[tid] = 0;
        __syncthreads();
        int above = 0;
        auto append = [&](u64* list, int which, bool in, float x, int v) {
            const u64 m = __ballot(in);
            if (!m) return;
            int at = 0;
            if (lane == 0) at = atomicAdd(&s.count[which], __popcll(m));
            at = __builtin_amdgcn_readfirstlane(at) + __popcll(m & ((1ull << lane) - 1));
            if (in && at < kWideList) list[at] = comp_of(x, v);
        };
        Loop::run(row, vocab, tid, [&](const float* x, int v) {
#pragma unroll
            for (int e = 0; e < SIDE; ++e) {
                const bool in = x[e] >= x_lo && is_kept(x[e], v + e, cut_x, cut_v);
                above += in && x[e] >= x_hi;
                append(all, 0, in, x[e], v + e);
                append(own, 1, in && x[e] < x_hi, x[e], v + e);
            }
        });
        above = block_count(s, above, tid);
        const int n_all = s.count[0], n_own = s.count[1];
        __syncthreads();
        if (n_all <= kWideList) {
            sort_list(all, n_all, tid);
            r.listed = n_all;
            const double scale = 0x1p50;
            static_assert(kListBits == 50);
            r.kept = UNIT ? (int)fmin(end, (double)n_all) : list_below(s, r, all, n_all, tid, [&](double) { return end * scale; });
            r.cut = all[r.kept - 1];
        } else if (n_own <= kWideList) {
            sort_list(own, n_own, tid);
            const int n = UNIT ? (int)fmin(end - before, (double)n_own) : list_below(s, r, own, n_own, tid, [&](double) { return (end - before) * 0x1p50; });
            r.kept = above + n;
            r.cut = own[n - 1];
        } else {
            refine<UNIT>(x_lo, x_hi, cut_x, cut_v, UNIT ? end - before : (end - before) * ldexp(exp_neg(b * r.bin_width), r.bits), weight);
            r.kept = -1;
        }
        __syncthreads();
    }

    // The same among the tokens of [x_lo, x_hi), in the bins' whole numbers, by their places in the order
    template <bool UNIT>
    __device__ __forceinline__ void refine(float x_lo, float x_hi, float cut_x, int cut_v, double left, BinWeight weight) {
        u64 lo = (u64)~(key_of(x_hi) - 1) << 24, hi = (u64)~key_of(x_lo) << 24 | 0xFFFFFF;
        for (;;) {
            int shift = 0;
            while ((hi - lo) >> shift >= kBins) ++shift;
            for (int i = tid; i < kBins; i += kThreads) s.big[i] = 0;
            __syncthreads();
            Loop::run(row, vocab, tid, [&](const float* x, int v) {
#pragma unroll
                for (int e = 0; e < SIDE; ++e) {
                    const u64 c = comp_of(x[e], v + e);
                    if (x[e] >= x_lo && x[e] < x_hi && is_kept(x[e], v + e, cut_x, cut_v) && c >= lo && c <= hi)
                        atomicAdd(&s.big[(c - lo) >> shift], UNIT ? 1ull : weight(bin_of(r, x[e]).f));
                }
            });
            __syncthreads();
            double before;
            const int b = last_below(s, tid, [&](int i) { return (double)s.big[i]; }, [&](double) { return left; }, before);
            left -= before;
            lo += (u64)b << shift;
            hi = min(hi, lo + ((1ull << shift) - 1));
            if (shift == 0) break;
        }
        r.cut = lo;
    }

    // keeps what is no less than x_m
    __device__ void at_least(u32 key) {
        const float x_m = from_key(key);
        if (r.listed >= 0) {
            int n = 0;
            for (int i = tid; i < r.kept; i += kThreads) n += logit_of(s.big[i]) >= x_m;
            n = block_count(s, n, tid);
            r.kept = n;
            r.cut = s.big[n - 1];
        } else if (logit_of(r.cut) < x_m) {
            r.cut = (u64)~key << 24 | 0xFFFFFF;
            r.kept = -1;
        }
    }

    __device__ void count() {
        const float cut_x = logit_of(r.cut);
        const int cut_v = token_of(r.cut);
        int n = 0;
        Loop::run(row, vocab, tid, [&](const float* x, int v) {
#pragma unroll
            for (int e = 0; e < SIDE; ++e) n += is_kept(x[e], v + e, cut_x, cut_v);
        });
        r.kept = block_count(s, n, tid);
    }

    // the token that u falls on, and ln of its share
    __device__ int draw(float u, float& logp) {
        u64* const seg = s.big + kWideList;
        const bool from_list = r.listed >= 0;
        const int bits = from_list ? kListBits : r.bits;
        const float cut_x = logit_of(r.cut);
        const int cut_v = token_of(r.cut);
        int shift = from_list ? 0 : SIDE == 1 ? 6 : SIDE == 4 ? 8 : 9;   // (a wave's step lies in one segment)
        while ((vocab - 1) >> shift >= kThreads) ++shift;
        int first = 0, size = vocab;                        // what the draw is known to fall into
        u64 target = 0, total = 0;
        int kept = 0;
        for (bool known = false;; known = true) {
            seg[tid] = 0;
            __syncthreads();
            if (from_list) {
                for (int i = tid; i < r.kept; i += kThreads) {
                    const u64 c = s.big[i];
                    const int v = token_of(c) - first;
                    if (v >= 0 && v < size) atomicAdd(&seg[v >> shift], weight_of(r, logit_of(c), bits));
                }
            } else if (!known) {
                Loop::run(row, vocab, tid, [&](const float* x, int v) {
                    u64 q = 0;
#pragma unroll
                    for (int e = 0; e < SIDE; ++e) {
                        if (!is_kept(x[e], v + e, cut_x, cut_v)) continue;
                        ++kept;
                        q += weight_of(r, x[e], bits);
                    }
                    q = wave_sum_u64(q);
                    if (lane == 0) atomicAdd(&seg[v >> shift], q);
                });
            } else {
                for (int i = tid; i < size; i += kThreads) {
                    const int v = first + i;
                    const float x = v < vocab ? to_f(row[v]) : -__builtin_inff();
                    if (v < vocab && is_kept(x, v, cut_x, cut_v)) atomicAdd(&seg[i >> shift], weight_of(r, x, bits));
                }
            }
            __syncthreads();
            const u64 mine = seg[tid], up = wave_scan_u64(mine);
            if (lane == 63) s.whole[wave] = up;
            __syncthreads();
            u64 before = up - mine, all = 0;
            for (int w = 0; w < kWaves; ++w) {
                if (w == wave) before += all;
                all += s.whole[w];
            }
            if (!known) {
                total = all;
                target = u > 0.f ? min((u64)((double)u * (double)total), total - 1) : 0;
            }
            if (before <= target && target < before + mine) {
                s.count[0] = tid;
                s.found = before;
            }
            __syncthreads();
            first += s.count[0] << shift;
            target -= s.found;
            size = 1 << shift;
            __syncthreads();
            if (shift == 0) break;
            shift = max(shift - 10, 0);
        }
        if (r.kept < 0) r.kept = block_count(s, kept, tid);
        logp = (float)(((double)to_f(row[first]) - (double)r.top) * r.inv - log((double)total * ldexp(1.0, -bits)));
        return first;
    }
};

// ---------------------------------------------------------------- one read of every logit
// A wave has a run of its own, 16 logits a lane at a time.  The first of them are the sample: of groups of 16 to 64 logits the largest, and of these 64 one
// by its rank, which about kWanted / vocab of all logits exceed; the sum's units come from the sample's largest, too.
template <typename T, bool VEC>
struct Run {
    static constexpr int SIDE = VEC ? 16 / (int)sizeof(T) : 1;
    static __device__ __forceinline__ int place(int e, int lane) { return (e / SIDE * 64 + lane) * SIDE + e % SIDE; }
    static __device__ __forceinline__ void load(const T* __restrict__ row, int v0, int end, int lane, float (&x)[kPer]) {
#pragma unroll
        for (int e = 0; e < kPer; e += SIDE) {
            const int v = v0 + place(e, lane);
            if (VEC && v + SIDE <= end) {
                load_n<SIDE == 1 ? 4 : SIDE>(row + v, x + e);
            } else {
#pragma unroll
                for (int f = 0; f < SIDE; ++f) x[e + f] = v + f < end ? to_f(row[v + f]) : -__builtin_inff();
            }
        }
    }
};
__device__ __forceinline__ float row16_max(float v) {      // of 16 lanes side by side, in all of them
    auto up = [](float x, auto ctrl) { return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, false))); };
    v = up(v, std::integral_constant<int, 0xB1>{});
    v = up(v, std::integral_constant<int, 0x4E>{});
    v = up(v, std::integral_constant<int, 0x141>{});
    return up(v, std::integral_constant<int, 0x140>{});
}

// Bound by the bytes for many rows of fp32, where nothing else is in the way: 778 MB in 155 us (the exponentials of rows with a top-p alone keep the vector units
// 68 % busy), with the masks filled on the way 350 + 350 MB in 136; by instructions for bf16 (64 rows 15 us: a logit costs what an fp32 one does).  The next step's loads are
// under way while a step is worked on.
template <typename T, bool VEC, bool FILL>
__global__ __launch_bounds__(kPartThreads) void k_filter_parts(FilterArgs a) {
    using R = Run<T, VEC>;
    __shared__ word2 s_pow[256];
    __shared__ float s_group[kGroups];
    __shared__ float s_bound;
    __shared__ double s_sum[kPartWaves];
    __shared__ float s_top[kPartWaves], s_least[kPartWaves];
    __shared__ int32_t s_live[kPartWaves], s_bad[kPartWaves], s_listed[kPartWaves];
    const int i = blockIdx.y, part = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const T* const row = (const T*)a.logits + (int64_t)i * a.row_stride;
    const int p0 = part * a.part_len, run = a.part_len / kPartWaves, v_begin = min(p0 + wave * run, a.vocab), v_end = min(v_begin + run, a.vocab);
    float next[kPer];
    R::load(row, v_begin, v_end, lane, next);
    s_pow[tid] = kPow.at[tid];
    const Params q = params_of(a, i / a.per);
    const bool all = !FILL && !a.in_place && !q.one && !q.by_count && !q.by_mass && !q.by_share;      // nothing is dropped: no list
    const bool want_sum = all || (q.by_mass && !q.by_count);
    // the sample
    static_assert(kPer == 16 && kGroups == 4 * 4 * kPartWaves);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        float m = next[4 * g];
        if (a.sample_len > 1) m = fmaxf(m, next[4 * g + 1]);
        if (a.sample_len > 2) m = fmaxf(fmaxf(m, next[4 * g + 2]), next[4 * g + 3]);
        m = row16_max(m);
        if ((lane & 15) == 0) s_group[wave * 16 + g * 4 + lane / 16] = m;
    }
    float least = __builtin_inff();
#pragma unroll
    for (int e = 0; e < kPer; ++e) least = fminf(least, next[e] > -__builtin_inff() ? next[e] : __builtin_inff());
    least = -wave_max_dpp(-least);
    if (lane == 0) s_least[wave] = least;
    if (tid == 0 && part == 0 && i == 0) *a.wide = 0;
    __syncthreads();
    const float group = s_group[lane];
    const float anchor = wave_max_dpp(group);
    if (wave == 0) {
        // the largest bound that so many groups reach, by the upper half of its bits (in short runs some groups miss lanes: their largest
        // says little; without a whole one everything is listed)
        const int from = p0 + lane / 16 * run, last = from + R::place(lane / 4 % 4 * 4 + a.sample_len - 1, lane % 4 * 16 + 15);
        const bool whole_group = last < min(from + run, a.vocab);
        const u32 key = whole_group || q.one ? key_of(group) : 0;
        const int there = __popcll(__ballot(whole_group));
        const int rank = q.one ? 1 : there == 0 ? kGroups + 1 : (a.sample_rank * there + kGroups - 1) / kGroups;
        u32 at = 0;
        for (u32 bit = 1u << 31; bit >= 1u << 16; bit >>= 1)
            if (__popcll(__ballot(key >= (at | bit))) >= rank) at |= bit;
        if (lane == 0) s_bound = at > key_of(-__builtin_inff()) ? from_key(at) : -__builtin_inff();
    }
    __syncthreads();
    // (a NaN among the sample leaves the bound to chance; the row is refused all the same)
    const float bound = all ? __builtin_inff() : s_bound, reach = fmaxf(bound, -3.4028234663852886e38f);      // (-infinity is not listed)
    const double unit = q.inv * 369.3299304675746;          // 256 / ln 2
    const double whole = anchor > -__builtin_inff() && anchor < __builtin_inff() ? rint((double)anchor * unit) : 0.0, start = 0x1.8p52 - whole;
    const bool sums = want_sum && q.good && q.inv > 1e-20 && fabs(whole) < 0x1p24;
    const float lowest = sums ? (float)((whole - 200000.0) / unit) : 0.f;       // 2^-781: a masked logit's weight is none
    const int64_t list = (((int64_t)i * a.n_parts + part) * kPartWaves + wave) * a.list_len;
    T* const out = FILL ? (T*)a.out + (int64_t)i * a.out_stride : nullptr;
    float top = -__builtin_inff();
    double sum = 0.0;
    int listed = 0, live = 0;
    bool bad = false;
    for (int v0 = v_begin; v0 < v_end; v0 += kStep) {
        float x[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = next[e];
        if (v0 + kStep < v_end) R::load(row, v0 + kStep, v_end, lane, next);
        if (FILL) {
#pragma unroll
            for (int e = 0; e < kPer; e += R::SIDE) {
                const int v = v0 + R::place(e, lane);
                constexpr u32 none = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
                if (VEC && a.out_aligned && v + R::SIDE <= v_end) *(uint4*)(out + v) = uint4{none, none, none, none};
                else
#pragma unroll
                    for (int f = 0; f < R::SIDE; ++f)
                        if (v + f < v_end) out[v + f] = from_f<T>(-__builtin_inff());
            }
        }
        float most = x[0], low = x[0];                      // (a NaN stays one)
#pragma unroll
        for (int e = 0; e < kPer; e += 2) {
            asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(most) : "v"(most), "v"(x[e]), "v"(x[e + 1]));
            asm("v_minimum3_f32 %0, %1, %2, %3" : "=v"(low) : "v"(low), "v"(x[e]), "v"(x[e + 1]));
        }
        bad |= !(most < __builtin_inff());
        top = fmaxf(top, most);
        if (__any(!(low > -__builtin_inff()))) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) live += __popcll(__ballot(x[e] > -__builtin_inff()));
        } else {
            live += kStep;
        }
        if (sums) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const double y = (double)fmaxf(x[e], lowest), big = __builtin_fma(y, unit, start);
                sum = times_power(s_pow, small_power(__builtin_fma(y, unit, start - big)), (u32)__builtin_bit_cast(u64, big), sum);
            }
        }
        if (!__any(most >= reach)) continue;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const bool in = x[e] >= reach;
            const u64 m = __ballot(in);
            if (!m) continue;
            const int at = listed + __builtin_amdgcn_mbcnt_hi((u32)(m >> 32), __builtin_amdgcn_mbcnt_lo((u32)m, 0));
            if (in && at < a.list_len) a.lists[list + at] = comp_of(x[e], v0 + R::place(e, lane));
            listed += __popcll(m);
        }
    }
    sum = wave_sum64_dpp(sum);
    top = wave_max_dpp(top);
    if (lane == 0) {
        s_sum[wave] = sum;
        s_top[wave] = top;
        s_live[wave] = live;
        s_listed[wave] = listed;
    }
    const bool any_bad = __any(bad);
    if (lane == 0) s_bad[wave] = any_bad;
    __syncthreads();
    if (tid != 0) return;
    Part o{};
    o.top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    o.sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    o.scale = whole * (0.69314718055994530942 / 256);
    o.bound = bound;
    o.least = fminf(fminf(s_least[0], s_least[1]), fminf(s_least[2], s_least[3]));
    for (int w = 0; w < kPartWaves; ++w) {
        o.live += s_live[w];
        o.bad |= s_bad[w];
        o.listed[w] = s_listed[w];
        if (s_listed[w] > a.list_len) o.bound = __builtin_inff();
    }
    // (weights up to 2^781 of the sample's largest: beyond that the sum says nothing)
    o.has_sum = sums && ((double)o.top - (double)anchor) * unit < 200000.0;
    if (o.live == 0) o.has_sum = 1, o.sum = 0.0, o.scale = -__builtin_inf();
    a.parts[(int64_t)i * a.n_parts + part] = o;
}

// ---------------------------------------------------------------- a row from its lists
template <int ROOM>
struct __attribute__((aligned(16))) ListShared {
    static constexpr int room = ROOM;
    u64 list[ROOM], weight[ROOM];
    u64 bins[kFinishBins];
    u32 counts[kFinishBins];
    u64 few_key[kFew], few_q[kFew], least, most;
    u64 red[kWaves];
    int32_t num[kWaves], few, n, bad;
};
template <typename S>
__device__ __forceinline__ void append_to(S& s, bool in, u64 c, int lane) {
    const u64 m = __ballot(in);
    if (!m) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(&s.n, __popcll(m));
    at = __builtin_amdgcn_readfirstlane(at) + __builtin_amdgcn_mbcnt_hi((u32)(m >> 32), __builtin_amdgcn_mbcnt_lo((u32)m, 0));
    if (in && at < S::room) s.list[at] = c;
}
using FinishShared = ListShared<kList>;
struct Found { u64 key, sum; };      // sum: up to it and with it

// Of n items with weights q (0: not there), in the order of their keys within [lo, hi]: the last whose sum of those before it is below `limit`
// (FEW: there are no more than kFew of them).
template <bool FEW, int NT, typename S, typename Key, typename Weight>
__device__ __forceinline__ Found last_item(S& s, int n, u64 lo, u64 hi, u64 limit, int tid, Key key, Weight weight) {
    const int lane = tid & 63;
    u64 sum = 0;
    if (FEW) {
        __syncthreads();
        if (tid == 0) s.few = 0;
        __syncthreads();
    }
    for (;;) {
        if (!FEW) {
        const int shift = max(0, 64 - 9 - __clzll((long long)(hi - lo)));
        static_assert(kFinishBins == 1 << 9);
        __syncthreads();                                    // (bins and few are still looked at)
        for (int i = tid; i < kFinishBins; i += NT) s.bins[i] = 0;
        if (tid == 0) {
            s.few = 0;
            s.least = ~0ull;
            s.most = 0;
        }
        __syncthreads();
#pragma unroll 4
        for (int i = tid; i < n; i += NT) {
            const u64 c = key(i), q = weight(i);
            if (c >= lo && c <= hi && q) atomicAdd(&s.bins[(c - lo) >> shift], q);
        }
        __syncthreads();
        // every wave for itself, 8 bins a lane
        constexpr int PER = kFinishBins / 64;
        u64 v[PER], mine = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) mine += v[e] = s.bins[PER * lane + e];
        const u64 up = wave_scan_u64(mine);
        u64 at = up - mine, before = 0, own = 0;
        int last = -1;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (v[e] && at < limit) {
                last = PER * lane + e;
                before = at;
                own = v[e];
            }
            at += v[e];
        }
        const u64 have = __ballot(last >= 0);               // (the first item's bin has nothing before it: none only where there are no items)
        if (!have) return Found{lo, sum};
        const int from = 63 - __clzll(have);
        const int b = __builtin_amdgcn_readlane(last, from);
        before = of_lane(before, from);
        own = of_lane(own, from);
        sum += before;
        limit -= before;
        lo += (u64)b << shift;
        hi = min(hi, lo + ((1ull << shift) - 1));
        if (shift == 0) return Found{lo, sum + own};
        }
#pragma unroll 4
        for (int i = tid; i < n; i += NT) {
            const u64 c = key(i), q = weight(i);
            if (c < lo || c > hi || !q) continue;
            const int place = atomicAdd(&s.few, 1);
            if (place < kFew) {
                s.few_key[place] = c;
                s.few_q[place] = q;
            }
            if (!FEW) {
                atomicMin(&s.least, c);
                atomicMax(&s.most, c);
            }
        }
        __syncthreads();
        const int few = s.few;
        if (!FEW && few > kFew) {                           // (equal logits lie far apart from others by their keys, close together by their indices)
            lo = s.least;
            hi = s.most;
            continue;
        }
        const u64 c = lane < few ? s.few_key[lane] : ~0ull, q = lane < few ? s.few_q[lane] : 0;
        u64 below = 0;
        int rank = 0;
        for (int j = 0; j < few; ++j) {
            const u64 c_j = of_lane(c, j), q_j = of_lane(q, j);
            const bool less = c_j < c;
            below += less ? q_j : 0;
            rank += less;
        }
        // the last of those that are kept
        const bool kept = lane < few && below < limit;
        const int l = __ffsll((unsigned long long)__ballot(kept && rank == __popcll(__ballot(kept)) - 1)) - 1;
        if (l < 0) return Found{lo, sum};                   // (no items)
        return Found{of_lane(c, l), sum + of_lane(below, l) + of_lane(q, l)};
    }
}
struct Sum { u64 q; int n; };
template <int NT, typename S>
__device__ __forceinline__ Sum block_sum(S& s, u64 q, int n, int tid) {
    q = wave_sum_u64(q);
    n = wave_sum_int(n);
    __syncthreads();
    if ((tid & 63) == 0) {
        s.red[tid >> 6] = q;
        s.num[tid >> 6] = n;
    }
    __syncthreads();
    Sum all{0, 0};
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        all.q += s.red[w];
        all.n += s.num[w];
    }
    return all;
}

// The cut of the n places of s.list (weights beside them) by count (k > 0), then by mass (p < 1) of what is left, or of `total` (in the weights' units; below 0: of
// what is left): one histogram of counts and weights for both, then the tokens of the bins that the two fall into.
enum { CUT_DONE, CUT_MANY, CUT_BEYOND };                    // MANY: a bin holds more than kFew; BEYOND: the list's mass does not reach the limit
struct ListCut { u64 cut, total; int kept, state; u64 listed; };     // total: weights of the kept ones; listed: of all
template <int NT, typename S>
__device__ __forceinline__ ListCut list_cut(S& s, int n, u64 lo, u64 hi, int k, double p, double total, int tid) {
    const int lane = tid & 63, shift = max(0, 64 - 9 - __clzll((long long)(hi - lo)));
    static_assert(kFinishBins == 1 << 9);
    __syncthreads();
    for (int i = tid; i < kFinishBins; i += NT) {
        s.bins[i] = 0;
        s.counts[i] = 0;
    }
    if (tid == 0) s.few = 0;
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < n; i += NT) {
        const u64 c = s.list[i], q = s.weight[i];
        if (c > hi) continue;
        atomicAdd(&s.bins[(c - lo) >> shift], q);
        atomicAdd(&s.counts[(c - lo) >> shift], 1u);
    }
    __syncthreads();
    // every wave for itself, 8 bins a lane
    constexpr int PER = kFinishBins / 64;
    u64 w[PER], w_own = 0, c_own = 0;
    u32 c[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        w_own += w[e] = s.bins[PER * lane + e];
        c_own += c[e] = s.counts[PER * lane + e];
    }
    const u64 w_up = wave_scan_u64(w_own), c_up = wave_scan_u64(c_own);
    ListCut out{hi, of_lane(w_up, 63), (int)of_lane(c_up, 63), CUT_DONE, of_lane(w_up, 63)};
    int held = -1, few = 0;                                 // the bin whose tokens lie in few_*
    u64 key = 0, q = 0, below = 0;
    int rank = 0;
    // the last bin whose count (weight) before it is below the limit, its tokens, and the last of those
    auto narrow = [&](bool by_count, u64 limit) {
        u64 w_at = w_up - w_own, c_at = c_up - c_own, w_before = 0, c_before = 0;
        int last = -1;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (c[e] && (by_count ? c_at : w_at) < limit) {
                last = PER * lane + e;
                w_before = w_at;
                c_before = c_at;
            }
            w_at += w[e];
            c_at += c[e];
        }
        const u64 have = __ballot(last >= 0);
        if (!have) {
            out.state = CUT_MANY;
            return;
        }
        const int from = 63 - __clzll(have), b = __builtin_amdgcn_readlane(last, from);
        w_before = of_lane(w_before, from);
        c_before = of_lane(c_before, from);
        if (b != held) {
            if (held >= 0) {
                __syncthreads();
                if (tid == 0) s.few = 0;
                __syncthreads();
            }
            held = b;
#pragma unroll 4
            for (int i = tid; i < n; i += NT) {
                const u64 at = s.list[i];
                if (at > hi || (int)((at - lo) >> shift) != b) continue;
                const int place = atomicAdd(&s.few, 1);
                if (place < kFew) {
                    s.few_key[place] = at;
                    s.few_q[place] = s.weight[i];
                }
            }
            __syncthreads();
            few = s.few;
            if (few > kFew) {
                out.state = CUT_MANY;
                return;
            }
            key = lane < few ? s.few_key[lane] : ~0ull;
            q = lane < few ? s.few_q[lane] : 0;
            below = 0;
            rank = 0;
            for (int j = 0; j < few; ++j) {
                const u64 key_j = of_lane(key, j), q_j = of_lane(q, j);
                const bool less = key_j < key;
                below += less ? q_j : 0;
                rank += less;
            }
        }
        const bool kept = lane < few && (by_count ? c_before + rank : w_before + below) < limit;
        const int l = __ffsll((unsigned long long)__ballot(kept && rank == __popcll(__ballot(kept)) - 1)) - 1;
        out.cut = of_lane(key, l & 63);
        out.kept = (int)c_before + __builtin_amdgcn_readlane(rank, l & 63) + 1;
        out.total = w_before + of_lane(below, l & 63) + of_lane(q, l & 63);
    };
    if (k > 0) narrow(true, (u64)k);
    if (p < 1.0 && out.state == CUT_DONE) {
        const double limit = ceil(p * (total < 0.0 ? (double)out.total : total));
        if (!((double)out.total >= limit)) out.state = CUT_BEYOND;
        else narrow(false, (u64)fmax(limit, 1.0));
    }
    return out;
}

__device__ __forceinline__ int list_length(const FilterArgs& a, int i, int tid) {      // of the thread's list
    return tid < a.n_parts * kPartWaves ? a.parts[(int64_t)i * a.n_parts + tid / kPartWaves].listed[tid % kPartWaves] : 0;
}
// A row's lists one behind the other in s.list, entries beyond `last` as none (~0): how many places, or -1 if they do not fit or one of them is not whole;
// s.n counts the others.  A thread a list (`own`: its length), then a thread an entry.
template <int NT, typename S>
__device__ __forceinline__ int read_lists(S& s, const FilterArgs& a, int i, int own, int tid, u64 last) {
    static_assert(kMostParts * kPartWaves <= NT && NT <= 2 * kFinishBins);
    const int lane = tid & 63, wave = tid >> 6;
    const u64* const lists = a.lists + (int64_t)i * a.n_parts * kPartWaves * a.list_len;
    // the sums of the lengths; bit 32 of a sum: a list that is not whole
    const u64 up = wave_scan_u64((u64)(u32)own | (own > a.list_len ? 1ull << 32 : 0));
    if (lane == 63) s.red[wave] = up;
    if (tid == 0) s.n = 0;
    __syncthreads();
    u64 before = 0, all = 0;
    for (int w = 0; w < NT / 64; ++w) {
        if (w == wave) before = all;
        all += s.red[w];
    }
    const int n = (int)(u32)all;
    if (all >> 32 || n > S::room) return -1;
    u32* const ends = (u32*)s.bins;
    ends[tid] = (u32)(before + up);
    __syncthreads();
    int valid = 0;
    constexpr int AHEAD = 4;
    for (int e0 = tid; e0 < n; e0 += AHEAD * NT) {
        int l[AHEAD] = {};                                  // lists that end at or before the entry
#pragma unroll
        for (int step = NT / 2; step > 0; step /= 2)
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (ends[l[j] + step - 1] <= (u32)(e0 + j * NT)) l[j] += step;
        u64 c[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int e = e0 + j * NT;
            c[j] = e < n ? lists[(int64_t)l[j] * a.list_len + (e - (l[j] > 0 ? (int)ends[l[j] - 1] : 0))] : ~0ull;
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int e = e0 + j * NT;
            if (e >= n) continue;
            s.list[e] = c[j] <= last ? c[j] : ~0ull;
            valid += c[j] <= last;
        }
    }
    valid = wave_sum_int(valid);
    if (lane == 0) atomicAdd(&s.n, valid);
    __syncthreads();
    return n;
}

// The first of the logits [p0, end) whose weights up to it sum to more than `target` (the last with any if none does): the sums of the waves' steps, then the
// logits of one step.  weight(x, v) is 0 where a token is not kept.
template <typename T, bool VEC, int NT, typename S, typename Weight>
__device__ __forceinline__ int draw_part(S& s, const T* row, int p0, int run, int end, u64 target, int tid, Weight weight) {
    using R = Run<T, VEC>;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), v_begin = min(p0 + wave * run, end), v_end = min(v_begin + run, end);
    const int steps = (run + kStep - 1) / kStep;            // of a wave
    __syncthreads();
    for (int i = tid; i < kFinishBins; i += NT) s.bins[i] = 0;
    __syncthreads();
    float next[kPer];
    R::load(row, v_begin, v_end, lane, next);
    for (int st = 0; st < steps; ++st) {
        const int v0 = v_begin + st * kStep;
        float x[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = next[e];
        if (v0 + kStep < v_end) R::load(row, v0 + kStep, v_end, lane, next);
        if (v0 >= v_end) break;
        u64 q = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) q += weight(x[e], v0 + R::place(e, lane));
        q = wave_sum_u64(q);
        if (lane == 0) s.bins[wave * steps + st] = q;
    }
    __syncthreads();
    constexpr int PER = kFinishBins / 64;
    u64 v[PER], mine = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) mine += v[e] = s.bins[PER * lane + e];
    const u64 up = wave_scan_u64(mine);
    u64 at = up - mine, before = 0;
    int last = -1;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        if (v[e] && at <= target) {
            last = PER * lane + e;
            before = at;
        }
        at += v[e];
    }
    const u64 have = __ballot(last >= 0);
    if (!have) return p0;
    const int from = 63 - __clzll(have), step = __builtin_amdgcn_readlane(last, from);
    target -= of_lane(before, from);
    // a few logits a thread
    constexpr int SPAN = kStep / NT;
    const int w = step / steps, first = p0 + w * run + step % steps * kStep, stop = min(min(p0 + (w + 1) * run, end), first + kStep), v0 = first + SPAN * tid;
    u64 q[SPAN], own = 0;
#pragma unroll
    for (int e = 0; e < SPAN; ++e) own += q[e] = v0 + e < stop ? weight(to_f(row[v0 + e]), v0 + e) : 0;
    const u64 sum = wave_scan_u64(own);
    __syncthreads();
    if (lane == 63) s.red[wave] = sum;
    __syncthreads();
    at = sum - own;
    for (int i = 0; i < wave; ++i) at += s.red[i];
    int token = -1;
#pragma unroll
    for (int e = 0; e < SPAN; ++e) {
        if (q[e] && at <= target) token = v0 + e;
        at += q[e];
    }
    for (int o = 32; o > 0; o >>= 1) token = max(token, __shfl_xor(token, o));
    if (lane == 0) s.num[wave] = token;
    __syncthreads();
    for (int i = 0; i < NT / 64; ++i) token = max(token, s.num[i]);
    return token;
}

// The sum of a row's weights in the largest's, from the lanes' parts
__device__ __forceinline__ double part_total(double sum, double scale, const RowState& r) {
    return wave_sum64_dpp(sum > 0.0 ? sum * exp_neg(scale - (double)r.top * r.inv) : 0.0);
}

// A workgroup a row, from its lists.  Bound by its chain: two dependent reads, then for each of top-k and top-p a histogram, its running sums and a comparison of the bin at the
// cut, about 15 barriers: 10 us for one row, 40 for 1280, five workgroups a compute unit (four, with lists of up to 2048: 12 for one row).
template <typename T, bool VEC, bool MASK>
__global__ __launch_bounds__(kFinishThreads) __attribute__((amdgpu_waves_per_eu(5))) void k_filter_finish(FilterArgs a) {
    __shared__ FinishShared s;
    const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const T* const row = (const T*)a.logits + (int64_t)i * a.row_stride;
    const int length = a.direct ? 0 : list_length(a, i, tid);
    const Params p = params_of(a, i / a.per);
    if (tid == 0) s.n = s.bad = 0;
    __syncthreads();
    // the list, and what is known of the row
    int live = 0, n = 0;
    bool bad = !p.good, whole = true, has_sum = true;       // whole: the list holds all that are not masked
    float top = -__builtin_inff(), bound = -__builtin_inff();
    float least = __builtin_inff();
    double part_sum = 0.0, part_scale = -__builtin_inf();   // the lane's part
    auto append = [&](bool in, u64 c) { append_to(s, in, c, lane); };
    if (a.direct) {
        bool nan = false;
        for (int v0 = 0; v0 < a.vocab; v0 += kFinishThreads) {
            const float x = v0 + tid < a.vocab ? to_f(row[v0 + tid]) : -__builtin_inff();
            nan |= !(x < __builtin_inff());
            top = fmaxf(top, x);
            append(x > -__builtin_inff(), comp_of(x, v0 + tid));
        }
        if (__any(nan) && lane == 0) s.bad = 1;
        top = wave_max_dpp(top);
        if (lane == 0) s.num[wave] = __builtin_bit_cast(int, top);
        __syncthreads();
        for (int w = 0; w < kFinishWaves; ++w) top = fmaxf(top, __builtin_bit_cast(float, s.num[w]));
        bad |= s.bad != 0;
        live = s.n;
    } else {
        static_assert(kMostParts == 64);
        const Part* const parts = a.parts + (int64_t)i * a.n_parts;
        bool no_sum = false, wrong = false;
        if (lane < a.n_parts) {
            const Part o = parts[lane];
            top = o.top;
            bound = o.bound;
            live = o.live;
            wrong = o.bad;
            no_sum = !o.has_sum;
            part_sum = o.sum;
            part_scale = o.scale;
            least = o.least;
        }
        bad |= __any(wrong) != 0;
        has_sum = !__any(no_sum);
        top = wave_max_dpp(top);
        bound = wave_max_dpp(bound);
        least = -wave_max_dpp(-least);
        live = wave_sum_int(live);
        if (bound < __builtin_inff()) n = read_lists<kFinishThreads>(s, a, i, length, tid, (u64)~key_of(bound) << 24 | 0xFFFFFF);
        if (n < 0) bound = __builtin_inff();
        whole = bound == -__builtin_inff();
    }
    // places of the list, some of them empty
    if (a.direct) n = s.n;
    const int valid = bound < __builtin_inff() ? s.n : 0;
    const bool nothing_listed = bound == __builtin_inff();
    bool wide = false;
    bad |= live == 0;
    RowState r{};
    r.top = top + 0.f;
    r.inv = p.inv;
    int token = -1, kept = 0;
    float logp = __builtin_nanf("");
    u64 cut = (1ull << 56) - 1, listed_q = 0;
    float x_m = -__builtin_inff();
    double total = 0.0;                                     // of all weights
    int type = -1;                                          // of a wide row that the kernels behind this one serve
    if (!bad) {
        const bool by_count = p.by_count && p.k < live, any = p.one || by_count || p.by_mass || p.by_share;
        const u64 lo = (u64)~key_of(r.top) << 24, hi = a.direct || whole ? ((1ull << 56) - 1) : (u64)~key_of(bound) << 24 | 0xFFFFFF;
        auto comp = [&](int e) { return s.list[e]; };
        auto weight = [&](int e) { return s.weight[e]; };
        bool held = whole, counted = false;                 // the list holds all that the filters so far keep; `by` counts them
        u64 counted_q = 0;
        if (p.by_share) x_m = from_key(first_key(r.top, lane, [&, most = -log((double)p.m)](float x) { return ((double)r.top - (double)x) * r.inv <= most; }));
        // the weights, 0 for an empty place; each is looked at by the thread that sets it, up to last_item's barriers
        if (!nothing_listed && (by_count || p.by_mass || !MASK)) {
#pragma unroll 4
            for (int e = tid; e < n; e += kFinishThreads) s.weight[e] = s.list[e] <= hi ? weight_of(r, logit_of(s.list[e]), kListBits) : 0;
        }
        if (nothing_listed) {
            wide = any || MASK || !has_sum;
        } else if (!wide) {
            if (p.one) {
                u64 first = ~0ull;
                for (int e = tid; e < n; e += kFinishThreads) first = min(first, s.list[e]);
                for (int o = 32; o > 0; o >>= 1) first = min(first, (u64)__shfl_xor(first, o));
                __syncthreads();
                if (lane == 0) s.red[wave] = first;
                __syncthreads();
                cut = min(min(s.red[0], s.red[1]), min(s.red[2], s.red[3]));
                held = true;
            }
            ListCut by{0, 0, 0, CUT_MANY, 0};
            const bool from_parts = p.by_mass && !by_count && !held;          // the mass is the whole row's
            if (from_parts && has_sum) total = part_total(part_sum, part_scale, r);
            if ((by_count && p.k <= valid) || (!by_count && p.by_mass && (held || has_sum))) {
                by = list_cut<kFinishThreads>(s, n, lo, hi, by_count ? p.k : 0, p.by_mass ? (double)p.p : 1.0, from_parts ? total * 0x1p50 : -1.0, tid);
                static_assert(kListBits == 50);
                if (by.state == CUT_DONE) {
                    cut = by.cut;
                    held = counted = true;
                } else if (by.state == CUT_BEYOND) {
                    wide = true;
                    listed_q = by.listed;
                }
            }
            if (by.state == CUT_MANY) {                     // (thousands of tokens at a cut: top-k and top-p one after the other)
                if (by_count) {
                    if (p.k <= valid) {
                        cut = last_item<false, kFinishThreads>(s, n, lo, hi, (u64)p.k, tid, comp, [](int) { return 1ull; }).key;
                        held = true;
                    } else if (!held) {
                        wide = true;
                    }
                }
                if (p.by_mass && !wide) {
                    u64 mine = 0;
                    for (int e = tid; e < n; e += kFinishThreads) mine += s.list[e] <= cut ? weight(e) : 0;
                    const u64 listed = listed_q = block_sum<kFinishThreads>(s, mine, 0, tid).q;
                    double limit = 0.0;
                    if (held) {
                        limit = ceil((double)p.p * (double)listed);
                    } else if (has_sum) {
                        limit = ceil((double)p.p * total * 0x1p50);
                        static_assert(kListBits == 50);
                        wide = !((double)listed >= limit);
                    } else {
                        wide = true;
                    }
                    if (!wide) {
                        cut = last_item<false, kFinishThreads>(s, n, lo, min(hi, cut), (u64)fmax(limit, 1.0), tid, comp, weight).key;
                        held = true;
                    }
                }
            }
            if (counted) {
                kept = by.kept;
                counted_q = by.total;
            }
            if (p.by_share && !wide) {
                if (x_m >= bound) held = true;
                const u64 least_kept = (u64)~key_of(x_m) << 24 | 0xFFFFFF;
                if (least_kept < cut) {
                    cut = least_kept;
                    counted = false;
                }
            }
            wide = wide || !held;
        }
        if (wide) {
            type = !any ? -1 : by_count ? (p.by_mass ? -1 : BY_COUNT) : p.by_mass ? (has_sum ? BY_MASS : -1) : p.by_share ? BY_SHARE : -1;
            if (type == BY_MASS) total = part_total(part_sum, part_scale, r);
            if (nothing_listed) listed_q = 0;
        } else if (nothing_listed) {                        // nothing is dropped: the part that the draw falls into, read again
            const double own = part_sum > 0.0 ? part_sum * exp_neg(part_scale - (double)r.top * r.inv) : 0.0, up = wave_scan64_dpp(own);
            const double total = lane64(up, 63), target = fmin(fmax((double)a.u[i], 0.0), 1.0) * total;
            const u64 past = __ballot(up > target), some = __ballot(own > 0.0);
            const int part = past ? __ffsll((unsigned long long)past) - 1 : 63 - __clzll(some);
            const int p0 = part * a.part_len, len = min(a.part_len, a.vocab - p0), bits = min(50, 62 - (32 - __clz(a.part_len)));
            const u64 within = (u64)(fmax(target - lane64(up - own, part), 0.0) * ldexp(1.0, bits));
            token = draw_part<T, VEC, kFinishThreads>(s, row, p0, a.part_len / kFinishWaves, p0 + len, within, tid, [&](float x, int) { return x > -__builtin_inff() ? max(weight_of(r, x, bits), (u64)1) : 0; });
            logp = (float)(((double)to_f(row[token]) - (double)r.top) * r.inv - log(total));
            kept = live;
        } else {
            if (!counted) {
                u64 q = 0;
                int c = 0;
                for (int e = tid; e < n; e += kFinishThreads) {
                    const bool in = s.list[e] <= cut;
                    c += in;
                    if (!MASK && in) q += weight(e);
                }
                const Sum all = block_sum<kFinishThreads>(s, q, c, tid);
                kept = all.n;
                counted_q = all.q;
            }
            if (!MASK) {
                const float u = a.u[i];
                const u64 limit = u > 0.f ? min((u64)((double)u * (double)counted_q), counted_q - 1) + 1 : 1;
                auto token_at = [&](int e) { return s.list[e] <= cut ? (u64)token_of(s.list[e]) << 32 | (u32)e : ~0ull; };
                const Found f = kept <= kFew ? last_item<true, kFinishThreads>(s, n, 0, ~0ull - 1, limit, tid, token_at, weight)
                                             : last_item<false, kFinishThreads>(s, n, 0, (u64)a.vocab << 32, limit, tid, token_at, weight);
                token = (int)(f.key >> 32);
                const float x = logit_of(s.list[(u32)f.key]);
                logp = p.one ? 0.f : (float)(((double)x - (double)r.top) * r.inv - log((double)counted_q * 0x1p-50));
            }
        }
    }
    const bool keep_all = MASK && !bad && !a.direct && !p.one && !(p.by_count && p.k < live) && !p.by_mass && !p.by_share;
    if (MASK) {
        T* const out = (T*)a.out + (int64_t)i * a.out_stride;
        const T none = from_f<T>(-__builtin_inff());
        const bool pass = bad && p.good;                    // (its logits are no distribution: they are passed on)
        if (bad) cut = 0;
        if (pass || a.direct) {
            if (!pass || !a.in_place)
                for (int v = tid; v < a.vocab; v += kFinishThreads) {
                    const T x = row[v];
                    out[v] = pass || (to_f(x) > -__builtin_inff() && comp_of(to_f(x), v) <= cut) ? x : none;
                }
        } else if (!bad && !wide && !keep_all && !a.in_place) {
            for (int e = tid; e < n; e += kFinishThreads)
                if (s.list[e] <= cut) out[token_of(s.list[e])] = row[token_of(s.list[e])];
        }
    }
    if (tid != 0) return;
    if (!a.direct) {
        RowOut o{};
        o.cut = cut;
        o.state = bad ? (p.good ? ROW_BAD : ROW_CUT) : keep_all ? ROW_CUT : !wide ? ROW_DONE : type < 0 ? ROW_SLOW : ROW_WIDE;
        o.type = type;
        o.top = r.top;
        o.ref = bound;
        o.least = least;
        o.listed = valid;
        o.listed_q = listed_q;
        o.total = total;
        o.x_m = x_m;
        o.found = -1;
        a.rows[i] = o;
        if (o.state == ROW_WIDE || o.state == ROW_SLOW) a.wide[1 + atomicAdd(a.wide, 1)] = i;
    }
    if (keep_all) kept = live;
    else if (wide) return;
    if (a.kept) a.kept[i] = kept;
    if (MASK) return;
    a.token[i] = token;
    if (a.logprob) a.logprob[i] = logp;
}

// ---------------------------------------------------------------- rows whose cut is beyond their lists
// 2^bits exp((x - ref) / temperature) to a whole number, x at most ref or little above it
struct TableWeight {
    const word2* pow;
    double ref, unit;
    u32 up;
    __device__ TableWeight(const word2* table, float of, double inv, int bits) : pow(table), ref((double)of), unit(inv * 369.3299304675746), up(256u * (u32)bits) {}
    __device__ __forceinline__ u64 operator()(float x) const {
        const double t = fmax(((double)x - ref) * unit, -900.0 * 256.0), big = t + 0x1.8p52;
        return __builtin_bit_cast(u64, times_power(pow, small_power(t - (big - 0x1.8p52)), (u32)__builtin_bit_cast(u64, big) + up, 0x1p52)) & 0xFFFFFFFFFFFFFull;
    }
};
// the range of a logit below `ref`, the first next to it
struct Ranges {
    float ref, per_unit;
    __device__ Ranges(const RowOut& o) : ref(o.ref < __builtin_inff() ? o.ref : o.top) {
        const float width = ref - o.least;
        per_unit = width > 0.f && width < __builtin_inff() ? (float)fmin((kRanges - 1) / (double)width, 1e38) : 1.f;
    }
    __device__ __forceinline__ int operator()(float x) const { return (int)fminf((ref - x) * per_unit, (float)(kRanges - 1)); }
};
__device__ __forceinline__ int sum_bits(int n) { return min(kListBits, 61 - (32 - __clz(n))); }      // n weights stay below 2^62
// Counts of the ranges by part, in 16 bits each.  Bound by the LDS atomics: 140 rows of 151936 20 us.
template <typename T, bool VEC>
__global__ __launch_bounds__(kPartThreads) void k_filter_bins(FilterArgs a) {
    using R = Run<T, VEC>;
    __shared__ u32 s_bins[kRanges];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int items = *a.wide * a.n_parts;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int i = a.wide[1 + item / a.n_parts], part = item % a.n_parts;
        RowOut& o = a.rows[i];
        if (o.type != BY_MASS && o.type != BY_COUNT) continue;
        const T* const row = (const T*)a.logits + (int64_t)i * a.row_stride;
        const int p0 = part * a.part_len, run = a.part_len / kPartWaves, v_begin = min(p0 + wave * run, a.vocab), v_end = min(v_begin + run, a.vocab);
        const Ranges range_of(o);
        const float below = o.ref;
        __syncthreads();
        for (int e = tid; e < kRanges; e += kPartThreads) s_bins[e] = 0;
        __syncthreads();
        float next[kPer];
        R::load(row, v_begin, v_end, lane, next);
        for (int v0 = v_begin; v0 < v_end; v0 += kStep) {
            float x[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) x[e] = next[e];
            if (v0 + kStep < v_end) R::load(row, v0 + kStep, v_end, lane, next);
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (x[e] < below && x[e] > -__builtin_inff()) atomicAdd(&s_bins[range_of(x[e])], 1u);
        }
        __syncthreads();
        // (16 bits a count: one that does not fit, of parts beyond 65535 logits, makes the ranges miss the cut, which k_filter_close sees)
        u32* const slices = a.slices + (int64_t)i * a.n_parts * (kRanges / 2);
        for (int e = tid; e < kRanges / 2; e += kPartThreads) slices[part * (kRanges / 2) + e] = min(s_bins[2 * e], 65535u) | min(s_bins[2 * e + 1], 65535u) << 16;
    }
}

// The ranges in which the cut may lie, by the counts times the weights at their middles: ranges are narrow (0.005 of a logit, 200 tokens, for 150,000 tokens
// over 10), so that a few are left for k_filter_gather, which has exact sums.  false: nothing is found.
struct RangeShared { double sum[2][kPartWaves]; int32_t at[2][kPartWaves]; };
__device__ __forceinline__ bool find_ranges(RangeShared& s, const FilterArgs& a, const RowOut& o, const Params& q, const u32* slices, double aside, int more, int tid, float& x_lo, float& x_hi) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Ranges range_of(o);
    const float below = o.ref;
    const bool count = o.type == BY_COUNT;
    // what the ranges hold, eight a thread, and where the limit falls
    constexpr int PER = kRanges / kPartThreads;
    static_assert(PER == 8);
    u32 each[PER] = {};
    constexpr int AHEAD = 16;
    for (int j0 = 0; j0 < a.n_parts; j0 += AHEAD) {
        uint4 m[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) m[j] = j0 + j < a.n_parts ? *(const uint4*)(slices + (j0 + j) * (kRanges / 2) + 4 * tid) : uint4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const u32 two[4] = {m[j].x, m[j].y, m[j].z, m[j].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                each[2 * e] += two[e] & 0xFFFF;
                each[2 * e + 1] += two[e] >> 16;
            }
        }
    }
    // a range's weight is about its count times the weight at its middle, and for all of them together the logits lie within an eighth of a range of the middles;
    // bf16's, which lie on a grid of their own, within 0.3 of one, and four ranges more (flat rows of 151936 bf16 logits missed their cut with an
    // eighth in 2 of 600, with 0.3 in 1 of 1400, with two more in 1 of 2800)
    const double limit = count ? (double)(q.k - o.listed) : (double)q.p * o.total - (double)o.listed_q * 0x1p-50;
    const double width = count ? 0.0 : q.inv / (double)range_of.per_unit, step = exp_neg(-width), spare = exp_neg(-aside * width), over = 1.0 / spare;
    double middle = count ? 1.0 : exp_neg(fmin(((double)range_of.ref - (double)o.top) * q.inv - (PER * tid + 0.5) * width, 0.0));
    double least = 0.0, most = 0.0, v_least[PER], v_most[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const bool rest = !count && PER * tid + e == kRanges - 1;          // (all that is below the others)
        least += v_least[e] = rest ? 0.0 : each[e] * middle * spare;
        most += v_most[e] = each[e] * middle * over;
        middle *= step;
    }
    const double up_least = wave_scan64_dpp(least), up_most = wave_scan64_dpp(most);
    if (lane == 63) {
        s.sum[0][wave] = up_least;
        s.sum[1][wave] = up_most;
    }
    __syncthreads();
    double at_least = up_least - least, at_most = up_most - most;
    for (int w = 0; w < wave; ++w) {
        at_least += s.sum[0][w];
        at_most += s.sum[1][w];
    }
    // the first range that may, and the first that must, reach the limit
    int b0 = kRanges, b1 = kRanges;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        at_least += v_least[e];
        at_most += v_most[e];
        if (at_most >= limit) b0 = min(b0, PER * tid + e);
        if (at_least >= limit) b1 = min(b1, PER * tid + e);
    }
    for (int f = 32; f > 0; f >>= 1) {
        b0 = min(b0, __shfl_xor(b0, f));
        b1 = min(b1, __shfl_xor(b1, f));
    }
    if (lane == 0) {
        s.at[0][wave] = b0;
        s.at[1][wave] = b1;
    }
    __syncthreads();
    b0 = min(min(s.at[0][0], s.at[0][1]), min(s.at[0][2], s.at[0][3]));
    b1 = min(min(min(s.at[1][0], s.at[1][1]), min(s.at[1][2], s.at[1][3])), kRanges - 1);
    const bool good = b0 < kRanges && limit > 0.0;
    b0 = max(b0 - more, 0);
    b1 = min(b1 + more, kRanges - 1);
    x_lo = from_key(first_key(range_of.ref, lane, [&](float x) { return range_of(x) <= b1; }));
    x_hi = b0 == 0 ? below : from_key(first_key(range_of.ref, lane, [&](float x) { return range_of(x) < b0; }));
    return good;
}

// The tokens of the ranges in which the cut may lie, and what lies above them, by part; every workgroup finds the ranges for itself.  Bound by the exponentials of
// what is kept: 140 rows of 151936 45 us.  (With a row's last workgroup finding the ranges in k_filter_bins, and here the cut, the fences around that took longer than either
// kernel's own work: 95 + 87 us against 20 + 45 + k_filter_close's 21.)
template <typename T, bool VEC>
__global__ __launch_bounds__(kPartThreads) void k_filter_gather(FilterArgs a) {
    using R = Run<T, VEC>;
    __shared__ word2 s_pow[256];
    __shared__ RangeShared s;
    __shared__ u64 s_q[kPartWaves];
    __shared__ int32_t s_above[kPartWaves], s_listed[kPartWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int items = *a.wide * a.n_parts;
    if ((int)blockIdx.x >= items) return;
    s_pow[tid] = kPow.at[tid];
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int i = a.wide[1 + item / a.n_parts], part = item % a.n_parts;
        RowOut& o = a.rows[i];
        const Params q = params_of(a, i / a.per);
        const T* const row = (const T*)a.logits + (int64_t)i * a.row_stride;
        const int p0 = part * a.part_len, run = a.part_len / kPartWaves, v_begin = min(p0 + wave * run, a.vocab), v_end = min(v_begin + run, a.vocab);
        float next[kPer];
        R::load(row, v_begin, v_end, lane, next);          // (on their way while the ranges are found)
        float x_lo = o.x_m, x_hi = o.x_m;
        int type = o.type;
        __syncthreads();
        if (type >= 0 && type != BY_SHARE) {
            if (!find_ranges(s, a, o, q, a.slices + (int64_t)i * a.n_parts * (kRanges / 2), sizeof(T) == 2 ? 0.3 : 0.125, sizeof(T) == 2 ? 4 : 0, tid, x_lo, x_hi)) type = -1;
            else if (o.x_m >= x_hi) type = BY_SHARE, x_lo = x_hi = o.x_m;          // min-p keeps less
        }
        if (part == 0 && tid == 0) {
            o.found = type;
            o.x_lo = x_lo;
            o.x_hi = x_hi;
        }
        if (type < 0) continue;
        const int bits = sum_bits(a.vocab);
        const TableWeight weight(s_pow, o.top, q.inv, bits);
        u64* const lists = a.lists + (int64_t)i * a.n_parts * kPartWaves * a.list_len;
        u64* const list = lists + (part * kPartWaves + wave) * (int64_t)a.list_len;
        u64 sum = 0;
        int above = 0, listed = 0;
        for (int v0 = v_begin; v0 < v_end; v0 += kStep) {
            float x[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) x[e] = next[e];
            if (v0 + kStep < v_end) R::load(row, v0 + kStep, v_end, lane, next);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                if (x[e] >= x_hi) {
                    ++above;
                    sum += weight(x[e]);
                }
                const bool in = x[e] >= x_lo && x[e] < x_hi;
                const u64 m = __ballot(in);
                if (!m) continue;
                const int at = listed + __builtin_amdgcn_mbcnt_hi((u32)(m >> 32), __builtin_amdgcn_mbcnt_lo((u32)m, 0));
                if (in && at < a.list_len) list[at] = comp_of(x[e], v0 + R::place(e, lane));
                listed += __popcll(m);
            }
        }
        sum = wave_sum_u64(sum);
        above = wave_sum_int(above);
        if (lane == 0) {
            s_q[wave] = sum;
            s_above[wave] = above;
            s_listed[wave] = listed;
        }
        __syncthreads();
        if (tid == 0) {
            Part& to = a.parts[(int64_t)i * a.n_parts + part];
            to.above = s_above[0] + s_above[1] + s_above[2] + s_above[3];
            for (int w = 0; w < kPartWaves; ++w) {
                to.above_q[w] = s_q[w];
                to.listed[w] = s_listed[w];
            }
        }
    }
}

// The cut of a row from what k_filter_gather left, and the draw; false: it does not lie there
struct CloseShared { ListShared<kCloseList> f; u64 part[kMostParts * kPartWaves]; word2 pow[256]; };
template <typename T, bool VEC, bool MASK>
__device__ __forceinline__ bool close_row(CloseShared& c_s, const FilterArgs& a, int i, RowOut& o, const Params& q, int tid) {
    auto& s = c_s.f;
    u64* const s_part = c_s.part;
    const int lane = tid & 63, run = a.part_len / kPartWaves, bits = sum_bits(a.vocab);
    const T* const row = (const T*)a.logits + (int64_t)i * a.row_stride;
    const float x_lo = o.x_lo, x_hi = o.x_hi;
    if (tid < 256) c_s.pow[tid] = kPow.at[tid];
    const TableWeight weight(c_s.pow, o.top, q.inv, bits);
    // the row from its parts
    if (tid < kMostParts * kPartWaves) s_part[tid] = tid < a.n_parts * kPartWaves ? a.parts[(int64_t)i * a.n_parts + tid / kPartWaves].above_q[tid % kPartWaves] : 0;
    __syncthreads();
    int n_above = lane < a.n_parts ? a.parts[(int64_t)i * a.n_parts + lane].above : 0;
    n_above = wave_sum_int(n_above);
    const int n = read_lists<kThreads>(s, a, i, list_length(a, i, tid), tid, (1ull << 56) - 1);
    if (n < 0) return false;
    u64 cut = (u64)~key_of(x_hi) << 24 | 0xFFFFFF;      // (x_hi itself is above)
    const u64 over_q = wave_sum_u64(s_part[lane] + s_part[lane + 64] + s_part[lane + 128] + s_part[lane + 192]);
    const double mass = ceil((double)q.p * o.total * ldexp(1.0, bits));
    // (where k_filter_gather took min-p for the filter that keeps less, that was by an estimate, or by counts that may have been cut off: the weights, and the count, from its
    // logit on say whether it is)
    bool good = o.found != BY_SHARE || (o.type == BY_MASS ? (double)over_q < mass : o.type != BY_COUNT || n_above <= q.k);
    if (o.found != BY_SHARE) {
        const bool count = o.found == BY_COUNT;
        u64 mine = 0;
        for (int e = tid; e < n; e += kThreads) mine += s.weight[e] = count ? 1 : weight(logit_of(s.list[e]));
        const u64 listed = block_sum<kThreads>(s, mine, 0, tid).q;
        // what the range may still keep; the cut lies in it if something, and no more than it has
        const double left = count ? (double)(q.k - n_above) : mass - (double)over_q;
        good = n > 0 && left >= 1.0 && left <= (double)listed;
        if (good)
            cut = last_item<false, kThreads>(s, n, (u64)~(key_of(x_hi) - 1) << 24, (u64)~key_of(x_lo) << 24 | 0xFFFFFF, (u64)left, tid,
                                             [&](int e) { return s.list[e]; }, [&](int e) { return s.weight[e]; }).key;
        if (q.by_share) cut = min(cut, (u64)~key_of(o.x_m) << 24 | 0xFFFFFF);
    }
    if (!good) return false;
    int kept = 0;
    for (int e = tid; e < n; e += kThreads) {
        const u64 c = s.list[e];
        if (c > cut) continue;
        ++kept;
        if (!MASK) atomicAdd(&s_part[token_of(c) / run], weight(logit_of(c)));
    }
    kept = block_sum<kThreads>(s, 0, kept, tid).n + n_above;
    int token = -1;
    float logp = 0.f;
    if (!MASK) {
        const float u = a.u[i];
        // a lane four waves' runs
        u64 each[4], own = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) own += each[e] = s_part[4 * lane + e];
        const u64 up = wave_scan_u64(own), total = of_lane(up, 63);
        u64 target = u > 0.f ? min((u64)((double)u * (double)total), total - 1) : 0;
        const int of = __ffsll((unsigned long long)__ballot(up > target)) - 1;
        target -= of_lane(up - own, of);
        int w = 0;
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            const u64 q_e = of_lane(each[e], of);
            if (w == e && target >= q_e) {
                target -= q_e;
                ++w;
            }
        }
        const int first = (4 * of + w) * run, end = min(first + run, a.vocab), share = (run / 16 + kWaves - 1) / kWaves * 16;
        const float cut_x = logit_of(cut);
        const int cut_v = token_of(cut);
        token = draw_part<T, VEC, kThreads>(s, row, first, share, end, target, tid,
                                            [&](float x, int v) { return x > cut_x || (x == cut_x && v <= cut_v) ? weight(x) : 0; });
        logp = (float)(((double)to_f(row[token]) - (double)o.top) * q.inv - log((double)total * ldexp(1.0, -bits)));
    }
    if (tid == 0) {
        o.cut = cut;
        o.state = ROW_CUT;
        if (a.kept) a.kept[i] = kept;
        if (!MASK) {
            a.token[i] = token;
            if (a.logprob) a.logprob[i] = logp;
        }
    }
    return true;
}

// The cut of a row whatever it is, from the row itself
template <typename T, bool VEC, bool MASK>
__device__ __forceinline__ void slow_row(Shared& s, const FilterArgs& a, int i, const Params& q, int tid) {
    Row<T, VEC> row{(const T*)a.logits + (int64_t)i * a.row_stride, a.vocab, tid, tid & 63, tid >> 6, s, RowState{}};
    RowState& r = row.r;
    row.look();
    r.inv = q.inv;
    const double range = (double)r.top - (double)r.least;
    r.per_unit = fmax(64.0 * r.inv, range > 0.0 ? (kBins - 1.5) / range : 1.0);
    r.bin_width = r.inv / r.per_unit;
    r.bits = min(50, 61 - (32 - __clz(a.vocab)));
    r.cut = (u64)~key_of(r.least) << 24 | 0xFFFFFF;
    r.kept = r.live;
    r.listed = -1;
    const int k = q.one ? 1 : q.by_count ? q.k : r.live;
    if (k < r.live) row.template select<true>([&](double) { return (double)k; });
    if (q.by_mass) {
        if (r.listed >= 0) {
            r.kept = list_below(s, r, s.big, r.kept, tid, [&](double total) { return (double)q.p * total; });
            r.cut = s.big[r.kept - 1];
        } else {
            row.template select<false>([&](double total) { return (double)q.p * total; });
        }
    }
    if (q.by_share) {
        const double most = -log((double)q.m);
        row.at_least(first_key(r.top, tid & 63, [&](float x) { return ((double)r.top - (double)x) * r.inv <= most; }));
    }
    int token = -1;
    float logp = 0.f;
    if (!MASK) token = row.draw(a.u[i], logp);
    else if (r.kept < 0) row.count();
    if (tid != 0) return;
    if (a.kept) a.kept[i] = r.kept;
    if (MASK) {
        a.rows[i].cut = r.cut;
        a.rows[i].state = ROW_CUT;
        return;
    }
    a.token[i] = token;
    if (a.logprob) a.logprob[i] = logp;
}

// The rows that k_filter_gather has read, and those that are left: a workgroup a row.  Bound by its chain, as k_filter_finish: 140 rows 21 us; a row that has to be
// read again (slow_row) 80 to 250.
template <typename T, bool VEC, bool MASK>
__global__ __launch_bounds__(kThreads) void k_filter_close(FilterArgs a) {
    __shared__ union { Shared slow; CloseShared close; } shared;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= *a.wide) return;
    const int i = a.wide[1 + blockIdx.x];
    RowOut& o = a.rows[i];
    const Params q = params_of(a, i / a.per);
    if (o.found >= 0) {
        if (close_row<T, VEC, MASK>(shared.close, a, i, o, q, tid)) return;
        __syncthreads();
    }
    slow_row<T, VEC, MASK>(shared.slow, a, i, q, tid);
}

// In place: what is dropped.  Else, of the rows that were not written from their lists, what is kept (k_filter_parts has filled the rest).  Bound by its accesses, an element a lane:
// 576 rows of 151936, a ninth of them flat and an eighth without any filter (their logits are written over the fill), 35 us, 38 MB read and 67 written.  In place nearly all of every
// row is written here: those 576 rows take 270 us in all instead of 241 apart, of bf16 179 instead of 171.
template <typename T, bool IN_PLACE>
__global__ __launch_bounds__(kPartThreads) void k_filter_apply(FilterArgs a) {
    const int i = blockIdx.y, state = a.rows[i].state;
    if (state != ROW_CUT && !(IN_PLACE && state == ROW_DONE)) return;
    const u64 cut = a.rows[i].cut;
    const int end = min((int)(blockIdx.x + 1) * a.part_len, a.vocab);
    const T* const row = (const T*)a.logits + (int64_t)i * a.row_stride;
    T* const out = (T*)a.out + (int64_t)i * a.out_stride;
    constexpr int AHEAD = 8;
    for (int v0 = blockIdx.x * a.part_len + threadIdx.x; v0 < end; v0 += AHEAD * kPartThreads) {
        T x[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (v0 + j * kPartThreads < end) x[j] = row[v0 + j * kPartThreads];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int v = v0 + j * kPartThreads;
            if (v >= end) continue;
            const bool in = to_f(x[j]) > -__builtin_inff() && comp_of(to_f(x[j]), v) <= cut;
            if (IN_PLACE && !in) out[v] = from_f<T>(-__builtin_inff());
            if (!IN_PLACE && in) out[v] = x[j];
        }
    }
}

// How a call is cut.  Measured with a top-k and a top-p, both ways, us:
//   one launch (rows are their own lists) | the lists: 1 row, 64, 1280 rows of 1024: 18.8 | 18.8, 21.3 | 20.5, 34.7 | 32.7; of 1280: 14.8 | 19.7, 23.9 | 21.6, 38.2 | 38.3; of
//     1536: 25.0 | 18.5, 26.7 | 21.3, 41.3 | 34.9; without filters 8.1 | 12.7 and 14.2 | 23.9 (1 and 1280 rows of 1024).
//   parts as here | of 16384 or more | of 4096, rows of 151936 fp32: 1 row 22.2 | 25.5 | 22.1, 64 rows 30.5 | 31.1 | 31.4, 256 rows 48.2 | 47.7 | 56.4, 1024 rows 154.5 | 154.1 | 172.5.
//   rows at multiples of 16 bytes | others (RowLoop and Run without VEC): 1280 rows of 151936 fp32 189 | 188, 64 rows bf16 29.0 | 35.9.
struct Plan { int direct, n_parts, part_len, list_len, sample_len, sample_rank; };
int most_parts(int vocab) { return std::min((vocab - 1) / kLeastPart + 1, kMostParts); }
int least_parts(int vocab) { return std::min((vocab - 1) / kPart + 1, kMostParts); }
Plan plan_of(int rows, int vocab) {
    Plan p{};
    p.direct = vocab <= kDirect;
    if (p.direct) return p;
    // parts of up to kPart logits; smaller ones, down to kLeastPart, where the rows alone do not fill the chip
    p.n_parts = std::max(least_parts(vocab), std::min(most_parts(vocab), kFillParts / rows));
    p.part_len = ((vocab - 1) / (p.n_parts * kPartWaves) / 16 + 1) * 16 * kPartWaves;    // (waves' runs alike, as whole vectors)
    // kWanted of the row, a share f of its logits: a group's largest lies among them with probability 1 - (1 - f)^n
    // (at most a fifth: the least of all groups' largest would now and then be low enough for lists to overflow; 64 rows of 3500: 59 us against 26)
    const double f = std::min((double)kWanted / vocab, 0.2);
    p.sample_len = f < 0.015 ? 4 : f < 0.03 ? 2 : 1;
    p.sample_rank = std::min(kGroups, std::max(1, (int)(kGroups * (1.0 - pow(1.0 - f, 16.0 * p.sample_len)) + 0.5)));
    // eight times what a wave should find, but no more than a row's lists may hold together
    p.list_len = std::max(128, std::min(kList / kPartWaves, (8 * kWanted / (p.n_parts * kPartWaves) + 15) / 16 * 16));
    return p;
}
size_t lists_bytes(const Plan& p, int rows) { return (size_t)rows * p.n_parts * kPartWaves * p.list_len * sizeof(u64); }
size_t slices_bytes(const Plan& p, int rows) { return (size_t)rows * p.n_parts * (kRanges / 2) * sizeof(u32); }
size_t parts_bytes(const Plan& p, int rows) { return (size_t)rows * p.n_parts * sizeof(Part); }

template <typename T, bool MASK>
tasc_status enqueue(FilterArgs a, int rows, void* workspace, hipStream_t st) {
    const bool vec = (((uintptr_t)a.logits | (uintptr_t)(a.row_stride * (int64_t)sizeof(T))) & 15) == 0;
    const Plan p = plan_of(rows, a.vocab);
    a.direct = p.direct;
    a.in_place = MASK && a.out == a.logits;
    const dim3 all((unsigned)rows), threads(kPartThreads), parts((unsigned)p.n_parts, (unsigned)rows);
    if (!p.direct) {
        a.parts = (Part*)workspace;
        a.rows = (RowOut*)((char*)workspace + parts_bytes(p, rows));
        a.lists = (u64*)((char*)a.rows + (size_t)rows * sizeof(RowOut));
        a.slices = (u32*)((char*)a.lists + lists_bytes(p, rows));
        a.wide = (int32_t*)((char*)a.slices + slices_bytes(p, rows));
        a.n_parts = p.n_parts;
        a.part_len = p.part_len;
        a.list_len = p.list_len;
        a.sample_len = p.sample_len;
        a.sample_rank = p.sample_rank;
        a.out_aligned = (((uintptr_t)a.out | (uintptr_t)(a.out_stride * (int64_t)sizeof(T))) & 15) == 0;
        if (MASK && !a.in_place) vec ? k_filter_parts<T, true, true><<<parts, threads, 0, st>>>(a) : k_filter_parts<T, false, true><<<parts, threads, 0, st>>>(a);
        else vec ? k_filter_parts<T, true, false><<<parts, threads, 0, st>>>(a) : k_filter_parts<T, false, false><<<parts, threads, 0, st>>>(a);
    }
    vec ? k_filter_finish<T, true, MASK><<<all, dim3(kFinishThreads), 0, st>>>(a) : k_filter_finish<T, false, MASK><<<all, dim3(kFinishThreads), 0, st>>>(a);
    if (!p.direct) {
        if (a.top_k || a.top_p || a.min_p) {
            const dim3 some((unsigned)std::min<int64_t>((int64_t)rows * p.n_parts, kWideGrid));
            vec ? k_filter_bins<T, true><<<some, threads, 0, st>>>(a) : k_filter_bins<T, false><<<some, threads, 0, st>>>(a);
            vec ? k_filter_gather<T, true><<<some, threads, 0, st>>>(a) : k_filter_gather<T, false><<<some, threads, 0, st>>>(a);
        }
        vec ? k_filter_close<T, true, MASK><<<all, dim3(kThreads), 0, st>>>(a) : k_filter_close<T, false, MASK><<<all, dim3(kThreads), 0, st>>>(a);
        if (MASK) a.in_place ? k_filter_apply<T, true><<<parts, threads, 0, st>>>(a) : k_filter_apply<T, false><<<parts, threads, 0, st>>>(a);
    }
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}

tasc_status check_rows(const char* who, const void* logits, tasc_dtype dtype, int64_t row_stride, int64_t rows, int32_t vocab) {
    TASC_REQUIRE(vocab >= 2 && vocab <= 1 << 24, "%s: vocab %d outside [2, 2^24]", who, vocab);
    TASC_REQUIRE(rows >= 0 && rows <= 65535, "%s: %lld rows outside [0, 65535]", who, (long long)rows);
    if (rows == 0) return TASC_OK;
    TASC_REQUIRE(logits, "%s: null argument", who);
    TASC_REQUIRE(dtype == TASC_F32 || dtype == TASC_BF16, "%s: dtype %d", who, (int)dtype);
    TASC_REQUIRE(row_stride >= vocab, "%s: rows of %d logits lie %lld apart", who, vocab, (long long)row_stride);
    TASC_REQUIRE((uintptr_t)logits % (dtype == TASC_F32 ? 4 : 2) == 0, "%s: logits must be aligned to their type", who);
    return TASC_OK;
}
tasc_status check_workspace(const char* who, void* workspace, size_t ws_bytes, int32_t rows, int32_t vocab) {
    const size_t need = tasc_sample_workspace_bytes(rows, vocab);
    if (need == 0) return TASC_OK;
    if (!workspace || ws_bytes < need) {
        tasc_set_error("%s: workspace of %zu of %zu bytes", who, workspace ? ws_bytes : 0, need);
        return TASC_ENOMEM;
    }
    TASC_REQUIRE(((uintptr_t)workspace & 15) == 0, "%s: the workspace must be 16-byte aligned", who);
    return TASC_OK;
}
// What a call reads and writes.  (The workspace holds rows' numbers that kernels go by.  A row's word may be written over one of its own that is read: that is done
// when all of the row's work is.)
struct Area { const char* name; const void* at; size_t bytes; bool words; };      // words: one of each row
template <size_t R, size_t W>
tasc_status check_apart(const char* who, const Area (&read)[R], const Area (&written)[W]) {
    auto apart = [](const Area& x, const Area& y) {
        return !x.at || !y.at || x.bytes == 0 || y.bytes == 0 || (uintptr_t)x.at + x.bytes <= (uintptr_t)y.at || (uintptr_t)y.at + y.bytes <= (uintptr_t)x.at;
    };
    for (const Area& w : written) {
        for (const Area& r : read)
            TASC_REQUIRE(apart(w, r) || (w.words && r.words && w.at == r.at && w.bytes == r.bytes), "%s: %s and %s overlap", who, w.name, r.name);
        for (const Area* v = written; v != &w; ++v) TASC_REQUIRE(apart(w, *v), "%s: %s and %s overlap", who, w.name, v->name);
    }
    return TASC_OK;
}
size_t rows_bytes(int64_t rows, int64_t row_stride, int32_t vocab, tasc_dtype dtype) { return (size_t)((rows - 1) * row_stride + vocab) * (dtype == TASC_F32 ? 4 : 2); }

}  // namespace

extern "C" size_t tasc_sample_workspace_bytes(int32_t rows, int32_t vocab) {
    if (rows < 1 || rows > 65535 || vocab < 2 || vocab > 1 << 24) return 0;
    const Plan p = plan_of(rows, vocab);
    if (p.direct) return 0;
    // so much that fewer rows, in smaller parts, find room, too: of the parts that any number of rows up to this one has, and of their lists
    const size_t n_parts = std::max(std::min((size_t)rows * most_parts(vocab), (size_t)kFillParts), (size_t)rows * least_parts(vocab));
    const size_t listed = kPartWaves * std::max(128 * n_parts, std::min(kList / kPartWaves * n_parts, 8 * kWanted / kPartWaves * (size_t)rows + 16 * n_parts));
    return n_parts * (sizeof(Part) + kRanges / 2 * sizeof(u32)) + listed * sizeof(u64) + (size_t)rows * sizeof(RowOut) + ((size_t)rows + 1) * sizeof(int32_t);
}

extern "C" tasc_status tasc_sample(const void* logits, tasc_dtype dtype, int64_t row_stride, int32_t rows, int32_t vocab, const float* temperature, const int32_t* top_k,
                                   const float* top_p, const float* min_p, const float* u, int32_t* token, float* logprob, int32_t* kept, void* workspace,
                                   size_t ws_bytes, void* stream) {
    tasc_status rc = check_rows("sample", logits, dtype, row_stride, rows, vocab);
    if (rc != TASC_OK || rows == 0) return rc;
    TASC_REQUIRE(u && token, "sample: null argument");
    rc = check_workspace("sample", workspace, ws_bytes, rows, vocab);
    if (rc != TASC_OK) return rc;
    const size_t n = (size_t)rows * 4;
    const Area read[] = {{"logits", logits, rows_bytes(rows, row_stride, vocab, dtype), false}, {"temperature", temperature, n, true}, {"top_k", top_k, n, true},
                         {"top_p", top_p, n, true}, {"min_p", min_p, n, true}, {"u", u, n, true}};
    const Area written[] = {{"token", token, n, true}, {"logprob", logprob, n, true}, {"kept", kept, n, true}, {"workspace", workspace, tasc_sample_workspace_bytes(rows, vocab), false}};
    rc = check_apart("sample", read, written);
    if (rc != TASC_OK) return rc;
    const FilterArgs a{logits, row_stride, 1, vocab, temperature, top_k, top_p, min_p, u, token, logprob, kept};
    return dtype == TASC_F32 ? enqueue<float, false>(a, rows, workspace, (hipStream_t)stream) : enqueue<BF16, false>(a, rows, workspace, (hipStream_t)stream);
}

tasc_status tasc_filter_apart(const char* who, const void* logits, size_t logits_bytes, int32_t batch, int32_t k, int32_t vocab, const float* temperature, const int32_t* top_k,
                              const float* top_p, const float* min_p, const void* out, size_t out_bytes, const int32_t* kept, const void* workspace) {
    const size_t n = (size_t)batch * 4;
    const Area read[] = {{"temperature", temperature, n, true}, {"top_k", top_k, n, true}, {"top_p", top_p, n, true}, {"min_p", min_p, n, true}};
    const Area written[] = {{"out", out, out_bytes, false}, {"kept", kept, n * (k + 1), true}, {"workspace", workspace, tasc_sample_workspace_bytes(batch * (k + 1), vocab), false}};
    const tasc_status rc = check_apart(who, read, written);
    if (rc != TASC_OK || out == logits) return rc;
    const Area from[] = {{"logits", logits, logits_bytes, false}}, beside[] = {written[1], written[2]};
    return check_apart(who, from, beside);
}

extern "C" tasc_status tasc_filter_logits(const void* logits, tasc_dtype dtype, int64_t row_stride, int32_t batch, int32_t k, int32_t vocab, const float* temperature,
                                          const int32_t* top_k, const float* top_p, const float* min_p, void* out, int64_t out_stride, int32_t* kept, void* workspace,
                                          size_t ws_bytes, void* stream) {
    TASC_REQUIRE(k >= 0 && k <= TASC_MAX_K, "filter_logits: k %d outside [0, %d]", k, TASC_MAX_K);
    const int64_t rows = (int64_t)batch * (k + 1);
    tasc_status rc = check_rows("filter_logits", logits, dtype, row_stride, rows, vocab);
    if (rc != TASC_OK || rows == 0) return rc;
    TASC_REQUIRE(out, "filter_logits: null argument");
    const size_t size = dtype == TASC_F32 ? 4 : 2;
    TASC_REQUIRE(out_stride >= vocab && (uintptr_t)out % size == 0, "filter_logits: rows of %d logits to write lie %lld apart, or are not aligned to their type", vocab,
                 (long long)out_stride);
    const uintptr_t from = (uintptr_t)logits, to = (uintptr_t)out, from_n = rows_bytes(rows, row_stride, vocab, dtype), to_n = rows_bytes(rows, out_stride, vocab, dtype);
    TASC_REQUIRE((out == logits && out_stride == row_stride) || from + from_n <= to || to + to_n <= from, "filter_logits: logits and out overlap without being one");
    rc = check_workspace("filter_logits", workspace, ws_bytes, (int32_t)rows, vocab);
    if (rc != TASC_OK) return rc;
    rc = tasc_filter_apart("filter_logits", logits, from_n, batch, k, vocab, temperature, top_k, top_p, min_p, out, to_n, kept, workspace);
    if (rc != TASC_OK) return rc;
    const FilterArgs a{logits, row_stride, k + 1, vocab, temperature, top_k, top_p, min_p, nullptr, nullptr, nullptr, kept, out, out_stride};
    return dtype == TASC_F32 ? enqueue<float, true>(a, (int)rows, workspace, (hipStream_t)stream) : enqueue<BF16, true>(a, (int)rows, workspace, (hipStream_t)stream);
}
