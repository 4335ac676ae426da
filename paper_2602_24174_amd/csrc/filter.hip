// Sampling under top-k, top-p and min-p from given random numbers, and the same filters as masked logits.
//
// A row's tokens in the order of their logits (equal ones by index) are whole numbers of 56 bits, `comp`: the logit's bits, turned so that
// the largest comes first, over the index.  Every filter keeps a prefix of that order, so all of them together come to one last comp, `cut`.
//
// A prefix is found by a histogram over the values, 4096 bins between the largest logit and the least: of counts for top-k, of weights for
// top-p.  The bin in which the prefix ends then has few tokens, which are gathered, sorted and summed one by one.  A bin of more than fits
// (ties of thousands, a vocabulary of millions) is cut into 4096 again, by comp, until one token is left.
//
// Weights are sums of whole numbers, which no order of the work changes: a bin's of 2^-F of the weight at its middle, so that a bin far from the
// largest is as exact as one next to it, a list's and the draw's of 2^-F of the largest.
#include "numeric.h"
#include <algorithm>

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 4096, kList = 2048;
constexpr int kListBits = 50;                              // a list's weights: 2^11 of them stay below 2^62

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
};

__device__ __forceinline__ u32 key_of(float x) {           // grows with x; -0 is 0
    const u32 b = __float_as_uint(x + 0.f);
    return b ^ ((u32)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_key(u32 s) { return __uint_as_float(s & 0x80000000u ? s ^ 0x80000000u : ~s); }
__device__ __forceinline__ u64 comp_of(float x, int v) { return (u64)~key_of(x) << 24 | (u32)v; }
__device__ __forceinline__ float logit_of(u64 comp) { return from_key(~(u32)(comp >> 24)); }
__device__ __forceinline__ int token_of(u64 comp) { return (int)(comp & 0xFFFFFF); }

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ u64 wave_scan_u64(u64 v, int lane) {          // inclusive
    for (int o = 1; o < 64; o <<= 1) {
        const u64 up = __shfl_up(v, o);
        if (lane >= o) v += up;
    }
    return v;
}
__device__ __forceinline__ u64 of_lane(u64 v, int l) {
    return (u64)(u32)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 | (u32)__builtin_amdgcn_readlane((int)(u32)v, l);
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
    u64 big[kBins];                  // a histogram; lists of kList; segments of the draw
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
__device__ __forceinline__ u32 first_key(const RowState& r, int lane, F holds) {
    const u32 most = key_of(r.top), none = key_of(-__builtin_inff());
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
    const u64 up = wave_scan_u64(mine, lane);
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
        const u32 lo = first_key(r, lane, [&](float x) { return bin_of(r, x).at <= b; });
        const u32 hi = b == 0 ? key_of(__builtin_inff()) : first_key(r, lane, [&](float x) { return bin_of(r, x).at < b; });
        const float x_lo = from_key(lo), x_hi = from_key(hi);
        u64 *const all = s.big, *const own = s.big + kList;
        if (tid < 2) s.count[tid] = 0;
        __syncthreads();
        int above = 0;
        auto append = [&](u64* list, int which, bool in, float x, int v) {
            const u64 m = __ballot(in);
            if (!m) return;
            int at = 0;
            if (lane == 0) at = atomicAdd(&s.count[which], __popcll(m));
            at = __builtin_amdgcn_readfirstlane(at) + __popcll(m & ((1ull << lane) - 1));
            if (in && at < kList) list[at] = comp_of(x, v);
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
        if (n_all <= kList) {
            sort_list(all, n_all, tid);
            r.listed = n_all;
            const double scale = 0x1p50;
            static_assert(kListBits == 50);
            r.kept = UNIT ? (int)fmin(end, (double)n_all) : list_below(s, r, all, n_all, tid, [&](double) { return end * scale; });
            r.cut = all[r.kept - 1];
        } else if (n_own <= kList) {
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

    // the token that u falls on, and ln of its share
    __device__ int draw(float u, float& logp) {
        u64* const seg = s.big + kList;
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
            const u64 mine = seg[tid], up = wave_scan_u64(mine, lane);
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

template <typename T, bool VEC, bool MASK>
__global__ __launch_bounds__(kThreads) void k_filter_rows(FilterArgs a) {
    __shared__ Shared s;
    const int i = blockIdx.x, b = i / a.per, tid = threadIdx.x;
    Row<T, VEC> row{(const T*)a.logits + (int64_t)i * a.row_stride, a.vocab, tid, tid & 63, tid >> 6, s, RowState{}};
    RowState& r = row.r;
    const float t = a.temperature ? a.temperature[b] : 1.f, p = a.top_p ? a.top_p[b] : 1.f, m = a.min_p ? a.min_p[b] : 0.f;
    int k = a.top_k ? a.top_k[b] : 0;
    bool good = row.look();
    good = good && t >= 0.f && p == p && m == m;
    int token = -1;
    float logp = __builtin_nanf("");
    r.kept = 0;
    if (good) {
        if (t == 0.f || p <= 0.f || m > 1.f) k = 1;         // the first alone
        r.inv = t > 0.f ? 1.0 / (double)t : 1.0;
        const double range = (double)r.top - (double)r.least;
        r.per_unit = fmax(64.0 * r.inv, range > 0.0 ? (kBins - 1.5) / range : 1.0);
        r.bin_width = r.inv / r.per_unit;
        r.bits = min(50, 61 - (32 - __clz(a.vocab)));
        r.cut = (u64)~key_of(r.least) << 24 | 0xFFFFFF;
        r.kept = r.live;
        r.listed = -1;
        const bool by_mass = p > 0.f && p < 1.f && k != 1;
        if (k > 0 && k < r.live) row.template select<true>([&](double) { return (double)k; });
        if (by_mass) {
            if (r.listed >= 0) {
                r.kept = list_below(s, r, s.big, r.kept, tid, [&](double total) { return (double)p * total; });
                r.cut = s.big[r.kept - 1];
            } else {
                row.template select<false>([&](double total) { return (double)p * total; });
            }
        }
        if (m > 0.f && m <= 1.f && k != 1) {
            const double most = -log((double)m);
            row.at_least(first_key(r, tid & 63, [&](float x) { return ((double)r.top - (double)x) * r.inv <= most; }));
        }
        if (!MASK) token = row.draw(a.u[i], logp);
    }
    if (MASK) {
        const float cut_x = good ? logit_of(r.cut) : 0.f;
        const int cut_v = good ? token_of(r.cut) : 0;
        int kept = 0;
        T* const out = (T*)a.out + (int64_t)i * a.out_stride;
        for (int v = tid; v < a.vocab; v += kThreads) {
            const T x = row.row[v];
            const bool in = good && row.is_kept(to_f(x), v, cut_x, cut_v);
            kept += in;
            out[v] = in || !good ? x : from_f<T>(-__builtin_inff());
        }
        if (r.kept < 0) r.kept = block_count(s, kept, tid);
    }
    if (tid != 0) return;
    if (a.kept) a.kept[i] = r.kept;
    if (MASK) return;
    a.token[i] = token;
    if (a.logprob) a.logprob[i] = logp;
}

template <typename T, bool MASK>
tasc_status enqueue(const FilterArgs& a, int rows, hipStream_t st) {
    const bool vec = (((uintptr_t)a.logits | (uintptr_t)(a.row_stride * (int64_t)sizeof(T))) & 15) == 0;
    vec ? k_filter_rows<T, true, MASK><<<dim3((unsigned)rows), dim3(kThreads), 0, st>>>(a) : k_filter_rows<T, false, MASK><<<dim3((unsigned)rows), dim3(kThreads), 0, st>>>(a);
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

}  // namespace

extern "C" size_t tasc_sample_workspace_bytes(int32_t rows, int32_t vocab) {
    if (rows < 1 || rows > 65535 || vocab < 2 || vocab > 1 << 24) return 0;
    return 16;
}

extern "C" tasc_status tasc_sample(const void* logits, tasc_dtype dtype, int64_t row_stride, int32_t rows, int32_t vocab, const float* temperature, const int32_t* top_k,
                                   const float* top_p, const float* min_p, const float* u, int32_t* token, float* logprob, int32_t* kept, void* workspace,
                                   size_t ws_bytes, void* stream) {
    tasc_status rc = check_rows("sample", logits, dtype, row_stride, rows, vocab);
    if (rc != TASC_OK || rows == 0) return rc;
    TASC_REQUIRE(u && token, "sample: null argument");
    rc = check_workspace("sample", workspace, ws_bytes, rows, vocab);
    if (rc != TASC_OK) return rc;
    const FilterArgs a{logits, row_stride, 1, vocab, temperature, top_k, top_p, min_p, u, token, logprob, kept, nullptr, 0};
    return dtype == TASC_F32 ? enqueue<float, false>(a, rows, (hipStream_t)stream) : enqueue<BF16, false>(a, rows, (hipStream_t)stream);
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
    const uintptr_t from = (uintptr_t)logits, to = (uintptr_t)out, from_n = ((rows - 1) * row_stride + vocab) * size, to_n = ((rows - 1) * out_stride + vocab) * size;
    TASC_REQUIRE((out == logits && out_stride == row_stride) || from + from_n <= to || to + to_n <= from, "filter_logits: logits and out overlap without being one");
    rc = check_workspace("filter_logits", workspace, ws_bytes, (int32_t)rows, vocab);
    if (rc != TASC_OK) return rc;
    const FilterArgs a{logits, row_stride, k + 1, vocab, temperature, top_k, top_p, min_p, nullptr, nullptr, nullptr, kept, out, out_stride};
    return dtype == TASC_F32 ? enqueue<float, true>(a, (int)rows, (hipStream_t)stream) : enqueue<BF16, true>(a, (int)rows, (hipStream_t)stream);
}
