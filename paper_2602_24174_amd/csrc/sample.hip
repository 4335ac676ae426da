// Verification of drafted tokens against the target's probabilities, from given random numbers (paper, subsection "Speculative
// Decoding").
//
// With w(v) = exp((logit(v) - max) / temperature) and Z = sum w, draft d of a row is accepted iff u q(d) Z < w(d); the first row whose draft is
// not draws from max(0, w / Z - q) (q given) or from w without d (q a point mass), the row behind the last draft from w: the lowest v with
// sum up to v > u' total.
//
// Two passes over a row at most: k_sample_parts reads every logit once and leaves, per segment of 4096 tokens, the maximum (of a greedy
// sequence its place, too) and sum w relative to it, without the row's draft (so that what remains after a rejection is a sum, not a difference); k_sample_pick, a workgroup
// per sequence, joins the segments, decides, finds the segment that the draw falls into and reads that one again.  Given q, k_sample_decide
// joins and decides, and k_sample_residual sums max(0, w / Z - q) over the segments of the rejected row in between.
//
// Exponentials and sums are fp64: the draw compares sums over the whole vocabulary with u' total, and with fp32's 2^-24 on each of 150,000
// terms a token in a few thousand would come out as its neighbour.  An fp64 fma has the rate of an fp32 one here.
#include "numeric.h"
#include <algorithm>

namespace {

constexpr int kSeg = 4096, kPartThreads = 256, kPer = kSeg / kPartThreads, kPickThreads = 1024, kMostSegs = 8;

// A segment: sum of its weights, without the row's draft, in units of exp(scale) (-infinity: nothing above -infinity in it), its largest logit
// and, of a greedy sequence, that one's lowest place
struct __attribute__((aligned(16))) Part { double sum, scale; float top; int32_t at; };

struct Row;
struct SampleArgs {
    const void* logits;
    int64_t row_stride;
    int32_t k, vocab, n_seg;
    const int32_t* drafts;           // [B, k]
    const float* probs;              // nullable [B, k, vocab]
    const float* temperature;        // nullable [B]
    const float* u;                  // [B, n_u, 2]
    int64_t n_u;
    const int32_t* n_emit;           // null: row i of a sequence takes pair i; else pair min(n_emit + i, n_u - 1)
    Part* parts;                     // [B (k + 1), n_seg]
    Row* decided;             // [B (k + 1)], given probs
    double* residual;                // [B, n_seg], given probs
    int32_t *accept_len, *emitted;
    float* logprob;
    TascSessDev d;                   // a session's step (n_emit is not null): commits what it emits, as k_argmax_accept does
    int32_t max_len;
};
__device__ __forceinline__ double random_of(const SampleArgs& a, int b, int i, int which) {
    const int64_t pair = a.n_emit ? min((int64_t)a.n_emit[b] + i, a.n_u - 1) : i;
    return (double)a.u[2 * (b * a.n_u + pair) + which];
}

// 1 / temperature; 1 for a greedy sequence (its sums only tell whether the row holds a NaN), NaN for a temperature that is none
__device__ __forceinline__ double inv_temperature(const SampleArgs& a, int b) {
    const float t = a.temperature ? a.temperature[b] : 1.f;
    return t > 0.f ? 1.0 / (double)t : t == 0.f ? 1.0 : __builtin_nan("");
}
__device__ __forceinline__ bool is_greedy(const SampleArgs& a, int b) { return a.temperature && a.temperature[b] == 0.f; }
__device__ __forceinline__ int draft_of(const SampleArgs& a, int b, int i) {     // -1: the row scores none
    const int d = i < a.k ? a.drafts[(int64_t)b * a.k + i] : -1;
    return d >= 0 && d < a.vocab ? d : -1;
}
// a logit over the temperature, in the units of a row's weights; the product is rounded as the scale's own was, so that equal logits
// come out equal however large they are
__device__ __forceinline__ double exponent(float logit, double inv, double scale) {
#pragma clang fp contract(off)
    const double y = (double)logit * inv;
    return y - scale;
}
template <typename T>
__device__ __forceinline__ const T* row_of(const SampleArgs& a, int b, int i) {
    return (const T*)a.logits + ((int64_t)b * (a.k + 1) + i) * a.row_stride;
}
// A thread's 16 logits of a segment: VEC, 16 bytes side by side at a time (rows start at multiples of 16 bytes), else thread by thread
template <typename T, bool VEC>
struct Segment {
    static constexpr int SIDE = VEC ? 16 / (int)sizeof(T) : 1;
    static __device__ __forceinline__ int place(int e, int tid) { return (e / SIDE * kPartThreads + tid) * SIDE + e % SIDE; }
    static __device__ __forceinline__ void load(const T* __restrict__ row, int v0, int vocab, int tid, float (&x)[kPer]) {
        if (VEC && v0 + kSeg <= vocab) {
#pragma unroll
            for (int e = 0; e < kPer; e += SIDE) load_n<SIDE == 1 ? 4 : SIDE>(row + v0 + place(e, tid), x + e);
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int v = v0 + place(e, tid);
                x[e] = v < vocab ? to_f(row[v]) : -__builtin_inff();
            }
        }
    }
};

// What bounds it is the exponentials, 16 a thread and segment: exp(y) = 2^(i / 256) exp(f ln 2 / 256) with i = rint(256 y / ln 2), the first factor out of a
// table of 256 in LDS with i / 256 added to its exponent, the second by the polynomial of degree 3 (|f| <= 1/2: its remainder is below
// (ln 2 / 512)^4 / 24 = 1.4e-13).  A wave's weights are relative to the power of 2^(1/256) next to its largest, so that y = x / temperature - i' ln 2 / 256
// takes one fma, the rounding is the addition of 1.5 2^52 in another, which leaves i in the lower word, and the table has i's lower bits
// taken out of its exponents before: 10 instructions an element (rint, conversion and ldexp have a quarter of the rate of a product).
// Waves that hold logits too far from their largest for that (masked ones, say), or so large that 2^-53 of them counts, take the loop behind it.
// us of this kernel, 1280 rows of 151936 fp32 logits: exp_neg, with the place of the maximum followed as it went, 250; a table of 64, rint, a
// conversion and ldexp 169; the second loop for all waves 151; as it is 138 (5.6 TB/s).
// SEVERAL: a workgroup takes kMostSegs segments side by side, the next one's logits under way while one's exponentials are computed, and its
// waves do not wait for each other before the last; the registers for it cost three of seven waves a SIMD.
template <typename T, bool VEC, bool SEVERAL>
__global__ __launch_bounds__(kPartThreads) __attribute__((amdgpu_waves_per_eu(SEVERAL ? 4 : 6))) void k_sample_parts(SampleArgs a) {
    using S = Segment<T, VEC>;
    constexpr int kWaves = kPartThreads / 64, kMost = SEVERAL ? kMostSegs : 1;
    __shared__ word2 s_pow[256];
    __shared__ float s_top[kMost * kWaves];
    __shared__ int32_t s_at[kMost * kWaves];
    __shared__ double s_sum[kMost * kWaves], s_scale[kMost * kWaves];
    const int r = blockIdx.y, b = r / (a.k + 1), i = r % (a.k + 1), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int s0 = blockIdx.x * kMost, n = SEVERAL ? min(kMost, a.n_seg - s0) : 1;
    const T* const row = row_of<T>(a, b, i);
    float next[kPer];
    S::load(row, s0 * kSeg, a.vocab, tid, next);
    static_assert(kPartThreads == 256, "a thread an entry");
    s_pow[tid] = kPow.at[tid];
    const double inv = inv_temperature(a, b), unit = inv * 369.3299304675746;     // 256 / ln 2
    const int d = draft_of(a, b, i);
    const bool greedy = is_greedy(a, b);
    __syncthreads();
    for (int g = 0; g < n; ++g) {
        const int v0 = (s0 + g) * kSeg;
        float x[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = next[e];
        if (SEVERAL && g + 1 < n) S::load(row, v0 + kSeg, a.vocab, tid, next);
        float top = x[0], least = x[0];
#pragma unroll
        for (int e = 0; e < kPer; e += 2) {                 // (fmaxf would quiet its operands first; a NaN is left out by either)
            asm("v_max3_f32 %0, %1, %2, %3" : "=v"(top) : "v"(top), "v"(x[e]), "v"(x[e + 1]));
            asm("v_min3_f32 %0, %1, %2, %3" : "=v"(least) : "v"(least), "v"(x[e]), "v"(x[e + 1]));
        }
        top = wave_max_dpp(top);
        const int place = g * kWaves + wave;
        if (greedy) {                                       // the lowest place of the maximum
            int32_t at = 0x7FFFFFFF;
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (x[e] == top) at = min(at, v0 + S::place(e, tid));
            for (int o = 32; o > 0; o >>= 1) at = min(at, __shfl_xor(at, o));
            if (lane == 0) s_at[place] = at;
        }
        const double whole = rint((double)top * unit);
        double sum = 0.0, scale;
        // (conditions that a NaN fails: such a wave takes the second loop, and so do those of the draft's segment)
        if (!__any(!((double)least * unit > whole - 600.0 * 369.0)) && fabs(whole) < 0x1p24 && (d < v0 || d >= v0 + kSeg)) {
            const double start = 0x1.8p52 - whole;
            scale = whole * (0.69314718055994530942 / 256);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const double y = (double)x[e], big = __builtin_fma(y, unit, start);
                sum = times_power(s_pow, small_power(__builtin_fma(y, unit, start - big)), (u32)__builtin_bit_cast(u64, big), sum);
            }
        } else {
            // y is no less than -1023 ln 2, where an entry's exponent and mantissa come out as zero: a masked token weighs exactly nothing
            const double base = top == -__builtin_inff() ? 0.0 : (double)top;
            scale = top == -__builtin_inff() ? -__builtin_inf() : base * inv;
            bool nan = inv != inv || top == __builtin_inff();
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                nan |= x[e] != x[e];
                const double t = fmax(((double)x[e] - base) * unit, -1023.0 * 256.0), big = t + 0x1.8p52;
                const bool none = v0 + S::place(e, tid) == d || x[e] == -__builtin_inff();
                sum += none ? 0.0 : times_power(s_pow, small_power(t - (big - 0x1.8p52)), (u32)__builtin_bit_cast(u64, big), 0.0);
            }
            if (nan) sum = __builtin_nan("");
        }
        sum = wave_sum64_dpp(sum);
        if (lane == 0) {
            s_top[place] = top;
            s_sum[place] = sum;
            s_scale[place] = scale;
        }
    }
    __syncthreads();
    // a segment's four waves joined by four lanes
    if (tid >= n * kWaves) return;
    float top = s_top[tid];
    double scale = s_scale[tid], sum = s_sum[tid];
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    double most = fmax(scale, __shfl_xor(scale, 1));
    most = fmax(most, __shfl_xor(most, 2));
    if (scale != -__builtin_inf()) sum *= exp_neg(scale - most);
    sum += __shfl_xor(sum, 2);
    sum += __shfl_xor(sum, 1);
    int32_t at = greedy && s_top[tid] == top ? s_at[tid] : 0x7FFFFFFF;
    at = min(at, __shfl_xor(at, 1));
    at = min(at, __shfl_xor(at, 2));
    if (tid % kWaves == 0) a.parts[(int64_t)r * a.n_seg + s0 + tid / kWaves] = Part{sum, most, top, at};
}

// What a row comes to: Z = others + w(draft), log Z, and the decision on its draft
struct Row { double scale, others, z, logz; float draft_logp; int32_t best, draft; int32_t ok, accept; };
// weight of a segment in units of exp(scale)
__device__ __forceinline__ double scaled(const Part& q, double scale) { return q.scale == -__builtin_inf() ? q.sum : q.sum * exp_neg(q.scale - scale); }

template <typename T>
// own: the lane's segment (number `lane`) as `scaled` gives it
__device__ __forceinline__ Row join_row(const SampleArgs& a, int b, int i, int lane, double& own) {
    Row o;
    o.draft = draft_of(a, b, i);
    const double inv = inv_temperature(a, b), chance = random_of(a, b, i, 0);
    const float logit = o.draft >= 0 ? to_f(row_of<T>(a, b, i)[o.draft]) : 0.f;      // (on their way while the segments are joined)
    const float prob = o.draft >= 0 && a.probs ? a.probs[((int64_t)b * a.k + i) * a.vocab + o.draft] : 1.f;
    const Part* p = a.parts + ((int64_t)b * (a.k + 1) + i) * a.n_seg;
    float top = -__builtin_inff();
    int32_t best = 0x7FFFFFFF;
    double scale = -__builtin_inf();
    Part mine{0.0, -__builtin_inf(), -__builtin_inff(), 0x7FFFFFFF};
    if (lane < a.n_seg) mine = p[lane];
    for (int s = lane; s < a.n_seg; s += 64) {
        const Part q = s == lane ? mine : p[s];
        scale = fmax(scale, q.scale);
        if (q.top > top || (q.top == top && q.at < best)) { top = q.top; best = q.at; }
    }
    const bool greedy = is_greedy(a, b);
    if (greedy) {                                           // the lowest place among the lanes that hold the maximum
        if (top != wave_max_dpp(top)) best = 0x7FFFFFFF;
        for (int f = 32; f > 0; f >>= 1) best = min(best, __shfl_xor(best, f));
    }
    scale = wave_max64_dpp(scale);
    o.scale = scale;
    o.best = best;
    double sum = own = lane < a.n_seg ? scaled(mine, scale) : 0.0;
    for (int s = lane + 64; s < a.n_seg; s += 64) sum += scaled(p[s], scale);
    o.others = wave_sum64_dpp(sum);
    // (a masked draft weighs nothing at any temperature: over an infinite one -infinity is no number)
    const double x = o.draft >= 0 ? exponent(logit, inv, scale) : 0.0, w = o.draft >= 0 && logit != -__builtin_inff() ? exp_neg(x) : 0.0;
    o.z = o.others + w;
    o.ok = o.z > 0.0 && o.z < __builtin_inf();
    if (greedy) {
        o.accept = o.ok && o.draft == o.best && chance * (double)prob < 1.0;
        o.draft_logp = 0.f;
        o.logz = 0.0;
    } else {
        o.accept = o.ok && o.draft >= 0 && chance * (double)prob * o.z < w;
        o.logz = log(o.z);
        o.draft_logp = (float)(x - o.logz);
    }
    return o;
}

// Given q: every row's decision, which the two kernels behind it look up
template <typename T>
__global__ __launch_bounds__(64) void k_sample_decide(SampleArgs a) {
    const int r = blockIdx.x;
    double own;
    const Row o = join_row<T>(a, r / (a.k + 1), r % (a.k + 1), threadIdx.x, own);
    if (threadIdx.x == 0) a.decided[r] = o;
}

// sum max(0, p - q) over a segment of the row that rejected its draft (others write nothing that is read)
template <typename T, bool VEC>
__global__ __launch_bounds__(kPartThreads) void k_sample_residual(SampleArgs a) {
    using S = Segment<T, VEC>;
    __shared__ word2 s_pow[256];
    __shared__ double s_sum[kPartThreads / 64];
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (is_greedy(a, b)) return;
    const Row* rows = a.decided + (int64_t)b * (a.k + 1);
    const u64 stops = __ballot(lane >= a.k || !rows[min(lane, a.k)].accept);
    const int m = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)stops) - 1);
    const Row o = rows[m];
    if (m >= a.k || o.draft < 0 || !o.ok) return;
    float x[kPer], q[kPer];
    S::load(row_of<T>(a, b, m), blockIdx.x * kSeg, a.vocab, tid, x);
    const float* probs = a.probs + ((int64_t)b * a.k + m) * a.vocab;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int v = blockIdx.x * kSeg + S::place(e, tid);
        q[e] = v < a.vocab ? probs[v] : 0.f;
    }
    s_pow[tid] = kPow.at[tid];
    __syncthreads();
    const double inv = inv_temperature(a, b), inv_z = 1.0 / o.z;
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const double t = fmax(exponent(x[e], inv, o.scale) * 369.3299304675746, -1023.0 * 256.0), big = t + 0x1.8p52;      // (as in k_sample_parts' second loop)
        const double w = times_power(s_pow, small_power(t - (big - 0x1.8p52)), (u32)__builtin_bit_cast(u64, big), 0.0);
        sum += fmax(w * inv_z - (double)q[e], 0.0);
    }
    sum = wave_sum64_dpp(sum);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    if (tid == 0) a.residual[(int64_t)b * a.n_seg + blockIdx.x] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

template <typename T, bool VEC>
__global__ __launch_bounds__(kPickThreads) void k_sample_pick(SampleArgs a) {
    __shared__ Row s_row[TASC_MAX_K + 1];
    __shared__ double s_wave[16];
    __shared__ double s_before, s_target;
    __shared__ int32_t s_seg, s_first[16], s_last[16];
    __shared__ double s_x;
    const int b = blockIdx.x, nq = a.k + 1, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_emit = a.n_emit ? a.n_emit[b] : 0;
    const bool frozen = a.n_emit && n_emit >= (int)a.d.counters[TASC_CTR_MAX_NEW];
    if (frozen) {                                          // has its tokens: emits nothing
        if (tid < nq) {
            if (a.emitted) a.emitted[(int64_t)b * nq + tid] = -1;
            if (a.logprob) a.logprob[(int64_t)b * nq + tid] = 0.f;
        }
        if (tid == 0) {
            if (a.accept_len) a.accept_len[b] = 0;
            if (b == 0) atomicAdd(&a.d.counters[2], 1ull);
        }
        return;
    }
    double own = 0.0;                                       // of the wave's row: the lane's segment
    if (wave < nq) {
        Row o;
        if (a.probs) o = a.decided[(int64_t)b * nq + wave];
        else o = join_row<T>(a, b, wave, lane, own);
        if (lane == 0) s_row[wave] = o;
    }
    __syncthreads();
    int m = 0;
    while (m < a.k && s_row[m].accept) ++m;
    const Row o = s_row[m];
    const bool greedy = is_greedy(a, b);
    int32_t token = -1;
    float logp = __builtin_nanf("");
    if (!o.ok) {
    } else if (greedy) {
        token = o.best;
        logp = 0.f;
    } else {
        const double inv = inv_temperature(a, b), u = random_of(a, b, m, 1);
        const Part* p = a.parts + ((int64_t)b * nq + m) * a.n_seg;
        const double* res = a.residual + (int64_t)b * a.n_seg;
        // which weights: 0 w, 1 w without the draft, 2 max(0, p - q); what a rejection leaves may round to nothing: then w
        if (wave == m) {
            int kind = o.draft < 0 ? 0 : a.probs ? 2 : 1;
            auto seg_sum = [&](int s) {
                if (s >= a.n_seg) return 0.0;
                if (kind == 2) return res[s];
                double v = s == lane && !a.probs ? own : scaled(p[s], o.scale);
                if (kind == 0 && o.draft >= 0 && o.draft / kSeg == s) v += o.z - o.others;
                return v;
            };
            double total = 0.0;
            for (int pass = 0; pass < 2; ++pass) {
                total = 0.0;
                for (int s = lane; s < a.n_seg; s += 64) total += seg_sum(s);
                total = wave_sum64_dpp(total);
                if (total > 0.0) break;
                kind = 0;
            }
            const double target = u * total;
            double before = 0.0, at_before = 0.0;
            int seg = -1, last = 0;
            double last_before = 0.0;
            for (int s0 = 0; s0 < a.n_seg && seg < 0; s0 += 64) {
                const double own = seg_sum(s0 + lane);
                const double up = wave_scan64_dpp(own);
                const u64 past = __ballot(before + up > target), some = __ballot(own > 0.0);
                if (some) {
                    const int l = 63 - __clzll(some);
                    last = s0 + l;
                    last_before = before + lane64(up - own, l);
                }
                if (past) {
                    const int l = __ffsll(past) - 1;
                    seg = s0 + l;
                    at_before = before + lane64(up - own, l);
                }
                before += lane64(up, 63);
            }
            if (lane == 0) {
                s_seg = (seg >= 0 ? seg : last) | kind << 28;
                s_before = seg >= 0 ? at_before : last_before;
                s_target = target;
            }
        }
        __syncthreads();
        const int seg = s_seg & 0xFFFFFFF, kind = s_seg >> 28;
        const T* row = row_of<T>(a, b, m);
        const double inv_z = 1.0 / o.z;
        const float* q = kind == 2 ? a.probs + ((int64_t)b * a.k + m) * a.vocab : nullptr;
        constexpr int SPAN = kSeg / kPickThreads;
        const int v0 = seg * kSeg + SPAN * tid;
        float logit[SPAN];
        if (VEC && v0 + SPAN <= a.vocab) {
            load_n<SPAN>(row + v0, logit);
        } else {
#pragma unroll
            for (int e = 0; e < SPAN; ++e) logit[e] = v0 + e < a.vocab ? to_f(row[v0 + e]) : -__builtin_inff();
        }
        double w[SPAN], x[SPAN], mine = 0.0;
#pragma unroll
        for (int e = 0; e < SPAN; ++e) {
            const int v = v0 + e;
            const bool in = v < a.vocab;
            x[e] = exponent(logit[e], inv, o.scale);
            w[e] = logit[e] == -__builtin_inff() ? 0.0 : exp_neg(x[e]);
            if (kind == 1 && v == o.draft) w[e] = 0.0;
            if (kind == 2 && in) w[e] = fmax(w[e] * inv_z - (double)q[v], 0.0);
            mine += w[e];
        }
        const double up = wave_scan64_dpp(mine);
        if (lane == 63) s_wave[wave] = up;
        __syncthreads();
        double sum = s_before + (up - mine);
        for (int i = 0; i < wave; ++i) sum += s_wave[i];
        int first = 0x7FFFFFFF, last = -1;                  // the first token past the target, the last with any weight
#pragma unroll
        for (int e = 0; e < SPAN; ++e) {
            sum += w[e];
            const int v = v0 + e;
            if (w[e] > 0.0) {
                last = v;
                if (sum > s_target && first == 0x7FFFFFFF) first = v;
            }
        }
        const u64 hits = __ballot(first != 0x7FFFFFFF), any = __ballot(last >= 0);      // (the tokens go up with the lanes and the waves)
        first = hits ? __builtin_amdgcn_readlane(first, __ffsll((unsigned long long)hits) - 1) : 0x7FFFFFFF;
        last = any ? __builtin_amdgcn_readlane(last, 63 - __clzll(any)) : -1;
        if (lane == 0) { s_first[wave] = first; s_last[wave] = last; }
        __syncthreads();
        first = s_first[lane & 15];
        last = s_last[lane & 15];
        const u32 hit = (u32)__ballot(first != 0x7FFFFFFF) & 0xFFFF, some = (u32)__ballot(last >= 0) & 0xFFFF;
        first = hit ? __builtin_amdgcn_readlane(first, __ffs(hit) - 1) : 0x7FFFFFFF;
        last = some ? __builtin_amdgcn_readlane(last, 31 - __clz(some)) : -1;
        token = first != 0x7FFFFFFF ? first : last;
#pragma unroll
        for (int e = 0; e < SPAN; ++e)
            if (token == v0 + e) s_x = x[e];
        __syncthreads();
        if (token >= 0) logp = (float)(s_x - o.logz);
    }
    if (tid < nq) {
        const int64_t at = (int64_t)b * nq + tid;
        if (a.emitted) a.emitted[at] = tid < m ? s_row[tid].draft : tid == m ? token : -1;
        if (a.logprob) a.logprob[at] = tid < m ? s_row[tid].draft_logp : tid == m ? logp : 0.f;
    }
    if (tid == 0 && a.accept_len) a.accept_len[b] = m;
    if (!a.n_emit) return;
    __syncthreads();                                       // (every wave has looked at n_emit)
    const int at = a.d.n_tok[b];
    // (a row without a distribution commits token 0, as the greedy acceptance does)
    if (tid <= m) a.d.tokens[(size_t)b * a.max_len + at + tid] = tid < m ? s_row[tid].draft : max(token, 0);
    __syncthreads();
    if (tid != 0) return;
    a.d.n_tok[b] = at + m + 1;
    a.d.cached[b] += m + 1;
    a.d.n_emit[b] = n_emit + m + 1;
    if (n_emit + m + 1 >= (int)a.d.counters[TASC_CTR_MAX_NEW]) atomicAdd(&a.d.counters[0], 1ull);
    if (b == 0) atomicAdd(&a.d.counters[2], 1ull);
    atomicAdd(&a.d.counters[3], (u64)m);
    atomicAdd(&a.d.counters[4], (u64)a.k);
    atomicAdd(&a.d.counters[8 + m], 1ull);
}

// the workspace: parts, decisions, residual sums
size_t parts_bytes(int batch, int k, int n_seg) { return (size_t)batch * (k + 1) * n_seg * sizeof(Part); }
size_t decided_bytes(int batch, int k) { return (size_t)batch * (k + 1) * sizeof(Row); }
int segments(int vocab) { return (vocab - 1) / kSeg + 1; }
// Several segments a workgroup from four rounds of them on (us of a call, one | several a workgroup: 1280 rows of 151936 fp32 logits 163 | 154,
// 640 84 | 85, 224 of bf16, with draft probabilities, 51 | 55).
bool several_segments(int64_t rows, int n_seg) { return rows * n_seg >= 24576; }

template <typename T>
tasc_status enqueue(const SampleArgs& a, int batch, hipStream_t st) {
    const bool vec = (((uintptr_t)a.logits | (uintptr_t)(a.row_stride * (int64_t)sizeof(T))) & 15) == 0;
    const bool several = several_segments((int64_t)batch * (a.k + 1), a.n_seg);
    const int per = several ? kMostSegs : 1;
    const dim3 grid((unsigned)((a.n_seg + per - 1) / per), (unsigned)(batch * (a.k + 1))), threads(kPartThreads);
    auto parts = several ? (vec ? &k_sample_parts<T, true, true> : &k_sample_parts<T, false, true>) : (vec ? &k_sample_parts<T, true, false> : &k_sample_parts<T, false, false>);
    parts<<<grid, threads, 0, st>>>(a);
    if (a.probs) {
        const dim3 of((unsigned)a.n_seg, (unsigned)batch);
        k_sample_decide<T><<<dim3((unsigned)(batch * (a.k + 1))), dim3(64), 0, st>>>(a);
        vec ? k_sample_residual<T, true><<<of, threads, 0, st>>>(a) : k_sample_residual<T, false><<<of, threads, 0, st>>>(a);
    }
    const dim3 seqs((unsigned)batch), many(kPickThreads);
    vec ? k_sample_pick<T, true><<<seqs, many, 0, st>>>(a) : k_sample_pick<T, false><<<seqs, many, 0, st>>>(a);
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}

}  // namespace

extern "C" size_t tasc_accept_sampled_workspace_bytes(int32_t batch, int32_t k, int32_t vocab) {
    if (batch < 1 || k < 0 || k > TASC_MAX_K || vocab < 2 || vocab > 1 << 24) return 0;
    const int n_seg = segments(vocab);
    return parts_bytes(batch, k, n_seg) + decided_bytes(batch, k) + (size_t)batch * n_seg * sizeof(double);
}

extern "C" tasc_status tasc_accept_sampled(const void* logits, tasc_dtype dtype, int64_t row_stride, int32_t batch, int32_t k, int32_t vocab, const int32_t* drafts,
                                           const float* draft_probs, const float* temperature, const float* u, int32_t* accept_len, int32_t* emitted, float* logprob,
                                           void* workspace, size_t ws_bytes, void* stream) {
    TASC_REQUIRE(k >= 0 && k <= TASC_MAX_K, "accept_sampled: k %d outside [0, %d]", k, TASC_MAX_K);
    TASC_REQUIRE(vocab >= 2 && vocab <= 1 << 24, "accept_sampled: vocab %d outside [2, 2^24]", vocab);
    TASC_REQUIRE(batch >= 0 && (int64_t)batch * (k + 1) <= 65535, "accept_sampled: %d sequences of %d rows are not 0 .. 65535 rows", batch, k + 1);
    if (batch == 0) return TASC_OK;
    TASC_REQUIRE(logits && u && accept_len && emitted && (drafts || k == 0), "accept_sampled: null argument");
    TASC_REQUIRE(dtype == TASC_F32 || dtype == TASC_BF16, "accept_sampled: dtype %d", (int)dtype);
    TASC_REQUIRE(row_stride >= vocab, "accept_sampled: rows of %d logits lie %lld apart", vocab, (long long)row_stride);
    TASC_REQUIRE((uintptr_t)logits % (dtype == TASC_F32 ? 4 : 2) == 0, "accept_sampled: logits must be aligned to their type");
    const size_t need = tasc_accept_sampled_workspace_bytes(batch, k, vocab);
    if (!workspace || ws_bytes < need) {
        tasc_set_error("accept_sampled: workspace of %zu of %zu bytes", workspace ? ws_bytes : 0, need);
        return TASC_ENOMEM;
    }
    TASC_REQUIRE(((uintptr_t)workspace & 15) == 0, "accept_sampled: the workspace must be 16-byte aligned");
    const int n_seg = segments(vocab);
    const SampleArgs a{logits, row_stride, k, vocab, n_seg, drafts, k > 0 ? draft_probs : nullptr, temperature, u, k + 1, nullptr, (Part*)workspace,
                       (Row*)((char*)workspace + parts_bytes(batch, k, n_seg)),
                       (double*)((char*)workspace + parts_bytes(batch, k, n_seg) + decided_bytes(batch, k)), accept_len, emitted, logprob, TascSessDev{}, 0};
    return dtype == TASC_F32 ? enqueue<float>(a, batch, (hipStream_t)stream) : enqueue<BF16>(a, batch, (hipStream_t)stream);
}

size_t tasc_sample_logits_bytes(int32_t batch, int32_t k, int32_t vocab) { return ((size_t)batch * (k + 1) * vocab * sizeof(float) + 255) / 256 * 256; }

tasc_status tasc_sample_step(const tasc_session* s, const TascVerifyTail& t, hipStream_t st) {
    const int vocab = s->model->desc.vocab, n_seg = segments(vocab);
    const TascSampled& p = *t.sampled;
    const TascFilters& f = p.filters;
    if (f.top_k || f.top_p || f.min_p) {
        const tasc_status rc = tasc_filter_logits(p.logits, TASC_F32, vocab, s->batch, t.k, vocab, p.temperature, f.top_k, f.top_p, f.min_p, p.logits, vocab, nullptr,
                                                  f.workspace, f.ws_bytes, st);
        if (rc != TASC_OK) return rc;
    }
    const SampleArgs a{p.logits, vocab, t.k, vocab, n_seg, t.drafts, nullptr, p.temperature, p.u, p.n_u, s->d.n_emit, (Part*)p.parts, nullptr, nullptr,
                       t.accept_len, t.emitted, p.logprob, s->d, s->max_len};
    return enqueue<float>(a, s->batch, st);
}
