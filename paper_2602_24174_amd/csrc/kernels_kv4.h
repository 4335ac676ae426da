// The 4-bit KV cache: its layout, and the kernels that write, read and attend over it.
//
// A token's head of HD channels (32, 64 or 128) is held in groups of min(HD, 64) channels: scale = bf16((hi - lo) * (1 / 15)), low = bf16(lo)
// with lo and hi the group's least and largest value (the steps in fp32), and per channel the whole number c in [0, 15] nearest to (value - low) / scale; it
// stands for low + scale c.  bf16 pairs take 4 bytes a group whatever the values' range (a bf16 key's least value is held exactly, the
// scale's rounding moves the largest by 15 2^-9 of a step), so a token of 128 channels takes 72 bytes where bf16 takes 256.
//
// Per page of 16 tokens and head: key numbers [16][HD / 2 bytes], value numbers [16][HD / 2], then {scale, low} as one word (scale in the
// upper half) [groups][16] of the keys and of the values.  The numbers lie as the lanes of the attention want them, all tokens alike:
//   keys    the four lanes that share a token own 1/4 of its bytes each, words of 8 channels, of every group as many: of 128 channels lane r
//           owns channels 16 r .. +16 and 64 + 16 r .. +16, of 64 16 r .. +16, of 32 8 r .. +8.  In a word channel e lies at bit
//           4 (e / 2) + 16 (e % 2), so that one shift and one mask give the pair (2 j, 2 j + 1) in the halves of a register.
//   values  the sixteen lanes of a token own 1/16 each: of 128 channels lane r owns 4 r .. +4 (lower half of its word) and 64 + 4 r .. +4
//           (upper), of 64 4 r .. +4, of 32 2 r .. +2; channels in order, 4 bits each.
// A token's bytes are its own (no byte holds two tokens), so rows are written without a look at their neighbours.
#pragma once
#include "numeric.h"
#include <algorithm>

typedef uint32_t kv4_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t kv4_u32x2 __attribute__((ext_vector_type(2)));
typedef float kv4_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 kv4_bf16x8 __attribute__((ext_vector_type(8)));

template <int HD>
struct Kv4Layout {
    static constexpr int GROUPS = HD == 128 ? 2 : 1, HALF = HD / 2;     // HALF: bytes of a token's numbers
    static constexpr int K = 0, V = 16 * HALF, KS = 32 * HALF, VS = KS + 64 * GROUPS, HEAD = KS + 128 * GROUPS;
};
inline int kv4_head_bytes(int hd) { return 16 * hd + 128 * (hd == 128 ? 2 : 1); }
inline bool kv4_head_dim_ok(int hd) { return hd == 32 || hd == 64 || hd == 128; }

// ---------------------------------------------------------------- numbers of a group
// {scale, low} of a group from its least and largest value; not a number for a group that holds an infinity or a NaN (or whose range
// is beyond fp32), so that every value of it reads as NaN
struct Kv4Range { float lo, hi; int finite; };
__device__ __forceinline__ Kv4Range kv4_range(const float (&x)[8]) {
    Kv4Range g{x[0], x[0], 1};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        g.lo = fminf(g.lo, x[e]);
        g.hi = fmaxf(g.hi, x[e]);
        g.finite &= fabsf(x[e]) < __builtin_inff();
    }
    return g;
}
__device__ __forceinline__ Kv4Range kv4_join(const Kv4Range& a, const Kv4Range& b) { return {fminf(a.lo, b.lo), fmaxf(a.hi, b.hi), a.finite & b.finite}; }
__device__ __forceinline__ Kv4Range kv4_from(const Kv4Range& g, int o) { return {__shfl_xor(g.lo, o), __shfl_xor(g.hi, o), __shfl_xor(g.finite, o)}; }   // lane ^ o's
__device__ __forceinline__ uint32_t kv4_scale_low(const Kv4Range& g) {
    const float scale = (g.hi - g.lo) * (1.0f / 15.0f);
    return g.finite && fabsf(scale) < __builtin_inff() ? f2bf_pair(g.lo, scale) : 0x7FC07FC0u;
}
__device__ __forceinline__ float kv4_scale(uint32_t sl) { return __uint_as_float(sl & 0xFFFF0000u); }
__device__ __forceinline__ float kv4_low(uint32_t sl) { return __uint_as_float(sl << 16); }
// The nearest whole number: the quotient is taken in 64 bits, where a quotient at a border (scale has 8 significant bits) comes out exact
// and one beside it on its own side.
__device__ __forceinline__ uint32_t kv4_number(float x, float scale, float low) {
    const double n = rint(((double)x - (double)low) / (double)scale);
    return scale > 0.f ? (uint32_t)fmin(fmax(n, 0.0), 15.0) : 0u;       // (0 where scale is 0 or NaN)
}
// a key word of 8 channels
__device__ __forceinline__ uint32_t kv4_key_word(const uint32_t (&c)[8]) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= c[e] << (4 * (e / 2) + 16 * (e % 2));
    return w;
}
__device__ __forceinline__ uint32_t kv4_value_word(const uint32_t (&c)[8]) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= c[e] << (4 * e);
    return w;
}
// byte of a token's key word that holds channels 8 blk .. +8
template <int HD>
__device__ __forceinline__ int kv4_key_byte(int blk) {
    if constexpr (HD == 128) return 16 * ((blk & 7) / 2) + 4 * (blk & 1) + 8 * (blk / 8);
    else return 4 * blk;
}
// writes the value numbers of channels 8 blk .. +8 of a token
template <int HD>
__device__ __forceinline__ void kv4_store_values(uint8_t* token, int blk, uint32_t w) {
    if constexpr (HD == 128) {                              // two lanes' halves of a word each
        uint16_t* p = reinterpret_cast<uint16_t*>(token + 8 * (blk & 7) + 2 * (blk / 8));
        p[0] = (uint16_t)w;
        p[2] = (uint16_t)(w >> 16);
    } else {
        *reinterpret_cast<uint32_t*>(token + 4 * blk) = w;
    }
}
template <int HD>
__device__ __forceinline__ uint32_t kv4_load_values(const uint8_t* token, int blk) {
    if constexpr (HD == 128) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(token + 8 * (blk & 7) + 2 * (blk / 8));
        return p[0] | (uint32_t)p[2] << 16;
    } else {
        return *reinterpret_cast<const uint32_t*>(token + 4 * blk);
    }
}
// Quantises 8 channels whose group has the given {scale, low} and writes them.
template <int HD>
__device__ __forceinline__ void kv4_put(uint8_t* head, int slot, int blk, bool value, const float (&x)[8], uint32_t sl) {
    using L = Kv4Layout<HD>;
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = kv4_number(x[e], kv4_scale(sl), kv4_low(sl));
    if (value) kv4_store_values<HD>(head + L::V + slot * L::HALF, blk, kv4_value_word(c));
    else *reinterpret_cast<uint32_t*>(head + L::K + slot * L::HALF + kv4_key_byte<HD>(blk)) = kv4_key_word(c);
    if (blk % 8 == 0) reinterpret_cast<uint32_t*>(head + (value ? L::VS : L::KS))[(HD == 128 ? blk / 8 : 0) * 16 + slot] = sl;
}

// ---------------------------------------------------------------- append and read
struct Kv4Rows {
    uint8_t* pool;
    int32_t n_pages, Hkv, rows;
    const int32_t* slots;
};

// One thread per 8 channels of a row's key or value head; the HD / 8 (8 at most) threads of a group find its range among themselves.
// Bound by bytes: 2 or 4 read and 1/2 written per value.  VEC: rows start at multiples of 16 bytes.
template <int HD, typename T, bool VEC>
__global__ __launch_bounds__(256) void k_kv4_append(Kv4Rows a, const T* __restrict__ k, const T* __restrict__ v, int64_t k_stride, int64_t v_stride) {
    constexpr int BLKS = HD / 8, SPAN = BLKS < 8 ? BLKS : 8;
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t unit = idx / BLKS;                       // (row, head)
    const int blk = (int)(idx % BLKS);
    const bool value = blockIdx.y != 0;
    const int64_t row = min(unit / a.Hkv, (int64_t)a.rows - 1);   // (all lanes take part in the exchange)
    const int head = (int)(unit % a.Hkv);
    const T* src = (value ? v + row * v_stride : k + row * k_stride) + head * HD + 8 * blk;
    float x[8];
    if constexpr (VEC) load8(src, x);
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_f(src[e]);
    }
    const int32_t slot = a.slots[row];
    Kv4Range g = kv4_range(x);
#pragma unroll
    for (int o = 1; o < SPAN; o *= 2) g = kv4_join(g, kv4_from(g, o));
    if (unit >= (int64_t)a.rows * a.Hkv || slot < 0 || slot / TASC_KV_BLOCK >= a.n_pages) return;
    uint8_t* const at = a.pool + ((size_t)(slot / TASC_KV_BLOCK) * a.Hkv + head) * Kv4Layout<HD>::HEAD;
    kv4_put<HD>(at, slot % TASC_KV_BLOCK, blk, value, x, kv4_scale_low(g));
}

// The values that slots hold, zeros for a slot outside the pool.
template <int HD, typename T>
__global__ __launch_bounds__(256) void k_kv4_read(Kv4Rows a, T* __restrict__ k, T* __restrict__ v) {
    using L = Kv4Layout<HD>;
    constexpr int BLKS = HD / 8;
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x, unit = idx / BLKS;
    if (unit >= (int64_t)a.rows * a.Hkv) return;
    const int blk = (int)(idx % BLKS), head = (int)(unit % a.Hkv);
    const int64_t row = unit / a.Hkv;
    const bool value = blockIdx.y != 0;
    const int32_t slot = a.slots[row];
    float x[8] = {};
    if (slot >= 0 && slot / TASC_KV_BLOCK < a.n_pages) {
        const uint8_t* at = a.pool + ((size_t)(slot / TASC_KV_BLOCK) * a.Hkv + head) * L::HEAD;
        const int t = slot % TASC_KV_BLOCK;
        const uint32_t sl = reinterpret_cast<const uint32_t*>(at + (value ? L::VS : L::KS))[(HD == 128 ? blk / 8 : 0) * 16 + t];
        const uint32_t w = value ? kv4_load_values<HD>(at + L::V + t * L::HALF, blk)
                                 : *reinterpret_cast<const uint32_t*>(at + L::K + t * L::HALF + kv4_key_byte<HD>(blk));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t c = w >> (value ? 4 * e : 4 * (e / 2) + 16 * (e % 2)) & 15u;
            x[e] = __builtin_fmaf((float)c, kv4_scale(sl), kv4_low(sl));
        }
    }
    T* const out = (value ? v : k) + unit * HD + 8 * blk;
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(out) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(out + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *reinterpret_cast<kv4_u32x4*>(out) = kv4_u32x4{f2bf_pair(x[0], x[1]), f2bf_pair(x[2], x[3]), f2bf_pair(x[4], x[5]), f2bf_pair(x[6], x[7])};
    }
}

// ---------------------------------------------------------------- attention
// Query row i of a sequence with n rows and L cached tokens (the rows' own among them) sees the keys at positions 0 .. L - n + i.
// S^T = K Q^T and O^T = V^T P^T in 16x16x32 bf16 products, keys as the first operand: the scores come out with a lane's four
// tokens side by side and one (row, head) pair a lane, which is how the second product wants the weights, so nothing is
// exchanged between lanes but the maximum of a pair's four lanes.
//   A number c enters the products as the bf16 value 16 + c, which is a shift and a mask away from its 4 bits (0x4180 | c << 3), and exact.
//   q . key = sum over groups of scale (q . (16 + c)) + (low - 16 scale) sum q        scales applied to the fp32 products
//   sum p value = sum (p scale) (16 + c) - 23.5 sum (p scale) + sum p (low + 7.5 scale)
//                                                                                     p scale rounded to bf16 (2^-8 relative at most, like the
//   output itself), the same rounded weights in the first two sums: a rounding then moves the output by (c - 7.5) scale, about the value's
//   distance from the middle of its group's range, and not by c scale
// Maxima, sums and products are fp32.  Tiles of 32 tokens at absolute positions, tile t to unit t % units (a unit: a wave of a key chunk), joined
// in a fixed order: a row's bits depend on neither the other rows nor the length beyond its own last key.
struct Kv4Attn {
    const uint8_t* pool;
    int32_t n_pages, max_pages, Hkv, H, batch, rows, max_rows, chunks;
    const BF16* q;
    BF16* out;
    int64_t q_stride, out_stride;      // elements from row to row
    const int32_t* table;              // [batch, max_pages]
    const int32_t* row_off;            // [batch + 1], or null:
    const int32_t* row0;               //   first row and rows of a sequence,
    const int32_t* n_rows;
    const int32_t* pos0;               //   the position of its first row
    const int32_t* kv_len;             // [batch] with row_off
    int32_t row_base;                  // first row of the launch in row0's count
    float scale;
    float* part_o;                     // [chunks, rows, H, HD], used if chunks > 1
    float* part_ml;                    // [chunks, rows, H, 2]
};
// Which units there are, and so in which order a row's keys are added: waves of a workgroup that share its pairs (1: none), key chunks
struct Kv4Order { int wk, chunks; };
// `pairs` (row, head) pairs of a KV head, a bound or what stands for it; split: waves share pairs in any case
inline Kv4Order kv4_order(int64_t batch, int kv_heads, int64_t pairs, int64_t max_kv, int most_chunks, bool split) {
    constexpr int64_t kCus = 256;
    Kv4Order o{4, 1};
    const int64_t heads = batch * kv_heads;
    if (!split && pairs >= 256 && (pairs + 255) / 256 * heads >= kCus) o.wk = 1;
    if (o.wk == 4) {
        const int64_t wgs = heads * ((pairs + 63) / 64);
        o.chunks = (int)std::clamp<int64_t>(std::min<int64_t>(2 * kCus / wgs, max_kv / 512), 1, most_chunks);
    }
    return o;
}
struct Kv4Attn;
// kv4.hip: enqueues the attention (a.chunks is set from the order)
tasc_status tasc_kv4_attend(Kv4Attn a, int hd, const Kv4Order& o, hipStream_t st);
struct Kv4Seq { int first, n, len; };
__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Attn& a, int b) {
    Kv4Seq s;
    if (a.row_off) {
        s.first = a.row_off[b];
        s.n = a.row_off[b + 1] - s.first;
        s.len = a.kv_len[b];
    } else {
        s.first = a.row0[b] - a.row_base;
        s.n = a.n_rows[b];
        s.len = a.pos0[b] + s.n;
    }
    s.n = min(s.n, a.max_rows);
    if (s.first < 0) s.n = 0;
    return s;
}

template <int HD>
struct Kv4Tile {                       // a tile's bytes of one lane: 32 tokens, pages p = 0, 1
    uint32_t kc[2][HD / 32];
    kv4_u32x4 ks[2][HD == 128 ? 2 : 1];
    uint32_t vc[2][4];
    kv4_u32x4 vs[2][HD == 128 ? 2 : 1];
};
template <int HD>
__device__ __forceinline__ void kv4_fetch(Kv4Tile<HD>& t, const uint8_t* __restrict__ head0, const uint8_t* __restrict__ head1, int lane) {
    using L = Kv4Layout<HD>;
    const int c = lane & 15, r = lane >> 4;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const uint8_t* h = p ? head1 : head0;
        const uint8_t* kp = h + L::K + c * L::HALF + r * (L::HALF / 4);
        if constexpr (HD == 128) {
            const kv4_u32x4 w = *reinterpret_cast<const kv4_u32x4*>(kp);
            t.kc[p][0] = w[0]; t.kc[p][1] = w[1]; t.kc[p][2] = w[2]; t.kc[p][3] = w[3];
        } else if constexpr (HD == 64) {
            const kv4_u32x2 w = *reinterpret_cast<const kv4_u32x2*>(kp);
            t.kc[p][0] = w[0]; t.kc[p][1] = w[1];
        } else {
            t.kc[p][0] = *reinterpret_cast<const uint32_t*>(kp);
        }
#pragma unroll
        for (int g = 0; g < L::GROUPS; ++g) {
            t.ks[p][g] = *reinterpret_cast<const kv4_u32x4*>(h + L::KS + 64 * g + 16 * r);
            t.vs[p][g] = *reinterpret_cast<const kv4_u32x4*>(h + L::VS + 64 * g + 16 * r);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint8_t* vp = h + L::V + (4 * r + i) * L::HALF + c * (L::HALF / 16);
            if constexpr (HD == 128) t.vc[p][i] = *reinterpret_cast<const uint32_t*>(vp);
            else if constexpr (HD == 64) t.vc[p][i] = *reinterpret_cast<const uint16_t*>(vp);
            else t.vc[p][i] = *vp;
        }
    }
}
// bits 4 j .. 4 j + 3 of both halves of w as the bf16 pair 16 + c
__device__ __forceinline__ uint32_t kv4_pair(uint32_t w, int j) {
    return ((j == 0 ? w << 3 : w >> (4 * j - 3)) & 0x00780078u) | 0x41804180u;
}
__device__ __forceinline__ float kv4_pair_sum(uint32_t p, float to) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(tasc_bf16x2, p), __builtin_bit_cast(tasc_bf16x2, 0x3F803F80u), to, false);
}
// maximum / sum over the four lanes that share lane % 16
__device__ __forceinline__ float kv4_quad_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float kv4_quad_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// MT: tiles of 16 (row, head) pairs a wave holds.  WK: waves of a workgroup that share its pairs and take the key tiles in turn (4), or
// 1: every wave has pairs of its own and all tiles.
template <int HD, int MT, int WK>
__global__ __launch_bounds__(256) void k_kv4_attention(Kv4Attn a) {
    using L = Kv4Layout<HD>;
    constexpr int G = L::GROUPS, KSTEPS = HD / 32, DT = HD / 16;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, r = lane >> 4;
    const int b = blockIdx.y / a.Hkv, h = blockIdx.y % a.Hkv, share = a.H / a.Hkv;
    const int tile = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const Kv4Seq sq = kv4_seq(a, b);
    const int n_pairs = sq.n * share, pair0 = (WK == 1 ? tile * 4 + wave : tile) * 16 * MT;
    if (pair0 >= n_pairs) return;                          // (WK 4: the whole workgroup)
    const int len = min(max(sq.len, 0), a.max_pages * TASC_KV_BLOCK);
    const int pair_last = min(pair0 + 16 * MT, n_pairs) - 1;
    const int first_last = sq.len - sq.n + pair0 / share, last_last = sq.len - sq.n + pair_last / share;   // last keys of the first and the last pair
    const int n_tiles = (min(last_last + 1, len) + 31) / 32;      // (a negative count: no key at all)

    int last[MT], row[MT], head[MT];
    kv4_bf16x8 fq[MT][KSTEPS];
    float qsum[MT][G];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int pair = pair0 + 16 * t + col;
        row[t] = sq.first + pair / share;
        head[t] = h * share + pair % share;
        const bool live = pair < n_pairs && row[t] < a.rows;
        last[t] = live ? sq.len - sq.n + pair / share : -1;
        if (!live) row[t] = -1;
#pragma unroll
        for (int g = 0; g < G; ++g) qsum[t][g] = 0.f;
#pragma unroll
        for (int i = 0; i < KSTEPS; ++i) {
            const int d = HD == 128 ? (i / 2) * 64 + 16 * r + 8 * (i & 1) : HD == 64 ? 16 * r + 8 * i : 8 * r;
            kv4_u32x4 w = {0, 0, 0, 0};
            if (live) w = *reinterpret_cast<const kv4_u32x4*>(a.q + (size_t)row[t] * a.q_stride + head[t] * HD + d);
            fq[t][i] = __builtin_bit_cast(kv4_bf16x8, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) qsum[t][HD == 128 ? i / 2 : 0] = kv4_pair_sum(w[e], qsum[t][HD == 128 ? i / 2 : 0]);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) qsum[t][g] = kv4_quad_sum(qsum[t][g]);
    }

    kv4_f32x4 acc[MT][DT];
    float m[MT], l[MT], ev[MT][G];                          // ev: sum p (low + 7.5 scale) - 23.5 sum (p scale), this lane's tokens
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        m[t] = -__builtin_inff();
        l[t] = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) ev[t][g] = 0.f;
#pragma unroll
        for (int j = 0; j < DT; ++j) acc[t][j] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float scale2 = a.scale * 1.44269504088896340736f;   // scores in powers of 2
    const int32_t* const tab = a.table + (size_t)b * a.max_pages;
    const size_t page_bytes = (size_t)a.Hkv * L::HEAD;
    const uint8_t* const pool = a.pool + (size_t)h * L::HEAD;
    const int units = WK * a.chunks, unit = WK == 1 ? chunk : chunk * WK + wave;
    // a page id outside the pool is not followed: its tokens are masked
    auto page_of = [&](int t, int p) { const int at = 2 * t + p; return at < a.max_pages ? __builtin_amdgcn_readfirstlane(tab[at]) : -1; };
    auto where = [&](int page) { return pool + (size_t)(page >= 0 && page < a.n_pages ? page : 0) * page_bytes; };

    Kv4Tile<HD> cur, nxt;
    int pg0 = -1, pg1 = -1;
    if (unit < n_tiles) {
        pg0 = page_of(unit, 0);
        pg1 = page_of(unit, 1);
        kv4_fetch<HD>(cur, where(pg0), where(pg1), lane);
    }
    for (int t = unit; t < n_tiles; t += units) {
        const int ng0 = t + units < n_tiles ? page_of(t + units, 0) : -1, ng1 = t + units < n_tiles ? page_of(t + units, 1) : -1;
        if (t + units < n_tiles) kv4_fetch<HD>(nxt, where(ng0), where(ng1), lane);
        const int at = 32 * t;
        const bool ok0 = pg0 >= 0 && pg0 < a.n_pages, ok1 = pg1 >= 0 && pg1 < a.n_pages;
        const bool whole = ok0 && ok1 && at + 31 <= first_last && at + 32 <= len;

        kv4_bf16x8 fk[2][KSTEPS];
        float ksc[2][G][4], kb[2][G][4];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) {
                const uint32_t w = cur.kc[p][i];
                fk[p][i] = __builtin_bit_cast(kv4_bf16x8, kv4_u32x4{kv4_pair(w, 0), kv4_pair(w, 1), kv4_pair(w, 2), kv4_pair(w, 3)});
            }
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float sc = kv4_scale(cur.ks[p][g][i]) * scale2, lo = kv4_low(cur.ks[p][g][i]) * scale2;
                    ksc[p][g][i] = sc;
                    kb[p][g][i] = __builtin_fmaf(-16.f, sc, lo);
                }
        }
        // value numbers of lane's tokens, channel by channel: pairs of tokens in a register
        kv4_bf16x8 fv[DT];
        {
            uint32_t pr[2][4];                              // [lower, upper half of the words][token pair]
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const uint32_t x = cur.vc[s / 2][2 * (s % 2)], y = cur.vc[s / 2][2 * (s % 2) + 1];
                pr[0][s] = (x & 0xFFFFu) | y << 16;
                pr[1][s] = x >> 16 | (y & 0xFFFF0000u);
            }
#pragma unroll
            for (int j = 0; j < DT; ++j)
                fv[j] = __builtin_bit_cast(kv4_bf16x8, kv4_u32x4{kv4_pair(pr[j / 4][0], j % 4), kv4_pair(pr[j / 4][1], j % 4),
                                                                 kv4_pair(pr[j / 4][2], j % 4), kv4_pair(pr[j / 4][3], j % 4)});
        }
        float vsc[2][G][4], vmid[2][G][4];
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    vsc[p][g][i] = kv4_scale(cur.vs[p][g][i]);
                    vmid[p][g][i] = __builtin_fmaf(7.5f, vsc[p][g][i], kv4_low(cur.vs[p][g][i]));
                }

#pragma unroll
        for (int u = 0; u < MT; ++u) {
            float s[2][4];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                kv4_f32x4 sg[G];
#pragma unroll
                for (int g = 0; g < G; ++g) sg[g] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KSTEPS; ++i) {
                    constexpr int per = G == 2 ? KSTEPS / 2 : KSTEPS;
                    sg[i / per] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fk[p][i], fq[u][i], sg[i / per], 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = kb[p][0][i] * qsum[u][0];
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        if (g > 0) v = __builtin_fmaf(kb[p][g][i], qsum[u][g], v);
                        v = __builtin_fmaf(ksc[p][g][i], sg[g][i], v);
                    }
                    s[p][i] = v;
                }
            }
            uint32_t keep = 0xFFu;                          // bit 4 p + i: the token counts
            if (!whole) {
                keep = 0;
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int pos = at + 16 * p + 4 * r + i;
                        const bool in = (p ? ok1 : ok0) && pos <= last[u] && pos < len;
                        keep |= (in ? 1u : 0u) << (4 * p + i);
                        if (!in) s[p][i] = -__builtin_inff();
                    }
            }
            float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            top = fmaxf(kv4_quad_max(top), m[u]);
            if (__any(top > m[u])) {
                const float f = top == m[u] ? 1.f : __builtin_amdgcn_exp2f(m[u] - top);   // (0 at the first key; a pair without one keeps -inf)
                l[u] *= f;
#pragma unroll
                for (int g = 0; g < G; ++g) ev[u][g] *= f;
#pragma unroll
                for (int j = 0; j < DT; ++j) acc[u][j] *= f;
                m[u] = top;
            }
            const float base = m[u] == -__builtin_inff() ? 0.f : m[u];
            float pw[2][4];
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    pw[p][i] = __builtin_amdgcn_exp2f(s[p][i] - base);
                    l[u] += pw[p][i];
                }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float ps[2][4];
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        ps[p][i] = pw[p][i] * vsc[p][g][i];
                        float mid = pw[p][i] * vmid[p][g][i];
                        if (!whole && !(keep >> (4 * p + i) & 1)) { ps[p][i] = 0.f; mid = 0.f; }    // (what lies there may be no number)
                        ev[u][g] += mid;
                    }
                const kv4_u32x4 w = {f2bf_pair(ps[0][0], ps[0][1]), f2bf_pair(ps[0][2], ps[0][3]), f2bf_pair(ps[1][0], ps[1][1]), f2bf_pair(ps[1][2], ps[1][3])};
                float rounded = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) rounded = kv4_pair_sum(w[e], rounded);
                ev[u][g] = __builtin_fmaf(-23.5f, rounded, ev[u][g]);
                const kv4_bf16x8 fp = __builtin_bit_cast(kv4_bf16x8, w);
#pragma unroll
                for (int j = g * (DT / G); j < (g + 1) * (DT / G); ++j) acc[u][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv[j], fp, acc[u][j], 0, 0, 0);
            }
        }
        cur = nxt;
        pg0 = ng0;
        pg1 = ng1;
    }

    // the four lanes' sums, and the channels' share of ev
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        l[t] = kv4_quad_sum(l[t]);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float e = kv4_quad_sum(ev[t][g]);
#pragma unroll
            for (int j = g * (DT / G); j < (g + 1) * (DT / G); ++j) acc[t][j] += e;
        }
    }
    if constexpr (WK > 1) {
        // the waves' results, (0 + 2) + (1 + 3): maxima first, then sums in units of the common one
        float* const sm = lds;                              // [4][16 MT]
        float* const sx = lds + 4 * 16 * MT;                // [2][MT * (DT * 4 + 1)][64]
        if (r == 0)
#pragma unroll
            for (int t = 0; t < MT; ++t) sm[wave * 16 * MT + 16 * t + col] = m[t];
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            float top = m[t];
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w * 16 * MT + 16 * t + col]);
            const float f = m[t] == top ? 1.f : __builtin_amdgcn_exp2f(m[t] - top);
            m[t] = top;
            l[t] *= f;
#pragma unroll
            for (int j = 0; j < DT; ++j) acc[t][j] *= f;
        }
        constexpr int SPAN = MT * (DT * 4 + 1);
#pragma unroll
        for (int half = 2; half >= 1; half /= 2) {
            if (wave >= half && wave < 2 * half) {
                float* to = sx + (size_t)(wave - half) * SPAN * 64 + lane;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
#pragma unroll
                    for (int j = 0; j < DT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) to[(t * (DT * 4 + 1) + 4 * j + e) * 64] = acc[t][j][e];
                    to[(t * (DT * 4 + 1) + 4 * DT) * 64] = l[t];
                }
            }
            __syncthreads();
            if (wave < half) {
                const float* from = sx + (size_t)wave * SPAN * 64 + lane;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
#pragma unroll
                    for (int j = 0; j < DT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t][j][e] += from[(t * (DT * 4 + 1) + 4 * j + e) * 64];
                    l[t] += from[(t * (DT * 4 + 1) + 4 * DT) * 64];
                }
            }
            __syncthreads();
        }
        if (wave != 0) return;
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        if (row[t] < 0) continue;
        // lane's channels: of tile j row 4 r + i, channel (HD 128, 64) 64 (j / 4) + 16 r + 4 i + j % 4, (32) 8 r + 2 i + j
        if (a.chunks == 1) {
            const float inv = l[t] > 0.f ? 1.f / l[t] : l[t];          // a pair without keys gives zeros (a NaN stays one)
            uint16_t* o = reinterpret_cast<uint16_t*>(a.out + (size_t)row[t] * a.out_stride + head[t] * HD);
            if constexpr (HD == 32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(o + 8 * r + 2 * i) = f2bf_pair(acc[t][0][i] * inv, acc[t][1][i] * inv);
            } else {
#pragma unroll
                for (int g = 0; g < DT / 4; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<kv4_u32x2*>(o + 64 * g + 16 * r + 4 * i) =
                            kv4_u32x2{f2bf_pair(acc[t][4 * g][i] * inv, acc[t][4 * g + 1][i] * inv), f2bf_pair(acc[t][4 * g + 2][i] * inv, acc[t][4 * g + 3][i] * inv)};
            }
        } else {
            const size_t at = ((size_t)chunk * a.rows + row[t]) * a.H + head[t];
            float* o = a.part_o + at * HD;
            if constexpr (HD == 32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(o + 8 * r + 2 * i) = make_float2(acc[t][0][i], acc[t][1][i]);
            } else {
#pragma unroll
                for (int g = 0; g < DT / 4; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<float4*>(o + 64 * g + 16 * r + 4 * i) =
                            make_float4(acc[t][4 * g][i], acc[t][4 * g + 1][i], acc[t][4 * g + 2][i], acc[t][4 * g + 3][i]);
            }
            if (r == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(m[t], l[t]);
        }
    }
}
template <int HD, int MT, int WK>
constexpr int kv4_attention_lds() { return WK == 1 ? 0 : (4 * 16 * MT + 2 * MT * (HD / 4 + 1) * 64) * 4; }

// The key chunks' results in chunk order; a workgroup per (sequence, row), a thread per 4 channels of a head at a time.
template <int HD>
__global__ __launch_bounds__(256) void k_kv4_merge(Kv4Attn a) {
    const Kv4Seq sq = kv4_seq(a, blockIdx.y);
    const int row = sq.first + blockIdx.x;
    if ((int)blockIdx.x >= sq.n || row >= a.rows) return;
    for (int idx = threadIdx.x; idx < a.H * (HD / 4); idx += 256) {
        const int head = idx / (HD / 4), d = 4 * (idx % (HD / 4));
        float top = -__builtin_inff();
        for (int c = 0; c < a.chunks; ++c) top = fmaxf(top, a.part_ml[2 * (((size_t)c * a.rows + row) * a.H + head)]);
        float l = 0.f;
        kv4_f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (int c = 0; c < a.chunks; ++c) {
            const size_t at = ((size_t)c * a.rows + row) * a.H + head;
            const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * at);
            const float f = ml.x == top ? 1.f : __builtin_amdgcn_exp2f(ml.x - top);
            l = __builtin_fmaf(ml.y, f, l);
            o += *reinterpret_cast<const kv4_f32x4*>(a.part_o + at * HD + d) * f;
        }
        const float inv = l > 0.f ? 1.f / l : l;
        *reinterpret_cast<kv4_u32x2*>(a.out + (size_t)row * a.out_stride + head * HD + d) = kv4_u32x2{f2bf_pair(o[0] * inv, o[1] * inv), f2bf_pair(o[2] * inv, o[3] * inv)};
    }
}
