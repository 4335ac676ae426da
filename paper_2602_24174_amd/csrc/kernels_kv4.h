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
#include "kv4_order.h"

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
// The whole numbers nearest to (x - low) / scale.  In fp32, (x - low) * (1 / scale) is off by less than 15 * 4 * 2^-24 + 2^-22 < 1e-5 of a step; a
// quotient nearer to a border than that is taken again in 64 bits, where one at a border (scale has 8 significant bits) comes out exact
// and one beside it on its own side.  (All of them in 64 bits: 16384 rows of 8 x 128 fp32 41 us.)
__device__ __forceinline__ void kv4_numbers(const float (&x)[8], uint32_t sl, uint32_t (&c)[8]) {
    const float scale = kv4_scale(sl), low = kv4_low(sl), inv = 1.0f / scale;
    bool doubt = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float q = (x[e] - low) * inv, n = rintf(q);
        doubt |= !(fabsf(q - n) < 0.49998f);               // (also where 1 / scale is infinite)
        c[e] = (uint32_t)fminf(fmaxf(n, 0.f), 15.f);
    }
    if (doubt) {
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = (uint32_t)fmin(fmax(rint(((double)x[e] - (double)low) / (double)scale), 0.0), 15.0);
    }
    if (!(scale > 0.f)) {                                   // 0 or NaN
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = 0;
    }
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
    kv4_numbers(x, sl, c);
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
// fp32 values: bound by bytes, 4 read and 1/2 written per value (16384 rows of 8 x 128: 153 MB in 31 us, 4.9 TB/s, the rate of a copy); bf16 ones
// by the quotients in 64 bits that 62 % of the waves take (fp32 2 %): 39 us.  VEC: rows start at multiples of 16 bytes.
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

// The values that slots hold, zeros for a slot outside the pool.  Bound by the bytes it writes (the same rows: 31 us).
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
//   sum p value = sum (p scale) (16 + c) + sum (p scale) (z - 16),  z = low / scale        p scale rounded to bf16 (2^-8 relative at most, like
//                                                                                     the output itself)
// The last of these sums is three rows of a 16 x 16 product of its own, z - 16 in three bf16 terms.  Maxima, sums and products are
// fp32.  Tiles of 32 tokens at absolute positions, chunk_tiles of them a key chunk, a chunk's dealt to
// the waves in turn, all joined in a fixed order: a row's bits depend on neither the other rows nor the length beyond its own last key.
// What bounds it: of long contexts with few pairs the read of the cache (2 sequences of up to 131072 tokens, 8 x 128: 227 MB in 54 us, 4.2 TB/s,
// where a stream of reads alone has 6.4), else the vector instructions around the products (exponentials, scales, numbers to bf16; 55 to 60 % of the
// busy time) and, with ragged lengths, compute units that are done before others.
struct Kv4Attn {
    const uint8_t* pool;
    int32_t n_pages, max_pages, Hkv, H, batch, rows, max_rows, chunks, chunk_tiles, row_waves;
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
// kv4.hip: enqueues the attention (a.chunks is set from the order)
tasc_status tasc_kv4_attend(Kv4Attn a, int hd, const Kv4Order& o, hipStream_t st);
struct Kv4Seq { int first, n, len; };
__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Attn& a, int b) {
    // The arrays may hold anything: rows that are not among the call's, or beyond max_rows, are left out; the last ones, whose tokens are no
    // other row's.  (Differences of numbers from 0 on: none overflows.)
    const int first = a.row_off ? a.row_off[b] : a.row0[b] - a.row_base, next = a.row_off ? a.row_off[b + 1] : first + a.n_rows[b];
    Kv4Seq s{0, 0, 0};
    if (first >= 0 && next > first && first < a.rows) {
        const int n = next - first, len = a.row_off ? max(a.kv_len[b], 0) : a.pos0[b] + n;
        s.first = first;
        s.n = min(min(n, a.max_rows), a.rows - first);
        s.len = max(len - (n - s.n), 0);                    // (below 0 as 0: the rows see nothing)
    }
    return s;
}

// A tile's bytes of one lane: 32 tokens, pages p = 0, 1.  The {scale, low} words are dealt over the lanes.
template <int HD>
struct Kv4Tile {
    uint32_t kc[2][HD / 32];
    uint32_t vc[2][4];
    uint32_t ks, vs;
};
// of two groups lane 32 p + 16 g + t has those of token t, page p; of one group 16 p + t, the upper half of the wave the same again
template <int HD>
__device__ __forceinline__ int kv4_scale_word(int lane) { return Kv4Layout<HD>::GROUPS == 2 ? lane & 31 : lane & 15; }
template <int HD>
__device__ __forceinline__ int kv4_scale_page(int lane) { return Kv4Layout<HD>::GROUPS == 2 ? lane >> 5 : (lane >> 4) & 1; }
template <int HD>
__device__ __forceinline__ void kv4_fetch(Kv4Tile<HD>& t, const uint8_t* __restrict__ head0, const uint8_t* __restrict__ head1, int lane) {
    using L = Kv4Layout<HD>;
    const uint32_t c = lane & 15, r = lane >> 4;
    const uint32_t k_at = L::K + c * L::HALF + r * (L::HALF / 4), v_at = L::V + 4 * r * L::HALF + c * (L::HALF / 16);   // (unsigned: offsets from a scalar base)
    {
        const uint8_t* h = (kv4_scale_page<HD>(lane) ? head1 : head0) + 4u * kv4_scale_word<HD>(lane);
        t.ks = *reinterpret_cast<const uint32_t*>(h + L::KS);
        t.vs = *reinterpret_cast<const uint32_t*>(h + L::VS);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const uint8_t* kp = (p ? head1 : head0) + k_at;
        if constexpr (HD == 128) {
            const kv4_u32x4 w = *reinterpret_cast<const kv4_u32x4*>(kp);
            t.kc[p][0] = w[0]; t.kc[p][1] = w[1]; t.kc[p][2] = w[2]; t.kc[p][3] = w[3];
        } else if constexpr (HD == 64) {
            const kv4_u32x2 w = *reinterpret_cast<const kv4_u32x2*>(kp);
            t.kc[p][0] = w[0]; t.kc[p][1] = w[1];
        } else {
            t.kc[p][0] = *reinterpret_cast<const uint32_t*>(kp);
        }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint8_t* vp = (p ? head1 : head0) + v_at + i * L::HALF;
            if constexpr (HD == 128) t.vc[p][i] = *reinterpret_cast<const uint32_t*>(vp);
            else if constexpr (HD == 64) t.vc[p][i] = *reinterpret_cast<const uint16_t*>(vp);
            else t.vc[p][i] = *vp;
        }
}
// Bits 4 j .. 4 j + 3 of both halves of w as the bf16 pair 16 + c.  The two constants come out of registers whose contents the compiler
// does not know: with literals it takes an and and an or, which have room for one each.
struct Kv4Bits { uint32_t mask, base; };
__device__ __forceinline__ Kv4Bits kv4_bits() {
    Kv4Bits k{0x00780078u, 0x41804180u};
    asm("" : "+s"(k.mask));
    asm("" : "+v"(k.base));
    return k;
}
__device__ __forceinline__ uint32_t kv4_pair(const Kv4Bits& k, uint32_t w, int j) { return ((j == 0 ? w << 3 : w >> (4 * j - 3)) & k.mask) | k.base; }
__device__ __forceinline__ float kv4_pair_sum(uint32_t p, float to) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(tasc_bf16x2, p), __builtin_bit_cast(tasc_bf16x2, 0x3F803F80u), to, false);
}
// (fmaxf quiets each operand by an instruction of its own first)
__device__ __forceinline__ float kv4_max3(float a, float b, float c) {
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
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
// What a tile's {scale, low} words come to, in LDS: every lane works out the tokens that it was dealt, all lanes read those of the products
// they hold (as each lane's own work it is a quarter of a tile's instructions).  A value low + scale c is scale (c + z), z = low / scale:
// the weights of the second product are p scale, rounded to bf16 once, and meet 16 + c in one matrix instruction and z - 16, as three bf16
// terms, in another, so that what the rounding takes from a weight it takes from the whole value.  (With p (low + 7.5 scale) as a product
// of its own, the two roundings of a weight differ, and the error against 64 bits is twice as large.)
template <int HD>
struct __attribute__((aligned(16))) Kv4Scales {
    static constexpr int G = Kv4Layout<HD>::GROUPS;
    float ks[2][G][16], kb[2][G][16], vs[2][G][16];    // by page, group, token
    uint16_t z[G][3][32], none[32];                     // (and zeros, the product's other rows) tokens in the order of the second product (4 of page 0, 4 of page 1 for each r)
};
// z - 16 in three terms, and the scale to go with it: where z is too large for them (its value is low then, to fp32's last place) or
// there is no scale, another pair with the same values
struct Kv4Z { float scale; uint16_t z[3]; };
__device__ __forceinline__ Kv4Z kv4_z(float scale, float low) {
    float z = low * __builtin_amdgcn_rcpf(scale);
    if (scale < 1.17549435e-38f && scale != 0.f) z = low / scale;               // (below the reciprocal's range)
    if (!(fabsf(z) <= 1073741824.f)) {                      // 2^30
        // (numbers are 0 where the scale is: 16 + c times low / 16 is the value, and z - 16 nothing)
        const bool none = scale == 0.f;
        z = none ? 16.f : 1073741824.f;
        scale = low * (none ? 1.f / 16.f : 1.f / 1073741824.f);
    }
    Kv4Z o;
    o.scale = scale;
    z -= 16.f;
#pragma unroll
    for (int i = 0; i < 3; ++i) {                           // 8 of the 24 bits each
        const uint32_t top = __float_as_uint(z) & 0xFFFF0000u;
        o.z[i] = (uint16_t)(top >> 16);
        z -= __uint_as_float(top);
    }
    return o;
}
constexpr float kKv4Grown = 8.f;                        // a maximum is followed once it grew by more than this power of 2
// Sums are taken of 2^-40 times the values from the first tile on that holds large ones (kKv4Large), for these have no room beside the weights
// (up to 2^8 each, of up to 2^30 tokens) and 16 + c: below that a sum is at most 2^38 (31 scale + |low - 16 scale|) < 2^111, and with the factor, of
// the largest values, 2^38 2^129.1 2^-40 < 2^128.  A power of 2: what ordinary tiles give is the same bits either way (products of a weight and
// a scale from 2^-86 on).
constexpr float kKv4Large = 0x1p70f, kKv4Less = 0x1p-40f, kKv4Room = 0x1p118f;

// What a wave holds: MT tiles of 16 (row, head) pairs of a KV head, with their queries and sums.
template <int HD, int MT>
struct Kv4Wave {
    static constexpr int G = Kv4Layout<HD>::GROUPS, KSTEPS = HD / 32, DT = HD / 16;
    kv4_bf16x8 fq[MT][KSTEPS];
    float qsum[MT][G];
    kv4_f32x4 acc[MT][DT], ev[MT];                          // ev rows 4 g .. 4 g + 2: sums of p scale (z - 16)'s terms
    float m[MT], l[MT], lim[MT];                            // lim: what a score may be above m (nothing yet: -infinity)
    float s[MT][2][4];                                      // a tile's scores, less m
    int last[MT];                                           // last key that the lane's pair sees
    int pair0, live, first_last;                            // first pair, tiles of pairs that hold any, last key of the first pair
    bool less;                                              // acc and ev are of 2^-40 times the values
    const Kv4Seq& sq;
    int h, share, n_pairs, lane, col, r;

    __device__ __forceinline__ Kv4Wave(const Kv4Seq& sequence, int kv_head, int heads_share, int first_pair, int lane_)
        : pair0(first_pair), sq(sequence), h(kv_head), share(heads_share), lane(lane_), col(lane_ & 15), r(lane_ >> 4) {
        n_pairs = sq.n * share;
        live = pair0 < n_pairs ? (min(pair0 + 16 * MT, n_pairs) - 1 - pair0) / 16 + 1 : 0;
        first_last = sq.len - sq.n + pair0 / share;
    }
    // tiles of 32 tokens with a key that any of the pairs sees (a negative count: none)
    __device__ __forceinline__ int tiles(int len) const {
        if (pair0 >= n_pairs) return 0;
        const int last_last = sq.len - sq.n + (min(pair0 + 16 * MT, n_pairs) - 1) / share;
        return (min(last_last + 1, len) + 31) / 32;
    }
    __device__ __forceinline__ bool pair(int t, int rows, int& row, int& head) const {
        const int pr = pair0 + 16 * t + col;
        row = sq.first + pr / share;
        head = h * share + pr % share;
        return pr < n_pairs && row < rows;
    }
    // the queries are asked for ..
    __device__ __forceinline__ void ask(const Kv4Attn& a) {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            int row, head;
            const bool there = pair(t, a.rows, row, head);
            last[t] = there ? sq.len - sq.n + (pair0 + 16 * t + col) / share : -1;
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) {
                const int d = HD == 128 ? (i / 2) * 64 + 16 * r + 8 * (i & 1) : HD == 64 ? 16 * r + 8 * i : 8 * r;
                kv4_u32x4 w = {0, 0, 0, 0};
                if (there) w = *reinterpret_cast<const kv4_u32x4*>(a.q + (size_t)row * a.q_stride + head * HD + d);
                fq[t][i] = __builtin_bit_cast(kv4_bf16x8, w);
            }
        }
    }
    // .. and looked at
    __device__ __forceinline__ void begin() {
        less = false;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
#pragma unroll
            for (int g = 0; g < G; ++g) qsum[t][g] = 0.f;
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) {
                const kv4_u32x4 w = __builtin_bit_cast(kv4_u32x4, fq[t][i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) qsum[t][HD == 128 ? i / 2 : 0] = kv4_pair_sum(w[e], qsum[t][HD == 128 ? i / 2 : 0]);
            }
#pragma unroll
            for (int g = 0; g < G; ++g) qsum[t][g] = kv4_quad_sum(qsum[t][g]);
            m[t] = 0.f;
            l[t] = 0.f;
            lim[t] = -__builtin_inff();
            ev[t] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < DT; ++j) acc[t][j] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // scores of page p's 16 tokens
    __device__ __forceinline__ void scores(int p, const kv4_bf16x8 (&fk)[KSTEPS], const Kv4Scales<HD>& sc) {
        kv4_f32x4 ks[G], kb[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            ks[g] = *reinterpret_cast<const kv4_f32x4*>(&sc.ks[p][g][4 * r]);
            kb[g] = *reinterpret_cast<const kv4_f32x4*>(&sc.kb[p][g][4 * r]);
        }
#pragma unroll
        for (int u = 0; u < MT; ++u) {
            if (MT > 1 && u >= live) break;                 // (a wave without pairs sees no tile)
            kv4_f32x4 sg[G];
#pragma unroll
            for (int g = 0; g < G; ++g) sg[g] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) {
                constexpr int per = KSTEPS / G;
                sg[i / per] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fk[i], fq[u][i], sg[i / per], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = -m[u];
#pragma unroll
                for (int g = 0; g < G; ++g) v = __builtin_fmaf(kb[g][i], qsum[u][g], v);
#pragma unroll
                for (int g = 0; g < G; ++g) v = __builtin_fmaf(ks[g][i], sg[g][i], v);
                s[u][p][i] = v;
            }
        }
    }
    // the tile's weights and their sums; at: its first position, whole: every pair sees all of it, ok0, ok1: its pages are in the pool, large:
    // some of its values are
    __device__ __forceinline__ void sums(const kv4_bf16x8 (&fv)[DT], const Kv4Scales<HD>& sc, int at, bool whole, bool ok0, bool ok1, bool large, int len) {
        kv4_bf16x8 fz[G];
        kv4_f32x4 vs[2][G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int k = col - 4 * g;
            fz[g] = *reinterpret_cast<const kv4_bf16x8*>(&sc.z[0][k >= 0 && k < 3 ? 3 * g + k : 3 * G][8 * r]);     // 3 G: the zeros
#pragma unroll
            for (int p = 0; p < 2; ++p) vs[p][g] = *reinterpret_cast<const kv4_f32x4*>(&sc.vs[p][g][4 * r]);
        }
        if (large || less) {
            if (!less) {
                less = true;
#pragma unroll
                for (int u = 0; u < MT; ++u) {
                    ev[u] *= kKv4Less;
#pragma unroll
                    for (int j = 0; j < DT; ++j) acc[u][j] *= kKv4Less;
                }
            }
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int p = 0; p < 2; ++p) vs[p][g] *= kKv4Less;
        }
#pragma unroll
        for (int u = 0; u < MT; ++u) {
            if (MT > 1 && u >= live) break;                 // (a wave without pairs sees no tile)
            if constexpr (MT > 1) __builtin_amdgcn_sched_barrier(0);
            if (!whole) {
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int upto = ((p ? ok1 : ok0) ? min(last[u], len - 1) : -1) - (at + 16 * p + 4 * r);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[u][p][i] = i > upto ? -__builtin_inff() : s[u][p][i];
                }
            }
            float top = kv4_max3(kv4_max3(s[u][0][0], s[u][0][1], s[u][0][2]), s[u][0][3], s[u][1][0]);
            top = kv4_max3(kv4_max3(top, s[u][1][1], s[u][1][2]), s[u][1][3], s[u][1][3]);
            if (__any(top > lim[u])) {
                top = kv4_quad_max(top);
                if (top > lim[u]) {                         // (the four lanes of a pair alike)
                    const float f = __builtin_amdgcn_exp2f(-top);
                    l[u] *= l[u] > 0.f ? f : 1.f;           // (zeros so far: f may be infinite)
                    if (lim[u] == kKv4Grown) {
                        ev[u] *= f;
#pragma unroll
                        for (int j = 0; j < DT; ++j) acc[u][j] *= f;
                    }
                    m[u] += top;
                    lim[u] = kKv4Grown;
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[u][p][i] -= top;
                }
            }
            float pw[2][4];
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    pw[p][i] = __builtin_amdgcn_exp2f(s[u][p][i]);
                    l[u] += pw[p][i];
                }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float ps[2][4];
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) ps[p][i] = pw[p][i] * vs[p][g][i];
                const kv4_u32x4 w = {f2bf_pair(ps[0][0], ps[0][1]), f2bf_pair(ps[0][2], ps[0][3]), f2bf_pair(ps[1][0], ps[1][1]), f2bf_pair(ps[1][2], ps[1][3])};
                const kv4_bf16x8 fp = __builtin_bit_cast(kv4_bf16x8, w);
                ev[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fz[g], fp, ev[u], 0, 0, 0);
#pragma unroll
                for (int j = g * (DT / G); j < (g + 1) * (DT / G); ++j) acc[u][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv[j], fp, acc[u][j], 0, 0, 0);
            }
        }
    }
    // the four lanes' sums, and the channels' share of ev
    __device__ __forceinline__ void end() {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            l[t] = kv4_quad_sum(l[t]);
            if (lim[t] != kKv4Grown) m[t] = -__builtin_inff();   // no key
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float e = __shfl((ev[t][0] + ev[t][1]) + ev[t][2], 16 * g + col);
#pragma unroll
                for (int j = g * (DT / G); j < (g + 1) * (DT / G); ++j) acc[t][j] += e;
            }
            // Back to the values themselves; a pair whose sums have no room for that (there are up to 512 to join) has the same mean with 2^-16 as
            // its weights' sum, and a maximum to go with it.  (What a pair does not see decides nothing here.)
            if (less) {
                float top = 0.f;
#pragma unroll
                for (int j = 0; j < DT; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(acc[t][j][i]));
                const bool room = !(kv4_quad_max(top) > kKv4Room * kKv4Less);
                const float f = room ? 1.f / kKv4Less : (0x1p-16f / kKv4Less) / l[t];
#pragma unroll
                for (int j = 0; j < DT; ++j) acc[t][j] *= f;
                if (!room) {
                    m[t] += __builtin_amdgcn_logf(l[t]) + 16.f;
                    l[t] = 0x1p-16f;
                }
            }
        }
    }
    // A lane's channels: of tile j row 4 r + i, channel (HD 128, 64) 64 (j / 4) + 16 r + 4 i + j % 4, (32) 8 r + 2 i + j: in items (i, group of
    // four tiles j) of as many neighbours
    static constexpr int QUADS = DT / 4 > 0 ? DT / 4 : 1, ITEMS = 4 * QUADS;
    __device__ __forceinline__ float4 quad(int t, int item) const {
        const int i = item / QUADS, j = 4 * (item % QUADS);
        return HD == 32 ? make_float4(acc[t][0][i], acc[t][1][i], 0.f, 0.f) : make_float4(acc[t][j][i], acc[t][j + 1][i], acc[t][j + 2][i], acc[t][j + 3][i]);
    }
    __device__ __forceinline__ int channel(int item) const { return HD == 32 ? 8 * r + 2 * (item / QUADS) : 64 * (item % QUADS) + 16 * r + 4 * (item / QUADS); }
    static __device__ __forceinline__ void store(const Kv4Attn& a, int row, int head, int d, const float4& o, float inv) {
        uint16_t* to = reinterpret_cast<uint16_t*>(a.out + (size_t)row * a.out_stride + head * HD + d);
        if constexpr (HD == 32) *reinterpret_cast<uint32_t*>(to) = f2bf_pair(o.x * inv, o.y * inv);
        else *reinterpret_cast<kv4_u32x2*>(to) = kv4_u32x2{f2bf_pair(o.x * inv, o.y * inv), f2bf_pair(o.z * inv, o.w * inv)};
    }
};
// a pair without keys gives zeros (a NaN stays one)
__device__ __forceinline__ float kv4_inverse(float l) { return l > 0.f ? 1.f / l : l; }

// the tile's {scale, low} words, which the lanes were dealt, into LDS; whether any of the values is large
template <int HD>
__device__ __forceinline__ bool kv4_work_scales(Kv4Scales<HD>& sc, uint32_t k_word, uint32_t v_word, float scale2, int at, bool whole, bool ok0, bool ok1, int len, int lane) {
    constexpr int G = Kv4Layout<HD>::GROUPS;
    const int p = kv4_scale_page<HD>(lane), g = kv4_scale_word<HD>(lane) / 16, tok = lane & 15;
    float ks = kv4_scale(k_word) * scale2, lo = kv4_low(k_word) * scale2, vs = kv4_scale(v_word), vl = kv4_low(v_word);
    const bool in = whole || ((p ? ok1 : ok0) && at + 16 * p + tok < len);      // (what lies elsewhere may be no number)
    if (!in) ks = lo = vs = vl = 0.f;
    if (!(fabsf(__builtin_fmaf(7.5f, vs, vl)) < __builtin_inff())) { ks = __builtin_nanf(""); vs = vl = 0.f; }   // values that are none: who sees the token gets NaN by its score
    const Kv4Z z = kv4_z(vs, vl);
    if (G == 2 || lane < 32) {
        (&sc.ks[0][0][0])[lane] = ks;
        (&sc.kb[0][0][0])[lane] = __builtin_fmaf(-16.f, ks, lo);
        (&sc.vs[0][0][0])[lane] = z.scale;
#pragma unroll
        for (int i = 0; i < 3; ++i) sc.z[g][i][(tok / 4) * 8 + 4 * p + tok % 4] = z.z[i];
    }
    return __any(__builtin_fmaf(16.f, vs, fabsf(vl)) > kKv4Large);
}
template <int HD>
__device__ __forceinline__ kv4_bf16x8 kv4_key_part(const Kv4Bits& bits, const Kv4Tile<HD>& t, int p, int i) {
    const uint32_t w = t.kc[p][i];
    return __builtin_bit_cast(kv4_bf16x8, kv4_u32x4{kv4_pair(bits, w, 0), kv4_pair(bits, w, 1), kv4_pair(bits, w, 2), kv4_pair(bits, w, 3)});
}
// the lane's tokens' value numbers, pairs of tokens in a register: [lower, upper half of the words][token pair]
template <int HD>
struct Kv4Values { uint32_t pr[HD == 128 ? 2 : 1][4]; };
template <int HD>
__device__ __forceinline__ Kv4Values<HD> kv4_values(const Kv4Tile<HD>& t) {
    Kv4Values<HD> v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t x = t.vc[e / 2][2 * (e % 2)], y = t.vc[e / 2][2 * (e % 2) + 1];
        v.pr[0][e] = __builtin_amdgcn_perm(y, x, 0x05040100u);
        if constexpr (HD == 128) v.pr[1][e] = __builtin_amdgcn_perm(y, x, 0x07060302u);
    }
    return v;
}
template <int HD>
__device__ __forceinline__ kv4_bf16x8 kv4_value_part(const Kv4Bits& bits, const Kv4Values<HD>& v, int j) {
    const uint32_t(&w)[4] = v.pr[j / 4];
    return __builtin_bit_cast(kv4_bf16x8, kv4_u32x4{kv4_pair(bits, w[0], j % 4), kv4_pair(bits, w[1], j % 4), kv4_pair(bits, w[2], j % 4), kv4_pair(bits, w[3], j % 4)});
}
// The ids of 32 tiles' pages, two lanes a tile, tile `from` and every `step`-th behind it: a look at the table is then no memory access.
// -1: behind the last tile, or outside the pool, where an id is not followed and its tokens are masked.
__device__ __forceinline__ int kv4_page_ids(const Kv4Attn& a, int b, int from, int step, int n_tiles, int lane) {
    const int t = from + (lane >> 1) * step, at = 2 * t + (lane & 1);
    int page = -1;
    if (t < n_tiles && at < a.max_pages) page = a.table[(size_t)b * a.max_pages + at];
    return page < a.n_pages ? page : -1;
}

// A step's rows: few pairs (up to 16 MT a wave).  (To work a tile out once for the two waves of 17 to 64 pairs, as k_kv4_attention_rows does, is
// no faster: 256 sequences of 5 rows, 16 / 2 heads, 29.7 | 29.6 us, 64 of 9 rows 34.3 | 33.9, and with 20 pairs 24.8 | 36.3: the barriers cost
// what the instructions save.)  KW waves share their pairs and take a key chunk's tiles in turn; a workgroup has a.row_waves times as
// many, each KW of them with pairs of their own (over the same keys, which they so find in the L1 cache).
template <int HD, int MT, int KW>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_kv4_attention(Kv4Attn a) {
    using W = Kv4Wave<HD, MT>;
    using L = Kv4Layout<HD>;
    constexpr int AHEAD = MT * HD >= 256 ? 1 : 2;           // tiles under way: as many as the registers of two waves a SIMD hold beside the sums
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, r = lane >> 4;
    // (the last waves have the fewest pairs; every second workgroup of a compute unit takes them the other way round, or the same SIMDs would
    // have the full ones every time)
    const int kw = wave % KW, turned = (blockIdx.y * gridDim.x + blockIdx.x) / 256 % 2, rw = turned ? a.row_waves - 1 - wave / KW : wave / KW;
    Kv4Scales<HD>& sc = reinterpret_cast<Kv4Scales<HD>*>(lds)[wave];
    const int b = blockIdx.y / a.Hkv, h = blockIdx.y % a.Hkv, share = a.H / a.Hkv;
    const int tile = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const Kv4Seq sq = kv4_seq(a, b);
    const int wg_pair = tile * a.row_waves * 16 * MT;
    if (wg_pair >= sq.n * share) return;                   // (the whole workgroup; a wave without pairs among them goes on without keys)
    W w(sq, h, share, wg_pair + rw * 16 * MT, lane);
    const int len = min(max(sq.len, 0), a.max_pages * TASC_KV_BLOCK);
    const int n_tiles = min(w.tiles(len), chunk + 1 < a.chunks ? (chunk + 1) * a.chunk_tiles : INT32_MAX);
    const size_t page_bytes = (size_t)a.Hkv * L::HEAD;
    const uint8_t* const pool = a.pool + (size_t)h * L::HEAD;
    const int first_tile = chunk * a.chunk_tiles + kw;
    int ids = kv4_page_ids(a, b, first_tile, KW, n_tiles, lane), ids_next = 0;
    auto where = [&](int page) { return pool + (size_t)max(page, 0) * page_bytes; };
    w.ask(a);
    // the first tiles are under way while the queries are looked at
    Kv4Tile<HD> tile_a, tile_b;
    int pa0 = __builtin_amdgcn_readlane(ids, 0), pa1 = __builtin_amdgcn_readlane(ids, 1);
    int pb0 = __builtin_amdgcn_readlane(ids, 2), pb1 = __builtin_amdgcn_readlane(ids, 3);
    kv4_fetch<HD>(tile_a, where(pa0), where(pa1), lane);   // (without tiles: page 0, not used)
    if constexpr (AHEAD == 2) kv4_fetch<HD>(tile_b, where(pb0), where(pb1), lane);
    w.begin();
    if (lane < 32) sc.none[lane] = 0;
    const Kv4Bits bits = kv4_bits();
    const float scale2 = a.scale * 1.44269504088896340736f;   // scores in powers of 2

    // one tile out of `cur`, whose registers then take the tile of the pages that come next
    auto work = [&](Kv4Tile<HD>& cur, int t, int pg0, int pg1, int ng0, int ng1) __attribute__((always_inline)) {
        const int at = 32 * t;
        const bool whole = pg0 >= 0 && pg1 >= 0 && at + 31 <= w.first_last && at + 32 <= len;
        const bool large = kv4_work_scales<HD>(sc, cur.ks, cur.vs, scale2, at, whole, pg0 >= 0, pg1 >= 0, len, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a wave's LDS accesses are in order: the compiler has to keep them so)
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            if constexpr (MT > 1) __builtin_amdgcn_sched_barrier(0);
            kv4_bf16x8 fk[W::KSTEPS];
#pragma unroll
            for (int i = 0; i < W::KSTEPS; ++i) fk[i] = kv4_key_part<HD>(bits, cur, p, i);
            w.scores(p, fk, sc);
        }
        if constexpr (MT > 1) __builtin_amdgcn_sched_barrier(0);
        const Kv4Values<HD> values = kv4_values<HD>(cur);
        if constexpr (MT > 1) __builtin_amdgcn_sched_barrier(0);
        kv4_fetch<HD>(cur, where(ng0), where(ng1), lane);
        kv4_bf16x8 fv[W::DT];
#pragma unroll
        for (int j = 0; j < W::DT; ++j) fv[j] = kv4_value_part<HD>(bits, values, j);
        w.sums(fv, sc, at, whole, pg0 >= 0, pg1 >= 0, large, len);
    };
    int k = 2 * AHEAD;                                      // place of the next tile's ids
    for (int t = first_tile; t < n_tiles; t += AHEAD * KW) {
        if (k == 2 * AHEAD) ids_next = kv4_page_ids(a, b, t + 32 * KW, KW, n_tiles, lane);   // (32 tiles ahead)
        if (k == 64) { ids = ids_next; k = 0; }
        const int na0 = __builtin_amdgcn_readlane(ids, k), na1 = __builtin_amdgcn_readlane(ids, k + 1);
        if constexpr (AHEAD == 2) {
            const int nb0 = __builtin_amdgcn_readlane(ids, k + 2), nb1 = __builtin_amdgcn_readlane(ids, k + 3);
            work(tile_a, t, pa0, pa1, na0, na1);
            if (t + KW < n_tiles) work(tile_b, t + KW, pb0, pb1, nb0, nb1);
            pb0 = nb0; pb1 = nb1;
        } else {
            work(tile_a, t, pa0, pa1, na0, na1);
        }
        pa0 = na0; pa1 = na1;
        k += 2 * AHEAD;
    }

    // every wave leaves its sums in LDS and joins a part of the channels, in wave order
    w.end();
    constexpr int ITEMS = W::ITEMS, SPAN = MT * ITEMS;
    float4* const sx = reinterpret_cast<float4*>(lds) + (size_t)rw * KW * SPAN * 64;                      // [KW][MT][ITEMS][64]
    float2* const sm = reinterpret_cast<float2*>(reinterpret_cast<float4*>(lds) + (size_t)a.row_waves * KW * SPAN * 64) + rw * KW * MT * 16;   // [KW][MT][16]
    __syncthreads();                                        // (the scales are read)
#pragma unroll
    for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int item = 0; item < ITEMS; ++item) sx[((kw * MT + t) * ITEMS + item) * 64 + lane] = w.quad(t, item);
        if (r == 0) sm[(kw * MT + t) * 16 + col] = make_float2(w.m[t], w.l[t]);
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        float part[KW], top = -__builtin_inff(), l = 0.f;
#pragma unroll
        for (int x = 0; x < KW; ++x) top = fmaxf(top, sm[(x * MT + t) * 16 + col].x);
#pragma unroll
        for (int x = 0; x < KW; ++x) {
            const float2 ml = sm[(x * MT + t) * 16 + col];
            part[x] = ml.x == top ? 1.f : __builtin_amdgcn_exp2f(ml.x - top);
            l = __builtin_fmaf(ml.y, part[x], l);
        }
        int row, head;
        if (!w.pair(t, a.rows, row, head)) continue;
        const float inv = kv4_inverse(l);
        const size_t at = ((size_t)chunk * a.rows + row) * a.H + head;
        constexpr int MINE = ITEMS / KW > 0 ? ITEMS / KW : 1;
        if (KW <= ITEMS || kw < ITEMS)
#pragma unroll
            for (int n = 0; n < MINE; ++n) {
                const int item = kw * MINE + n, d = w.channel(item);
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int x = 0; x < KW; ++x) {
                    const float4 v = sx[((x * MT + t) * ITEMS + item) * 64 + lane];
                    o.x = __builtin_fmaf(v.x, part[x], o.x);
                    o.y = __builtin_fmaf(v.y, part[x], o.y);
                    o.z = __builtin_fmaf(v.z, part[x], o.z);
                    o.w = __builtin_fmaf(v.w, part[x], o.w);
                }
                if (a.chunks == 1) {
                    W::store(a, row, head, d, o, inv);
                } else {
                    float* to = a.part_o + at * HD + d;
                    if constexpr (HD == 32) *reinterpret_cast<float2*>(to) = make_float2(o.x, o.y);
                    else *reinterpret_cast<float4*>(to) = o;
                }
            }
        if (a.chunks > 1 && kw == 0 && r == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(top, l);
    }
}
// LDS of a workgroup of `waves` waves
template <int HD, int MT, int KW>
int kv4_attention_lds(int waves) {
    const int scales = waves * (int)sizeof(Kv4Scales<HD>), join = waves * MT * ((HD >= 64 ? HD / 16 : 4) * 64 * 16 + 16 * 8);
    return scales > join ? scales : join;
}

// A prompt's rows: enough pairs that every wave has 32 of its own and sees all of their keys.  What a tile comes to before it meets
// a query (numbers as bf16, scales) is a third of a wave's instructions, so the four waves of a workgroup work out a tile each, a
// fragment of a product's operand a KB of LDS, and all of them take the four.
template <int HD>
struct Kv4Staged {
    kv4_u32x4 key[2][HD / 32][64], value[HD / 16][64];
    Kv4Scales<HD> scales;
};
constexpr int kKv4RowWaves = 4;
template <int HD>
__global__ __launch_bounds__(64 * kKv4RowWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_kv4_attention_rows(Kv4Attn a) {
    constexpr int MT = 2, WAVES = kKv4RowWaves;
    using W = Kv4Wave<HD, MT>;
    using L = Kv4Layout<HD>;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Kv4Staged<HD>* const staged = reinterpret_cast<Kv4Staged<HD>*>(lds);                 // [WAVES]
    // The last pairs see the most keys: those of all heads begin first, and a head goes from one XCD to the next (head by head: 113 us for
    // 4 prompts of up to 2048 rows, 12 heads, where this takes 104; a head on one XCD, whose prompt may be the short one: 133).  Every second
    // 256 workgroups, one a compute unit, come the other way round, so that long ones share theirs with short ones (8 prompts of up to 1024
    // rows 69 -> 65 us, 16 of 400 24.9 -> 23.9, the 4 of 2048 alike).
    const int layer = blockIdx.x / 256, id = layer % 2 == 1 && (layer + 1) * 256 <= (int)gridDim.x ? (2 * layer + 1) * 256 - 1 - (int)blockIdx.x : (int)blockIdx.x;
    const int heads = a.batch * a.Hkv, turned = id / heads, head = (id % heads + turned) % heads, b = head / a.Hkv, h = head % a.Hkv, share = a.H / a.Hkv;
    const Kv4Seq sq = kv4_seq(a, b);
    const int n_pairs = sq.n * share, n_wgs = (n_pairs + 16 * MT * WAVES - 1) / (16 * MT * WAVES), turn = n_wgs - 1 - turned;
    if (turn < 0) return;
    W w(sq, h, share, (turn * WAVES + wave) * 16 * MT, lane);
    const int len = min(max(sq.len, 0), a.max_pages * TASC_KV_BLOCK);
    const int mine = w.tiles(len);
    const int n_tiles = (min(sq.len - sq.n + (min((turn + 1) * WAVES * 16 * MT, n_pairs) - 1) / share + 1, len) + 31) / 32;    // of the workgroup
    const size_t page_bytes = (size_t)a.Hkv * L::HEAD;
    const uint8_t* const pool = a.pool + (size_t)h * L::HEAD;
    auto where = [&](int page) { return pool + (size_t)max(page, 0) * page_bytes; };
    int ids = kv4_page_ids(a, b, wave, WAVES, n_tiles, lane), ids_next = 0, k = 0;
    w.ask(a);
    Kv4Tile<HD> tile;
    int pg0 = __builtin_amdgcn_readlane(ids, 0), pg1 = __builtin_amdgcn_readlane(ids, 1);
    kv4_fetch<HD>(tile, where(pg0), where(pg1), lane);
    w.begin();
    if (lane < 32) staged[wave].scales.none[lane] = 0;
    const Kv4Bits bits = kv4_bits();
    const float scale2 = a.scale * 1.44269504088896340736f;
    __shared__ int s_ok[WAVES];                             // pages of a tile that are in the pool: bits 0, 1; large values: bit 2
    for (int t0 = 0; t0 < n_tiles; t0 += WAVES) {
        {
            Kv4Staged<HD>& to = staged[wave];
            const int t = t0 + wave;
            const bool inside = pg0 >= 0 && pg1 >= 0 && 32 * t + 32 <= len;
            const bool large = kv4_work_scales<HD>(to.scales, tile.ks, tile.vs, scale2, 32 * t, inside, pg0 >= 0, pg1 >= 0, len, lane);
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < W::KSTEPS; ++i) to.key[p][i][lane] = __builtin_bit_cast(kv4_u32x4, kv4_key_part<HD>(bits, tile, p, i));
            const Kv4Values<HD> values = kv4_values<HD>(tile);
#pragma unroll
            for (int j = 0; j < W::DT; ++j) to.value[j][lane] = __builtin_bit_cast(kv4_u32x4, kv4_value_part<HD>(bits, values, j));
            if (lane == 0) s_ok[wave] = (pg0 >= 0 ? 1 : 0) | (pg1 >= 0 ? 2 : 0) | (large ? 4 : 0);
        }
        // the next four tiles are under way while these are worked on
        k += 2;
        if (k == 2) ids_next = kv4_page_ids(a, b, t0 + wave + 32 * WAVES, WAVES, n_tiles, lane);
        if (k == 64) { ids = ids_next; k = 0; }
        pg0 = __builtin_amdgcn_readlane(ids, k);
        pg1 = __builtin_amdgcn_readlane(ids, k + 1);
        kv4_fetch<HD>(tile, where(pg0), where(pg1), lane);
        __syncthreads();
        for (int n = 0; n < WAVES && t0 + n < mine; ++n) {
            const Kv4Staged<HD>& from = staged[n];
            const int at = 32 * (t0 + n), ok = __builtin_amdgcn_readfirstlane(s_ok[n]);
            const bool whole = (ok & 3) == 3 && at + 31 <= w.first_last && at + 32 <= len;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                kv4_bf16x8 fk[W::KSTEPS];
#pragma unroll
                for (int i = 0; i < W::KSTEPS; ++i) fk[i] = __builtin_bit_cast(kv4_bf16x8, from.key[p][i][lane]);
                w.scores(p, fk, from.scales);
            }
            kv4_bf16x8 fv[W::DT];
#pragma unroll
            for (int j = 0; j < W::DT; ++j) fv[j] = __builtin_bit_cast(kv4_bf16x8, from.value[j][lane]);
            w.sums(fv, from.scales, at, whole, ok & 1, (ok >> 1) & 1, (ok >> 2) & 1, len);
        }
        __syncthreads();
    }
    w.end();
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        int row, q_head;
        if (!w.pair(t, a.rows, row, q_head)) continue;
        const float inv = kv4_inverse(w.l[t]);
#pragma unroll
        for (int item = 0; item < W::ITEMS; ++item) W::store(a, row, q_head, w.channel(item), w.quad(t, item), inv);
    }
}
template <int HD>
int kv4_attention_rows_lds() { return kKv4RowWaves * (int)sizeof(Kv4Staged<HD>); }

// The key chunks' results joined: HD / 4 lanes a (row, head) pair, four channels each.  A workgroup has 1024 / HD pairs of a sequence's row,
// or, of many chunks (SPLIT), one, whose chunks its 1024 / HD parts take in turn (64 chunks of 64 pairs: 9.6 -> 4.8 us).
template <int HD, bool SPLIT>
__global__ __launch_bounds__(256) void k_kv4_merge(Kv4Attn a) {
    constexpr int LANES = HD / 4, PARTS = 256 / LANES;
    __shared__ kv4_f32x4 s_o[SPLIT ? PARTS : 1][LANES];
    __shared__ float2 s_ml[SPLIT ? PARTS : 1];
    const Kv4Seq sq = kv4_seq(a, blockIdx.y);
    const int i = blockIdx.x % a.max_rows, row = sq.first + i, part = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int head = SPLIT ? blockIdx.x / a.max_rows : blockIdx.x / a.max_rows * PARTS + part;
    if (i >= sq.n || row >= a.rows || head >= a.H) return;  // (of SPLIT the whole workgroup)
    const size_t step = (size_t)a.rows * a.H, at = (size_t)row * a.H + head;
    const int c0 = SPLIT ? part : 0, by = SPLIT ? PARTS : 1;
    float top = -__builtin_inff(), l = 0.f;
#pragma unroll 8
    for (int c = c0; c < a.chunks; c += by) top = fmaxf(top, a.part_ml[2 * (c * step + at)]);
    kv4_f32x4 o = {0.f, 0.f, 0.f, 0.f};
    auto join = [&](const float2& ml, const kv4_f32x4& x) {
        const float f = ml.x == top ? 1.f : __builtin_amdgcn_exp2f(ml.x - top);
        l = __builtin_fmaf(ml.y, f, l);
        o += x * f;
    };
#pragma unroll 8
    for (int c = c0; c < a.chunks; c += by)
        join(*reinterpret_cast<const float2*>(a.part_ml + 2 * (c * step + at)), *reinterpret_cast<const kv4_f32x4*>(a.part_o + (c * step + at) * HD + 4 * lane));
    if constexpr (SPLIT) {
        s_o[part][lane] = o;
        if (lane == 0) s_ml[part] = make_float2(top, l);
        __syncthreads();
        if (part > 0) return;
        for (int n = 0; n < PARTS; ++n) top = fmaxf(top, s_ml[n].x);
        l = 0.f;
        o = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < PARTS; ++n) join(s_ml[n], s_o[n][lane]);
    }
    const float inv = kv4_inverse(l);
    *reinterpret_cast<kv4_u32x2*>(a.out + (size_t)row * a.out_stride + head * HD + 4 * lane) = kv4_u32x2{f2bf_pair(o[0] * inv, o[1] * inv), f2bf_pair(o[2] * inv, o[3] * inv)};
}
