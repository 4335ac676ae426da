// Storage types, vector loads and wave sums that the kernels share.
#pragma once
#include "tasc_internal.h"
#include <type_traits>

struct BF16 { uint16_t v; };

__device__ inline float bf2f(uint32_t bits16) { return __uint_as_float(bits16 << 16); }
// fp32 -> bf16, round to nearest even: the hardware conversion of gfx950 (v_cvt_pk_bf16_f32), one instruction per pair
typedef __attribute__((ext_vector_type(2))) float tasc_f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 tasc_bf16x2;
__device__ inline uint32_t f2bf_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(tasc_f32x2{lo, hi}, tasc_bf16x2));
}
__device__ inline uint16_t f2bf(float f) { return (uint16_t)(f2bf_pair(f, 0.f) & 0xFFFFu); }
__device__ inline float to_f(float v) { return v; }
__device__ inline float to_f(BF16 v) { return bf2f(v.v); }
template <typename T> __device__ inline T from_f(float f);
template <> __device__ inline float from_f<float>(float f) { return f; }
template <> __device__ inline BF16 from_f<BF16>(float f) { return BF16{f2bf(f)}; }

__device__ inline void load8(const float* __restrict__ p, float* o) {
    float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w; o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
}
__device__ inline void load8(const BF16* __restrict__ p, float* o) {
    uint4 u = *reinterpret_cast<const uint4*>(p);
    o[0] = bf2f(u.x & 0xFFFFu); o[1] = bf2f(u.x >> 16); o[2] = bf2f(u.y & 0xFFFFu); o[3] = bf2f(u.y >> 16);
    o[4] = bf2f(u.z & 0xFFFFu); o[5] = bf2f(u.z >> 16); o[6] = bf2f(u.w & 0xFFFFu); o[7] = bf2f(u.w >> 16);
}

__device__ inline void load4(const float* __restrict__ p, float* o) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
}
__device__ inline void load4(const BF16* __restrict__ p, float* o) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    o[0] = bf2f(u.x & 0xFFFFu); o[1] = bf2f(u.x >> 16); o[2] = bf2f(u.y & 0xFFFFu); o[3] = bf2f(u.y >> 16);
}

template <int VEC, typename T>
__device__ inline void load_n(const T* __restrict__ p, float* o) {
    if constexpr (VEC == 8) load8(p, o);
    else load4(p, o);
}

__device__ inline float wave_sum(float v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ inline float wave_max(float v) {
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// Sum over the 64 lanes with DPP row operations (a few cycles each; the ds_bpermute path of __shfl_xor costs an LDS
// round trip per step).  The lanes are added in a fixed order, the same for every call.
__device__ __forceinline__ float wave_sum_dpp(float v) {
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, false));    // quad_perm [1,0,3,2]
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, false));    // quad_perm [2,3,0,1]
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x141, 0xF, 0xF, false));   // row_half_mirror
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x140, 0xF, 0xF, false));   // row_mirror
    // every lane now holds the sum of its row of 16; rows 0..3 are lanes 0-15, 16-31, 32-47, 48-63
    const float r0 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 0));
    const float r1 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 16));
    const float r2 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 32));
    const float r3 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 48));
    return (r0 + r1) + (r2 + r3);
}
// The same for a maximum, and for a sum of 64 bits
__device__ __forceinline__ float wave_max_dpp(float v) {
    auto up = [](float x, auto ctrl) { return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, false))); };
    v = up(v, std::integral_constant<int, 0xB1>{});
    v = up(v, std::integral_constant<int, 0x4E>{});
    v = up(v, std::integral_constant<int, 0x141>{});
    v = up(v, std::integral_constant<int, 0x140>{});
    auto row = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); };
    return fmaxf(fmaxf(row(0), row(16)), fmaxf(row(32), row(48)));
}
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double lane64_dpp(double v) {   // 0 where the lane has no source
    const u64 b = __builtin_bit_cast(u64, v);
    const u32 lo = __builtin_amdgcn_update_dpp(0, (int)(u32)b, CTRL, ROWS, 0xF, false), hi = __builtin_amdgcn_update_dpp(0, (int)(u32)(b >> 32), CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(double, (u64)hi << 32 | lo);
}
__device__ __forceinline__ double lane64(double v, int l) {  // l: the same in all lanes
    const u64 b = __builtin_bit_cast(u64, v);
    return __builtin_bit_cast(double, (u64)(u32)__builtin_amdgcn_readlane((int)(u32)(b >> 32), l) << 32 | (u32)__builtin_amdgcn_readlane((int)(u32)b, l));
}
template <typename Op>
__device__ __forceinline__ double wave_all64_dpp(double v, Op op) {
    v = op(v, lane64_dpp<0xB1>(v));
    v = op(v, lane64_dpp<0x4E>(v));
    v = op(v, lane64_dpp<0x141>(v));
    v = op(v, lane64_dpp<0x140>(v));
    return op(op(lane64(v, 0), lane64(v, 16)), op(lane64(v, 32), lane64(v, 48)));
}
__device__ __forceinline__ double wave_sum64_dpp(double v) { return wave_all64_dpp(v, [](double x, double y) { return x + y; }); }
__device__ __forceinline__ double wave_max64_dpp(double v) { return wave_all64_dpp(v, [](double x, double y) { return fmax(x, y); }); }
__device__ __forceinline__ double wave_scan64_dpp(double v) {   // sums of the lanes up to each
    v += lane64_dpp<0x111>(v);                              // row_shr 1, 2, 4, 8
    v += lane64_dpp<0x112>(v);
    v += lane64_dpp<0x114>(v);
    v += lane64_dpp<0x118>(v);
    v += lane64_dpp<0x142, 0xA>(v);                         // lane 15 of the row before, into rows 1 and 3
    v += lane64_dpp<0x143, 0xC>(v);                         // lane 31, into rows 2 and 3
    return v;
}

// exp(x) for x <= 1 (NaN stays one): x = n ln 2 + r, |r| <= ln 2 / 2, and the Taylor polynomial of degree 11, whose remainder is below
// (ln 2 / 2)^12 / 12! = 6.3e-15
__device__ __forceinline__ double exp_neg(double x) {
    x = x < -1000.0 ? -1000.0 : x;                         // (an underflow either way; -infinity has no n)
    const double n = rint(x * 1.4426950408889634074);
    double r = __builtin_fma(n, -0x1.62e42fefa4000p-1, x);            // ln 2 in 40 bits, and the rest
    r = __builtin_fma(n, 0x1.8432a1b0e2634p-43, r);
    double p = 1.0 / 39916800.0;
    p = __builtin_fma(p, r, 1.0 / 3628800.0);
    p = __builtin_fma(p, r, 1.0 / 362880.0);
    p = __builtin_fma(p, r, 1.0 / 40320.0);
    p = __builtin_fma(p, r, 1.0 / 5040.0);
    p = __builtin_fma(p, r, 1.0 / 720.0);
    p = __builtin_fma(p, r, 1.0 / 120.0);
    p = __builtin_fma(p, r, 1.0 / 24.0);
    p = __builtin_fma(p, r, 1.0 / 6.0);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return ldexp(p, (int)n);
}

// Exponentials by a table: 2^(n / 256) p, n in the low word of a double
typedef uint32_t word2 __attribute__((ext_vector_type(2)));
// 2^(i / 256), by the series of the exponential
constexpr double pow2_256(int i) {
    const double x = i * (0.69314718055994530942 / 256);
    double sum = 1.0, term = 1.0;
    for (int k = 1; k < 30; ++k) sum += term *= x / k;
    return sum;
}
struct PowTable { word2 at[256]; };                   // lower word, upper word less i << 12 (what i adds there beside i / 256 << 20)
constexpr PowTable pow_table() {
    PowTable t{};
    for (int i = 0; i < 256; ++i) {
        const u64 b = __builtin_bit_cast(u64, pow2_256(i));
        t.at[i] = word2{(u32)b, (u32)(b >> 32) - ((u32)i << 12)};
    }
    return t;
}
static __device__ const PowTable kPow = pow_table();
// p 2^(m / 256)
__device__ __forceinline__ double times_power(const word2* pow, double p, u32 m, double plus) {
    const word2 w = pow[m & 255];
    return __builtin_fma(p, __builtin_bit_cast(double, word2{w[0], w[1] + (m << 12)}), plus);
}
__device__ __forceinline__ double small_power(double f) {  // 2^(f / 256)
    double p = 0x1.c6b08d704a0c0p-29;
    p = __builtin_fma(p, f, 0x1.ebfbdff82c58fp-19);
    p = __builtin_fma(p, f, 0x1.62e42fefa39efp-9);
    return __builtin_fma(p, f, 1.0);
}
