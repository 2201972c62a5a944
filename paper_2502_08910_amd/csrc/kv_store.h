// KV caches in the storages that the library writes and reads (ihip_kv_store), and the 4-bit row format.
#pragma once

#include "common.h"

namespace ihip {

// A store as kernels see it: strides in bytes
struct StoreView {
    uint8_t *k, *v;
    int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st;
    uint8_t *ks, *vs;            // MX4: the four scale bytes of the row at byte o stand at o / 16
    float k_scale, v_scale;      // E4M3
    PagedView paged;             // block_table == nullptr: stride b goes from sequence to sequence
};
int32_t check_store(const char *who, const ihip_kv_store *store, const ihip_shape &for_lengths, StoreView *view);
// `whole`: with positions and tokens seen; otherwise the weights alone
int32_t check_track(const char *who, const ihip_kv_track *track, int64_t rows, bool whole);
int32_t check_packed(const char *who, const ihip_packed *p);
// `before`, decay and the weights [heads, rows] that they go into: arrays that are the same or apart
int32_t check_before(const char *who, const float *before, float decay, const ihip_kv_track *track, int64_t heads);
// Arrays that have bytes in common and do not begin together
inline bool overlap_in_part(const void *x, int64_t x_bytes, const void *y, int64_t y_bytes)
{
    const uintptr_t a = (uintptr_t)x, b = (uintptr_t)y;
    return a != b && a < b + (uintptr_t)y_bytes && b < a + (uintptr_t)x_bytes;
}

// ---- MX4 ----------------------------------------------------------------------
// 2^(s - 127) of a scale byte; what the converters take as their scale (only its exponent counts there).  255, which is an infinity here, is
// NaN to them: all codes widen to NaN, 0 too (checked on the card with codes of 0 and of any kind).
__device__ inline float mx4_scale(uint32_t s) { return __uint_as_float(s << 23); }

// One byte of codes (in byte SEL of w) -> two bf16, exact: E2M1 times a power of two is a bf16 number
template <int SEL>
__device__ inline uint32_t mx4_pair(uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}
// a lane's eight codes -> eight bf16
__device__ inline uint4 mx4_to_bf16x8(uint32_t w, float scale)
{
    return make_uint4(mx4_pair<0>(w, scale), mx4_pair<1>(w, scale), mx4_pair<2>(w, scale), mx4_pair<3>(w, scale));
}

// Eight elements a lane, 32 of them in four neighbouring lanes: their scale byte, and this lane's eight codes.  The largest
// magnitude is taken as an integer, so that NaN and infinity come out on top; 2^e is the smallest power of two with which it is
// at most 7 = 1.75 * 4, kept to 2^-100 .. 2^125 (6 times which bf16 still holds).  v_cvt_scalef32_pk_fp4_f32 divides by the scale (exact), rounds to nearest, ties to even, and stops at 6
// (compared with the comparisons of the definition at every multiple of 2^-9 up to 8).
__device__ inline uint32_t mx4_quantise(const float (&f)[8], uint32_t &scale_byte)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true));     // quad_perm [1,0,3,2]
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, true));     // quad_perm [2,3,0,1]
    const int e = (int)(top >> 23) - ((top & 0x7fffffu) <= 0x600000u ? 2 : 1);                    // biased by 127
    const bool finite = top < 0x7f800000u;
    scale_byte = finite ? (uint32_t)min(max(e, 27), 252) : 255u;
    const float s = mx4_scale(finite ? scale_byte : 127u);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], s, 3);
    return finite ? w : 0u;
}

// ---- rotation -----------------------------------------------------------------
// Four (even, odd) pairs turned in place, fp32, every product and sum rounded on its own: what is rounded to 4 or 8 bits next does not
// depend on which of them the compiler would fuse.
__device__ inline void turn_f32x8(float (&f)[8], const float4 c, const float4 sn)
{
#pragma clang fp contract(off)
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {sn.x, sn.y, sn.z, sn.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float e = f[2 * i], o = f[2 * i + 1];
        f[2 * i] = e * cc[i] - o * ss[i];
        f[2 * i + 1] = e * ss[i] + o * cc[i];
    }
}

// ---- E4M3 ---------------------------------------------------------------------
// value / scale, kept inside the format's range (NaN stays NaN), to nearest, ties to even
__device__ inline uint2 e4m3_quantise(const float (&f)[8], float scale)
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = f[i] / scale;
        x[i] = y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
    }
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}

}  // namespace ihip
