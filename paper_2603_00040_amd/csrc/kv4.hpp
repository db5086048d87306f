// Attention over the NVFP4 cache with Q and P unquantized: what its kernels share (ragged.hip, sparse.hip).  The cached values of a lane's part of a
// key as operands of the matrix instruction, the factor of a row of Q, and the reference of a row's exponents.
#pragma once
#include "common.hpp"
#include "nvfp4.hpp"

namespace aq {

// The reference that a row's exponents are taken against, in powers of two, is set where the row's largest probability becomes 2^kTop, and follows the running
// maximum only when that would make it more than 2^kTopMost, just below what fp16 holds: most tiles need no rescaling of O, though some row of 32 has a
// new maximum in most of the first fifty tiles.  The higher the one, the smaller the probabilities that keep all their bits; the nearer to the other, the more
// often O is rescaled where scores spread widely (six prompts, four channels of K times 20, kTopMost 15: kTop 7 225 us, 9 226, 11 229; scores of deviation 1: even).
constexpr float kTop = 11.0f, kTopMost = 15.9f;
// The score up to which that holds (no score beyond, whatever is rounded here): a tile's largest is compared as it comes out of the product.
__device__ inline float score_up_to(float m, float c_row) { return fmaf(fabsf(m), -0x1p-20f, m + (kTopMost - 0x1p-10f)) * __builtin_amdgcn_rcpf(c_row); }

// Codes and scale bytes of D / 4 values of one key: lane (key cc of 16, group g) holds d = (D/4) g .. + D/4 - 1.  (The scale bytes as the dword that they
// lie in: of a narrower load the compiler makes the widening an instruction of its own, which waits for the load wherever it puts it.)
template <int D> struct Raw { uint32_t w[D / 32]; uint32_t sc; };
template <int D>
__device__ inline Raw<D> load_raw(const unsigned char* part /* K or V part of a page's head */, int key, int g)
{
    Raw<D> r;
    if constexpr (D == 128) {
        const uint4v c = *reinterpret_cast<const uint4v*>(part + key * 64 + 16 * g);
        r.w[0] = c[0]; r.w[1] = c[1]; r.w[2] = c[2]; r.w[3] = c[3];
        r.sc = *reinterpret_cast<const uint32_t*>(part + 128 * 64 + key * 8 + 4 * (g >> 1));
    } else {
        const uint2v c = *reinterpret_cast<const uint2v*>(part + key * 32 + 8 * g);
        r.w[0] = c[0]; r.w[1] = c[1];
        r.sc = *reinterpret_cast<const uint32_t*>(part + 128 * 32 + key * 4);
    }
    return r;
}
// The block scales of those values as an fp16 pair (one for D = 64).  Not live: 0, whatever the bytes are (a stale scale byte may be NaN).
template <int D>
__device__ inline half2v scales_of(const Raw<D>& r, int g, bool live)
{
    const uint32_t sc = r.sc >> (D == 128 ? 16 * (g & 1) : 8 * g);
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(live ? sc : 0u, 1.0f, false);
}
// Values 8 s .. 8 s + 7 of the lane's as fp16.
template <int D>
__device__ inline half8 values8(const Raw<D>& r, half2v sc, int s)
{
    const half_t sv = (D == 128 && s >= 2) ? sc[1] : sc[0];
    const half2v sc2 = {sv, sv};
    const uint32_t w = r.w[s];
    uint4v v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0) * sc2);
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1) * sc2);
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2) * sc2);
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3) * sc2);
    return __builtin_bit_cast(half8, v);
}

// The largest magnitude of 8 N bf16 values: without their signs they are ordered as whole numbers are.
template <int N>
__device__ inline float largest_of(const uint4v (&x)[N])
{
    typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
    ushort2v m = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2v, x[i][j] & 0x7FFF7FFFu));
    return __uint_as_float((uint32_t)max(m[0], m[1]) << 16);
}
// The power of two that brings a row's largest magnitude to [2^14, 2^15), and its inverse (magnitudes below 2^-112 count as that).  The factor of the
// scores times the inverse is kept a normal number: where it would be less, scores differ by less than 2^-90, but a masked one times 0 would be a NaN.
constexpr float kLeastFactor = 0x1p-126f;
__device__ inline void row_factor(float amax, float& f, float& inv)
{
    const uint32_t e = max(__float_as_uint(amax) >> 23, 15u);
    f = __uint_as_float((268u - e) << 23);
    inv = __uint_as_float((e - 14u) << 23);
}

}  // namespace aq
