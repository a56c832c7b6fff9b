// Quantization of a vector to 8 bits, for the writers of 8-bit caches (ffd_kv8.hip has the format and the argument for
// its exactness).
#pragma once

#include "ffd_device.h"

namespace ffd {

// Codes of dims 2 i, 2 i + 1 in words w[i] of a vector with these absmax bits, four codes a word of out; zeros where the
// absmax is not finite (absmax is what is kept of it).
template <int WORDS>
__device__ __forceinline__ void encode_words(const uint32_t (&w)[WORDS], uint32_t bits, uint32_t (&out)[WORDS / 2], uint32_t& absmax) {
#pragma clang fp contract(off)          // the argument above names the fused product
    const bool finite = bits < 0x7f80u;
    absmax = finite ? bits : 0x7fc0u;
    const uint32_t keep = finite && bits != 0 ? 0xffffffffu : 0u;
    int E;
    const float m = frexpf(bf16_to_f32((uint16_t)bits), &E);
    const float hi = 127.f / m, lo = fmaf(-hi, m, 127.f) / m;
#pragma unroll
    for (int i = 0; i < WORDS / 2; ++i) {
        uint32_t n[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t word = w[2 * i + (e >> 1)];
            const float x = ldexpf(e & 1 ? bf16_hi(word) : bf16_lo(word), -E);
            n[e] = __float_as_uint(fmaf(x, hi, x * lo) + 12582912.f);
        }
        const uint32_t a = __builtin_amdgcn_perm(n[1], n[0], 0x0c0c0400u), b = __builtin_amdgcn_perm(n[3], n[2], 0x0c0c0400u);
        out[i] = (a | b << 16) & keep;
    }
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_u16(uint32_t x) {
    return pk_max_u16(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false));
}

// Codes (16 bytes) and absmax bits of a vector from this lane's 16 dims; the vector's eight lanes call it together.
__device__ __forceinline__ uint4 encode_slice(const uint4 (&raw)[2], uint32_t& absmax) {
    const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
    uint32_t m2 = w[0] & 0x7fff7fffu, out[4];
#pragma unroll
    for (int i = 1; i < 8; ++i) m2 = pk_max_u16(m2, w[i] & 0x7fff7fffu);
    m2 = dpp_max_u16<kDppHalfMirror>(dpp_max_u16<kDppXor2>(dpp_max_u16<kDppXor1>(m2)));
    encode_words(w, max(m2 & 0xffffu, m2 >> 16), out, absmax);
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// The same from this lane's eight dims, by the vector's 16 lanes.
__device__ __forceinline__ uint2 encode_eighth(const uint4& raw, uint32_t& absmax) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    uint32_t m2 = w[0] & 0x7fff7fffu, out[2];
#pragma unroll
    for (int i = 1; i < 4; ++i) m2 = pk_max_u16(m2, w[i] & 0x7fff7fffu);
    m2 = dpp_max_u16<kDppRor8>(dpp_max_u16<kDppRor4>(dpp_max_u16<kDppXor2>(dpp_max_u16<kDppXor1>(m2))));
    encode_words(w, max(m2 & 0xffffu, m2 >> 16), out, absmax);
    return make_uint2(out[0], out[1]);
}

}  // namespace ffd
