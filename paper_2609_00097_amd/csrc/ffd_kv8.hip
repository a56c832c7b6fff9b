// The 8-bit KV cache for gfx950: writing tokens into it and reading it back.
//
// Format. A token's key or value x (128 bf16 dims of one KV head) is kept as M = max |x_d|, which is a bf16
// value, and n_d = rint(127 x_d / M) in [-127, 127] (half to even); x~_d = n_d M / 127. M = 0 has n = 0. A token
// with an infinity or a NaN keeps M = NaN and n = 0, so that it reads back as NaN in every dim.
//
// Exactness of n. M is scaled to [1/2, 1) by its exponent and x with it (exact, but for dims so far below M that
// n = 0). 127 / M is held as hi + lo (lo from the remainder of the division), q = fma(x, hi, x lo) is the quotient
// Q rounded to fp32, so a Q that is a tie (an fp32 value) is hit exactly. With X the 8-bit significand of x a Q that
// is no tie lies at least Q / (254 X) > 2^-16 Q from every tie, far more than q is off. The rounding to an integer is
// the addition of 1.5 * 2^23, whose low byte is n in two's complement.
// Exactness of the read. x = (n * fl(1/127)) * M is within 2^-22 of n M / 127, which lies at least 2^-17 from every
// midpoint of bf16 values unless it is a bf16 value itself (127 divides M n only if it divides n or M's significand,
// and then the quotient has 8 bits): the bf16 result is the correctly rounded one.
//
// Bound: HBM (a written vector: 256 bytes read, 130 written; a read one the other way round), or the launch. Measured: one
// token of 2 KV heads written 2.2 us, of 32 x 8 4.8; 2 x 2K tokens of 8 KV heads 6.9 (3.5 TB/s; over with its first round
// of loads); 2 x 11.8K tokens read back 27 us (5.4 TB/s), 1 x 128K 137 (5.9).
#include "ffd_kernels.h"
#include "ffd_kv8.h"

namespace ffd {

// A workgroup writes 32 vectors of one sequence: 2^tok_shift tokens of 32 / 2^tok_shift KV heads, eight lanes each,
// key and value. With as many tokens as there are, up to 32, the absmaxes of a head leave side by side.
__global__ __launch_bounds__(kThreads) void write_kv8_kernel(WriteKv8Args a) {
    const int tid = threadIdx.x, s8 = tid & 7, i = tid >> 3;
    const int b = blockIdx.z;
    const int h = (int)(blockIdx.y << (5 - a.tok_shift)) + (i >> a.tok_shift);
    const int t = (int)(blockIdx.x << a.tok_shift) + (i & ((1 << a.tok_shift) - 1));
    const int count = a.counts ? min(a.counts[b], a.T) : a.T;
    const long long at = (long long)a.start[b] + t;
    if (h >= a.Hkv || t >= count || at < 0 || at >= a.Lcap) return;         // a vector's eight lanes together
    const uint4* kp = reinterpret_cast<const uint4*>(a.k_new + b * a.ks[0] + t * a.ks[1] + h * a.ks[2]) + 2 * s8;
    const uint4* vp = reinterpret_cast<const uint4*>(a.v_new + b * a.vs[0] + t * a.vs[1] + h * a.vs[2]) + 2 * s8;
    const uint4 kraw[2] = {kp[0], kp[1]}, vraw[2] = {vp[0], vp[1]};
    const size_t row = ((size_t)b * a.Hkv + h) * a.Lcap + at;
    uint32_t m;
    reinterpret_cast<uint4*>(a.k_codes)[row * 8 + s8] = encode_slice(kraw, m);
    if (s8 == 0) a.k_absmax[row] = (uint16_t)m;
    reinterpret_cast<uint4*>(a.v_codes)[row * 8 + s8] = encode_slice(vraw, m);
    if (s8 == 0) a.v_absmax[row] = (uint16_t)m;
}

// A workgroup reads back kReadTokens tokens of one (sequence, KV head), keys and values, 16 lanes a token: 8 codes
// in, 16 bytes out each, so that every access of a wave is whole rows. All of a thread's loads are asked for first (128K
// tokens: 151 us with one token after the other, 138 so). Rows behind the sequence's last token of the window repeat
// that one's load, and a workgroup that has no other reads nothing (4 sequences of up to 64K, eight KV heads: none empty
// 278 us, lengths spread over all 251, all empty 185).
__global__ __launch_bounds__(kThreads) void read_kv8_kernel(ReadKv8Args a) {
    constexpr int kSteps = kReadTokens / 16;
    const int l16 = threadIdx.x & 15, n = a.t_end - a.t_begin;
    const size_t bh = (size_t)blockIdx.z * a.Hkv + blockIdx.y;
    const int i0 = blockIdx.x * kReadTokens + (threadIdx.x >> 4);
    const int len = a.seq_lens ? min(max(a.seq_lens[blockIdx.z], 0), a.Lcap) : a.Lcap;
    const int shown = min(n, len - a.t_begin);          // tokens of the window that there are, none if not positive
    uint2 c[2][kSteps] = {};
    uint16_t m[2][kSteps] = {};
    if ((int)blockIdx.x * kReadTokens < shown) {
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const size_t row = bh * a.Lcap + a.t_begin + min(i0 + 16 * u, shown - 1);
            c[0][u] = reinterpret_cast<const uint2*>(a.k_codes)[row * 16 + l16];
            c[1][u] = reinterpret_cast<const uint2*>(a.v_codes)[row * 16 + l16];
            m[0][u] = a.k_absmax[row];
            m[1][u] = a.v_absmax[row];
        }
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const int i = i0 + 16 * u;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const uint32_t w[2] = {c[which][u].x, c[which][u].y};
            const float M = bf16_to_f32(m[which][u]);
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float x0 = (float)(int8_t)(w[e >> 2] >> (8 * (e & 3))) * (1.f / 127.f) * M;
                const float x1 = (float)(int8_t)(w[e >> 2] >> (8 * (e & 3) + 8)) * (1.f / 127.f) * M;
                o[e >> 1] = i < shown ? pack_bf16(x0, x1) : 0u;
            }
            uint16_t* dst = which ? a.v : a.k;
            if (i < n) reinterpret_cast<uint4*>(dst)[(bh * n + i) * 16 + l16] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

}  // namespace ffd
