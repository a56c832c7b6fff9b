// New queries, keys and values of a ragged batch on their way to attention over a paged cache: norms per head, rotation,
// and keys and values to their places, in one pass.
//
// Mathematics, in fp32 with one rounding to bf16 at the end: y = x / sqrt(mean(x^2) + eps) * w over the 128 dims of a
// query's or key's head (w null: y = x); then, for each of the rope_dims / 2 pairs (a, b) of dims, the rotation
// (a cos - b sin, b cos + a sin) by the angle of the token's position, whose cosine and sine come from the caller's table
// (computing them here would take 64 bits for far positions, and the table's row is read once for all heads of a token).
// Pairs are (d, d + rope_dims / 2), or neighbours (2 d, 2 d + 1). A key is rounded to bf16 before its 8-bit codes are taken
// (ffd_kv8.hip), so that they are those of the same key written by ffd_write_kv8.
//
// Bound: HBM (256 bytes read and written per vector), for few tokens the chain of starts, length, page and vector.
#include "ffd_kv8.h"
#include "ffd_paged.h"

namespace ffd {

namespace {

// Sequence of a row of the batch: the number of sequences that end at or before it, found by the wave 64 at a time, a range
// that is 64 times smaller with each look.
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int B, int row, int lane) {
    int low = 0, count = B;                     // ends low .. low + count - 1 are open, those before are at or before the row
    while (count > 0) {
        const int step = (count + 63) / 64;
        const int i = (lane + 1) * step - 1;    // the last of this lane's `step` ends
        const bool passed = i < count && q_start[low + min(i, count - 1) + 1] <= row;
        const int whole = __popcll(__ballot(passed));
        low += whole * step;
        count = step == 1 ? 0 : min(step, count - whole * step);
    }
    return low;
}

struct Vec {
    float x[16];
};

__device__ __forceinline__ Vec load_vec(const uint16_t* p, int s8) {
    const uint4* at = reinterpret_cast<const uint4*>(p) + 2 * s8;
    const uint4 a = at[0], b = at[1];
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    Vec v;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v.x[2 * i] = bf16_lo(w[i]);
        v.x[2 * i + 1] = bf16_hi(w[i]);
    }
    return v;
}

}  // namespace

// Eight lanes a vector, 16 dims each; a wave's eight vectors belong to one token. A token's Hq + 2 Hkv vectors are taken by
// a.parts (a multiple of eight) such groups in turn, so that with many tokens a group reads its row of the table once for several heads.
template <bool I8, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void write_paged_kernel(WritePagedArgs a) {
    const int lane = threadIdx.x & 63, s8 = lane & 7;
    const int waves = a.parts >> 3;
    const long long wave = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int row = __builtin_amdgcn_readfirstlane((int)(wave / waves));
    const int part = (int)(wave - (long long)row * waves) * 8 + (lane >> 3);
    if (row >= a.T) return;
    const int b = sequence_of(a.q_start, a.B, row, lane);
    if (b >= a.B) return;
    const int first = a.q_start[b], last = min(a.q_start[b + 1], a.T);
    const int len = a.seq_lens[b];
    if (row < first) return;
    const int place = min(max(len, 0), kMaxLen) - (last - row);
    const int position = a.positions ? a.positions[row] : place;

    float cs[16], sn[16];
    const int half = a.rope_dims >> 1, lanes = half >> 4;      // lanes of the first members of the pairs
    if (a.rope && 16 * s8 < a.rope_dims) {
        const bool in = position >= 0 && position < a.rope_rows;
        const float* c = a.rope + (size_t)(in ? position : 0) * a.rope_dims;
        if constexpr (INTERLEAVED) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 x = *reinterpret_cast<const float4*>(c + 8 * s8 + 4 * i), y = *reinterpret_cast<const float4*>(c + half + 8 * s8 + 4 * i);
                cs[4 * i] = x.x, cs[4 * i + 1] = x.y, cs[4 * i + 2] = x.z, cs[4 * i + 3] = x.w;
                sn[4 * i] = y.x, sn[4 * i + 1] = y.y, sn[4 * i + 2] = y.z, sn[4 * i + 3] = y.w;
            }
        } else {
            const int at = 16 * (s8 < lanes ? s8 : s8 - lanes);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 x = *reinterpret_cast<const float4*>(c + at + 4 * i), y = *reinterpret_cast<const float4*>(c + half + at + 4 * i);
                cs[4 * i] = x.x, cs[4 * i + 1] = x.y, cs[4 * i + 2] = x.z, cs[4 * i + 3] = x.w;
                sn[4 * i] = y.x, sn[4 * i + 1] = y.y, sn[4 * i + 2] = y.z, sn[4 * i + 3] = y.w;
            }
        }
#pragma unroll
        for (int i = 0; i < (INTERLEAVED ? 8 : 16); ++i) {
            cs[i] = in ? cs[i] : NAN;
            sn[i] = in ? sn[i] : NAN;
        }
        if (!INTERLEAVED && s8 < lanes) {       // the first of a pair takes away what the second adds
#pragma unroll
            for (int i = 0; i < 16; ++i) sn[i] = -sn[i];
        }
    }

    const bool cached = place >= 0 && place < (a.pages.max_pages << a.pages.page_shift);
    const int entry = cached ? page_entry(a.pages, b, place) : -1;
    const bool there = page_there(a.pages, entry);
    const int Hq = a.q ? a.Hq : 0, vectors = Hq + 2 * a.Hkv;
    for (int v = part; v < vectors; v += a.parts) {             // the eight lanes of a vector together
        const bool is_q = v < Hq, is_k = !is_q && v < Hq + a.Hkv;
        const int head = is_q ? v : is_k ? v - Hq : v - Hq - a.Hkv;
        if (!is_q && !there) continue;
        const uint16_t* from = is_q ? a.q + row * a.qs[0] + head * a.qs[1] : is_k ? a.k + row * a.ks[0] + head * a.ks[1] : a.v + row * a.vs[0] + head * a.vs[1];
        uint4 raw[2];
        if (is_q || is_k) {
            Vec x = load_vec(from, s8);
            const uint16_t* weight = is_q ? a.q_weight : a.k_weight;
            if (weight) {
                const Vec w = load_vec(weight, s8);
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) sum = fmaf(x.x[i], x.x[i], sum);
                sum += dpp_f<kDppXor1>(sum);
                sum += dpp_f<kDppXor2>(sum);
                sum += dpp_f<kDppHalfMirror>(sum);
                const float inv = 1.f / sqrtf(sum * (1.f / kD) + a.eps);
#pragma unroll
                for (int i = 0; i < 16; ++i) x.x[i] = x.x[i] * inv * w.x[i];
            }
            if (a.rope) {
                if constexpr (INTERLEAVED) {
                    if (16 * s8 < a.rope_dims) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float p = x.x[2 * i], r = x.x[2 * i + 1];
                            x.x[2 * i] = p * cs[i] - r * sn[i];
                            x.x[2 * i + 1] = r * cs[i] + p * sn[i];
                        }
                    }
                } else {
                    const int other = (lane & ~7) | (s8 < lanes ? s8 + lanes : 16 * s8 < a.rope_dims ? s8 - lanes : s8);
                    Vec y;
#pragma unroll
                    for (int i = 0; i < 16; ++i) y.x[i] = __shfl(x.x[i], other);
                    if (16 * s8 < a.rope_dims) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) x.x[i] = x.x[i] * cs[i] + y.x[i] * sn[i];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
                raw[i] = make_uint4(pack_bf16(x.x[8 * i], x.x[8 * i + 1]), pack_bf16(x.x[8 * i + 2], x.x[8 * i + 3]),
                                    pack_bf16(x.x[8 * i + 4], x.x[8 * i + 5]), pack_bf16(x.x[8 * i + 6], x.x[8 * i + 7]));
        } else {
            const uint4* p = reinterpret_cast<const uint4*>(from) + 2 * s8;
            raw[0] = p[0];
            raw[1] = p[1];
        }
        if (is_q) {
            uint4* to = reinterpret_cast<uint4*>(a.q_out + ((size_t)row * a.Hq + head) * kD) + 2 * s8;
            to[0] = raw[0];
            to[1] = raw[1];
            continue;
        }
        const size_t at = page_row(a.pages, a.Hkv, head, entry, place);
        uint8_t* tokens = const_cast<uint8_t*>(is_k ? a.pages.kv.k : a.pages.kv.v);
        if constexpr (I8) {
            uint32_t m;
            reinterpret_cast<uint4*>(tokens)[at * 8 + s8] = encode_slice(raw, m);
            if (s8 == 0) const_cast<uint16_t*>(is_k ? a.pages.kv.k_absmax : a.pages.kv.v_absmax)[at] = (uint16_t)m;
        } else {
            reinterpret_cast<uint4*>(tokens)[at * 16 + 2 * s8] = raw[0];
            reinterpret_cast<uint4*>(tokens)[at * 16 + 2 * s8 + 1] = raw[1];
        }
    }
}

template __global__ void write_paged_kernel<false, false>(WritePagedArgs);
template __global__ void write_paged_kernel<false, true>(WritePagedArgs);
template __global__ void write_paged_kernel<true, false>(WritePagedArgs);
template __global__ void write_paged_kernel<true, true>(WritePagedArgs);

}  // namespace ffd
