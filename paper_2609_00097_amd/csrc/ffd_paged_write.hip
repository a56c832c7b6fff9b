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
// Bound: HBM (256 bytes read and written per vector): 7K tokens of 32 + 2 x 8 heads with norms and rotation 41 us, 4.0 TB/s. For few
// tokens the chain of starts, length, page and vector, 4.5 us; the vectors are asked for before it. 16 lanes a vector: with eight, and
// the vectors asked for behind the chain, the 7K tokens took 47 us where this took 45. A wave's loads are whole rows, and the other half of a pair is eight lanes away, which is a DPP rotation.
#include "ffd_kv8.h"
#include "ffd_paged.h"
#include "ffd_tile.h"

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

// A lane's eight dims of a vector.
struct Vec {
    float x[8];
};
__device__ __forceinline__ Vec floats(const uint4& r) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    Vec v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v.x[2 * i] = bf16_lo(w[i]);
        v.x[2 * i + 1] = bf16_hi(w[i]);
    }
    return v;
}

}  // namespace

// 16 lanes a vector; a wave's four vectors belong to one token. A token's Hq + 2 Hkv vectors are taken by a.parts (a multiple
// of four) such groups in turn, so that with many tokens a group reads its row of the table once for several heads.
template <bool I8, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void write_paged_kernel(WritePagedArgs a) {
    const int lane = threadIdx.x & 63, c = lane & 15;          // dims 8 c ..
    const int waves = a.parts >> 2;
    const long long wave = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int row = __builtin_amdgcn_readfirstlane((int)(wave / waves));
    const int part = (int)(wave - (long long)row * waves) * 4 + (lane >> 4);
    if (row >= a.T) return;
    // This group's heads: part, part + a.parts, .. of queries, keys and values in a row.
    const int Hq = a.q ? a.Hq : 0, turns = Hq > part ? (Hq - part + a.parts - 1) / a.parts : 0;
    const int k0 = part + turns * a.parts - Hq, k_turns = a.Hkv > k0 ? (a.Hkv - k0 + a.parts - 1) / a.parts : 0, v0 = k0 + k_turns * a.parts - a.Hkv;
    constexpr int U = 4, V = 2;                 // queries, keys and values asked for together
    const v4u* qp = reinterpret_cast<const v4u*>(a.q + row * a.qs[0] + part * a.qs[1]) + c;
    const v4u* kp = reinterpret_cast<const v4u*>(a.k + row * a.ks[0]) + c;
    const v4u* vp = reinterpret_cast<const v4u*>(a.v + row * a.vs[0]) + c;
    v4u q[U], k[V], v[V];
    // (unconditional, the last head again behind it)
    auto load_q = [&](int h) {
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = qp[(int64_t)(min(h + u * a.parts, Hq - 1) - part) * (a.qs[1] >> 3)];
    };
    auto load_kv = [&](v4u (&x)[V], const v4u* p, int h, int64_t stride) {
#pragma unroll
        for (int u = 0; u < V; ++u) x[u] = p[min(h + u * a.parts, a.Hkv - 1) * (stride >> 3)];
    };
    if (part < Hq) load_q(part);                // before the chain of sequence, length, position and page
    load_kv(k, kp, k0, a.ks[1]);
    load_kv(v, vp, v0, a.vs[1]);
    asm volatile("" ::: "memory");
    const int b = sequence_of(a.q_start, a.B, row, lane);
    if (b >= a.B) return;
    const int first = a.q_start[b], last = min(a.q_start[b + 1], a.T);
    const int len = a.seq_lens[b];
    if (row < first) return;
    const int place = min(max(len, 0), kMaxLen) - (last - row);
    const int position = a.positions ? a.positions[row] : place;

    // Dims 8 c .. are rotated if c < chunks; where pairs are half of the dims apart, with those of the lane `apart` further or
    // before. The first of a pair takes away what the second adds.
    float cs[8], sn[8];
    const int chunks = a.rope_dims >> 3, apart = chunks >> 1;
    if (a.rope) {
        const bool in = position >= 0 && position < a.rope_rows, begins = INTERLEAVED || c < apart;
        const float* table = a.rope + (size_t)(in ? position : 0) * a.rope_dims;
        const int at = c < chunks ? INTERLEAVED ? 4 * c : 8 * (begins ? c : c - apart) : 0;
#pragma unroll
        for (int i = 0; i < (INTERLEAVED ? 1 : 2); ++i) {
            const float4 x = *reinterpret_cast<const float4*>(table + at + 4 * i), y = *reinterpret_cast<const float4*>(table + 8 * apart + at + 4 * i);
            const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                cs[4 * i + e] = in ? xs[e] : NAN;
                sn[4 * i + e] = in ? begins ? -ys[e] : ys[e] : NAN;
            }
        }
    }
    const bool cached = place >= 0 && place < (a.pages.max_pages << a.pages.page_shift);
    const int entry = cached ? page_entry(a.pages, b, place) : -1;
    const bool there = page_there(a.pages, entry);
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    const uint4 qw = a.q_weight ? reinterpret_cast<const uint4*>(a.q_weight)[c] : none, kw = a.k_weight ? reinterpret_cast<const uint4*>(a.k_weight)[c] : none;

    auto turned = [&](const uint4& raw, bool norm, const uint4& weight) {       // the 16 lanes of a vector together
        Vec x = floats(raw);
        if (norm) {
            const Vec w = floats(weight);
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(x.x[i], x.x[i], sum);
            const float inv = 1.f / sqrtf(row16_sum(sum) * (1.f / kD) + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) x.x[i] = x.x[i] * inv * w.x[i];
        }
        if (a.rope) {
            if constexpr (INTERLEAVED) {
                if (c < chunks) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = x.x[2 * i], r = x.x[2 * i + 1];
                        x.x[2 * i] = p * cs[i] + r * sn[i];
                        x.x[2 * i + 1] = r * cs[i] - p * sn[i];
                    }
                }
            } else {
                Vec y;                          // the other one of each pair
                if (apart == 8) {               // uniform: all dims
#pragma unroll
                    for (int i = 0; i < 8; ++i) y.x[i] = dpp_f<kDppRor8>(x.x[i]);
                } else {
                    const int other = (lane & ~15) | (c < apart ? c + apart : c < chunks ? c - apart : c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y.x[i] = __shfl(x.x[i], other);
                }
                if (c < chunks) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x.x[i] = x.x[i] * cs[i] + y.x[i] * sn[i];
                }
            }
        }
        return make_uint4(pack_bf16(x.x[0], x.x[1]), pack_bf16(x.x[2], x.x[3]), pack_bf16(x.x[4], x.x[5]), pack_bf16(x.x[6], x.x[7]));
    };
    auto store_kv = [&](const uint8_t* tokens, const uint16_t* absmax, int head, const uint4& raw) {
        const size_t at = page_row(a.pages, a.Hkv, head, entry, place);
        if constexpr (I8) {
            uint32_t m;
            reinterpret_cast<uint2*>(const_cast<uint8_t*>(tokens))[at * 16 + c] = encode_eighth(raw, m);
            if (c == 0) const_cast<uint16_t*>(absmax)[at] = (uint16_t)m;
        } else {
            reinterpret_cast<uint4*>(const_cast<uint8_t*>(tokens))[at * 16 + c] = raw;
        }
    };
    uint4* out = reinterpret_cast<uint4*>(a.q_out + (size_t)row * a.Hq * kD) + c;
    for (int h = part; h < Hq; h += U * a.parts) {
        if (h != part) load_q(h);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (h + u * a.parts < Hq) out[(h + u * a.parts) * 16] = turned(__builtin_bit_cast(uint4, q[u]), a.q_weight != nullptr, qw);
    }
    if (!there) return;
    for (int h = k0; h < a.Hkv; h += V * a.parts) {
        if (h != k0) load_kv(k, kp, h, a.ks[1]);
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (h + u * a.parts < a.Hkv) store_kv(a.pages.kv.k, a.pages.kv.k_absmax, h + u * a.parts, turned(__builtin_bit_cast(uint4, k[u]), a.k_weight != nullptr, kw));
    }
    for (int h = v0; h < a.Hkv; h += V * a.parts) {
        if (h != v0) load_kv(v, vp, h, a.vs[1]);
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (h + u * a.parts < a.Hkv) store_kv(a.pages.kv.v, a.pages.kv.v_absmax, h + u * a.parts, __builtin_bit_cast(uint4, v[u]));
    }
}

template __global__ void write_paged_kernel<false, false>(WritePagedArgs);
template __global__ void write_paged_kernel<false, true>(WritePagedArgs);
template __global__ void write_paged_kernel<true, false>(WritePagedArgs);
template __global__ void write_paged_kernel<true, true>(WritePagedArgs);

}  // namespace ffd
