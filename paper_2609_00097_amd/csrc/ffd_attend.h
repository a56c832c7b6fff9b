// Attention of many query rows over one cache for gfx950: decode over an 8-bit cache (own_decode_kernel) and the
// attention of a whole batch over its shared prefix (prefix_kernel, bf16 or 8-bit).
//
// Mathematics. z_t = scale q . k_t, out = sum_t e^(z_t - m) v_t / sum_t e^(z_t - m) with the running maximum m of an
// online softmax (in powers of two: z2 = z log2 e), fp32 throughout but for the operands of the matrix instructions.
// 8-bit keys and values are n M / 127: the integers n are bf16 values, M / 127 of a key multiplies its score and that
// of a value its probability, so nothing is rounded by the conversion.
//
// Mapping. A wave takes 32 tokens at a time and 16 CT query rows. Scores are computed transposed, S^T = K Q^T, by
// v_mfma_f32_16x16x32_bf16: lane (n, g) = (lane & 15, lane >> 4) holds, of query row n, tokens 4g .. 4g + 3 of both
// 16-token halves. These eight are the contraction indices 8g .. 8g + 7 that the lane has to hold of P^T in
// O^T = V^T P^T, so the probabilities stay in their registers, and the running maximum and the rescaling of O^T are
// per lane too: no LDS and no barrier in the loop. The other operand takes, for its dim, the same eight tokens: lane
// (n, g) loads dims 8n .. 8n + 7 of these eight rows (a row per 16 lanes, 256 or 128 contiguous bytes) and sorts them
// by dim in registers; it serves all CT tiles. The next tile's keys are requested once this one's scores are done,
// its values once this one's are sorted.
//
// The waves of a workgroup take the 32-token tiles of its run in turn and are joined in LDS at its end: one partial
// state per query row and workgroup.
//
// Bound: HBM (260 bytes a token and KV head in 8 bits, 512 in bf16), for short caches the chain of lengths, queries, first
// tile and join, 5 us. Measured, by the card: 4 x 128K tokens in 8 bits, 32 and 8 heads, 186 to 196 us (5.85 to 5.55 TB/s); 16
// sequences of 1 to 64K, eight heads per KV head, 217 to 225 (5.5); 32 sequences of 500 to 8K 68 (4.7); 1 x 32K 16 (4.2).
// Staging the tokens in LDS for all waves of a workgroup, as for many rows, has nothing to share here: a token is used by
// one wave.
#pragma once

#include <cfloat>

#include "ffd_balance.h"
#include "ffd_device.h"
#include "ffd_kernels.h"

namespace ffd {

constexpr int kTile = 32;                      // tokens a wave takes at a time
constexpr int kRound = kTile * kWaves;         // and a workgroup
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// max and sum over the four lanes n, n + 16, n + 32, n + 48
__device__ __forceinline__ float groups_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The high halves of two floats: bf16 where the floats are bf16 values (small integers here).
__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
template <int BYTE>
__device__ __forceinline__ float byte_value(uint32_t w) { return (float)(int8_t)(w >> (8 * BYTE)); }

// Eight codes as eight bf16 values.
__device__ __forceinline__ v8bf expand8(uint32_t a, uint32_t b) {
    uint4 r;
    r.x = high_halves(byte_value<0>(a), byte_value<1>(a));
    r.y = high_halves(byte_value<2>(a), byte_value<3>(a));
    r.z = high_halves(byte_value<0>(b), byte_value<1>(b));
    r.w = high_halves(byte_value<2>(b), byte_value<3>(b));
    return __builtin_bit_cast(v8bf, r);
}

// A tile's keys: the operand of half t and step s holds, in lane (n, g), token 16 t + n's dims at key_dim(s, g).
template <bool I8> __device__ __forceinline__ constexpr int key_dim(int s, int g) { return I8 ? 32 * g + 8 * s : 32 * s + 8 * g; }
template <bool I8> struct KeyTile;
template <> struct KeyTile<false> {
    uint4 k[2][4];
    __device__ __forceinline__ void load(const KvSource& kv, size_t tok0, int last, int n, int g) {
        const uint8_t* base = kv.k + tok0 * (2 * kD);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t off = (uint32_t)min(16 * t + n, last) * (2 * kD) + 16 * g;
#pragma unroll
            for (int s = 0; s < 4; ++s) k[t][s] = *reinterpret_cast<const uint4*>(base + off + 64 * s);
        }
    }
    // Half t's rows from row[t] on.
    __device__ __forceinline__ void load_halves(const KvSource& kv, const size_t (&row)[2], int n, int g) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint8_t* base = kv.k + row[t] * (2 * kD);
#pragma unroll
            for (int s = 0; s < 4; ++s) k[t][s] = *reinterpret_cast<const uint4*>(base + (uint32_t)(n * (2 * kD) + 16 * g + 64 * s));
        }
    }
    __device__ __forceinline__ v8bf operand(int t, int s) const { return __builtin_bit_cast(v8bf, k[t][s]); }
};
template <> struct KeyTile<true> {
    uint4 k[2][2];
    uint2 m[2];                                 // absmaxes of tokens 16 t + 4 g ..
    __device__ __forceinline__ void load(const KvSource& kv, size_t tok0, int last, int n, int g) {
        const uint8_t* base = kv.k + tok0 * kD;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t off = (uint32_t)(16 * t + n) * kD + 32 * g;
            k[t][0] = *reinterpret_cast<const uint4*>(base + off);
            k[t][1] = *reinterpret_cast<const uint4*>(base + off + 16);
            m[t] = *reinterpret_cast<const uint2*>(kv.k_absmax + tok0 + 16 * t + 4 * g);
        }
    }
    __device__ __forceinline__ void load_halves(const KvSource& kv, const size_t (&row)[2], int n, int g) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint8_t* base = kv.k + row[t] * kD;
            const uint32_t off = (uint32_t)(n * kD + 32 * g);
            k[t][0] = *reinterpret_cast<const uint4*>(base + off);
            k[t][1] = *reinterpret_cast<const uint4*>(base + off + 16);
            m[t] = *reinterpret_cast<const uint2*>(kv.k_absmax + row[t] + 4 * g);
        }
    }
    __device__ __forceinline__ v8bf operand(int t, int s) const {
        const uint4 w = k[t][s >> 1];
        return s & 1 ? expand8(w.z, w.w) : expand8(w.x, w.y);
    }
};

// absmax r of four
__device__ __forceinline__ float absmax_of(uint2 m, int r) {
    const uint32_t w = r < 2 ? m.x : m.y;
    return r & 1 ? bf16_hi(w) : bf16_lo(w);
}

// A tile's values: lane (n, g) loads dims 8n .. 8n + 7 of its eight tokens; operand i is dim 8n + i of them.
__device__ __forceinline__ int value_token(int e, int g) { return (e < 4 ? 0 : 12) + 4 * g + e; }
template <bool I8> struct ValueTile;
template <> struct ValueTile<false> {
    uint4 v[8];
    __device__ __forceinline__ void load(const KvSource& kv, size_t tok0, int last, int n, int g) {
        const uint8_t* base = kv.v + tok0 * (2 * kD);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = *reinterpret_cast<const uint4*>(base + (uint32_t)min(value_token(e, g), last) * (2 * kD) + 16 * n);
    }
    __device__ __forceinline__ void load_halves(const KvSource& kv, const size_t (&row)[2], int n, int g) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = *reinterpret_cast<const uint4*>(kv.v + row[e >> 2] * (2 * kD) + (uint32_t)((4 * g + (e & 3)) * (2 * kD) + 16 * n));
    }
    __device__ __forceinline__ void operands(v8bf (&f)[8]) const {
        uint32_t w[8][4];                       // [dim][token pair]
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t a[4] = {v[2 * p].x, v[2 * p].y, v[2 * p].z, v[2 * p].w};
            const uint32_t b[4] = {v[2 * p + 1].x, v[2 * p + 1].y, v[2 * p + 1].z, v[2 * p + 1].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[2 * j][p] = __builtin_amdgcn_perm(b[j], a[j], 0x05040100u);
                w[2 * j + 1][p] = __builtin_amdgcn_perm(b[j], a[j], 0x07060302u);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __builtin_bit_cast(v8bf, make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]));
    }
    __device__ __forceinline__ bool all_finite() const {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m = pk_max_u16(m, pk_max_u16(v[e].x & 0x7fff7fffu, v[e].y & 0x7fff7fffu));
            m = pk_max_u16(m, pk_max_u16(v[e].z & 0x7fff7fffu, v[e].w & 0x7fff7fffu));
        }
        return max(m & 0xffffu, m >> 16) < 0x7f80u;
    }
    // Rows at and behind `end` of the tile to zero.
    __device__ __forceinline__ void clear_from(int end, int g) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (value_token(e, g) >= end) v[e] = make_uint4(0u, 0u, 0u, 0u);
    }
    // Rows that are not `alive` (bit e: row e of this lane) to zero.
    __device__ __forceinline__ void keep(uint32_t alive) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!(alive >> e & 1)) v[e] = make_uint4(0u, 0u, 0u, 0u);
    }
    // Infinities and NaN to zero.
    __device__ __forceinline__ void make_finite() {
        auto fix = [](uint32_t w) {
            w = (w & 0x7f80u) == 0x7f80u ? w & 0xffff0000u : w;
            return (w & 0x7f800000u) == 0x7f800000u ? w & 0xffffu : w;
        };
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = make_uint4(fix(v[e].x), fix(v[e].y), fix(v[e].z), fix(v[e].w));
    }
};
template <> struct ValueTile<true> {
    uint2 v[8];
    uint2 m[2];
    __device__ __forceinline__ void load(const KvSource& kv, size_t tok0, int last, int n, int g) {
        const uint8_t* base = kv.v + tok0 * kD;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = *reinterpret_cast<const uint2*>(base + (uint32_t)value_token(e, g) * kD + 8 * n);
#pragma unroll
        for (int t = 0; t < 2; ++t) m[t] = *reinterpret_cast<const uint2*>(kv.v_absmax + tok0 + 16 * t + 4 * g);
    }
    __device__ __forceinline__ void load_halves(const KvSource& kv, const size_t (&row)[2], int n, int g) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = *reinterpret_cast<const uint2*>(kv.v + row[e >> 2] * kD + (uint32_t)((4 * g + (e & 3)) * kD + 8 * n));
#pragma unroll
        for (int t = 0; t < 2; ++t) m[t] = *reinterpret_cast<const uint2*>(kv.v_absmax + row[t] + 4 * g);
    }
    template <int BYTE>
    __device__ __forceinline__ v8bf column(bool second) const {
        uint32_t w[4];
#pragma unroll
        for (int p = 0; p < 4; ++p)
            w[p] = high_halves(byte_value<BYTE>(second ? v[2 * p].y : v[2 * p].x),
                               byte_value<BYTE>(second ? v[2 * p + 1].y : v[2 * p + 1].x));
        return __builtin_bit_cast(v8bf, make_uint4(w[0], w[1], w[2], w[3]));
    }
    __device__ __forceinline__ void operands(v8bf (&f)[8]) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f[4 * h] = column<0>(h);
            f[4 * h + 1] = column<1>(h);
            f[4 * h + 2] = column<2>(h);
            f[4 * h + 3] = column<3>(h);
        }
    }
};

// State of 16 CT query rows: lane (n, g) holds of row n of tile c the maximum (of z2), its own tokens' share of the
// sum, and o[c][i][r] = dim 32 g + 8 r + i of the unnormalised output.
template <int CT>
struct RowState {
    float m[CT], l[CT];
    v4f o[CT][8];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            m[c] = -INFINITY;
            l[c] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[c][i] = v4f{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ bool all_finite() const {
        float x = 0.f;                          // stays zero where every o is finite
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) x = fmaf(o[c][i][r], 0.f, x);
        return x == 0.f;
    }
};

// What the instruction cannot do in a tile that some rows see only in part, or with a probability's low part: infinities
// and NaN among the values of a token reach the rows that see it and no other (zero times infinity would reach all).
// The values have been made finite; here they are added to the rows that see them, token by token.
template <int CT>
__device__ __forceinline__ void add_nonfinite(RowState<CT>& st, const uint16_t* v, int t0, int rows, const int (&lim)[CT], int g) {
#pragma unroll 1
    for (int t = t0; t < min(t0 + kTile, rows); ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = bf16_to_f32(v[(size_t)t * kD + 32 * g + 8 * r + i]);
                if (!(fabsf(x) < INFINITY)) {
#pragma unroll
                    for (int c = 0; c < CT; ++c)
                        if (t < lim[c]) st.o[c][i][r] += x;
                }
            }
    }
}

// Attends over tokens [begin, end) of kv: this wave's tiles of every round. `rows` (end of the tokens that any
// lane's row sees) clamps the rows read: those behind it may hold anything. Row n of tile c sees tokens below lim[c];
// tiles that end at or before `full` are seen whole by every row. zscale turns a product into z2.
//
// Probabilities are given to the instruction as p = hi + lo, both bf16, so that they are rounded to 2^-16 and not to
// 2^-8: kSpareRows: rows n and n + 8 are the same query, one with hi and the other with lo, and all see `rows` tokens;
// kTwoParts: two instructions. A lo may be zero or negative, so that an infinite value becomes NaN with it: kTwoPartsFinite
// takes infinities and NaN out of every tile, not only of those that are masked, for the caller to repeat a run with
// where kTwoParts left anything that is not finite (to look for them in each tile would cost all other runs).
enum Parts { kSpareRows, kTwoParts, kTwoPartsFinite };
template <int CT, bool I8, Parts PARTS>
__device__ __forceinline__ void attend(RowState<CT>& st, const v8bf (&q)[CT][4], const KvSource& kv, int begin, int end,
                                       int rows, const int (&lim)[CT], int full, float zscale, int wave, int n, int g) {
    int t0 = begin + kTile * wave;
    if (t0 >= end) return;
    KeyTile<I8> kt;
    ValueTile<I8> vt;
    // The queries are waited for here (vmcnt(0)): first used inside the loop, they would be waited for there, together
    // with the loads that the loop has just issued.
    __builtin_amdgcn_s_waitcnt(0x0f70);
    kt.load(kv, t0, rows - 1 - t0, n, g);
    vt.load(kv, t0, rows - 1 - t0, n, g);
    while (true) {
        const int next = t0 + kRound < end ? t0 + kRound : t0;
        v4f s[CT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int c = 0; c < CT; ++c) s[c][t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const v8bf a = kt.operand(t, k);
#pragma unroll
                for (int c = 0; c < CT; ++c) s[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[c][k], s[c][t], 0, 0, 0);
            }
        }
        float zs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (I8) zs[e] = absmax_of(kt.m[e >> 2], e & 3) * zscale;
            else zs[e] = zscale;
        }
        kt.load(kv, next, rows - 1 - next, n, g);

        v8bf p[CT], lo[CT];
        float vs[8];
        if constexpr (I8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) vs[e] = absmax_of(vt.m[e >> 2], e & 3) * (1.f / 127.f);
        }
        const bool masked = t0 + kTile > full;          // uniform
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = s[c][e >> 2][e & 3] * zs[e];
            bool any = true;
            if (masked) {
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = t0 + value_token(e, g) < lim[c] ? z[e] : -INFINITY;
                any = t0 < lim[c];
            }
            float mn = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
            mn = fmaxf(st.m[c], groups_max(mn));
            if (any) mn = fmaxf(mn, -FLT_MAX);          // finite once a token is seen, also where all scores are NaN
            if (__ballot(mn != st.m[c]) != 0) {         // uniform
                const float corr = mn == st.m[c] ? 1.f : exp2_hw(st.m[c] - mn);
                st.m[c] = mn;
                st.l[c] *= corr;
#pragma unroll
                for (int i = 0; i < 8; ++i) st.o[c][i] *= corr;
            }
            const float m0 = mn == -INFINITY ? 0.f : mn;
            float x[8], sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = exp2_hw(z[e] - m0);
                sum += x[e];
                if constexpr (I8) x[e] = masked && !(t0 + value_token(e, g) < lim[c]) ? 0.f : x[e] * vs[e];
            }
            st.l[c] += sum;
            uint32_t w[4], low[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
                low[e] = pack_bf16(x[2 * e] - bf16_lo(w[e]), x[2 * e + 1] - bf16_hi(w[e]));
                if constexpr (PARTS == kSpareRows) w[e] = n < 8 ? w[e] : low[e];
            }
            p[c] = __builtin_bit_cast(v8bf, make_uint4(w[0], w[1], w[2], w[3]));
            if constexpr (PARTS != kSpareRows) lo[c] = __builtin_bit_cast(v8bf, make_uint4(low[0], low[1], low[2], low[3]));
        }
        if constexpr (PARTS == kSpareRows && !I8) {
            if (masked) vt.clear_from(rows - t0, g);        // behind the last token: zero times infinity
        } else if constexpr (!I8) {
            if ((masked || PARTS == kTwoPartsFinite) && __ballot(!vt.all_finite()) != 0) {
                vt.make_finite();
                add_nonfinite<CT>(st, reinterpret_cast<const uint16_t*>(kv.v), t0, rows, lim, g);
            }
        }
        v8bf f[8];
        vt.operands(f);
        vt.load(kv, next, rows - 1 - next, n, g);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < CT; ++c) st.o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], p[c], st.o[c][i], 0, 0, 0);
        if constexpr (PARTS != kSpareRows) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int c = 0; c < CT; ++c) st.o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], lo[c], st.o[c][i], 0, 0, 0);
        }
        t0 += kRound;
        if (t0 >= end) break;
    }
}

// Joins the waves' states in LDS: afterwards acc[0] + acc[1] is the workgroup's output of a row, m and l per wave
// still apart.
constexpr int kAccPad = kD + 4;                // rows on 16 bytes, four banks apart
template <int CT>
struct JoinLds {
    float m[kWaves][16 * CT];
    float l[kWaves][16 * CT];
    alignas(16) float acc[2][16 * CT][kAccPad];
};

template <int CT>
__device__ __forceinline__ void join_waves(JoinLds<CT>& lds, RowState<CT>& st, int wave, int n, int g) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const float l = groups_sum(st.l[c]);
        if (g == 0) {
            lds.m[wave][16 * c + n] = st.m[c];
            lds.l[wave][16 * c + n] = l;
        }
    }
    __syncthreads();
    float f[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        float M = lds.m[0][16 * c + n];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) M = fmaxf(M, lds.m[w][16 * c + n]);
        f[c] = st.m[c] == -INFINITY ? 0.f : exp2_hw(st.m[c] - M);
    }
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {      // waves 2 and 3 leave theirs, 0 and 1 add to it
        if ((wave < 2) == (turn == 1)) {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float4* at = reinterpret_cast<float4*>(&lds.acc[wave & 1][16 * c + n][32 * g + 8 * r]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float4 x = make_float4(st.o[c][4 * h][r] * f[c], st.o[c][4 * h + 1][r] * f[c],
                                               st.o[c][4 * h + 2][r] * f[c], st.o[c][4 * h + 3][r] * f[c]);
                        if (turn == 1) {
                            const float4 y = at[h];
                            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
                        }
                        at[h] = x;
                    }
                }
        }
        __syncthreads();
    }
}

// (m, l) of a joined row, m in natural units as the merges expect it
template <int CT>
__device__ __forceinline__ void joined_ml(const JoinLds<CT>& lds, int row, float& m, float& l) {
    float M = lds.m[0][row];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, lds.m[w][row]);
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float mw = lds.m[w][row];
        if (mw != -INFINITY) l = fmaf(exp2_hw(mw - M), lds.l[w][row], l);
    }
    m = M * 0.69314718055994531f;
}

// A query row as the second operand of S^T. (Rows that no query has repeat one; nothing reads their results.)
template <bool I8>
__device__ __forceinline__ void load_query(v8bf (&q)[4], const uint16_t* row, int g) {
#pragma unroll
    for (int s = 0; s < 4; ++s) q[s] = __builtin_bit_cast(v8bf, *reinterpret_cast<const uint4*>(row + key_dim<I8>(s, g)));
}

// Decode over an 8-bit (I8) or bf16 cache: workgroup wg takes a run of blocks of a (sequence, KV head), as in
// dense_decode_kernel. The group's G <= 8 queries are rows 0 .. G - 1 and, for the low halves of the probabilities,
// 8 .. 8 + G - 1. WHOLE: a workgroup takes all of its pair's tokens (no table, S = 1) and writes the result itself.
template <bool I8, bool WHOLE = false>
__device__ __forceinline__ void own_decode(const OwnArgs& a, JoinLds<1>& lds, int wg) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int g = lane >> 4, n = lane & 15;
    const bool balanced = !WHOLE && a.table != nullptr;
    int kvh, b, L, jb, je, s = 0;
    if (balanced) {
        if (!balanced_share(a, wg, lane, b, kvh, L, jb, je)) return;
        b = __builtin_amdgcn_readfirstlane(b);
        kvh = __builtin_amdgcn_readfirstlane(kvh);
        jb = __builtin_amdgcn_readfirstlane(jb);
        je = __builtin_amdgcn_readfirstlane(je);
    } else {
        s = wg % a.S;
        kvh = wg / a.S % a.Hkv;
        b = wg / a.S / a.Hkv;
        L = min(max(a.seq_lens[b], 0), a.Lcap);
        const int nblk = (L + kBlock - 1) / kBlock, bps = (nblk + a.S - 1) / a.S;
        jb = min(s * bps, nblk);
        je = min(jb + bps, nblk);
    }
    const int G = a.G, hq0 = kvh * G;
    const size_t bh = (size_t)b * a.Hkv + kvh;
    const size_t row0 = bh * (size_t)a.Lcap, bytes = I8 ? kD : 2 * kD;
    const KvSource kv{a.kv.k + row0 * bytes, a.kv.v + row0 * bytes, I8 ? a.kv.k_absmax + row0 : nullptr,
                      I8 ? a.kv.v_absmax + row0 : nullptr};
    v8bf q[1][4];
    load_query<I8>(q[0], a.q + ((size_t)b * a.Hq + hq0 + min(n & 7, G - 1)) * kD, g);
    RowState<1> st;
    st.clear();
    const int lim[1] = {L};
    attend<1, I8, kSpareRows>(st, q, kv, kBlock * jb, min(kBlock * je, L), L, lim, L, a.scale * kLog2e / (I8 ? 127.f : 1.f), wave, n, g);
    join_waves(lds, st, wave, n, g);
    const size_t out0 = balanced ? (size_t)wg * G : ((size_t)b * a.Hq + hq0) * a.S + s;
    const size_t stride = balanced ? 1 : a.S;
    for (int i = tid; i < G * kD; i += kThreads) {
        const int h = i >> 7, d = i & (kD - 1);
        const size_t row = out0 + h * stride;
        const float hi = lds.acc[0][h][d] + lds.acc[1][h][d], lo = lds.acc[0][h + 8][d] + lds.acc[1][h + 8][d];
        const float o = fabsf(hi) < INFINITY ? hi + lo : hi;                // a low half may be zero: not times infinity
        if constexpr (WHOLE) {
            float m, l;
            joined_ml(lds, h, m, l);
            const bool any = m != -INFINITY;
            a.out[row * kD + d] = f32_to_bf16(any ? o / l : 0.f);
            if (d == 0 && a.lse) a.lse[row] = any ? m + logf(l) : -INFINITY;
        } else {
            a.part_acc[row * kD + d] = o;
            if (d == 0) {
                float m, l;
                joined_ml(lds, h, m, l);
                a.part_m[row] = m;
                a.part_l[row] = l;
            }
        }
    }
}

}  // namespace ffd
