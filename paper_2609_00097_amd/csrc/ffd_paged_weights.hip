// The attention weights that cached tokens get from the new ones: w_j = sum over the queries i of a KV head's group that see
// token j of e^(z_ij - lse_i), z and lse as of the attention (ffd_paged.h has the scores and what is seen). A sum has one
// order and one place, so that results do not change from call to call.
//
// Mapping. A workgroup keeps the keys of 128 tokens of a (sequence, KV head) in registers, 32 a wave, and goes through the
// query rows that may see them, 16 at a time, with S^T = K Q^T as in ffd_attend.h: lane (n, g) adds up its eight tokens' weights
// from row n, and the 16 lanes of a group are joined at the end.
//
// Bound: HBM where few queries count (256 bytes a token and KV head), else the exponentials and the matrix cores.
#include "ffd_paged.h"

namespace ffd {

namespace {

struct WeightsItem {
    ChunkSeq seq;
    int b, kvh, block;
};
// Item number `wanted` of the batch: blocks of kRound tokens by (sequence, KV head).
__device__ __forceinline__ bool weights_item(const ChunkWeightsArgs& a, long long wanted, int lane, WeightsItem& it) {
    long long before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const ChunkSeq s = chunk_seq(a, min(b0 + lane, a.B - 1));
        const int blocks = b0 + lane < a.B ? (min(s.L, a.Lcap) + kRound - 1) / kRound : 0;
        const int incl = wave_inclusive_scan(blocks);
        const long long first = before + (long long)(incl - blocks) * a.Hkv;
        const uint64_t hit = __ballot(wanted >= first && wanted < first + (long long)blocks * a.Hkv);
        if (hit != 0) {
            const int src = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hit));
            it.b = b0 + src;
            it.seq.q0 = __builtin_amdgcn_readlane(s.q0, src);
            it.seq.n = __builtin_amdgcn_readlane(s.n, src);
            it.seq.L = __builtin_amdgcn_readlane(s.L, src);
            it.seq.pre = __builtin_amdgcn_readlane(s.pre, src);
            const int count = __builtin_amdgcn_readlane(blocks, src);
            const int at = (int)(wanted - before - (long long)__builtin_amdgcn_readlane(incl - blocks, src) * a.Hkv);
            it.kvh = __builtin_amdgcn_readfirstlane(at / count);
            it.block = __builtin_amdgcn_readfirstlane(at) - it.kvh * count;
            return true;
        }
        before += (long long)__builtin_amdgcn_readlane(incl, 63) * a.Hkv;
    }
    return false;
}

}  // namespace

template <bool I8, bool RULED>
__global__ __launch_bounds__(kThreads, 3) void chunk_weights_kernel(ChunkWeightsArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int g = lane >> 4, n = lane & 15, gs = __builtin_ctz(a.G);
    const ScoreRule rule = score_rule(a, I8, 0);
    WeightsItem it;
    for (long long wanted = blockIdx.x; weights_item(a, wanted, lane, it); wanted += gridDim.x) {
        const int cached = min(it.seq.L, a.Lcap), place = it.seq.L - it.seq.n, pre = it.seq.pre;
        const int t0 = it.block * kRound + kTile * wave;
        if (t0 >= cached) continue;
        const int entry[2] = {page_entry(a.pages, it.b, t0), page_entry(a.pages, it.b, t0 + 16)};
        size_t row[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) row[t] = page_row(a.pages, a.Hkv, it.kvh, page_there(a.pages, entry[t]) ? entry[t] : 0, t0 + 16 * t);
        KeyTile<I8> kt;
        kt.load_halves(a.pages.kv, row, n, g);
        uint32_t alive = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (page_there(a.pages, entry[e >> 2]) && t0 + value_token(e, g) < cached) alive |= 1u << e;
        const bool whole = __ballot(alive != 0xffu) == 0;
        // new tokens [from, to) count and may see something of this tile
        int from = a.last > 0 ? max(it.seq.n - a.last, 0) : 0, to = it.seq.n;
        if (t0 >= pre) {
            from = max(from, t0 - place);
            if (a.window > 0) to = (int)min((long long)to, (long long)t0 + kTile - 1 + a.window - place);
        }
        const int r1 = to << gs, hq0 = it.kvh * a.G;
        v8bf q[4];
        float lse2, slope2;
        int at;
        auto load_row = [&](int r) {
            const int x = min(r + n, r1 - 1), tok = x >> gs, head = hq0 + (x & (a.G - 1));
            const size_t i = (size_t)(it.seq.q0 + tok) * a.Hq + head;
            load_query<I8>(q, a.q + i * kD, g);
            lse2 = a.lse[i] * kLog2e;
            at = place + tok;
            slope2 = RULED && a.slopes ? a.slopes[head] * kLog2e : 0.f;
        };
        float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (from < to) load_row(from << gs);
        for (int r = from << gs; r < r1; r += 16) {
            v4f s[2] = {v4f{0.f, 0.f, 0.f, 0.f}, v4f{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kt.operand(t, k), q[k], s[t], 0, 0, 0);
            const float lse_now = lse2, slope_now = slope2;
            const int at_now = at;
            if (r + 16 < r1) load_row(r + 16);
            const int low = place + (r >> gs), high = place + (min(r + 15, r1 - 1) >> gs);
            const bool masked = !whole || r + 16 > r1 ||
                                !((t0 + kTile <= low + 1 && (a.window <= 0 || t0 > high - a.window)) || t0 + kTile <= pre);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float z = s[e >> 2][e & 3] * rule.zscale;
                if constexpr (I8) z *= absmax_of(kt.m[e >> 2], e & 3);
                if constexpr (RULED) {
                    if (rule.cap2 != 0.f) z = capped(z, rule.cap2);
                    z = fmaf(-slope_now, fabsf((float)(at_now - t0 - value_token(e, g))), z);
                }
                float p = exp2_hw(z - lse_now);
                if (masked) p = r + n < r1 && (alive >> e & 1) && sees(at_now, t0 + value_token(e, g), a.window, pre) ? p : 0.f;
                sum[e] += p;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = row16_sum(sum[e]);
        if (n < 2) {                            // half n of the tile
            const int j = t0 + 16 * n + 4 * g;
            const size_t to0 = ((size_t)it.b * a.Hkv + it.kvh) * a.Lcap + j;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (j + e >= cached) continue;
                const float x = n == 0 ? sum[e] : sum[e + 4];
                a.weights[to0 + e] = a.previous && j + e < place ? a.previous[to0 + e] + x : x;
            }
        }
    }
}

template __global__ void chunk_weights_kernel<false, false>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<false, true>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<true, false>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<true, true>(ChunkWeightsArgs);

}  // namespace ffd
