// The attention weights that cached tokens get from the new ones: w_j = sum over the queries i of a KV head's group that see
// token j of e^(z_ij - lse_i), z and lse as of the attention (ffd_paged.h has the scores and what is seen). A sum has one
// order and one place, so that results do not change from call to call.
//
// Mapping. Work in the order (sequence, KV head, token), in units of 128 tokens, is given out in equal shares of consecutive
// units (MANY: a unit each). For a (sequence, KV head) of its share a workgroup takes 128 tokens at a time, 32 a wave, and puts
// the query rows that count into LDS, 128 of them at a time. With the keys of its 32 tokens in registers a wave goes through the
// rows, 16 by 16, with S^T = K Q^T as in ffd_attend.h: lane (n, g) adds up its eight tokens' weights from row n, and the 16 lanes of
// a group are joined at the end. Where 128 rows are all, they stay, the waves need no barrier, and the next keys are asked for
// early. MANY: two places for rows, one filled from memory by loads straight to LDS while the other is used (8K new tokens of one
// prompt 1712 -> 763 us, 5 x 1K on 8K 847 -> 498).
//
// Bound: HBM where few queries count (256 bytes a token and KV head: one token of 16 sequences on 8K 49 us, 5.5 TB/s). 8K new tokens of
// one prompt: the units of its first tokens, which all rows see, while those of its last ones are long done: all 512 begin at once,
// two a CU, and the CUs are busy for 58 % of the time; in that time the matrix cores for 28 %, vector instructions for 53, LDS for 16
// (0.36 PFLOP/s of products).
#include <type_traits>

#include "ffd_paged.h"
#include "ffd_tile.h"

namespace ffd {

namespace {

constexpr int kRowsAtOnce = 128;
template <int N>
struct WeightsLds {
    alignas(16) uint8_t q[N][kRowsAtOnce * 2 * kD];
    float lse2[N][kRowsAtOnce];
};

// Units [first, last) of a (sequence, KV head).
struct WeightsItem {
    ChunkSeq seq;
    int b, kvh, first, last;
};

// A wave's 32 tokens: their pages' rows, which of this lane's eight tokens there are, and what the four that it writes had.
struct WeightsTile {
    int t0;
    uint32_t alive;
    size_t row[2];
    float4 old;
};

// 16 bytes a lane from memory straight to LDS, where a wave's 64 pieces lie one after the other from lds_at on (the same in all
// lanes). The compiler does not count this load.
__device__ __forceinline__ void rows_to_lds(uint32_t lds_at, const uint8_t* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds_at), "v"(from) : "memory", "m0");
}

}  // namespace

template <bool I8, bool RULED, bool MANY>
__global__ __launch_bounds__(kThreads, MANY ? 2 : 3) void chunk_weights_kernel(ChunkWeightsArgs a) {
    __shared__ WeightsLds<MANY ? 2 : 1> lds;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int g = lane >> 4, n = lane & 15, gs = __builtin_ctz(a.G);
    const int unit = kRound << a.unit_shift;
    auto load = [&](int b0, ChunkSeq& s) {      // units of this lane's sequence
        s = chunk_seq(a, min(b0 + lane, a.B - 1));
        return b0 + lane < a.B ? (min(s.L, a.Lcap) + unit - 1) / unit * a.Hkv : 0;
    };
    int all = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        ChunkSeq s;
        all += __builtin_amdgcn_readlane(wave_inclusive_scan(load(b0, s)), 63);
    }
    const Shares shares(all, a.slots);
    const int begin = shares.begin(blockIdx.x), stop = shares.begin(blockIdx.x + 1);
    for (int u = begin; u < stop;) {            // uniform
        if (u != begin) __syncthreads();            // the rows in LDS are done with
        WeightsItem it{};
        for (int b0 = 0, before = 0; b0 < a.B; b0 += 64) {
            ChunkSeq s;
            const int mine = load(b0, s), incl = wave_inclusive_scan(mine), at = before + incl - mine;
            const uint64_t hit = __ballot(u >= at && u < at + mine);
            if (hit != 0) {
                const int src = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hit));
                it.b = b0 + src;
                it.seq.q0 = __builtin_amdgcn_readlane(s.q0, src);
                it.seq.n = __builtin_amdgcn_readlane(s.n, src);
                it.seq.L = __builtin_amdgcn_readlane(s.L, src);
                it.seq.pre = __builtin_amdgcn_readlane(s.pre, src);
                const int count = __builtin_amdgcn_readlane(mine, src) / a.Hkv, in = __builtin_amdgcn_readfirstlane(u) - __builtin_amdgcn_readlane(at, src);
                it.kvh = in / count;
                it.first = in - it.kvh * count;
                it.last = min(count, it.first + stop - u);
                break;
            }
            before += __builtin_amdgcn_readlane(incl, 63);
        }
        u += it.last - it.first;
        const ScoreRule rule = score_rule(a, I8, it.kvh * a.G + (n & (a.G - 1)));
        const int cached = min(it.seq.L, a.Lcap), place = it.seq.L - it.seq.n, pre = it.seq.pre;
        const int first = it.first * unit, end = min(it.last * unit, cached), hq0 = it.kvh * a.G;
        struct Entries {
            int e[2];
        };
        auto entries_at = [&](int t0) {
            return Entries{{uniform_page_entry(a.pages, it.b, t0), uniform_page_entry(a.pages, it.b, t0 + 16)}};
        };
        auto tile_of = [&](int t0, const Entries& entries) {
            WeightsTile x;
            x.t0 = t0;
            x.alive = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bool there = page_there(a.pages, entries.e[t]);
                x.row[t] = page_row(a.pages, a.Hkv, it.kvh, there ? entries.e[t] : 0, t0 + 16 * t);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x.alive |= (uint32_t)(there & (t0 + value_token(4 * t + i, g) < cached)) << (4 * t + i);
            }
            return x;
        };
        // new tokens [from, to) count and may see something of tokens [t0, t1)
        auto rows_for = [&](int t0, int t1, int& from, int& to) {
            from = a.last > 0 ? max(it.seq.n - a.last, 0) : 0;
            to = it.seq.n;
            if (t0 >= pre) {
                from = max(from, t0 - place);
                if (a.window > 0) to = (int)min((long long)to, (long long)t1 - 1 + a.window - place);
            }
        };
        // What lanes n < 2 will add to: asked for with the keys, since a load waits for all loads before it.
        auto load_old = [&](WeightsTile& x) {
            x.old = make_float4(0.f, 0.f, 0.f, 0.f);
            const int j = x.t0 + 16 * n + 4 * g;
            if (a.previous && n < 2 && j < cached) x.old = *reinterpret_cast<const float4*>(a.previous + ((size_t)it.b * a.Hkv + it.kvh) * a.Lcap + j);
        };
        int from, to;
        rows_for(first, end, from, to);
        const int r0 = from << gs, rows = from < to ? (to - from) << gs : 0;
        // rows r0 + at .. into LDS; those behind the last one repeat it
        auto stage = [&](int at) {
#pragma unroll
            for (int i = 0; i < kRowsAtOnce * 16 / kThreads; ++i) {
                const int row = (tid >> 4) + 16 * i;
                if (at + row >= rows + 15) break;
                const int r = r0 + min(at + row, rows - 1);
                const size_t from_row = (size_t)(it.seq.q0 + (r >> gs)) * a.Hq + hq0 + (r & (a.G - 1));
                *reinterpret_cast<v4u*>(&lds.q[0][row * (2 * kD) + 16 * key_chunk(row, tid & 15)]) =
                    *reinterpret_cast<const v4u*>(a.q + from_row * kD + 8 * (tid & 15));
                if ((tid & 15) == 0) lds.lse2[0][row] = a.lse[from_row] * kLog2e;
            }
        };
        // The same without a register between, asked for here and there after a wait and a barrier: a wave brings 32 rows, four a
        // load, each piece from the chunk that belongs to its place. This thread's row's lse comes with them.
        auto bring = [&](int at, int buffer) {
#pragma unroll
            for (int i = 0; i < kRowsAtOnce / kWaves / 4; ++i) {
                const int row = (kRowsAtOnce / kWaves) * wave + 4 * i, mine = row + (lane >> 4), r = r0 + min(at + mine, rows - 1);
                const size_t from_row = (size_t)(it.seq.q0 + (r >> gs)) * a.Hq + hq0 + (r & (a.G - 1));
                rows_to_lds((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&lds.q[buffer][row * (2 * kD)],
                            reinterpret_cast<const uint8_t*>(a.q + from_row * kD + 8 * key_chunk(mine, lane & 15)));
            }
            const int r = r0 + min(at + (tid & (kRowsAtOnce - 1)), rows - 1);
            return a.lse[(size_t)(it.seq.q0 + (r >> gs)) * a.Hq + hq0 + (r & (a.G - 1))];
        };
        float sum[8];
        // the weights that rows [at, at + kRowsAtOnce) give this wave's tile
        auto add_rows = [&](const KeyTile<I8>& kt, const WeightsTile& tile, int at, int buffer) {
            v8bf keys[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) keys[t][k] = kt.operand(t, k);
            float km[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (I8) km[e] = absmax_of(kt.m[e >> 2], e & 3) * rule.zscale;
                else km[e] = rule.zscale;
            }
            const bool whole = __ballot(tile.alive != 0xffu) == 0;
            int lowest, highest;
            rows_for(tile.t0, tile.t0 + kTile, lowest, highest);
            lowest = max(((lowest - from) << gs) - at, 0) & ~15;
            highest = min(((highest - from) << gs) - at, kRowsAtOnce);
            auto tiles = [&](int r, auto count) {       // row tiles r, r + 16: two are each other's latency
                constexpr int N = decltype(count)::value;
                v4f s[N][2];
                float lse2[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    lse2[i] = lds.lse2[buffer][r + 16 * i + n];
                    s[i][0] = s[i][1] = v4f{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const v8bf q = *reinterpret_cast<const v8bf*>(&lds.q[buffer][(r + 16 * i + n) * (2 * kD) + 16 * key_chunk(n, key_dim<I8>(k, g) / 8)]);
#pragma unroll
                        for (int t = 0; t < 2; ++t) s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(keys[t][k], q, s[i][t], 0, 0, 0);
                    }
                const int tok = from + ((at + r) >> gs), low = place + tok, high = place + min(tok + ((16 * N - 1) >> gs), to - 1), t0 = tile.t0;
                const bool masked = !whole || at + r + 16 * N > rows ||
                                    !((t0 + kTile <= low + 1 && (a.window <= 0 || t0 > high - a.window)) || t0 + kTile <= pre);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int row = at + r + 16 * i + n, mine = place + from + (row >> gs);
                    float p[8];
                    if constexpr (RULED) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[e] = s[i][e >> 2][e & 3] * km[e];
                        if (rule.cap2 != 0.f) cap_all(p, rule);
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[e] = exp2_hw(fmaf(-rule.slope2, fabsf((float)(mine - t0 - value_token(e, g))), p[e]) - lse2[i]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[e] = exp2_hw(fmaf(s[i][e >> 2][e & 3], km[e], -lse2[i]));
                    }
                    if (masked) {
                        const uint32_t row_there = row < rows;
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            p[e] = row_there & (tile.alive >> e) & (uint32_t)sees(mine, t0 + value_token(e, g), a.window, pre) ? p[e] : 0.f;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += p[e];
                }
            };
            int r = lowest;
            for (; r + 16 < highest; r += 32) tiles(r, std::integral_constant<int, 2>());
            if (r < highest) tiles(r, std::integral_constant<int, 1>());
        };
        auto finish = [&](const WeightsTile& tile) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = row16_sum(sum[e]);
            const int j = tile.t0 + 16 * n + 4 * g;
            if (n >= 2 || j >= cached) return;      // half n of the tile
            const float old[4] = {tile.old.x, tile.old.y, tile.old.z, tile.old.w};
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (j + e < place ? old[e] : 0.f) + (n == 0 ? sum[e] : sum[e + 4]);
            float* to_weights = a.weights + ((size_t)it.b * a.Hkv + it.kvh) * a.Lcap + j;
            if (j + 4 <= cached) {
                *reinterpret_cast<float4*>(to_weights) = make_float4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (j + e < cached) to_weights[e] = w[e];
            }
        };

        KeyTile<I8> kt;
        if (rows <= kRowsAtOnce) {
            int t0 = first + kTile * wave;
            // behind the end: a tile that is there, unused
            auto within = [&](int t) { return min(t, end - 1) & ~(kTile - 1); };
            WeightsTile tile = tile_of(within(t0), entries_at(within(t0)));
            Entries entries = entries_at(within(t0 + kRound));
            kt.load_halves(a.pages.kv, tile.row, n, g);
            load_old(tile);
            if (rows > 0) stage(0);
            __syncthreads();
            while (t0 < end) {
                const int next = t0 + kRound;
                KeyTile<I8> kn;
                WeightsTile next_tile = tile_of(within(next), entries);
                entries = entries_at(within(next + kRound));
                kn.load_halves(a.pages.kv, next_tile.row, n, g);
                load_old(next_tile);
                asm volatile("" ::: "memory");      // here, not where they are used
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.f;
                if (rows > 0) add_rows(kt, tile, 0, 0);
                finish(tile);
                kt = kn;
                tile = next_tile;
                t0 = next;
            }
            continue;
        }
        for (int t0 = first + kTile * wave; t0 - kTile * wave < end; t0 += kRound) {            // all waves alike, for the barriers
            WeightsTile tile = tile_of(t0, entries_at(t0));
            if (t0 < end) kt.load_halves(a.pages.kv, tile.row, n, g);
            load_old(tile);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            if constexpr (MANY) {
                // rows that some of the 128 tokens may count for
                int lowest, highest;
                rows_for(t0 - kTile * wave, min(t0 - kTile * wave + kRound, end), lowest, highest);
                const int begin_row = max((lowest - from) << gs, 0) / kRowsAtOnce * kRowsAtOnce, end_row = min((highest - from) << gs, rows);
                float lse = 0.f;
                if (begin_row < end_row) lse = bring(begin_row, 0);
                for (int at = begin_row, buffer = 0; at < end_row; at += kRowsAtOnce, buffer ^= 1) {       // uniform
                    wait_for_loads();
                    if (tid < kRowsAtOnce) lds.lse2[buffer][tid] = lse * kLog2e;
                    __syncthreads();
                    if (at + kRowsAtOnce < end_row) lse = bring(at + kRowsAtOnce, buffer ^ 1);
                    if (t0 < end) add_rows(kt, tile, at, buffer);
                }
                __syncthreads();
            } else {
                for (int at = 0; at < rows; at += kRowsAtOnce) {
                    stage(at);
                    __syncthreads();
                    if (t0 < end) add_rows(kt, tile, at, 0);
                    __syncthreads();
                }
            }
            if (t0 < end) finish(tile);
        }
    }
}

template __global__ void chunk_weights_kernel<false, false, false>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<false, false, true>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<false, true, false>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<false, true, true>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<true, false, false>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<true, false, true>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<true, true, false>(ChunkWeightsArgs);
template __global__ void chunk_weights_kernel<true, true, true>(ChunkWeightsArgs);

}  // namespace ffd
