// Attention of chunks of new tokens over a paged bf16 cache for gfx950 (ffd_attend.h has the mathematics, ffd_paged.h which tokens a
// query sees and how the work is cut; ffd_paged_rows.hip takes the sequences with few query rows, ffd_paged_tile8.hip 8-bit
// caches): tiles of 256 query rows of a KV head, new tokens by query heads, in eight waves of 32 rows, and the cache's tokens from
// memory straight to LDS, 64 at a time.
//
// Mapping: S^T = K Q^T by v_mfma_f32_32x32x16_bf16; lane (n, h) = (lane & 31, lane >> 5) has row n and tokens 8 a + 4 h + i (a, i =
// 0 .. 3) of a sub-tile of 32, which are its contraction indices in O^T = V^T P^T, so probabilities stay where they are made.
// LDS holds rows of 256 bytes with their chunks in the orders of ffd_tile.h; V is read by transposing reads.
//
// A wave takes a step for each sub-tile t, in two halves, so that the matrix cores always have products that wait for nothing:
// first the scores of t + 1 beside the exponentials of t, then the products of t - 1 beside the largest score of t + 1. The
// maximum is settled between two steps; where it grows (by more than 2^8, or at first) the sum is scaled at once and o after the
// products that are still to come. Operands are read two products ahead; a step's first ones at the end of the step before. A
// workgroup meets once a tile, in the middle of its first step (`turn`), with two places for keys and three for values.
//
// Probabilities enter the second product rounded to bf16, in one part: a second part would cost half as much again of a product
// that the matrix cores bound (the few-row kernel, which memory bounds, has two). So that the roundings cancel where they are
// alike (equal scores, one token with most of the weight), a row is divided by the sum of the rounded probabilities; the exact
// sum is kept beside it for the lse.
//
// Pages: 16 tokens lie together, so a wave's load is one page's, whose entry is read a tile ahead. Values of pages that are not
// there, and behind what any query sees, become zeros in LDS, in the tiles that have such. An infinity or NaN among the values of
// tokens that some rows see and others do not turns results into NaN; a workgroup that finds a result not finite repeats
// its run with all of them taken out of the tiles, and adds them at the end to the rows that see them.
//
// Bound: the issue of instructions by two waves a SIMD (without any matrix instruction two thirds of the time are left, without
// the loads, or the barrier, all of it) beside the matrix cores, which 512 operations a query row and token keep busy for 47 to 49 % of it.
// Against two teams of waves with matrix and softmax phases in turn and tokens staged in registers, eight KV heads of four:
// 8K tokens 620 -> 585 us, 512 on 32K 309 -> 291, 3800 in a window of 1024 with a cap, twice, 252 -> 229; with the queries asked for
// beside the first tile's page and results out in whole rows 562 us (0.97 PFLOP/s) and 287.
// Not kept: the waves of a SIMD half a step apart (8K 599), operands three products ahead (589), four waves of 64 rows (763).
#include <type_traits>

#include "ffd_paged.h"
#include "ffd_tile.h"

namespace ffd {

namespace {

constexpr int kTThreads = kChunkTileThreads;
constexpr int kTokens = 64;                     // tokens of a tile
constexpr int kShift = kChunkTileShift;
constexpr int kTileBytes = kTokens * 2 * kD;
constexpr int kMarks = 1024;
static_assert(kTokens == 1 << kShift);

struct alignas(2 * kTileBytes) TileLds {
    uint8_t keys[2][kTileBytes];                // places that differ in one bit of the address
    uint8_t values[3][kTileBytes];
    uint32_t nonfinite[kMarks / 32];            // bits: runs of tiles that have an infinity or NaN among their values
};

// 16 bytes a lane from memory straight to LDS, where a wave's 64 pieces lie one after the other; `lds_at` and `base` are the
// same in all lanes. The compiler does not count this load: whoever needs it waits with wait_for_loads() and a barrier. (As a
// builtin it would be taken to be in the way of every read of LDS, and waited for there.)
__device__ __forceinline__ void load_to_lds(uint32_t lds_at, const uint8_t* base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds_at), "v"(offset), "s"(base) : "memory", "m0");
}

template <int N> using Int = std::integral_constant<int, N>;
enum : int { kNoCap, kNearOnly, kAnyCap };       // scores that are capped with the exponential: none, all of them small ones, any

}  // namespace

template <bool RULED>
__global__ __launch_bounds__(kTThreads, 2) void chunk_tile_kernel(ChunkAttendArgs a) {
    __shared__ TileLds lds;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int n = lane & 31, h = lane >> 5;
    ChunkItem it;
    if (!chunk_item<kChunkTileRows, kShift>(a, blockIdx.x, lane, it)) return;
    const int gs = __builtin_ctz(a.G), step = kChunkTileRows >> gs, tok0 = it.tile * step;
    const int tok1 = min(tok0 + step, it.seq.n) - 1, live_rows = (tok1 - tok0 + 1) << gs;
    const int hq0 = it.kvh * a.G, place = it.seq.L - it.seq.n, cached = min(it.seq.L, a.Lcap);
    write_record(a, it, tok0, live_rows);
    const ChunkSpan span = chunk_span<kShift>(a, it.seq, tok0, tok1);
    const int first = (int)((long long)span.count * it.run / it.cuts), last = (int)((long long)span.count * (it.run + 1) / it.cuts);

    // this lane's row; behind the last one it is that one again, whose results are not written
    const int r = 32 * wave + n, tok = tok0 + (min(r, live_rows - 1) >> gs), head = hq0 + (r & (a.G - 1));
    const bool live = r < live_rows;
    const size_t row_at = (size_t)(it.seq.q0 + tok) * a.Hq + head;
    const int at = place + tok;
    const ScoreRule rule = score_rule(a, false, head);
    // the wave's first and last place, and the tile from which on none of its rows sees a token
    const int low = place + tok0 + ((32 * wave) >> gs), high = place + min(tok0 + ((32 * wave + 31) >> gs), tok1);
    const int wave_end = 32 * wave < live_rows ? max(min(max(high + 1, it.seq.pre), cached), 0) : 0;
    const int high_block = (wave_end + kTokens - 1) >> kShift;
    const int mine_last = max(first, min(last, high_block <= span.prefix ? high_block : max(high_block - span.skip, span.prefix)));
    // 32 tokens from t0 on are seen whole by every row of the wave if they are there, t0 <= whole_to and t0 > whole_from or
    // t0 <= prefix_to
    const int whole_to = min(max(low + 1, it.seq.pre), cached) - 32, whole_from = a.window > 0 ? high - a.window : INT32_MIN, prefix_to = it.seq.pre - 32;

    auto token0 = [&](int u) { return span.block(min(u, last - 1)) << kShift; };
    uint32_t ring = 0;                          // four bits a tile, which 16-token groups are there, by its number mod 4
    // A wave brings eight rows of a tile, four a load. The entries of a tile's four groups lie in lanes 0 .. 3.
    const int my_row = 8 * wave + (lane >> 4);
    uint32_t key_from[2], value_from[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = my_row + 4 * j, in = (4 * j + (lane >> 4)) * (2 * kD);
        key_from[j] = in + 16 * key_chunk(r, lane & 15);
        value_from[j] = in + 16 * value_chunk<false>(r, lane & 15);
    }
    // (whether they are the table's is seen where they are used, so that the load is waited for there)
    auto load_entries = [&](int u) {
        const int page = (max(token0(u), 0) + 16 * (lane & 3)) >> a.pages.page_shift;            // (no tile: the first page's)
        return a.pages.table[(size_t)it.b * a.pages.max_pages + min(page, a.pages.max_pages - 1)];
    };
    const int first_entries = load_entries(first);
    v8bf q[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) q[k] = __builtin_bit_cast(v8bf, *reinterpret_cast<const v4u*>(a.q + row_at * kD + 16 * k + 8 * h));
    asm volatile("" ::: "memory");              // on their way while the first tile's page is awaited
    auto load_rows = [&](const uint8_t* tile, const uint8_t* pages, size_t row, const uint32_t (&from)[2]) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            load_to_lds((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)(tile + (8 * wave + 4 * j) * (2 * kD)), pages + row * (2 * kD), from[j]);
    };
    int entries = 0;                            // of the tile whose keys are asked for next
    size_t row = 0;                             // this wave's, of the tile whose keys were asked for last
    auto bring_keys = [&](int u) {
        const int shift = 4 * (u & 3), known = (token0(u) + 16 * (lane & 3)) >> a.pages.page_shift < a.pages.max_pages ? entries : -1;
        const int e = __builtin_amdgcn_readlane(known, wave >> 1);
        ring = (ring & ~(15u << shift)) | ((uint32_t)__ballot(page_there(a.pages, known)) & 15u) << shift;
        row = page_row(a.pages, a.Hkv, it.kvh, page_there(a.pages, e) ? e : 0, token0(u) + 8 * wave);
        entries = load_entries(u + 1);
        load_rows(lds.keys[u & 1], a.pages.kv.k, row, key_from);
    };
    // Rows that nobody sees to zero (zero times infinity); `careful`: infinities and NaN of the others too.
    int mark_shift = 0;                         // tiles of a mark
    while ((last - first) >> mark_shift >= kMarks) ++mark_shift;
    auto fix_rows = [&](int u, uint8_t* values, bool careful) {
        const int t0 = token0(u);
        const uint32_t there = ring >> (4 * (u & 3)) & 15u;
        if (!careful && there == 15u && t0 + kTokens <= span.end) return;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = my_row + 4 * j;
            v4u* p = reinterpret_cast<v4u*>(values + r * (2 * kD) + 16 * (lane & 15));
            v4u x = *p;
            if (!((there >> (wave >> 1)) & (uint32_t)(t0 + r < span.end) & 1u)) x = v4u{0, 0, 0, 0};
            const uint32_t big = pk_max_u16(pk_max_u16(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), pk_max_u16(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
            if (careful && max(big & 0xffffu, big >> 16) >= 0x7f80u) {
                atomicOr(&lds.nonfinite[(u - first) >> mark_shift >> 5], 1u << ((u - first) >> mark_shift & 31));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t lo = (x[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu, hi = (x[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u;
                    x[i] &= lo | hi;
                }
            }
            *p = x;
        }
    };

    v16f o[4], s[2];                            // 32 dims each; scores by sub-tile of 32 tokens mod 2
    v8bf p[2][2];                               // [sub-tile mod 2][16 tokens]
    float m, l, rounded;

    const int i16 = lane & 15;
    const int v_row = 4 * h + (i16 >> 2), v_c = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
    // Places of the operands in LDS, kept for the tiles at hand: of the keys that the next scores take, of the values that the
    // next products take. Operand j of a sub-tile: keys' dims 16 j .., or 32 dims 32 (j & 3) .. of values' tokens 16 (j >> 2) ..
    using Lds = __attribute__((address_space(3))) const uint8_t*;
    uint32_t key_at[8], value_at[4][2];
    auto keys_at = [&](int u) {
        const uint32_t keys = (uint32_t)(uintptr_t)(Lds)lds.keys[u & 1] + n * (2 * kD) + 16 * key_chunk(n, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) key_at[j] = keys ^ (j << 5);
    };
    auto key_operand = [&](int half, int j) { return *reinterpret_cast<__attribute__((address_space(3))) const v8bf*>((Lds)(uintptr_t)key_at[j] + half * 32 * 2 * kD); };
    auto value_operand = [&](int half, int j) {
        v4s v[2];
#pragma unroll
        for (int z = 0; z < 2; ++z)
            v[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(
                (uintptr_t)(value_at[j & 3][z] + (16 * (j >> 2) + 8 * z + 32 * half) * 2 * kD)));
        return __builtin_bit_cast(v8bf, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto values_at = [&](const uint8_t* values) {
        const uint32_t x = (uint32_t)(uintptr_t)(Lds)values + v_row * (2 * kD) + 16 * value_chunk<false>(v_row, v_c) + 8 * (i16 & 1);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int z = 0; z < 2; ++z) value_at[d][z] = x ^ (d << 6) ^ (z << 5);
    };
    auto add_product = [&](int j, const v8bf& operand, const v8bf (&prob)[2]) {
        o[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand, prob[j >> 2], o[j & 3], 0, 0, 0);
    };

    // Sub-tile t's products x on their way to scores: the largest of the row (in powers of two), whether any is seen; rules and
    // masks are applied where there are any, else x stays the product (`raw`), to be scaled, and capped, with the exponential.
    float top = -INFINITY;
    bool raw = true, near = false;              // near: all of the wave's products are of scores up to half of the cap
    auto rules_and_masks = [&](int t, v16f& x, bool whole) {
        asm volatile("");                       // a branch around all this, not selections after it
        const int t0 = token0(t >> 1) + 32 * (t & 1), rel = at - t0 - 4 * h;
        if constexpr (RULED) {
            x *= rule.zscale;
            if (rule.cap2 != 0.f) cap_scores(x, rule);
            if (a.slopes) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = fmaf(-rule.slope2, fabsf((float)rel - (float)(8 * (i >> 2) + (i & 3))), x[i]);
            }
        }
        bool any = true;
        if (!whole) {
            const uint32_t there = ring >> (4 * ((t >> 1) & 3) + 2 * (t & 1)) & 3u;
            const int end = cached - t0 - 4 * h;
            const int high = min(rel, end - 1), low = a.window > 0 ? rel - a.window : INT32_MIN, prefix = min(it.seq.pre - t0 - 4 * h, end);
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = 8 * (i >> 2) + (i & 3);
                const uint32_t seen = (uint32_t)(((k <= high) & (k > low)) | (k < prefix)) & (there >> (i >> 3));
                x[i] = seen & 1 ? x[i] : -INFINITY;
                some |= seen;
            }
            any = halves_max(some & 1 ? 1.f : 0.f) > 0.f;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, x[i]);
        top = any ? fmaxf(halves_max(mx) * (RULED ? 1.f : rule.zscale), -FLT_MAX) : -INFINITY;
        raw = false;
    };
    // The reference m up to the largest score of sub-tile t. The products of t - 1 are still to come with the old one: o follows
    // after them.
    float corr = 1.f;
    uint64_t grown = 0;                         // lanes whose reference has grown
    auto settle = [&]() {
        grown = __ballot(top > m + kSlack);
        if (grown == 0) return;
        const float mn = top > m + kSlack ? top : m;
        corr = mn == m ? 1.f : exp2_hw(m - mn);
        m = mn;
        l *= corr;
        rounded *= corr;
    };

    v8bf kf[3], vf[3];                          // operands on their way: two products ahead
    // First half of a step: the probabilities of a sub-tile, beside them the scores of the next one, which is half `half` of its tile.
    auto exponentials = [&](v16f& now, v16f& next, v8bf (&probs)[2], auto half, auto capping) {
        constexpr int H = decltype(half)::value;
        constexpr int CAP = decltype(capping)::value;
        const float scale = RULED && CAP == kNoCap && !raw ? 1.f : rule.zscale;
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < 16; ++i) next[i] = 0.f;
        // With each product the arguments of pair j + 2, the exponentials of pair j, sum and rounding of pair j - 1, so that none
        // waits for the one before it.
        float sum[2] = {0.f, 0.f}, x[3][2], e[2][2];
        auto arguments = [&](int j) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float z = now[2 * j + i];
                if constexpr (CAP == kNearOnly) x[j % 3][i] = fmaf(z * scale, near_cap(z * scale, rule), -ref);
                else if constexpr (CAP == kAnyCap) x[j % 3][i] = capped(z * scale, rule) - ref;
                else x[j % 3][i] = fmaf(z, scale, -ref);
            }
        };
        auto round_pair = [&](int j) {
            uint32_t w0 = pack_bf16(e[j & 1][0], e[j & 1][1]);
            asm volatile("" : "+v"(w0));
            sum[0] += e[j & 1][0];
            sum[1] += e[j & 1][1];
            rounded = pair_sum(w0, rounded);
            v4u w = __builtin_bit_cast(v4u, probs[j >> 2]);
            w[j & 3] = w0;
            probs[j >> 2] = __builtin_bit_cast(v8bf, w);
        };
        arguments(0);
        arguments(1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j < 6) kf[(j + 2) % 3] = key_operand(H, j + 2);
            else vf[j - 6] = value_operand(H, j - 6);           // of the sub-tile before this one: the other half of its tile
            next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j % 3], q[j], next, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) e[j & 1][i] = exp2_hw(x[j % 3][i]);
            if (j < 6) arguments(j + 2);
            if (j > 0) round_pair(j - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        round_pair(7);
        l += sum[0] + sum[1];
        asm volatile("" : "+v"(l), "+v"(rounded));        // here, not where they are needed
    };
    auto probabilities = [&](v16f& now, v16f& next, v8bf (&probs)[2], auto half) {
        if (RULED && raw && rule.cap2 != 0.f) {
            if (near) exponentials(now, next, probs, half, Int<kNearOnly>());
            else exponentials(now, next, probs, half, Int<kAnyCap>());
        } else {
            exponentials(now, next, probs, half, Int<kNoCap>());
        }
    };
    // Second half: the products of the sub-tile before, beside them the largest of the next one, t; then the first operands
    // of the step to come, from half `half` of its keys' tile.
    auto second = [&](int t, v16f& next, v8bf (&before)[2], auto half, auto products) {
        constexpr bool P = decltype(products)::value;
        constexpr int H = decltype(half)::value;
        const int t0 = token0(t >> 1) + 32 * (t & 1);
        const uint32_t there = ring >> (4 * ((t >> 1) & 3) + 2 * (t & 1)) & 3u;
        const bool whole = (there == 3u) & (t0 <= whole_to) & ((t0 > whole_from) | (t0 <= prefix_to)), plain = whole & !(RULED && a.slopes);
        float mx[4], abs_mx[4], up_to = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (P) {
                if (j < 6) vf[(j + 2) % 3] = value_operand(1 - H, j + 2);
                else kf[j - 6] = key_operand(H, j - 6);
                add_product(j, vf[j % 3], before);
            } else if (j >= 6) {
                kf[j - 6] = key_operand(H, j - 6);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (j == 2) mx[i] = fmaxf(next[4 * i], next[4 * i + 1]);
                if (j == 3) mx[i] = fmaxf(fmaxf(mx[i], next[4 * i + 2]), next[4 * i + 3]);
                if constexpr (RULED) {
                    if (j == 2) abs_mx[i] = fmaxf(fabsf(next[4 * i]), fabsf(next[4 * i + 1]));
                    if (j == 3) abs_mx[i] = fmaxf(fmaxf(abs_mx[i], fabsf(next[4 * i + 2])), fabsf(next[4 * i + 3]));
                }
            }
            if (j == 4) mx[0] = fmaxf(fmaxf(mx[0], mx[1]), mx[2]);
            if (j == 5) mx[0] = fmaxf(mx[0], mx[3]);
            if (j == 6) up_to = halves_max(mx[0]);
            if (j == 7) up_to *= rule.zscale;
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (RULED) {
            if (rule.cap2 != 0.f) {
                up_to = capped(up_to, rule);
                near = __ballot(fmaxf(fmaxf(abs_mx[0], abs_mx[1]), fmaxf(abs_mx[2], abs_mx[3])) * rule.zscale > kNearCap) == 0;
            }
        }
        top = fmaxf(up_to, -FLT_MAX);           // NaN: of no weight for the reference
        raw = true;
        if ((grown != 0) | !plain) {            // uniform
            asm volatile("");
            if (grown != 0) {
#pragma unroll
                for (int d = 0; d < 4; ++d) o[d] *= corr;
            }
            if (!plain) rules_and_masks(t, next, whole);
        }
    };
    // They reach the rows that see them at the end, when o is scaled no more.
    auto add_nonfinite = [&]() {
#pragma unroll 1
        for (int u = first; u < last; ++u) {
            const int mark = (u - first) >> mark_shift;
            if (!(__builtin_amdgcn_readfirstlane(lds.nonfinite[mark >> 5]) >> (mark & 31) & 1)) continue;
            const int t0 = token0(u);
#pragma unroll 1
            for (int t = t0; t < min(t0 + kTokens, span.end); ++t) {
                const int entry = page_entry(a.pages, it.b, t);
                if (!page_there(a.pages, entry)) continue;
                const uint16_t* row = reinterpret_cast<const uint16_t*>(a.pages.kv.v) + page_row(a.pages, a.Hkv, it.kvh, entry, t) * kD + 4 * h;
                const bool seen = sees(at, t, a.window, it.seq.pre);
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float x = bf16_to_f32(row[32 * d + 8 * (i >> 2) + (i & 3)]);
                        o[d][i] += !(fabsf(x) < INFINITY) & seen ? x : 0.f;
                    }
            }
        }
    };

    for (bool careful = false;; careful = true) {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
#pragma unroll
        for (int y = 0; y < 2; ++y) p[1][y] = __builtin_bit_cast(v8bf, v4u{0, 0, 0, 0});
        m = -INFINITY;
        l = rounded = 0.f;
        grown = 0;
        if (tid < kMarks / 32) lds.nonfinite[tid] = 0;
        if (first < last) {
            entries = first_entries;
            __syncthreads();                    // a careful run: the first one's reads are done
            uint8_t *before = lds.values[0], *now = lds.values[1], *after = lds.values[2];      // values of tiles u - 1, u, u + 1
            for (int i = tid; i < kTileBytes / 16; i += kTThreads) reinterpret_cast<v4u*>(before)[i] = v4u{0, 0, 0, 0};
            bring_keys(first);
            wait_for_loads();
            asm volatile("" : "+v"(entries));
            __syncthreads();
            load_rows(now, a.pages.kv.v, row, value_from);
            if (first + 1 < last) bring_keys(first + 1);
            // In the middle of the first step of tile u: its values and the next one's keys are there; those after them are asked for,
            // to the places of the values of u - 2 and the keys of u, which are done with.
            auto turn = [&](int u) {
                wait_for_loads();
                asm volatile("" : "+v"(entries));       // counted as there from here on, not after the next loads
                fix_rows(u, now, careful);
                __syncthreads();
                if (u + 1 < last) load_rows(after, a.pages.kv.v, row, value_from);
                if (u + 2 < last) bring_keys(u + 2);
            };
            auto rotate = [&]() {
                uint8_t* x = before;
                before = now, now = after, after = x;
            };
            constexpr Int<0> kFirst{};
            constexpr Int<1> kSecond{};
            int u = first;
            if (first < mine_last) {
                keys_at(first);
                values_at(before);
                kf[0] = key_operand(0, 0), kf[1] = key_operand(0, 1);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j < 6) kf[(j + 2) % 3] = key_operand(0, j + 2);
                    s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j % 3], q[j], s[0], 0, 0, 0);
                }
                second(2 * u, s[0], p[1], kSecond, std::false_type());
                for (; u < mine_last; ++u) {
                    settle();
                    probabilities(s[0], s[1], p[0], kSecond);
                    turn(u);
#pragma unroll
                    for (int j = 0; j < 8; ++j) key_at[j] ^= kTileBytes;
                    second(2 * u + 1, s[1], p[1], kFirst, std::true_type());
                    values_at(now);
                    settle();
                    probabilities(s[1], s[0], p[1], kFirst);
                    second(2 * u + 2, s[0], p[0], kSecond, std::true_type());
                    rotate();
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) add_product(j, value_operand(1, j), p[1]);
            }
            for (; u < last; ++u) {
                turn(u);
                rotate();
            }
        }
        if (careful) {
            add_nonfinite();                    // the last turn's barrier is behind all marks
            __syncthreads();
            break;
        }
        float x = 0.f;                          // stays zero where every o is finite
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) x = fmaf(o[d][i], 0.f, x);
        if (!__syncthreads_or(x != 0.f)) break;
    }

    // Out through LDS, which nobody reads any more, 8 KB a wave, so that rows go out whole: rows of 256 bytes, their 16-byte chunks
    // XORed with the row against bank conflicts.
    const float sum = halves_sum(l), rounded_sum = halves_sum(rounded);
    const bool any = m != -INFINITY;
    const float ln = m * 0.69314718055994531f;
    uint8_t* mine = lds.keys[0] + wave * (32 * 256);
    const int row4 = lane >> 4, chunk = lane & 15;
    auto place_of = [&](int row, int chunk) { return row * 256 + 16 * (chunk ^ (row & 15)); };
    if (it.part >= 0) {
        const float f = rounded_sum > 0.f ? sum / rounded_sum : 1.f;            // (0 of 0: all scores are minus infinity)
        const size_t to = (size_t)it.part * kChunkTileRows + 32 * wave;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int d = 0; d < 2; ++d)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const v16f& x = o[2 * half + d];
                    *reinterpret_cast<float4*>(mine + place_of(n, 8 * d + 2 * b + h)) = make_float4(x[4 * b] * f, x[4 * b + 1] * f, x[4 * b + 2] * f, x[4 * b + 3] * f);
                }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = 4 * i + row4;
                const float4 x = *reinterpret_cast<const float4*>(mine + place_of(row, chunk));
                if (32 * wave + row < live_rows) *reinterpret_cast<float4*>(a.parts.acc + (to + row) * kD + 64 * half + 4 * chunk) = x;
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (h == 0 && live) {
            a.parts.m[to + n] = ln;
            a.parts.l[to + n] = sum;
        }
        return;
    }
    const float inv = any ? 1.f / rounded_sum : 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const uint2 w = make_uint2(pack_bf16(o[d][4 * b] * inv, o[d][4 * b + 1] * inv), pack_bf16(o[d][4 * b + 2] * inv, o[d][4 * b + 3] * inv));
            *reinterpret_cast<uint2*>(mine + place_of(n, 4 * d + b) + 8 * h) = any ? w : make_uint2(0u, 0u);
        }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = 32 * wave + 4 * i + row4;
        const uint4 x = *reinterpret_cast<const uint4*>(mine + place_of(4 * i + row4, chunk));
        if (row < live_rows) *reinterpret_cast<uint4*>(a.out + ((size_t)(it.seq.q0 + tok0 + (row >> gs)) * a.Hq + hq0 + (row & (a.G - 1))) * kD + 8 * chunk) = x;
    }
    if (h == 0 && live && a.lse) a.lse[row_at] = any ? ln + logf(sum) : -INFINITY;
}

template __global__ void chunk_tile_kernel<false>(ChunkAttendArgs);
template __global__ void chunk_tile_kernel<true>(ChunkAttendArgs);

}  // namespace ffd
