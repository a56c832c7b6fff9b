// Attention of few new tokens a sequence over a paged cache (ffd_attend.h has the mathematics and the mapping of a wave,
// ffd_paged.h which tokens a query sees and how the work is cut): tiles of 16 or 32 query rows of a KV head, new tokens by
// query heads, and runs of 128-token blocks of the cache; a wave takes 32 of a block's tokens, straight from memory.
//
// Probabilities enter the second product in two bf16 parts (2^-16), which costs nothing where memory bounds.
//
// Bound: HBM, 512 bytes a token and KV head (8 bits: 260), for short caches the chain of lengths, pages, first tile and join.
// One token of 32 sequences, eight KV heads, with the merge: on 4K 101 us (5.3 TB/s; 8 bits 50, 5.4), on 32K 703 us (6.1 TB/s; 388, 5.6),
// of one sequence on 4K 12.8 us. Equal shares instead of runs of one length for all tiles: one chunk beside 15 decoding sequences 197
// -> 172 us, 37 tokens of three prompts 39 -> 16 (with tiles of 16 rows 13.5). Pages through the scalar cache: their wait does not
// drain the loads that are under way.
#include "ffd_paged.h"

namespace ffd {

namespace {

constexpr int kRowsShift = kChunkRowsShift;     // blocks of kRound tokens
static_assert(kRound == 1 << kRowsShift);
constexpr int kWholeShift = 8;                  // a unit of more blocks than a tile that is not cut has
static_assert(2 * kWholeBlocks < 1 << kWholeShift);

// The pages of a wave's 32 tokens: first rows of both 16-token halves, whether they are there.
struct TilePages {
    int entry[2];
    __device__ __forceinline__ void load(const PagedKv& p, int b, int t0) {
        entry[0] = uniform_page_entry(p, b, t0);
        entry[1] = uniform_page_entry(p, b, t0 + 16);
    }
    __device__ __forceinline__ void rows(const PagedKv& p, int Hkv, int kvh, int t0, size_t (&row)[2], bool (&there)[2]) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            there[t] = page_there(p, entry[t]);
            row[t] = page_row(p, Hkv, kvh, there[t] ? entry[t] : 0, t0 + 16 * t);
        }
    }
};

// Infinities and NaN among the values, which have been made zeros in the operand, reach the rows that see them.
template <int CT>
__device__ __forceinline__ void add_seen_nonfinite(RowState<CT>& st, const KvSource& kv, const size_t (&row)[2], const bool (&there)[2], int t0,
                                                   int end, const int (&at)[CT], int window, int pre, int g) {
#pragma unroll 1
    for (int t = 0; t < kTile && t0 + t < end; ++t) {
        if (!(t < 16 ? there[0] : there[1])) continue;
        const uint16_t* v = reinterpret_cast<const uint16_t*>(kv.v) + ((t < 16 ? row[0] : row[1]) + (t & 15)) * kD + 32 * g;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = bf16_to_f32(v[8 * r + i]);
                if (!(fabsf(x) < INFINITY)) {
#pragma unroll
                    for (int c = 0; c < CT; ++c)
                        if (sees(at[c], t0 + t, window, pre)) st.o[c][i][r] += x;
                }
            }
    }
}

// Where a tile's queries are and what they may see, per lane: the place of the row of tile c.
template <int CT>
struct Rows {
    int at[CT];
    float slope2[CT];
    int low, high;              // the first and the last place, of all rows
};

// Blocks [first, last) of the span. finite: infinities and NaN are taken out of every tile, see attend().
template <int CT, bool I8, bool RULED>
__device__ __forceinline__ void attend_pages(const ChunkAttendArgs& a, RowState<CT>& st, const v8bf (&q)[CT][4], const Rows<CT>& rows,
                                             const ScoreRule& rule, const ChunkItem& it, const ChunkSpan& span, int first, int last,
                                             bool finite, int wave, int n, int g) {
    if (first >= last) return;
    const int cached = min(it.seq.L, a.Lcap), pre = it.seq.pre, window = a.window;
    auto token = [&](int u) { return span.block(u) * kRound + kTile * wave; };
    // A wave's tile behind what any query sees is loaded all the same, from page 0 if its own is not there.
    TilePages pages, next_pages;
    size_t row[2];
    bool there[2];
    int t0 = token(first);
    pages.load(a.pages, it.b, t0);
    next_pages.load(a.pages, it.b, token(min(first + 1, last - 1)));
    KeyTile<I8> kt;
    ValueTile<I8> vt;
    __builtin_amdgcn_s_waitcnt(0x0f70);         // vmcnt(0): see attend()
    pages.rows(a.pages, a.Hkv, it.kvh, t0, row, there);
    kt.load_halves(a.pages.kv, row, n, g);
    vt.load_halves(a.pages.kv, row, n, g);
    for (int u = first; u < last; ++u) {
        const int t1 = token(min(u + 1, last - 1));
        size_t next[2];
        bool next_there[2];
        next_pages.rows(a.pages, a.Hkv, it.kvh, t1, next, next_there);
        v4f s[CT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int c = 0; c < CT; ++c) s[c][t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const v8bf x = kt.operand(t, k);
#pragma unroll
                for (int c = 0; c < CT; ++c) s[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[c][k], s[c][t], 0, 0, 0);
            }
        }
        float zs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (I8) zs[e] = absmax_of(kt.m[e >> 2], e & 3) * rule.zscale;
            else zs[e] = rule.zscale;
        }
        kt.load_halves(a.pages.kv, next, n, g);
        next_pages.load(a.pages, it.b, token(min(u + 2, last - 1)));

        // every row sees the whole tile, or not
        const bool behind = t0 + kTile <= rows.low + 1 && (window <= 0 || t0 > rows.high - window);
        const bool masked = !((behind || t0 + kTile <= pre) && t0 + kTile <= cached && there[0] && there[1]);
        uint32_t alive = 0xffu;                 // this lane's tokens that any row may see
        if (masked) {
            alive = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                alive |= (uint32_t)(there[e >> 2] & (t0 + value_token(e, g) < span.end)) << e;
        }
        float vs[8];
        if constexpr (I8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) vs[e] = absmax_of(vt.m[e >> 2], e & 3) * (1.f / 127.f);
        }
        v8bf p[CT], lo[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            float z[8];
            uint32_t seen = 0xffu;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = s[c][e >> 2][e & 3] * zs[e];
            if constexpr (RULED) {
                if (rule.cap2 != 0.f) cap_all(z, rule);
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = fmaf(-rows.slope2[c], fabsf((float)(rows.at[c] - t0 - value_token(e, g))), z[e]);
            }
            if (masked) {
                seen = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t x = (alive >> e) & (uint32_t)sees(rows.at[c], t0 + value_token(e, g), window, pre);
                    z[e] = x ? z[e] : -INFINITY;
                    seen |= x << e;
                }
            }
            float mn = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
            mn = fmaxf(st.m[c], groups_max(seen ? fmaxf(mn, -FLT_MAX) : mn));        // finite once a token is seen, also where all scores are NaN
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
                if constexpr (I8) x[e] = seen >> e & 1 ? x[e] * vs[e] : 0.f;
            }
            st.l[c] += sum;
            uint32_t w[4], low[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
                low[e] = pack_bf16(x[2 * e] - bf16_lo(w[e]), x[2 * e + 1] - bf16_hi(w[e]));
            }
            p[c] = __builtin_bit_cast(v8bf, make_uint4(w[0], w[1], w[2], w[3]));
            lo[c] = __builtin_bit_cast(v8bf, make_uint4(low[0], low[1], low[2], low[3]));
        }
        if constexpr (!I8) {
            if (masked) vt.keep(alive);
            if ((masked || finite) && __ballot(!vt.all_finite()) != 0) {
                vt.make_finite();
                add_seen_nonfinite<CT>(st, a.pages.kv, row, there, t0, span.end, rows.at, window, pre, g);
            }
        }
        v8bf f[8];
        vt.operands(f);
        row[0] = next[0];
        row[1] = next[1];
        there[0] = next_there[0];
        there[1] = next_there[1];
        t0 = t1;
        // The next values are asked for here, or behind the products where that would spill (8 tokens on 32K 45 us with spills, 39
        // so; 32 sequences of 8K in 8 bits 114 and 109), and not, where the compiler would have them, at their use in the next turn
        // (of which there is none after the last one).
        constexpr bool kEarly = CT == 1 && !I8;
        if constexpr (kEarly) {
            vt.load_halves(a.pages.kv, row, n, g);
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < CT; ++c) st.o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], p[c], st.o[c][i], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < CT; ++c) st.o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], lo[c], st.o[c][i], 0, 0, 0);
        if constexpr (!kEarly) {
            vt.load_halves(a.pages.kv, row, n, g);
            asm volatile("" ::: "memory");
        }
    }
}

}  // namespace

// Work in the order (sequence, tile, KV head, block), a tile of a sequence counted as its longest one, in equal shares of
// consecutive blocks, one for each workgroup: a share is the end of one tile, whole tiles, and the beginning of another. A tile
// that is whole in a share goes to the outputs, else the workgroup leaves at most two partial states: 2 w + 1 of the tile
// that it begins, 2 w of one that another began.
template <int CT, bool I8, bool RULED>
__global__ __launch_bounds__(kThreads, CT == 1 && I8 ? 3 : 2) void chunk_rows_kernel(ChunkAttendArgs a) {
    __shared__ JoinLds<CT> lds;
    constexpr int kRows = 16 * CT;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int g = lane >> 4, n = lane & 15, wg = blockIdx.x;
    const int gs = __builtin_ctz(a.G), step = kRows >> gs;
    ChunkPlan<kRows, kRowsShift> plan;
    auto units = [&](int shift) { return (plan.blocks + (1 << shift) - 1) >> shift; };           // of a tile
    // a tile without blocks is one unit, for its empty rows to be written
    auto work = [&](int shift) { return plan.tiles * max(units(shift), 1) * a.Hkv; };
    int all = 0, pairs = 0, tiles = 0;
    bool over[2] = {false, false};              // a tile of more than kWholeBlocks, of more than twice as many
    for (int b0 = (a.B - 1) & ~63; b0 >= 0; b0 -= 64) {         // backwards, to end at the first ones
        plan.load(a, b0, lane);
        all += __builtin_amdgcn_readlane(wave_inclusive_scan(work(a.unit_shift)), 63);
        pairs += __builtin_amdgcn_readlane(wave_inclusive_scan(work(a.unit_shift + 1)), 63);
        tiles += __builtin_amdgcn_readlane(wave_inclusive_scan(plan.tiles * a.Hkv), 63);
#pragma unroll
        for (int i = 0; i < 2; ++i) over[i] |= __ballot(plan.blocks > kWholeBlocks << i) != 0;
    }
    // Short tiles are not cut (longer ones where there are many), others, where there is a workgroup for every two blocks, into these.
    const bool whole = !over[0] || (!over[1] && 4 * tiles >= a.slots);
    const int shift = whole ? kWholeShift : pairs <= a.slots ? a.unit_shift + 1 : a.unit_shift;
    if (whole) all = tiles;
    else if (shift != a.unit_shift) all = pairs;
    const Shares shares(all, a.slots);
    const int begin = shares.begin(wg), end = shares.begin(wg + 1);
    int u = begin;
    bool begun = false;                         // a tile that another workgroup ends
    while (u < end) {                           // uniform
        ChunkItem it{};
        int tile_units = 1, at = 0, before = 0;
        for (int b0 = 0; b0 < a.B; b0 += 64) {
            if (b0 > 0 || u != begin) plan.load(a, b0, lane);          // (kept, it would cost the loop registers)
            const int mine = work(shift), incl = wave_inclusive_scan(mine), first = before + incl - mine;
            const uint64_t hit = __ballot(u >= first && u < first + mine);
            if (hit != 0) {
                const int src = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hit));
                it.b = b0 + src;
                plan.give(it.seq, src);
                tile_units = max(__builtin_amdgcn_readlane(units(shift), src), 1);
                at = __builtin_amdgcn_readfirstlane(u) - __builtin_amdgcn_readlane(first, src);
                break;
            }
            before += __builtin_amdgcn_readlane(incl, 63);
        }
        const int pair = at / tile_units, from = at - pair * tile_units, to = min(tile_units, from + end - u);
        it.tile = pair / a.Hkv;
        it.kvh = pair - it.tile * a.Hkv;
        it.part = from == 0 && to == tile_units ? -1 : 2 * wg + (from == 0 ? 1 : 0);
        u += to - from;
        const int tok0 = it.tile * step, live = min(kRows, (it.seq.n - tok0) << gs);
        const int hq0 = it.kvh * a.G, place = it.seq.L - it.seq.n;
        if (it.part >= 0 && from == 0) {
            begun = true;
            if (tid == 0) a.parts.records[wg] = make_int4(it.seq.q0 + tok0, it.kvh, live, shares.of(u - to + tile_units - 1) - wg + 1);
        }
        v8bf q[CT][4];
        Rows<CT> rows;
        const ScoreRule rule = score_rule(a, I8, hq0);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const int r = min(16 * c + n, live - 1), tok = tok0 + (r >> gs), head = hq0 + (r & (a.G - 1));
            load_query<I8>(q[c], a.q + ((size_t)(it.seq.q0 + tok) * a.Hq + head) * kD, g);
            rows.at[c] = place + tok;
            rows.slope2[c] = RULED && a.slopes ? slope_in_twos(a.slopes[head]) : 0.f;
        }
        const int tok1 = min(tok0 + step, it.seq.n) - 1;
        rows.low = place + tok0;
        rows.high = place + tok1;
        const ChunkSpan span = chunk_span<kRowsShift>(a, it.seq, tok0, tok1);
        const int first = (int)min((long long)span.count, (long long)from << shift), last = (int)min((long long)span.count, (long long)to << shift);
        RowState<CT> st;
        for (bool finite = false;; finite = true) {
            st.clear();
            attend_pages<CT, I8, RULED>(a, st, q, rows, rule, it, span, first, last, finite, wave, n, g);
            if (I8 || finite || __ballot(!st.all_finite()) == 0) break;
        }
        join_waves(lds, st, wave, n, g);
        for (int i = tid; i < live * (kD / 4); i += kThreads) {
            const int r = i >> 5, d4 = i & 31;
            const float4 x = *reinterpret_cast<const float4*>(&lds.acc[0][r][4 * d4]);
            const float4 y = *reinterpret_cast<const float4*>(&lds.acc[1][r][4 * d4]);
            const float4 o = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
            if (it.part >= 0) {
                const size_t to = (size_t)it.part * kRows + r;
                *reinterpret_cast<float4*>(a.parts.acc + to * kD + 4 * d4) = o;
                if (d4 == 0) joined_ml(lds, r, a.parts.m[to], a.parts.l[to]);
            } else {
                const size_t to = (size_t)(it.seq.q0 + tok0 + (r >> gs)) * a.Hq + hq0 + (r & (a.G - 1));
                float m, l;
                joined_ml(lds, r, m, l);
                const bool any = m != -INFINITY;
                const float inv = any ? 1.f / l : 0.f;
                const uint2 w = any ? make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv)) : make_uint2(0u, 0u);
                *reinterpret_cast<uint2*>(a.out + to * kD + 4 * d4) = w;
                if (d4 == 0 && a.lse) a.lse[to] = any ? m + logf(l) : -INFINITY;
            }
        }
        if (u < end) __syncthreads();           // the next tile takes the join's place
    }
    if (!begun && tid == 0) a.parts.records[wg] = make_int4(0, 0, 0, 0);
}

// Joins the runs of the row tiles that were cut: a workgroup takes 16 or 32 rows of one tile and 32 dims, eight lanes a row;
// where there are fewer rows several groups of lanes share a row's runs, eight of which are asked for together. Bound: latency (4 us
// for a few tiles, 10 for 64 tiles of 256 rows in four runs each).
__global__ __launch_bounds__(kThreads) void chunk_merge_kernel(ChunkMergeArgs a) {
    struct State {
        float m, l;
    };
    __shared__ State states[32];
    __shared__ float4 sums[32][8];
    const bool second = (int)blockIdx.x >= a.wgs;
    const ChunkParts& x = second ? a.parts[1] : a.parts[0];
    const int slice_rows = chunk_merge_rows(x.rows), slices = 4 * (x.rows / slice_rows);
    const int wg = second ? blockIdx.x - a.wgs : blockIdx.x, part = wg / slices, slice = wg % slices;
    const int4 record = x.records[part];
    if (record.w == 0 || (x.total && part >= x.total[0])) return;           // not the first run of a tile, or not used
    const int live = min(record.z - slice_rows * (slice >> 2), slice_rows), cuts = record.w;
    // part of run s
    const int first = x.total ? part : 2 * part + 1, second_run = x.total ? part + a.Hkv : 2 * part + 2, step = x.total ? a.Hkv : 2;
    if (live <= 0 || second_run + (cuts - 2) * step >= x.count) return;
    int shift = 5;                              // 2^shift rows
    while (shift > 0 && live <= 1 << (shift - 1)) --shift;
    const int d4 = 8 * (slice & 3) + (threadIdx.x & 7), group = threadIdx.x >> 3;
    const int r = group & ((1 << shift) - 1), k = group >> shift, groups = 32 >> shift;
    const int row0 = slice_rows * (slice >> 2) + min(r, live - 1);
    float M = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto fold = [&](float m, float pl, const float4& y) {
        if (m == -INFINITY) return;                             // a run that saw nothing
        const float Mn = fmaxf(M, m), c = M == -INFINITY ? 0.f : __expf(M - Mn), w = __expf(m - Mn);
        M = Mn;
        l = fmaf(w, pl, l * c);
        o = make_float4(fmaf(w, y.x, o.x * c), fmaf(w, y.y, o.y * c), fmaf(w, y.z, o.z * c), fmaf(w, y.w, o.w * c));
    };
    constexpr int U = 8;                        // rows asked for together
    for (int s0 = k; s0 < cuts; s0 += U * groups) {
        float m[U], pl[U];
        float4 y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = min(s0 + u * groups, cuts - 1);
            const size_t row = (size_t)(s == 0 ? first : second_run + (s - 1) * step) * x.rows + row0;
            m[u] = x.m[row];
            pl[u] = x.l[row];
            y[u] = *reinterpret_cast<const float4*>(x.acc + row * kD + 4 * d4);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) fold(s0 + u * groups < cuts ? m[u] : -INFINITY, pl[u], y[u]);
    }
    if (groups > 1) {                           // uniform
        if ((threadIdx.x & 7) == 0) states[group] = State{M, l};
        sums[group][threadIdx.x & 7] = o;
        __syncthreads();
        if (k > 0) return;
        for (int i = 1; i < groups; ++i) fold(states[group + (i << shift)].m, states[group + (i << shift)].l, sums[group + (i << shift)][threadIdx.x & 7]);
    }
    if (r >= live) return;
    const bool any = M != -INFINITY;
    const float inv = any ? 1.f / l : 0.f;
    const int gs = __builtin_ctz(a.G);
    const size_t to = (size_t)(record.x + (row0 >> gs)) * a.Hq + record.y * a.G + (row0 & (a.G - 1));
    *reinterpret_cast<uint2*>(a.out + to * kD + 4 * d4) =
        any ? make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv)) : make_uint2(0u, 0u);
    if (d4 == 0 && a.lse) a.lse[to] = any ? M + logf(l) : -INFINITY;
}

template __global__ void chunk_rows_kernel<1, false, false>(ChunkAttendArgs);
template __global__ void chunk_rows_kernel<1, false, true>(ChunkAttendArgs);
template __global__ void chunk_rows_kernel<1, true, false>(ChunkAttendArgs);
template __global__ void chunk_rows_kernel<1, true, true>(ChunkAttendArgs);
template __global__ void chunk_rows_kernel<2, false, false>(ChunkAttendArgs);
template __global__ void chunk_rows_kernel<2, false, true>(ChunkAttendArgs);
template __global__ void chunk_rows_kernel<2, true, false>(ChunkAttendArgs);
template __global__ void chunk_rows_kernel<2, true, true>(ChunkAttendArgs);

}  // namespace ffd
