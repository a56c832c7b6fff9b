// Attention of few new tokens a sequence over a paged cache (ffd_attend.h has the mathematics and the mapping of a wave,
// ffd_paged.h which tokens a query sees and how the work is cut): tiles of 16 or 32 query rows of a KV head, new tokens by
// query heads, and runs of 128-token blocks of the cache; a wave takes 32 of a block's tokens, straight from memory.
//
// Probabilities enter the second product in two bf16 parts (2^-16), which costs nothing where memory bounds.
//
// Bound: HBM, 512 bytes a token and KV head (8 bits: 260), for short caches the chain of lengths, pages, first tile and join.
#include "ffd_paged.h"

namespace ffd {

namespace {

constexpr int kRowsShift = kChunkRowsShift;     // blocks of kRound tokens
static_assert(kRound == 1 << kRowsShift);

// The pages of a wave's 32 tokens: first rows of both 16-token halves, whether they are there.
struct TilePages {
    int entry[2];
    __device__ __forceinline__ void load(const PagedKv& p, int b, int t0) {
        entry[0] = page_entry(p, b, t0);
        entry[1] = page_entry(p, b, t0 + 16);
    }
    __device__ __forceinline__ bool there(const PagedKv& p, int t) const { return page_there(p, entry[t]); }
    __device__ __forceinline__ void rows(const PagedKv& p, int Hkv, int kvh, int t0, size_t (&row)[2]) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) row[t] = page_row(p, Hkv, kvh, there(p, t) ? entry[t] : 0, t0 + 16 * t);
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

// Blocks [first, last) of the span. FINITE: infinities and NaN are taken out of every tile, see attend().
template <int CT, bool I8, bool RULED, bool FINITE>
__device__ __forceinline__ void attend_pages(const ChunkAttendArgs& a, RowState<CT>& st, const v8bf (&q)[CT][4], const Rows<CT>& rows,
                                             const ScoreRule& rule, const ChunkItem& it, const ChunkSpan& span, int first, int last,
                                             int wave, int n, int g) {
    if (first >= last) return;
    const int cached = min(it.seq.L, a.Lcap), pre = it.seq.pre, window = a.window;
    auto token = [&](int u) { return span.block(u) * kRound + kTile * wave; };
    // A wave's tile behind what any query sees is loaded all the same, from page 0 if its own is not there.
    TilePages pages, next_pages;
    size_t row[2];
    int t0 = token(first);
    pages.load(a.pages, it.b, t0);
    next_pages.load(a.pages, it.b, token(min(first + 1, last - 1)));
    KeyTile<I8> kt;
    ValueTile<I8> vt;
    __builtin_amdgcn_s_waitcnt(0x0f70);         // vmcnt(0): see attend()
    pages.rows(a.pages, a.Hkv, it.kvh, t0, row);
    kt.load_halves(a.pages.kv, row, n, g);
    vt.load_halves(a.pages.kv, row, n, g);
    for (int u = first; u < last; ++u) {
        const bool there[2] = {pages.there(a.pages, 0), pages.there(a.pages, 1)};
        const int t1 = token(min(u + 1, last - 1));
        size_t next[2];
        next_pages.rows(a.pages, a.Hkv, it.kvh, t1, next);
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
        pages = next_pages;
        next_pages.load(a.pages, it.b, token(min(u + 2, last - 1)));

        // every row sees the whole tile, or not
        const bool behind = t0 + kTile <= rows.low + 1 && (window <= 0 || t0 > rows.high - window);
        const bool masked = !((behind || t0 + kTile <= pre) && t0 + kTile <= cached && there[0] && there[1]);
        uint32_t alive = 0xffu;                 // this lane's tokens that any row may see
        if (masked) {
            alive = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (there[e >> 2] && t0 + value_token(e, g) < span.end) alive |= 1u << e;
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
            for (int e = 0; e < 8; ++e) {
                z[e] = s[c][e >> 2][e & 3] * zs[e];
                if constexpr (RULED) {
                    if (rule.cap2 != 0.f) z[e] = capped(z[e], rule.cap2);
                    z[e] = fmaf(-rows.slope2[c], fabsf((float)(rows.at[c] - t0 - value_token(e, g))), z[e]);
                }
            }
            if (masked) {
                seen = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool x = (alive >> e & 1) && sees(rows.at[c], t0 + value_token(e, g), window, pre);
                    z[e] = x ? z[e] : -INFINITY;
                    seen |= x ? 1u << e : 0u;
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
            if ((masked || FINITE) && __ballot(!vt.all_finite()) != 0) {
                vt.make_finite();
                add_seen_nonfinite<CT>(st, a.pages.kv, row, there, t0, span.end, rows.at, window, pre, g);
            }
        }
        v8bf f[8];
        vt.operands(f);
        row[0] = next[0];
        row[1] = next[1];
        t0 = t1;
        vt.load_halves(a.pages.kv, row, n, g);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < CT; ++c) st.o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], p[c], st.o[c][i], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < CT; ++c) st.o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], lo[c], st.o[c][i], 0, 0, 0);
    }
}

}  // namespace

template <int CT, bool I8, bool RULED>
__global__ __launch_bounds__(kThreads, CT == 1 ? 3 : 2) void chunk_rows_kernel(ChunkAttendArgs a) {
    __shared__ JoinLds<CT> lds;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int g = lane >> 4, n = lane & 15;
    ChunkItem it;
    if (!chunk_item<16 * CT, kRowsShift>(a, blockIdx.x, lane, it) || it.part >= a.max_parts) return;
    const int gs = __builtin_ctz(a.G), step = (16 * CT) >> gs, tok0 = it.tile * step;
    const int live = min(16 * CT, (it.seq.n - tok0) << gs);
    const int hq0 = it.kvh * a.G, place = it.seq.L - it.seq.n;
    v8bf q[CT][4];
    Rows<CT> rows;
    ScoreRule rule = score_rule(a, I8, hq0);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int r = min(16 * c + n, live - 1), tok = tok0 + (r >> gs), head = hq0 + (r & (a.G - 1));
        load_query<I8>(q[c], a.q + ((size_t)(it.seq.q0 + tok) * a.Hq + head) * kD, g);
        rows.at[c] = place + tok;
        rows.slope2[c] = RULED && a.slopes ? a.slopes[head] * kLog2e : 0.f;
    }
    const int tok1 = min(tok0 + step, it.seq.n) - 1;
    rows.low = place + tok0;
    rows.high = place + tok1;
    const ChunkSpan span = chunk_span<kRowsShift>(a, it.seq, tok0, tok1);
    const int first = (int)((long long)span.count * it.run / it.cuts), last = (int)((long long)span.count * (it.run + 1) / it.cuts);
    RowState<CT> st;
    st.clear();
    attend_pages<CT, I8, RULED, false>(a, st, q, rows, rule, it, span, first, last, wave, n, g);
    if (!I8 && __ballot(!st.all_finite()) != 0) {
        st.clear();
        attend_pages<CT, I8, RULED, true>(a, st, q, rows, rule, it, span, first, last, wave, n, g);
    }
    join_waves(lds, st, wave, n, g);
    for (int i = tid; i < live * (kD / 4); i += kThreads) {
        const int r = i >> 5, d4 = i & 31;
        const float4 x = *reinterpret_cast<const float4*>(&lds.acc[0][r][4 * d4]);
        const float4 y = *reinterpret_cast<const float4*>(&lds.acc[1][r][4 * d4]);
        const float4 o = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
        if (it.part >= 0) {
            const size_t to = (size_t)it.part * (16 * CT) + r;
            *reinterpret_cast<float4*>(a.part_acc + to * kD + 4 * d4) = o;
            if (d4 == 0) joined_ml(lds, r, a.part_m[to], a.part_l[to]);
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
}

// Joins the runs of the row tiles that were cut: a workgroup takes eight rows of one tile, 32 lanes a row.
template <int ROWS, int SHIFT>
__global__ __launch_bounds__(kThreads) void chunk_merge_kernel(ChunkAttendArgs a) {
    const int tid = threadIdx.x, lane = tid & 63;
    constexpr int kSlices = ROWS / 8;
    const int pair = blockIdx.x / kSlices, slice = blockIdx.x % kSlices;
    // the pair-th (sequence, tile, KV head) of those that are cut
    ChunkPlan<ROWS, SHIFT> plan;
    plan.load(a, 0, lane);
    const int C = plan.run_blocks(a, lane);
    int before = 0, parts_before = 0, b = -1, q0, n, tiles, cuts, first_part, at;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        if (b0 > 0) plan.load(a, b0, lane);
        const int mine = plan.cuts_for(C), pairs = mine > 1 ? plan.tiles * a.Hkv : 0, parts = pairs * mine;
        const int incl = wave_inclusive_scan(pairs), parts_incl = wave_inclusive_scan(parts), first = before + incl - pairs;
        const uint64_t hit = __ballot(pair >= first && pair < first + pairs);
        if (hit != 0) {
            const int src = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hit));
            b = b0 + src;
            q0 = __builtin_amdgcn_readlane(plan.seq.q0, src);
            n = __builtin_amdgcn_readlane(plan.seq.n, src);
            tiles = __builtin_amdgcn_readlane(plan.tiles, src);
            cuts = __builtin_amdgcn_readlane(mine, src);
            first_part = parts_before + __builtin_amdgcn_readlane(parts_incl - parts, src);
            at = pair - __builtin_amdgcn_readlane(first, src);
            break;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
        parts_before += __builtin_amdgcn_readlane(parts_incl, 63);
    }
    if (b < 0) return;
    const int turn = at / a.Hkv, kvh = at - turn * a.Hkv, tile = tiles - 1 - turn;
    const int gs = __builtin_ctz(a.G), tok0 = tile * (ROWS >> gs), live = min(ROWS, (n - tok0) << gs);
    const int r = 8 * slice + (tid >> 5), d4 = tid & 31;
    if (r >= live) return;
    const int part0 = first_part + turn * cuts * a.Hkv + kvh;
    if (part0 + (cuts - 1) * a.Hkv >= a.max_parts) return;
    auto row_of = [&](int s) { return (size_t)(part0 + s * a.Hkv) * ROWS + r; };
    float M = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int U = 4;
    for (int s0 = 0; s0 < cuts; s0 += U) {
        float m[U], pl[U];
        float4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t row = row_of(min(s0 + u, cuts - 1));
            m[u] = s0 + u < cuts ? a.part_m[row] : -INFINITY;
            pl[u] = a.part_l[row];
            x[u] = *reinterpret_cast<const float4*>(a.part_acc + row * kD + 4 * d4);
        }
        float Mn = M;
#pragma unroll
        for (int u = 0; u < U; ++u) Mn = fmaxf(Mn, m[u]);
        if (Mn == -INFINITY) continue;
        const float c = M == -INFINITY ? 0.f : __expf(M - Mn);
        M = Mn;
        l *= c;
        o = make_float4(o.x * c, o.y * c, o.z * c, o.w * c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (m[u] == -INFINITY) continue;            // a run that saw nothing
            const float w = __expf(m[u] - M);
            l = fmaf(w, pl[u], l);
            o = make_float4(fmaf(w, x[u].x, o.x), fmaf(w, x[u].y, o.y), fmaf(w, x[u].z, o.z), fmaf(w, x[u].w, o.w));
        }
    }
    const bool any = M != -INFINITY;
    const float inv = any ? 1.f / l : 0.f;
    const size_t to = (size_t)(q0 + tok0 + (r >> gs)) * a.Hq + kvh * a.G + (r & (a.G - 1));
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
template __global__ void chunk_merge_kernel<16, kRowsShift>(ChunkAttendArgs);
template __global__ void chunk_merge_kernel<32, kRowsShift>(ChunkAttendArgs);
template __global__ void chunk_merge_kernel<kChunkTileRows, kChunkTileShift>(ChunkAttendArgs);

}  // namespace ffd
