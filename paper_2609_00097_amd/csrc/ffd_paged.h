// Paged caches and ragged batches of new tokens: what the kernels over them share.
//
// Sequence b has L = seq_lens[b] tokens, the last n = q_start[b + 1] - q_start[b] of them new: new token t has the place
// i = L - n + t. Its query sees token j < min(L, Lcap) if j <= i and (no window, or i - j < window), or if j < prefix_lens[b],
// and if j's page is there. All numbers come from the device and are clamped where they are read, so that no table, length
// or start leads outside the buffers.
#pragma once

#include "ffd_attend.h"

namespace ffd {

constexpr int kMaxLen = 1 << 30;               // longer lengths count as this

struct ChunkSeq {
    int q0, n, L, pre;
};

__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkArgs& a, int b) {
    ChunkSeq s;
    const int first = a.q_start[b], last = a.q_start[b + 1], len = a.seq_lens[b];
    s.pre = a.prefix_lens ? a.prefix_lens[b] : 0;
    s.q0 = min(max(first, 0), a.T);
    s.n = min(max(last, s.q0), a.T) - s.q0;
    s.L = min(max(len, 0), kMaxLen);
    s.pre = min(max(s.pre, 0), min(s.L, a.Lcap));
    return s;
}

// Blocks of 2^SHIFT tokens that hold what new tokens [first, last] of a sequence see: block(i), i < count.
struct ChunkSpan {
    int prefix, skip, count;
    int end;                    // behind the last token that any of them sees
    __device__ __forceinline__ int block(int i) const { return i < prefix ? i : i + skip; }
};
template <int SHIFT>
__device__ __forceinline__ ChunkSpan chunk_span(const ChunkArgs& a, const ChunkSeq& s, int first, int last) {
    const int cached = min(s.L, a.Lcap), place = s.L - s.n;
    ChunkSpan p;
    p.end = max(min(max(place + last + 1, s.pre), cached), 0);
    const int from = a.window > 0 ? max(place + first - a.window + 1, 0) : 0;
    const int high = (p.end + (1 << SHIFT) - 1) >> SHIFT;
    p.prefix = min((s.pre + (1 << SHIFT) - 1) >> SHIFT, high);
    const int low = min(max(from >> SHIFT, p.prefix), high);
    p.skip = low - p.prefix;
    p.count = high - p.skip;
    return p;
}

// Whether a query at place i sees token j (of a page that is there, below min(L, Lcap)). Without branches: eight or 32 of these in
// a row would become as many jumps.
__device__ __forceinline__ bool sees(int i, int j, int window, int pre) {
    return (((j <= i) & ((window <= 0) | (i - j < window))) | (j < pre)) != 0;
}

// Row of (token j, KV head kvh) in the pages: first row of the 16-token group that holds j, given its page's entry.
__device__ __forceinline__ size_t page_row(const PagedKv& p, int Hkv, int kvh, int entry, int j) {
    return (((size_t)entry * Hkv + kvh) << p.page_shift) + (j & ((1 << p.page_shift) - 1));
}
__device__ __forceinline__ bool page_there(const PagedKv& p, int entry) { return (unsigned)entry < (unsigned)p.num_pages; }
// Entry of the page that holds token j; -1 behind the table's row.
__device__ __forceinline__ int page_entry(const PagedKv& p, int b, int j) {
    const int i = j >> p.page_shift;
    const int e = p.table[(size_t)b * p.max_pages + min(i, p.max_pages - 1)];
    return i < p.max_pages ? e : -1;
}

// The same for a token that all lanes agree on, through the scalar cache: the entry is waited for by itself and not, as a
// vector load's result, behind all loads that are under way.
__device__ __forceinline__ int uniform_page_entry(const PagedKv& p, int b, int j) {
    const int i = __builtin_amdgcn_readfirstlane(j >> p.page_shift);
    const auto* table = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p.table));
    const int e = table[(size_t)__builtin_amdgcn_readfirstlane(b) * p.max_pages + min(i, p.max_pages - 1)];
    return i < p.max_pages ? e : -1;
}

// The batch's work, laid out by every wave alone, 64 sequences at a time. A sequence's n G query rows of a KV head are row
// tiles of ROWS rows.
struct ChunkItem {
    ChunkSeq seq;
    int b, kvh, tile, run, cuts;
    int part;                   // number of the partial state, -1: the tile is whole
};
template <int ROWS, int SHIFT>
struct ChunkPlan {
    ChunkSeq seq;               // this lane's sequence of the 64 at hand
    int tiles, blocks;          // of a tile at most
    __device__ __forceinline__ void load(const ChunkAttendArgs& a, int b0, int lane) {
        const int b = b0 + lane;
        seq = chunk_seq(a, min(b, a.B - 1));
        const long long rows = (long long)seq.n * a.G;
        tiles = blocks = 0;
        if (b < a.B && rows > a.rows_above && rows <= a.rows_upto) {
            tiles = (int)((rows + ROWS - 1) / ROWS);
            const int step = ROWS / a.G;
            // of the last tile, as if it saw all before it, but within a window no more than a tile's first and last place span
            const ChunkSpan all = chunk_span<SHIFT>(a, seq, (tiles - 1) * step, seq.n - 1);
            blocks = all.count + all.skip;
            if (a.window > 0) blocks = min(blocks, all.prefix + ((a.window + step - 2) >> SHIFT) + 2);
        }
    }
    __device__ __forceinline__ void give(ChunkSeq& s, int src) const {
        s.q0 = __builtin_amdgcn_readlane(seq.q0, src);
        s.n = __builtin_amdgcn_readlane(seq.n, src);
        s.L = __builtin_amdgcn_readlane(seq.L, src);
        s.pre = __builtin_amdgcn_readlane(seq.pre, src);
    }
    __device__ __forceinline__ int cuts_for(int C) const { return max((blocks + C - 1) / C, 1); }
    // C of chunk_item, with the first 64 sequences loaded
    __device__ __forceinline__ int run_blocks(const ChunkAttendArgs& a, int lane) {
        long long all = 0, count = 0;
        for (int b0 = 0; b0 < a.B; b0 += 64) {
            if (b0 > 0) load(a, b0, lane);
            all += (long long)tiles * blocks;
            count += tiles;
        }
        if (a.B > 64) load(a, 0, lane);
#pragma unroll
        for (int x = 32; x; x >>= 1) {
            all += __shfl_xor(all, x);
            count += __shfl_xor(count, x);
        }
        all *= a.Hkv;
        count *= a.Hkv;
        const long long spare = max(max((long long)a.slots - count, (long long)a.slots / 2), 1LL);
        const int C = (int)min(max((all + spare - 1) / spare, 1LL), (long long)(INT32_MAX / 2));
        if (a.B > 64 || count >= a.slots) return C;
        // A workgroup has its CU to itself, so the smallest C whose items fill the slots once; the lanes try 64.
        const int least = (int)max(all / a.slots, 1LL), mine = least + (int)((long long)(C - least) * (lane + 1) / 64);
        long long items = 0;
        for (uint64_t left = __ballot(tiles > 0); left; left &= left - 1) {
            const int src = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(left));
            const int n = __builtin_amdgcn_readlane(blocks, src);
            items += (long long)__builtin_amdgcn_readlane(tiles, src) * max((n + mine - 1) / mine, 1);
        }
        const uint64_t fit = __ballot(items * a.Hkv <= a.slots);
        return fit ? __builtin_amdgcn_readlane(mine, __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(fit))) : C;
    }
};

// Large tiles: each tile's blocks (of 2^SHIFT tokens) are cut into `cuts` runs, the same number for all tiles of a sequence: as few
// runs as keep the longest tile's at or below C blocks, where C gives each of the slots that whole tiles leave, or of half of all
// slots, an equal part of all blocks. So there are at most max(slots, slots / 2 + tiles * Hkv) items and, a tile that is cut
// being longer than C, at most `slots` parts. Items of a sequence are in the order (tile from the last one, which sees most, on;
// run; KV head). The item of workgroup wg; false: there is none. Workgroup 0 leaves the number of parts for the merge.
template <int ROWS, int SHIFT>
__device__ __forceinline__ bool chunk_item(const ChunkAttendArgs& a, int wg, int lane, ChunkItem& it) {
    ChunkPlan<ROWS, SHIFT> plan;
    plan.load(a, 0, lane);
    const int C = plan.run_blocks(a, lane);
    int before = 0, parts_before = 0;
    bool found = false;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        if (b0 > 0) plan.load(a, b0, lane);
        const int cuts = plan.cuts_for(C), items = plan.tiles * cuts * a.Hkv, parts = cuts > 1 ? items : 0;
        const int incl = wave_inclusive_scan(items), first = before + incl - items;
        const int parts_incl = wave_inclusive_scan(parts);
        const uint64_t hit = __ballot(wg >= first && wg < first + items);
        if (hit != 0) {
            const int src = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hit));
            it.b = b0 + src;
            plan.give(it.seq, src);
            it.cuts = __builtin_amdgcn_readlane(cuts, src);
            const int at = __builtin_amdgcn_readfirstlane(wg) - __builtin_amdgcn_readlane(first, src);
            const int rest = at / a.Hkv;
            it.kvh = at - rest * a.Hkv;
            const int turn = rest / it.cuts;
            it.run = rest - turn * it.cuts;
            it.tile = __builtin_amdgcn_readlane(plan.tiles, src) - 1 - turn;
            it.part = -1;
            if (it.cuts > 1) it.part = parts_before + __builtin_amdgcn_readlane(parts_incl - parts, src) + at;
            found = it.part < a.parts.count;
            if (wg != 0) return found;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
        parts_before += __builtin_amdgcn_readlane(parts_incl, 63);
    }
    if (wg == 0 && threadIdx.x == 0) a.parts.total[0] = min(parts_before, a.parts.count);
    return found;
}
__device__ __forceinline__ void write_record(const ChunkAttendArgs& a, const ChunkItem& it, int tok0, int live) {
    if (it.part >= 0 && threadIdx.x == 0) a.parts.records[it.part] = make_int4(it.seq.q0 + tok0, it.kvh, live, it.run == 0 ? it.cuts : 0);
}

// Units 0 .. all - 1 of work in equal shares (they differ by one unit at most) of consecutive units, as many as there are
// workgroups. Products below 2^52.
struct Shares {
    int all, count;
    double r_all, r_count;
    __device__ __forceinline__ Shares(int units, int slots)
        : all(units), count(min(slots, max(units, 1))), r_all(reciprocal((double)max(units, 1))), r_count(reciprocal((double)count)) {}
    __device__ __forceinline__ int begin(int w) const {
        return __builtin_amdgcn_readfirstlane(w >= count ? all : (int)floor_div((long long)w * all, count, r_count));
    }
    // the share that unit u belongs to
    __device__ __forceinline__ int of(int u) const {
        return __builtin_amdgcn_readfirstlane((int)floor_div((long long)(u + 1) * count - 1, all, r_all));
    }
};

// What a product s = q.k becomes, in powers of two: z2 = log2(e) (cap tanh(scale s / cap) - slope |i - j|). An 8-bit key's product is
// multiplied by its M before and by 1 / 127 within `scale`.
//
// With y = scale s / cap and x = 2 log2(e) y: tanh(y) = 1 - 2 / (1 + 2^x) has no overflow and keeps infinities and NaN, but is up to
// 2^-22 off, of scores far below the cap as of others. So up to |y| = 1/2 it is y times a polynomial of degree four in y^2, the
// interpolation of tanh(y) / y at the Chebyshev points of y^2 in [0, 1/4] (1.4e-8 off), whose coefficients come in terms of x and with
// the cap multiplied in (near_caps).
struct ScoreRule {
    float zscale;               // without a cap: scale log2(e); with one: 2 scale log2(e) / cap
    float cap2;                 // cap log2(e), or 0
    float slope2;               // this lane's row's slope log2(e)
    float near[5];
};
constexpr float kNearCap = 1.4426950408889634f;                         // x of y = 1/2
constexpr double kTanhNear[5] = {0.9999999867573891, -0.33333067944418876, 0.13324750504729285, -0.05298423882487847, 0.017131344424267444};
// finite, for the distance of zero
__device__ __forceinline__ float slope_in_twos(float slope) { return fminf(fmaxf(slope * kLog2e, -FLT_MAX), FLT_MAX); }
__device__ __forceinline__ ScoreRule score_rule(const ChunkArgs& a, bool i8, int head) {
    ScoreRule r;
    const float scale = i8 ? a.scale / 127.f : a.scale;
    r.zscale = a.cap > 0.f ? fminf(scale * 2.f * kLog2e / a.cap, FLT_MAX) : scale * kLog2e;
    r.cap2 = a.cap * kLog2e;
    r.slope2 = a.slopes ? slope_in_twos(a.slopes[head]) : 0.f;
#pragma unroll
    for (int i = 0; i < 5; ++i) r.near[i] = a.cap_near[i];
    return r;
}
// x = zscale s; of scores up to half of the cap, factor of x
__device__ __forceinline__ float near_cap(float x, const ScoreRule& r) {
    const float u = x * x;
    return fmaf(u, fmaf(u, fmaf(u, fmaf(u, r.near[4], r.near[3]), r.near[2]), r.near[1]), r.near[0]);
}
__device__ __forceinline__ float capped(float x, const ScoreRule& r) {
    float far = r.cap2 * fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + exp2_hw(x)), 1.f), near = x * near_cap(x, r);
    asm volatile("" : "+v"(far), "+v"(near));   // a selection, not a branch for each score
    return fabsf(x) <= kNearCap ? near : far;
}
// Several at once: the polynomial alone where the wave has no others.
template <int N, typename X>
__device__ __forceinline__ void cap_several(X& x, const ScoreRule& r) {
    float largest = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) largest = fmaxf(largest, fabsf(x[i]));
    if (__ballot(largest > kNearCap) == 0) {    // uniform
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= near_cap(x[i], r);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = capped(x[i], r);
    }
}
template <int N> __device__ __forceinline__ void cap_all(float (&x)[N], const ScoreRule& r) { cap_several<N>(x, r); }
template <typename V> __device__ __forceinline__ void cap_scores(V& x, const ScoreRule& r) { cap_several<16>(x, r); }       // v16f

}  // namespace ffd
