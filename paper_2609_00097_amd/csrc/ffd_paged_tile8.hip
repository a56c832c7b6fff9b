// Attention of chunks of new tokens over a paged 8-bit cache for gfx950 (ffd_paged_tile.hip is the same over bf16): tiles of 256
// query rows of a KV head, for which the cache's tokens are staged in LDS, 64 at a time, as bf16.
//
// Mapping, phases and LDS layout are those of ffd_prefix.hip with eight row groups: wave w holds rows 32 w .. 32 w + 31; S^T = K Q^T
// by v_mfma_f32_32x32x16_bf16, lane (n, h) = (lane & 31, lane >> 5) with row n and tokens 8 a + 4 h + i (a, i = 0 .. 3) of each 32,
// which are its contraction indices in O^T = V^T P^T; two teams of four waves, one wave of each on every SIMD, are one phase
// apart, so that one's matrix instructions run beside the other's softmax and staging. Codes take registers on their way, which
// the order of the bf16 kernel does not have.
//
// Probabilities are multiplied by M / 127 of their value and enter the second product in two bf16 parts, hi + lo: rounded to 2^-16. One
// part (2^-8) does not average out where one token has most of the weight or equal scores meet equal M, and the bf16 kernel's remedy, a
// row divided by the sum of what the rounded ones stand for, takes 127 / M of every token here and as much time: a prompt of 8K, eight
// KV heads of four, 724 us with one part, 866 with that divisor, 877 with two; two of 4K in a window of 1024 under a cap 315, 357 and 338.
//
// Pages: 16 tokens lie together, so a thread's load is one page's, whose entry is read a tile ahead; codes of pages that are not
// there, and behind what any query sees, have M = 0.
//
// Bound: the phases' instructions, matrix and softmax ones in turn on each SIMD: a prompt of 8K 859 to 877 us (0.64 PFLOP/s of the
// operator's products), 512 tokens on 32K 421 to 435 us.
#include "ffd_paged.h"
#include "ffd_tile.h"

namespace ffd {

namespace {

constexpr int kTThreads = kChunkTileThreads;
constexpr int kTeam = kTThreads / 2;
constexpr int kTokens = 64;                     // tokens of a tile
constexpr int kShift = kChunkTileShift;
constexpr int kPart = kTokens / 2;              // tokens that a team stages
static_assert(kTokens == 1 << kShift);

struct TileLds {
    alignas(16) uint8_t keys[2][kTokens * 2 * kD];
    alignas(16) uint8_t values[2][kTokens * 2 * kD];
    alignas(16) float km[4][kTokens];           // 8 bits: M / 127 of keys and values
    alignas(16) float vm[4][kTokens];
    int nonfinite[4];                           // last tile with this index mod 4 that has an infinity or NaN as value
};

// A tile's place and pages: the rows of this team's two 16-token groups, and which of the tile's four are there.
struct TileAt {
    int t0;
    uint32_t there;
    size_t row[2];
};

// A team's half of a tile on its way from memory to LDS, in registers.
struct Staged {
    v4u k, v;
    uint32_t m;                                 // absmax of a key (threads below kPart) or value (the next kPart)
    __device__ __forceinline__ void load(v4u& x, const uint8_t* from, const TileAt& at, int id) {
        const size_t row = (id >> 7 ? at.row[1] : at.row[0]) + ((id >> 3) & 15);
        x = *reinterpret_cast<const v4u*>(from + row * kD + 16 * (id & 7));
    }
    __device__ __forceinline__ void load_keys(const KvSource& kv, const TileAt& at, int id) {
        load(k, kv.k, at, id);
        m = 0;                                  // the values' absmaxes come with the keys: they are needed with the scores
        if (id < 2 * kPart) {
            const int t = id & (kPart - 1);
            m = (id < kPart ? kv.k_absmax : kv.v_absmax)[(t >> 4 ? at.row[1] : at.row[0]) + (t & 15)];
        }
    }
    __device__ __forceinline__ void load_values(const KvSource& kv, const TileAt& at, int id) { load(v, kv.v, at, id); }
    static __device__ __forceinline__ void expand(uint8_t* tile, int row, int c, bool keys, const v4u& w) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int at = keys ? key_chunk(row, c + x) : value_chunk<true>(row, c + x);
            *reinterpret_cast<v8bf*>(tile + row * (2 * kD) + 16 * at) = expand8(w[2 * x], w[2 * x + 1]);
        }
    }
    __device__ __forceinline__ void store_keys(TileLds& lds, int u, const TileAt& at, int end, int part, int id) const {
        expand(lds.keys[u & 1], kPart * part + (id >> 3), 2 * (id & 7), true, k);
        if (id < 2 * kPart) {
            const int t = kPart * part + (id & (kPart - 1));
            const bool alive = (at.there >> (t >> 4) & 1) && at.t0 + t < end;
            const float x = alive ? bf16_to_f32((uint16_t)m) * (1.f / 127.f) : 0.f;
            const bool finite = fabsf(x) < INFINITY;
            if (id < kPart) {
                lds.km[u & 3][t] = x;
            } else {
                lds.vm[u & 3][t] = finite ? x : 0.f;
                if (!finite) lds.nonfinite[u & 3] = u;
            }
        }
    }
    __device__ __forceinline__ void store_values(TileLds& lds, int u, const TileAt&, int, int part, int id) const {
        expand(lds.values[u & 1], kPart * part + (id >> 3), 2 * (id & 7), false, v);
    }
};

// What a lane's row sees of a tile, token c of the tile counted from 4 h: c <= high and c > low, or c < prefix.
struct Limits {
    int high, low, prefix;
};

// Infinities and NaN among the values of tile [t0, t0 + kTokens), which are zeros in LDS: added to the rows that see them.
__device__ __forceinline__ void add_nonfinite(v16f (&o)[4], const ChunkAttendArgs& a, const ChunkItem& it, int t0, int end, const Limits& see, int h) {
#pragma unroll 1
    for (int t = 0; t < kTokens && t0 + t < end; ++t) {
        const int entry = page_entry(a.pages, it.b, t0 + t);
        if (!page_there(a.pages, entry)) continue;
        const size_t at = page_row(a.pages, a.Hkv, it.kvh, entry, t0 + t);
        const float x = bf16_to_f32(a.pages.kv.v_absmax[at]);
        const int c = t - 4 * h;
        const bool seen = (c <= see.high && c > see.low) || c < see.prefix;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] += !(fabsf(x) < INFINITY) && seen ? x : 0.f;
    }
}

}  // namespace

template <bool RULED>
__global__ __launch_bounds__(kTThreads, 2) void chunk_tile8_kernel(ChunkAttendArgs a) {
    __shared__ TileLds lds;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int n = lane & 31, h = lane >> 5;
    ChunkItem it;
    if (!chunk_item<kChunkTileRows, kShift>(a, blockIdx.x, lane, it)) return;
    const int team = wave >> 2, part = team, id = tid & (kTeam - 1);
    const int gs = __builtin_ctz(a.G), step = kChunkTileRows >> gs, tok0 = it.tile * step;
    const int tok1 = min(tok0 + step, it.seq.n) - 1, live_rows = (tok1 - tok0 + 1) << gs;
    const int hq0 = it.kvh * a.G, place = it.seq.L - it.seq.n, cached = min(it.seq.L, a.Lcap);
    write_record(a, it, tok0, live_rows);
    const ChunkSpan span = chunk_span<kShift>(a, it.seq, tok0, tok1);
    const int first = (int)((long long)span.count * it.run / it.cuts), last = (int)((long long)span.count * (it.run + 1) / it.cuts);

    // this lane's row
    const int r = 32 * wave + n;
    const bool live = r < live_rows;
    const int tok = tok0 + (min(r, live_rows - 1) >> gs), head = hq0 + (r & (a.G - 1));
    const size_t row_at = (size_t)(it.seq.q0 + tok) * a.Hq + head;
    const int at = place + tok;
    v8bf q[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        const v4u x = *reinterpret_cast<const v4u*>(a.q + row_at * kD + 16 * s + 8 * h);
        q[s] = __builtin_bit_cast(v8bf, live ? x : v4u{0, 0, 0, 0});
    }
    const ScoreRule rule = score_rule(a, true, head);
    const float zscale = RULED ? 1.f : a.scale * kLog2e;               // of what the maximum is taken of
    // the wave's first and last place, and the tile from which on none of its rows sees a token
    const bool any_row = 32 * wave < live_rows;
    const int low = place + tok0 + ((32 * wave) >> gs), high = place + min(tok0 + ((32 * wave + 31) >> gs), tok1);
    const int wave_end = any_row ? max(min(max(high + 1, it.seq.pre), cached), 0) : 0;
    const int high_block = (wave_end + kTokens - 1) >> kShift;
    const int mine_last = max(first, min(last, high_block <= span.prefix ? high_block : max(high_block - span.skip, span.prefix)));

    if (tid < 4) lds.nonfinite[tid] = -1;
    v16f o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    // pages: the entries of a tile's four groups lie in the lanes, two tiles ahead of the loads by them
    auto token0 = [&](int u) { return span.block(min(u, last - 1)) << kShift; };
    auto load_entries = [&](int u) { return page_entry(a.pages, it.b, token0(u) + 16 * (lane & 3)); };
    uint32_t ring = 0;                          // four bits a tile, which groups are there, by its number mod 4
    auto place_of = [&](int u, int entries) {
        TileAt x;
        x.t0 = token0(u);
        x.there = (uint32_t)__ballot(page_there(a.pages, entries)) & 15u;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int e = __builtin_amdgcn_readlane(entries, 2 * part + j);
            x.row[j] = page_row(a.pages, a.Hkv, it.kvh, page_there(a.pages, e) ? e : 0, x.t0 + 16 * (2 * part + j));
        }
        const int s = 4 * (u & 3);
        ring = (ring & ~(15u << s)) | x.there << s;
        return x;
    };

    // this lane's places in a tile: its key row's chunk for step 0, and its piece of a transposing read of dims 0 .. 31
    const uint32_t k_at = n * (2 * kD) + 16 * key_chunk(n, h);
    const int i16 = lane & 15;
    const int v_row = 4 * h + (i16 >> 2), v_c = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
    const uint32_t v_at = v_row * (2 * kD) + 16 * value_chunk<true>(v_row, v_c) + 8 * (i16 & 1);

    v16f s[2];
    v8bf p[4], p_low[4];
    auto value_operand = [&](const uint8_t* values, int y, int d) {
        v4s v[2];
#pragma unroll
        for (int z = 0; z < 2; ++z)
            v[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(
                values + (v_at ^ (d << 6) ^ (z << 5)) + (16 * y + 8 * z) * 2 * kD));
        return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // s = K Q^T of tile u; the next four key operands are on their way from LDS while four are used
    v8bf kf[2][4];
    auto read_key_operands = [&](int u, int j) {
        const uint8_t* keys = lds.keys[u & 1];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            kf[j & 1][e] = *reinterpret_cast<const v8bf*>(keys + ((k_at ^ (((j & 1) * 4 + e) << 5)) + (j >> 1) * 32 * 2 * kD));
    };
    auto scores = [&](int u) {
#pragma unroll
        for (int j = 1; j < 5; ++j) {
            if (j < 4) read_key_operands(u, j);
            __builtin_amdgcn_sched_barrier(0);
            const int x = (j - 1) >> 1, k = (j - 1) & 1;
            if (k == 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k][e], q[4 * k + e], s[x], 0, 0, 0);
        }
    };
    auto read_scales = [&](v4f (&x)[2][4], const float* from) {
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int b = 0; b < 4; ++b) x[y][b] = *reinterpret_cast<const v4f*>(from + 32 * y + 8 * b + 4 * h);
    };
    auto limits = [&](int t0) {
        Limits see;
        const int rel = at - t0 - 4 * h, behind = cached - t0 - 4 * h;
        see.high = min(rel, behind - 1);
        see.low = a.window > 0 ? rel - a.window : INT32_MIN;
        see.prefix = min(it.seq.pre - t0 - 4 * h, behind);
        return see;
    };

    // p = the probabilities of tile u against the maximum m, which follows the running one; their sum into l.
    auto softmax = [&](int u) {
        const int t0 = token0(u);
        const uint32_t there = ring >> (4 * (u & 3)) & 15u;
        v4f scales[2][4];
        read_scales(scales, lds.km[u & 3]);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[x][i] *= scales[x][i >> 2][i & 3];
        if constexpr (RULED) {
            const float scale = rule.zscale * 127.f;                            // 1 / 127 is in the scales here
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[x][i] *= scale;
            if (rule.cap2 != 0.f) {
#pragma unroll
                for (int x = 0; x < 2; ++x) cap_scores(s[x], rule);
            }
            if (a.slopes) {
                const float rel = (float)(at - t0 - 4 * h);
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[x][i] = fmaf(-rule.slope2, fabsf(rel - (float)(32 * x + 8 * (i >> 2) + (i & 3))), s[x][i]);
            }
        }
        const bool behind = t0 + kTokens <= low + 1 && (a.window <= 0 || t0 > high - a.window);
        bool any = true;
        if (!((behind || t0 + kTokens <= it.seq.pre) && t0 + kTokens <= cached && there == 15u)) {
            const Limits see = limits(t0);
            uint32_t some = 0;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int c = 32 * x + 8 * (i >> 2) + (i & 3);
                    const uint32_t seen = (uint32_t)(((c <= see.high) & (c > see.low)) | (c < see.prefix)) & (there >> (2 * x + (i >> 3)));
                    s[x][i] = seen & 1 ? s[x][i] : -INFINITY;
                    some |= seen;
                }
            any = halves_max(some & 1 ? 1.f : 0.f) > 0.f;
        }
        float mx[4];                                    // four chains, as for the sum below
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[i] = s[0][i];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx[i & 3] = fmaxf(mx[i & 3], s[x][i]);
        const float top = halves_max(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]))) * zscale;
        const bool up = any && (m == -INFINITY || !(top <= m + kSlack));                // NaN: up
        if (__ballot(up) != 0) {
            const float mn = up ? fmaxf(fmaxf(m, top), -FLT_MAX) : m;                   // finite once a token is seen
            const float corr = mn == m ? 1.f : exp2_hw(m - mn);
            m = mn;
            l *= corr;
#pragma unroll
            for (int d = 0; d < 4; ++d) o[d] *= corr;
        }
        const float m0 = m == -INFINITY ? 0.f : m;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        read_scales(scales, lds.vm[u & 3]);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float e[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                e[i] = exp2_hw(fmaf(s[x][i], zscale, -m0));
                sum[i & 3] += e[i];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) e[i] *= scales[x][i >> 2][i & 3];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                uint32_t w[4], low[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    w[k] = pack_bf16(e[8 * y + 2 * k], e[8 * y + 2 * k + 1]);
                    low[k] = pack_bf16(e[8 * y + 2 * k] - bf16_lo(w[k]), e[8 * y + 2 * k + 1] - bf16_hi(w[k]));
                }
                p[2 * x + y] = __builtin_bit_cast(v8bf, v4u{w[0], w[1], w[2], w[3]});
                p_low[2 * x + y] = __builtin_bit_cast(v8bf, v4u{low[0], low[1], low[2], low[3]});
            }
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    // o += V^T P^T of tile u, and the infinities and NaN among its values
    auto products = [&](int u) {
        const uint8_t* values = lds.values[u & 1];
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const v8bf v = __builtin_bit_cast(v8bf, value_operand(values, y, d));
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[y], o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p_low[y], o[d], 0, 0, 0);
            }
    };
    auto nonfinite = [&](int u) {
        if (__builtin_amdgcn_readfirstlane(lds.nonfinite[u & 3]) == u) {
            const int t0 = token0(u);
            add_nonfinite(o, a, it, t0, span.end, limits(t0), h);
        }
    };

    __syncthreads();
    if (first < last) {
        Staged st, head_keys;
        const int e0 = load_entries(first), e1 = load_entries(first + 1);
        int entries = load_entries(first + 2);
        TileAt before = place_of(first, e0), now = before;
        head_keys.load_keys(a.pages.kv, now, id);
        st.load_values(a.pages.kv, now, id);
        now = place_of(first + 1, e1);
        st.load_keys(a.pages.kv, now, id);
        head_keys.store_keys(lds, first, before, span.end, part, id);
        // this team's half of the keys of tile u and the values of u - 1 to LDS; those after them are asked for. Behind the
        // run's end its last tile is staged again.
        auto stage = [&](int u) {
            st.store_keys(lds, u, now, span.end, part, id);
            st.store_values(lds, u - 1, before, span.end, part, id);
            before = now;
            now = place_of(u + 1, entries);
            entries = load_entries(u + 2);
            st.load_keys(a.pages.kv, now, id);
            st.load_values(a.pages.kv, before, id);
        };
        __syncthreads();
        if (team == 1) {
            stage(first + 1);
            __syncthreads();
        }
        // a tile's two phases: scores after the products of the tile before, then softmax
        auto vector_phase = [&](int u) {
            __syncthreads();
            softmax(u);
            stage(u + 1 + team);
            __syncthreads();
        };
        if (first < mine_last) {
            read_key_operands(first, 0);
            scores(first);
            vector_phase(first);
            for (int u = first + 1; u < mine_last; ++u) {
                read_key_operands(u, 0);
                products(u - 1);
                scores(u);
                nonfinite(u - 1);
                vector_phase(u);
            }
            products(mine_last - 1);
            nonfinite(mine_last - 1);
        }
        for (int u = mine_last; u <= last; ++u) {
            __syncthreads();
            if (u < last) stage(u + 1 + team);
            __syncthreads();
        }
        if (team == 0) __syncthreads();
    }

    l = halves_sum(l);
    if (!live) return;
    const float ln = m * 0.69314718055994531f;
    if (it.part >= 0) {
        const size_t to = (size_t)it.part * kChunkTileRows + r;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<float4*>(a.parts.acc + to * kD + 32 * d + 8 * b + 4 * h) =
                    make_float4(o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]);
        if (h == 0) {
            a.parts.m[to] = ln;
            a.parts.l[to] = l;
        }
        return;
    }
    const bool any = m != -INFINITY;
    const float inv = any ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const uint2 w = make_uint2(pack_bf16(o[d][4 * b] * inv, o[d][4 * b + 1] * inv), pack_bf16(o[d][4 * b + 2] * inv, o[d][4 * b + 3] * inv));
            *reinterpret_cast<uint2*>(a.out + row_at * kD + 32 * d + 8 * b + 4 * h) = any ? w : make_uint2(0u, 0u);
        }
    if (h == 0 && a.lse) a.lse[row_at] = any ? ln + logf(l) : -INFINITY;
}

template __global__ void chunk_tile8_kernel<false>(ChunkAttendArgs);
template __global__ void chunk_tile8_kernel<true>(ChunkAttendArgs);

}  // namespace ffd
