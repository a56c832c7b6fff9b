// A batch's attention over its shared prefix for gfx950, for more than 32 query rows per KV head (ffd_attend.h has
// the mathematics; ffd_attend.hip serves fewer rows and short prefixes): tokens staged in LDS once for all rows of a
// workgroup.
//
// Bound. A prefix token costs 512 bytes (8 bits: 260) and 768 operations per query row, 256 of them for the second part
// of its probability: up to about 128 rows HBM's, beyond them the matrix cores'. Next to these, a score costs about ten
// VALU slots (scale and subtract, exponential, maximum, sum, two conversions), as much time as its matrix instructions.
// Measured, by the card, eight KV heads, of which about 13 us are the start, the join of the token groups and the partial
// rows: in bf16, 64 rows on 80K tokens 67 to 69 us (4.9 TB/s), on 64K 128 rows 66 to 71 (4.0 TB/s), 256 105 to 110 (960
// TFLOP/s, the second part's included), 512 201 to 239 as the clock allows (1020 to 860); in 8 bits, on 128K 64 rows 76 to
// 81 us (3.5 TB/s), 128 122 to 130 (840 to 790 TFLOP/s), on 64K 256 rows 116 to 124 (890 to 830).
//
// Mapping. Eight waves: RW row groups of 32 query rows by 8 / RW token groups. Scores are computed transposed by
// v_mfma_f32_32x32x16_bf16, S^T = K Q^T: lane (n, h) = (lane & 31, lane >> 5) holds, of query row n, tokens
// 8 a + 4 h + i (a, i = 0 .. 3) of a 32-token tile, which are just the contraction indices it has to hold of P^T in
// O^T = V^T P^T: the probabilities never leave their registers, and maximum, sum and rescaling are per lane. V^T
// comes out of LDS by transposing reads (a 16-lane group gets, of four rows of 16 values, four of one column each).
// Rows of 256 bytes lie in LDS as 16-byte chunks in an order that depends on the row (xor), so that the lanes of a
// read, which all read the same columns of different rows, spread over the banks.
//
// 8-bit codes become bf16 integers on their way into LDS; M / 127 of a key multiplies its score, that of a value its
// probability. The maximum that the exponents are taken against follows the running one only when that has grown by
// 2^8, so that the accumulators are rarely rescaled.
//
// Probabilities are given to the instruction in two bf16 parts, p = hi + lo, as for small tiles: rounded to 2^-16, so that
// a result is as exact, and the same but for the order of sums, whatever number of rows it is computed with. One part
// (2^-8) would save 8 us of 66 for 128 rows, 17 of 105 for 256, 8 of 76 for 64 in 8 bits, but its error does not average
// out where many scores are equal, or where one token has most of the weight and the exponents' reference lags behind its
// score: up to 2^-8 of the values, as much again as the rounding of the output.
//
// Three ways to keep a CU's SIMDs, two waves each, on loads, matrix and vector instructions at once, by what there is
// most of. bf16, 64 rows (the plain loop): the loads; every wave does all there is to do to a tile, then stages its
// part of the next, one barrier a tile. 8 bits, 64 and 128 rows (roles): the conversion of the codes; four waves, one on
// each SIMD, stage, the others attend (64 rows on 128K tokens, probabilities in one part: 75 us in phases, 68 so). All
// else: phases.
//
// Phases. A tile has a matrix phase (the values' product of the tile before, then this one's scores) and a vector
// phase (softmax; staging), each closed by a barrier. The two teams of four waves, one wave of each on every SIMD, are
// one phase apart, so that one's matrix instructions and LDS reads run beside the other's vector instructions. In
// phase number 2 u, team 0 has the matrix phase of tile u and team 1 the vector phase of tile u - 1; in 2 u + 1 team 0
// the vector phase of u, team 1 the matrix phase of u. The keys of tile u are read in phases 2 u and 2 u + 1, its
// values in 2 u + 2 and 2 u + 3. Each team stages half of the rows in its vector phases: team 1 the keys of tile u + 1
// and the values of u in phase 2 u, team 0 the same in 2 u + 1, which is after the last read of tiles u - 1 and u - 2,
// whose places they take, and before their first use. The loads for them are issued one vector phase earlier.
#include "ffd_tile.h"

namespace ffd {

namespace {

constexpr int kPThreads = kPrefixTileThreads;

template <int RW, bool I8>
struct PrefixShape {
    static constexpr bool kRoles = I8 && RW <= 4;                       // waves 4 .. 7 stage, waves 0 .. 3 do the rest
    static constexpr bool kPhased = RW > 2 && !kRoles;
    static constexpr int kMathWaves = kRoles ? 4 : 8;
    static constexpr int kTokenGroups = kMathWaves / RW;
    static constexpr int kSub = kRoles || kPhased ? 2 : 1;              // 32-token tiles of a wave
    static constexpr int kTokens = 32 * kSub * kTokenGroups;            // tokens of a tile of the workgroup
    static constexpr int kRows = 32 * RW;
    static constexpr int kBytes = kTokens * 2 * kD;                     // of a tile's keys, or values, in LDS
    static constexpr int kParts = kRoles ? 1 : 2;                       // teams that stage a tile
    static constexpr int kPartTokens = kTokens / kParts;
    static constexpr int kLoads = kPartTokens / 16;                     // 16-byte chunks of bf16 keys per thread
};
constexpr int kTeam = kPThreads / 2;           // threads of a team, four waves
constexpr int kJoinPad = kD + 4;

template <int RW, bool I8>
struct PrefixLds {
    using Sh = PrefixShape<RW, I8>;
    union {
        struct {
            alignas(16) uint8_t keys[2][Sh::kBytes];
            alignas(16) uint8_t values[2][Sh::kBytes];
        };
        float join[Sh::kTokenGroups > 1 ? Sh::kRows : 1][kJoinPad];
    };
    alignas(16) float km[4][Sh::kTokens];                               // 8 bits: M / 127 of keys and values
    alignas(16) float vm[4][Sh::kTokens];
    int nonfinite[4];                          // last tile with this index mod 4 that has an infinity or NaN as value
    int longest[8];                            // each wave's; apart from m, which a run without tiles writes next, no barrier between
    float m[8][32], l[8][32];
};

// A team's part of a tile on its way from memory to LDS, in registers: rows [part kPartTokens, ..) of the tile. `last` is
// the last row of the tile that any query sees; rows behind it repeat it.
template <int RW, bool I8> struct Staged;
template <int RW> struct Staged<RW, false> {
    using Sh = PrefixShape<RW, false>;
    v4u k[Sh::kLoads], v[Sh::kLoads];
    static __device__ __forceinline__ int row_of(int j, int part, int id) { return part * Sh::kPartTokens + (id >> 4) + j * (kTeam / 16); }
    static __device__ __forceinline__ void load(v4u (&x)[Sh::kLoads], const uint8_t* from, int t0, int last, int part, int id) {
        const uint8_t* base = from + (size_t)t0 * (2 * kD);
#pragma unroll
        for (int j = 0; j < Sh::kLoads; ++j)
            x[j] = *reinterpret_cast<const v4u*>(base + (uint32_t)min(row_of(j, part, id), last) * (2 * kD) + 16 * (id & 15));
    }
    __device__ __forceinline__ void load_keys(const KvSource& kv, int t0, int last, int part, int id) { load(k, kv.k, t0, last, part, id); }
    __device__ __forceinline__ void load_values(const KvSource& kv, int t0, int last, int part, int id) { load(v, kv.v, t0, last, part, id); }
    __device__ __forceinline__ void store_keys(PrefixLds<RW, false>& lds, int u, int, int part, int id) const {
#pragma unroll
        for (int j = 0; j < Sh::kLoads; ++j) {
            const int row = row_of(j, part, id);
            *reinterpret_cast<v4u*>(&lds.keys[u & 1][row * (2 * kD) + 16 * key_chunk(row, id & 15)]) = k[j];
        }
    }
    __device__ __forceinline__ void store_values(PrefixLds<RW, false>& lds, int u, int part, int id) const {
#pragma unroll
        for (int j = 0; j < Sh::kLoads; ++j) {
            const int row = row_of(j, part, id);
            v4u x = v[j];
            const uint32_t big = pk_max_u16(pk_max_u16(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), pk_max_u16(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
            if (max(big & 0xffffu, big >> 16) >= 0x7f80u) {
                lds.nonfinite[u & 3] = u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t lo = (x[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu, hi = (x[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u;
                    x[i] &= lo | hi;
                }
            }
            *reinterpret_cast<v4u*>(&lds.values[u & 1][row * (2 * kD) + 16 * value_chunk<false>(row, id & 15)]) = x;
        }
    }
};
template <int RW> struct Staged<RW, true> {
    using Sh = PrefixShape<RW, true>;
    static constexpr int kLoads = Sh::kLoads / 2;
    static constexpr int kScales = Sh::kPartTokens;
    static_assert(2 * kScales <= kTeam, "one absmax per thread");
    v4u k[kLoads], v[kLoads];
    uint32_t m;                                 // absmax of a key (threads below kScales) or value (the next kScales)
    static __device__ __forceinline__ int row_of(int j, int part, int id) { return part * Sh::kPartTokens + (id >> 3) + j * (kTeam / 8); }
    static __device__ __forceinline__ void load(v4u (&x)[kLoads], const uint8_t* from, int t0, int last, int part, int id) {
        const uint8_t* base = from + (size_t)t0 * kD;
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            x[j] = *reinterpret_cast<const v4u*>(base + (uint32_t)min(row_of(j, part, id), last) * kD + 16 * (id & 7));
    }
    static __device__ __forceinline__ void expand(uint8_t* tile, int row, int c, bool keys, const v4u& w) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int at = keys ? key_chunk(row, c + x) : value_chunk<true>(row, c + x);
            *reinterpret_cast<v8bf*>(tile + row * (2 * kD) + 16 * at) = expand8(w[2 * x], w[2 * x + 1]);
        }
    }
    __device__ __forceinline__ void load_keys(const KvSource& kv, int t0, int last, int part, int id) {
        load(k, kv.k, t0, last, part, id);
        m = 0;                                  // the values' absmaxes come with the keys: they are needed with the scores
        if (id < 2 * kScales)
            m = (id < kScales ? kv.k_absmax : kv.v_absmax)[(size_t)t0 + min(part * kScales + (id & (kScales - 1)), last)];
    }
    __device__ __forceinline__ void load_values(const KvSource& kv, int t0, int last, int part, int id) { load(v, kv.v, t0, last, part, id); }
    __device__ __forceinline__ void store_keys(PrefixLds<RW, true>& lds, int u, int last, int part, int id) const {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) expand(lds.keys[u & 1], row_of(j, part, id), 2 * (id & 7), true, k[j]);
        if (id < 2 * kScales) {
            const int t = part * kScales + (id & (kScales - 1));
            const float x = t <= last ? bf16_to_f32((uint16_t)m) * (1.f / 127.f) : 0.f;
            const bool finite = fabsf(x) < INFINITY;
            if (id < kScales) {
                lds.km[u & 3][t] = x;
            } else {
                lds.vm[u & 3][t] = finite ? x : 0.f;
                if (!finite) lds.nonfinite[u & 3] = u;
            }
        }
    }
    __device__ __forceinline__ void store_values(PrefixLds<RW, true>& lds, int u, int part, int id) const {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) expand(lds.values[u & 1], row_of(j, part, id), 2 * (id & 7), false, v[j]);
    }
};

// Infinities and NaN among the values of tokens [begin, end), which are zeros in LDS (zero times infinity would reach
// rows that do not see the token): added to the rows that see them. An absmax that is NaN makes a whole row NaN.
template <bool I8>
__device__ __forceinline__ void add_nonfinite(v16f (&o)[4], const KvSource& kv, int begin, int end, int lim, int h) {
#pragma unroll 1
    for (int t = begin; t < end; ++t) {
        const uint16_t* row = I8 ? kv.v_absmax + t : reinterpret_cast<const uint16_t*>(kv.v) + (size_t)t * kD + 4 * h;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = bf16_to_f32(row[I8 ? 0 : 32 * d + 8 * (i >> 2) + (i & 3)]);
                o[d][i] += !(fabsf(x) < INFINITY) && t < lim ? x : 0.f;
            }
    }
}

// Sequences that use different parts of the prefix, in order of their lengths: then the waves of a tile end together
// and a tile is as long as its own sequences need. The tiles get workgroups by their lengths. Computed by every
// workgroup alone; `writes`: this one leaves the places for the merge. False, and nothing changed, where all
// lengths are equal; else lds.vm holds the order, tile is this workgroup's (-1: none) and mine its tile's workgroups.
template <int RW, bool I8>
__device__ __forceinline__ bool sort_by_length(const PrefixArgs& a, PrefixLds<RW, I8>& lds, bool writes, int w, int& tile, PrefixPlace& mine) {
    static_assert(sizeof(lds.km) >= kPrefixSortSeqs * sizeof(int) && sizeof(lds.vm) >= kPrefixSortSeqs * sizeof(int));
    const int tid = threadIdx.x;
    int* lens = reinterpret_cast<int*>(lds.km);
    int* order = reinterpret_cast<int*>(lds.vm);
    auto clamped = [&](int x) { return min(max(x, 0), a.Pcap); };
    const int len = clamped(a.prefix_lens[min(tid, a.B - 1)]), len0 = clamped(a.prefix_lens[0]);
    if (tid < kPrefixSortSeqs) lens[tid] = tid < a.B ? len : -1;
    const bool differ = __syncthreads_or(len != len0);
    int place = tid;
    if (differ) {
        place = 0;
        for (int j = 0; j < a.B; j += 4) {              // lens is padded with -1
            const int4 x = *reinterpret_cast<const int4*>(lens + j);
            place += (x.x > len) | (x.x == len & j < tid);
            place += (x.y > len) | (x.y == len & j + 1 < tid);
            place += (x.z > len) | (x.z == len & j + 2 < tid);
            place += (x.w > len) | (x.w == len & j + 3 < tid);
        }
        if (tid < a.B) order[place] = tid;
        __syncthreads();
    }
    const int step = PrefixShape<RW, I8>::kRows / a.G;      // sequences per tile, the first of them the longest
    if (!differ) {
        if (writes && tid < a.B) a.places[tid] = PrefixPlace{tid / step, a.tiles, a.S, tid};
        return false;
    }
    // one workgroup for every tile that has tokens, the others in proportion to the tiles' units
    long long all = 0;
    int used = 0;
    for (int t = 0; t < a.tiles; ++t) {
        const int units = (lens[order[t * step]] + PrefixShape<RW, I8>::kTokens - 1) / PrefixShape<RW, I8>::kTokens;
        all += units;
        used += units > 0;
    }
    const long long spare = (long long)a.S * a.tiles - used;
    tile = -1;
    int first = 0;
    for (int t = 0; t < a.tiles; ++t) {
        const int units = (lens[order[t * step]] + PrefixShape<RW, I8>::kTokens - 1) / PrefixShape<RW, I8>::kTokens;
        const int count = units > 0 ? 1 + (int)((double)(units * spare) / (double)all) : 0;
        if (writes && tid < a.B && place / step == t) a.places[tid] = PrefixPlace{first, 1, count, place};
        if (w >= first && w < first + count) {
            tile = t;
            mine = PrefixPlace{first, 1, count, 0};
        }
        first += count;
    }
    tile = __builtin_amdgcn_readfirstlane(tile);
    return true;
}

}  // namespace

template <int RW, bool I8>
__global__ __launch_bounds__(kPThreads, 2) void prefix_tile_kernel(PrefixArgs a) {
    using Sh = PrefixShape<RW, I8>;
    constexpr bool kGuess = RW < 8 && !I8;      // 256 rows: the runs may follow the lengths; 8 bits: no registers to spare
    __shared__ PrefixLds<RW, I8> lds;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int n = lane & 31, h = lane >> 5;
    const int rg = wave % RW, tg = wave % Sh::kMathWaves / RW;
    // Workgroups of one run but different tiles read the same tokens: they are eight apart, on one XCD (consecutive
    // workgroups go to the eight XCDs in turn). Where sequences are sorted by length the tiles have runs of their own, and
    // each XCD reads what its workgroups need (two tiles, of which the second ends at half of 268 MB: 404 MB).
    const int slot = (int)(blockIdx.x >> 3) % a.tiles;
    const int pair = (int)(blockIdx.x >> 3) / a.tiles * 8 + (int)(blockIdx.x & 7);
    if (pair >= a.Hkv * a.S) return;
    const int kvh = pair / a.S, w = pair % a.S * a.tiles + slot;        // workgroup w of this KV head
    const int rows = a.B * a.G, gs = __builtin_ctz(a.G);
    PrefixPlace mine{slot, a.tiles, a.S, 0};
    int tile = slot;
    const size_t row0 = (size_t)kvh * a.Pcap, bytes = I8 ? kD : 2 * kD;
    const KvSource kv{a.kv.k + row0 * bytes, a.kv.v + row0 * bytes, I8 ? a.kv.k_absmax + row0 : nullptr,
                      I8 ? a.kv.v_absmax + row0 : nullptr};
    const int team = wave >> 2, part = Sh::kParts == 2 ? team : 0, id = tid & (kTeam - 1);
    // equal runs of whole tiles, the first ones one longer
    auto run_begin = [&](int tokens, int run, int S, int& count) {
        const int units = (tokens + Sh::kTokens - 1) / Sh::kTokens, each = units / S, more = units - each * S;
        count = each + (run < more);
        return each * run + min(run, more);
    };

    // queries and lengths, asked for together
    int r = tile * Sh::kRows + 32 * rg + n, b = min(r >> gs, a.B - 1);
    v4u qw[8];
    auto load_queries = [&]() {
        const uint16_t* qrow = a.q + ((size_t)b * a.Hq + kvh * a.G + (r & (a.G - 1))) * kD + 8 * h;
#pragma unroll
        for (int s = 0; s < 8; ++s) qw[s] = *reinterpret_cast<const v4u*>(qrow + 16 * s);
    };
    load_queries();
    int len = a.prefix_lens[b];
    if constexpr (RW == 8) {
        if (a.places && sort_by_length(a, lds, kvh == 0 && w == 0, w, tile, mine)) {
            if (tile < 0) return;                       // lengths leave this workgroup without work
            const int* order = reinterpret_cast<const int*>(lds.vm);
            r = tile * Sh::kRows + 32 * rg + n;
            b = order[min(r >> gs, a.B - 1)];
            load_queries();
            len = a.prefix_lens[b];
        }
    }
    // The first tile is asked for before the lengths are there, as it is if they are the capacity (whole calls in turn
    // on one card, four times: 32 sequences on 32K tokens 67.8 us with two dependent loads at the start, 66.4 so; 64 rows on
    // 96K 90.9 and 88.6).
    Staged<RW, I8> st, head;
    int guess = -1;
    if constexpr (kGuess) {
        int count;
        guess = run_begin(a.Pcap, pair % a.S, a.S, count);
        const int last = a.Pcap - 1 - guess * Sh::kTokens;
        if (count == 0 || last < Sh::kTokens - 1) guess = -1;
        const int u = max(guess, 0);
        head.load_keys(kv, u * Sh::kTokens, max(last, 0), part, id);
        if constexpr (!Sh::kPhased) head.load_values(kv, u * Sh::kTokens, max(last, 0), part, id);
    }
    const int run = (w - mine.first) / mine.stride, S = mine.count;
    const bool live = r < rows;
    if (tid < 4) lds.nonfinite[tid] = -1;
    v8bf q[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) q[s] = __builtin_bit_cast(v8bf, live ? qw[s] : v4u{0, 0, 0, 0});
    // longest use of the prefix among the workgroup's rows, and this wave's longest and shortest
    const int lim = live ? min(max(len, 0), a.Pcap) : 0;
    int longest = lim, shortest = live ? lim : INT32_MAX;
#pragma unroll
    for (int x = 16; x; x >>= 1) {
        longest = max(longest, __shfl_xor(longest, x));
        shortest = min(shortest, __shfl_xor(shortest, x));
    }
    longest = __builtin_amdgcn_readfirstlane(longest);
    shortest = __builtin_amdgcn_readfirstlane(shortest);
    if (lane == 0) lds.longest[wave] = longest;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) all = max(all, lds.longest[w]);
    all = __builtin_amdgcn_readfirstlane(all);
    int count;
    const int first = run_begin(all, run, S, count), last = first + count;
    const bool guessed = kGuess && guess == first && (first + 1) * Sh::kTokens <= all;      // uniform

    const float zscale = a.scale * kLog2e;
    v16f o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    // this lane's places in a tile: its key row's chunk for step 0, and its piece of a transposing read of dims 0 .. 31
    const int wave_row = tg * 32 * Sh::kSub;
    const uint32_t k_at = (wave_row + n) * (2 * kD) + 16 * key_chunk(n, h);
    const int i16 = lane & 15;
    const int v_row = 4 * h + (i16 >> 2), v_c = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
    const uint32_t v_at = (wave_row + v_row) * (2 * kD) + 16 * value_chunk<I8>(v_row, v_c) + 8 * (i16 & 1);

    v16f s[Sh::kSub];
    v8bf p[2 * Sh::kSub], lo[2 * Sh::kSub];
    auto first_token = [&](int u) { return u * Sh::kTokens + wave_row; };

    // With 32 tokens per wave there are registers to ask for a tile's first value operands with its scores; read where
    // they are used, they are another latency of LDS in the wave's chain.
    constexpr bool kEarly = Sh::kSub == 1;
    v4f km[Sh::kSub][4], vm[Sh::kSub][4];
    v8s head_values[4];
    int flag = 0;
    auto read_scales = [&](v4f (&x)[Sh::kSub][4], const float* from) {
#pragma unroll
        for (int y = 0; y < Sh::kSub; ++y)
#pragma unroll
            for (int b = 0; b < 4; ++b) x[y][b] = *reinterpret_cast<const v4f*>(from + wave_row + 32 * y + 8 * b + 4 * h);
    };
    auto value_operand = [&](const uint8_t* values, int y, int d) {
        v4s v[2];
#pragma unroll
        for (int z = 0; z < 2; ++z)
            v[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(
                values + (v_at ^ (d << 6) ^ (z << 5)) + (16 * y + 8 * z) * 2 * kD));
        return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    };

    // s = K Q^T of tile u; the next four key operands are on their way from LDS while four are used. The first four can
    // be asked for earlier.
    v8bf kf[2][4];
    auto read_key_operands = [&](int u, int j) {
        const uint8_t* keys = lds.keys[u & 1];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            kf[j & 1][e] = *reinterpret_cast<const v8bf*>(keys + ((k_at ^ (((j & 1) * 4 + e) << 5)) + (j >> 1) * 32 * 2 * kD));
    };
    auto scores = [&](int u) {
        if constexpr (kEarly) flag = lds.nonfinite[u & 3];
#pragma unroll
        for (int j = 1; j < 2 * Sh::kSub + 1; ++j) {
            if (j < 2 * Sh::kSub) read_key_operands(u, j);
            __builtin_amdgcn_sched_barrier(0);
            const int x = (j - 1) >> 1, k = (j - 1) & 1;
            if (k == 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k][e], q[4 * k + e], s[x], 0, 0, 0);
        }
        if constexpr (kEarly) {
#pragma unroll
            for (int d = 0; d < 4; ++d) head_values[d] = value_operand(lds.values[u & 1], 0, d);
        }
    };

    // p = the probabilities of tile u against the maximum m, which follows the running one; their sum into l.
    auto softmax = [&](int u) {
        const int w0 = first_token(u);
        if constexpr (I8) {
            read_scales(km, lds.km[u & 3]);
#pragma unroll
            for (int x = 0; x < Sh::kSub; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[x][i] *= km[x][i >> 2][i & 3];
        }
        if (w0 + 32 * Sh::kSub > shortest) {
            const int rel = lim - w0 - 4 * h;           // tokens 32 x + 8 b + i below it are seen
#pragma unroll
            for (int x = 0; x < Sh::kSub; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[x][i] = 32 * x + 8 * (i >> 2) + (i & 3) < rel ? s[x][i] : -INFINITY;
        }
        float mx[4];                                    // four chains, as for the sum below
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[i] = s[0][i];
#pragma unroll
        for (int x = 0; x < Sh::kSub; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx[i & 3] = fmaxf(mx[i & 3], s[x][i]);
        const float top = halves_max(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]))) * zscale;
        const bool up = w0 < lim && (m == -INFINITY || !(top <= m + kSlack));           // NaN: up
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
        if constexpr (I8) read_scales(vm, lds.vm[u & 3]);
#pragma unroll
        for (int x = 0; x < Sh::kSub; ++x) {
            float e[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                e[i] = exp2_hw(fmaf(s[x][i], zscale, -m0));
                sum[i & 3] += e[i];
            }
            if constexpr (I8) {
#pragma unroll
                for (int i = 0; i < 16; ++i) e[i] *= vm[x][i >> 2][i & 3];
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                uint32_t w[4], low[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float x0 = e[8 * y + 2 * k], x1 = e[8 * y + 2 * k + 1];
                    w[k] = pack_bf16(x0, x1);
                    low[k] = pack_bf16(x0 - bf16_lo(w[k]), x1 - bf16_hi(w[k]));
                }
                p[2 * x + y] = __builtin_bit_cast(v8bf, v4u{w[0], w[1], w[2], w[3]});
                lo[2 * x + y] = __builtin_bit_cast(v8bf, v4u{low[0], low[1], low[2], low[3]});
            }
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };

    // o += V^T P^T of tile u, and the infinities and NaN among its values.
    auto products = [&](int u) {
        const uint8_t* values = lds.values[u & 1];
#pragma unroll
        for (int y = 0; y < 2 * Sh::kSub; ++y)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const v8s f = y == 0 && kEarly ? head_values[d] : value_operand(values, y, d);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, f), p[y], o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, f), lo[y], o[d], 0, 0, 0);
            }
    };
    auto nonfinite = [&](int u) {
        if constexpr (!kEarly) flag = lds.nonfinite[u & 3];
        const int w0 = first_token(u);
        if (__builtin_amdgcn_readfirstlane(flag) == u) add_nonfinite<I8>(o, kv, w0, min(w0 + 32 * Sh::kSub, all), lim, h);
    };
    // the tile from which on this wave's rows see no token any more
    const int mine_last = max(first, min(last, (longest - wave_row + Sh::kTokens - 1) / Sh::kTokens));

    // Staging. Behind the run's end its last tile is staged again: with a branch around loads or stores the wait for
    // one tile's registers would fall on the next one's loads.
    auto last_row = [&](int u) { return all - 1 - u * Sh::kTokens; };
    auto load_keys = [&](Staged<RW, I8>& x, int u) { u = min(u, last - 1); x.load_keys(kv, u * Sh::kTokens, last_row(u), part, id); };
    auto load_values = [&](Staged<RW, I8>& x, int u) { u = min(u, last - 1); x.load_values(kv, u * Sh::kTokens, last_row(u), part, id); };
    auto store_keys = [&](const Staged<RW, I8>& x, int u) { x.store_keys(lds, u, last_row(min(u, last - 1)), part, id); };
    auto store_values = [&](const Staged<RW, I8>& x, int u) { x.store_values(lds, u, part, id); };
    if (first < last) {
        if constexpr (Sh::kRoles) {
            if (team == 1) {
                // two tiles under way, in turn in the two sets of registers
                auto refill = [&](Staged<RW, I8>& x, int u) {
                    store_keys(x, u);
                    store_values(x, u);
                    load_keys(x, u + 2);
                    load_values(x, u + 2);
                    __syncthreads();
                };
                load_keys(head, first);
                load_values(head, first);
                load_keys(st, first + 1);
                load_values(st, first + 1);
                refill(head, first);
                for (int u = first; u < last; u += 2) {
                    refill(st, u + 1);
                    if (u + 1 < last) refill(head, u + 2);
                }
            } else {
                __syncthreads();
                for (int u = first; u < mine_last; ++u) {
                    read_key_operands(u, 0);
                    scores(u);
                    softmax(u);
                    products(u);
                    nonfinite(u);
                    __syncthreads();
                }
                for (int u = mine_last; u < last; ++u) __syncthreads();
            }
        } else if constexpr (Sh::kPhased) {
            if (!guessed) load_keys(head, first);
            load_values(st, first);
            load_keys(st, first + 1);
            store_keys(head, first);
            // this team's half of the keys of tile u and the values of u - 1 to LDS; those after them are asked for
            auto stage = [&](int u) {
                store_keys(st, u);
                store_values(st, u - 1);
                load_keys(st, u + 1);
                load_values(st, u);
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
        } else {
            if (!guessed) {
                load_keys(head, first);
                load_values(head, first);
            }
            load_keys(st, first + 1);
            load_values(st, first + 1);
            store_keys(head, first);
            store_values(head, first);
            __syncthreads();
            for (int u = first; u < last; ++u) {
                if (u < mine_last) {
                    read_key_operands(u, 0);
                    scores(u);
                    softmax(u);
                    products(u);
                    nonfinite(u);
                }
                store_keys(st, u + 1);
                store_values(st, u + 1);
                load_keys(st, u + 2);
                load_values(st, u + 2);
                __syncthreads();
            }
        }
    }

    // token groups joined in LDS, then one partial row per query row
    l = halves_sum(l);
    const size_t out0 = ((size_t)kvh * a.S * a.tiles + w) * Sh::kRows;
    const bool math = wave < Sh::kMathWaves;
    if constexpr (Sh::kTokenGroups > 1) {
        if (h == 0) {
            lds.m[wave][n] = m;
            lds.l[wave][n] = l;
        }
        __syncthreads();
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int x = 0; x < Sh::kTokenGroups; ++x) M = fmaxf(M, lds.m[x * RW + rg][n]);
#pragma unroll
        for (int x = 0; x < Sh::kTokenGroups; ++x) {
            const float mx = lds.m[x * RW + rg][n];
            if (mx != -INFINITY) L = fmaf(exp2_hw(mx - M), lds.l[x * RW + rg][n], L);
        }
        const float f = m == -INFINITY ? 0.f : exp2_hw(m - M);
#pragma unroll
        for (int x = Sh::kTokenGroups - 1; x >= 0; --x) {
            if (math && tg == x) {
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        float4* at = reinterpret_cast<float4*>(&lds.join[32 * rg + n][32 * d + 8 * b + 4 * h]);
                        float4 y = make_float4(o[d][4 * b] * f, o[d][4 * b + 1] * f, o[d][4 * b + 2] * f, o[d][4 * b + 3] * f);
                        if (x < Sh::kTokenGroups - 1) {
                            const float4 z = *at;
                            y = make_float4(y.x + z.x, y.y + z.y, y.z + z.z, y.w + z.w);
                        }
                        *at = y;
                    }
            }
            __syncthreads();
        }
        const int count = min(Sh::kRows, rows - tile * Sh::kRows);
        for (int i = tid; i < count * (kD / 4); i += kPThreads)
            *reinterpret_cast<float4*>(a.part_acc + (out0 + (i >> 5)) * kD + 4 * (i & 31)) =
                *reinterpret_cast<const float4*>(&lds.join[i >> 5][4 * (i & 31)]);
        if (math && tg == 0 && h == 0 && live) {
            a.part_m[out0 + 32 * rg + n] = M * 0.69314718055994531f;
            a.part_l[out0 + 32 * rg + n] = L;
        }
    } else {
        if (math && live) {
            const size_t row = out0 + 32 * rg + n;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    *reinterpret_cast<float4*>(a.part_acc + row * kD + 32 * d + 8 * b + 4 * h) =
                        make_float4(o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]);
            if (h == 0) {
                a.part_m[row] = m * 0.69314718055994531f;
                a.part_l[row] = l;
            }
        }
    }
}

template __global__ void prefix_tile_kernel<2, false>(PrefixArgs);
template __global__ void prefix_tile_kernel<4, false>(PrefixArgs);
template __global__ void prefix_tile_kernel<8, false>(PrefixArgs);
template __global__ void prefix_tile_kernel<2, true>(PrefixArgs);
template __global__ void prefix_tile_kernel<4, true>(PrefixArgs);
template __global__ void prefix_tile_kernel<8, true>(PrefixArgs);

}  // namespace ffd
