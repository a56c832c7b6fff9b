// C ABI of the paged cache: argument checks, the attention's cut into kernels and workgroups, launches.
#include <algorithm>
#include <cmath>

#include "ffd_host.h"
#include "ffd_paged.h"

using namespace ffd;

namespace {

constexpr int kMaxCapacity = 1 << 28;
constexpr int kMaxTokens = 1 << 24;
constexpr float kNoCapFrom = 0x1p100f;          // a cap that no score comes near: none, and nothing under- or overflows

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int check_heads(int Hq, int Hkv, int D) {
    if (Hq <= 0 || Hkv <= 0 || Hq % Hkv) return FFD_ERR_INVALID_ARGUMENT;
    const int G = Hq / Hkv;
    if (Hkv > 65535 || (G != 1 && G != 2 && G != 4 && G != 8) || D != FFD_HEAD_DIM) return FFD_ERR_UNSUPPORTED;
    return FFD_OK;
}

int check_batch(int B, int T, int heads) {
    if (B < 0 || T < 0) return FFD_ERR_INVALID_ARGUMENT;
    if (B > 65535 || T > kMaxTokens || (long long)T * heads >= 1LL << 28) return FFD_ERR_UNSUPPORTED;
    return FFD_OK;
}
bool pairs_fit(int B, int Hkv) { return (long long)B * Hkv <= 1LL << 20; }

// The cache's shape and pointers; *i8: 8-bit pages.
int check_paged(const ffd_paged* c, bool* i8) {
    if (!c) return FFD_ERR_INVALID_ARGUMENT;
    if (c->num_pages <= 0 || c->max_pages <= 0 || c->page <= 0 || (c->page & (c->page - 1))) return FFD_ERR_INVALID_ARGUMENT;
    if (c->page < 16 || c->page > 256 || (long long)c->max_pages * c->page > kMaxCapacity) return FFD_ERR_UNSUPPORTED;
    int bits;
    const int st = check_kv(&c->pages, false, &bits);
    if (st != FFD_OK) return st;
    if (!c->page_table || !aligned4(c->page_table)) return FFD_ERR_INVALID_ARGUMENT;
    *i8 = bits == 8;
    return FFD_OK;
}

PagedKv paged_of(const ffd_paged& c) {
    return PagedKv{source_of(c.pages), c.page_table, c.num_pages, __builtin_ctz(c.page), c.max_pages};
}

int check_rules(const ffd_score_rules* r) {
    if (!r) return FFD_OK;
    if (!(r->softcap >= 0.f) || std::isinf(r->softcap) || r->window < 0) return FFD_ERR_INVALID_ARGUMENT;
    if (!aligned4(r->slopes) || !aligned4(r->prefix_lens)) return FFD_ERR_INVALID_ARGUMENT;
    return FFD_OK;
}

ChunkArgs chunk_args(const void* q, const ffd_paged& c, const int32_t* q_start, const int32_t* seq_lens,
                     const ffd_score_rules* rules, int B, int T, int Hq, int Hkv, float softmax_scale) {
    ChunkArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.pages = paged_of(c);
    a.q_start = q_start;
    a.seq_lens = seq_lens;
    a.B = B, a.T = T, a.Hq = Hq, a.Hkv = Hkv, a.G = Hq / Hkv, a.Lcap = c.max_pages * c.page;
    a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)FFD_HEAD_DIM);
    if (rules) {
        a.prefix_lens = rules->prefix_lens;
        a.slopes = rules->slopes;
        a.window = std::min(rules->window, kMaxLen);
        if (rules->window > kMaxLen) a.window = 0;              // as wide as no length is
        a.cap = rules->softcap < kNoCapFrom ? rules->softcap : 0.f;
        double x = 1.0;                         // tanh(y) = y P(y^2) with y = x ln(2) / 2, times cap log2(e)
        for (int i = 0; i < 5; ++i, x *= M_LN2 * M_LN2 / 4) a.cap_near[i] = (float)(a.cap / 2.0 * x * kTanhNear[i]);
    }
    return a;
}

// One kernel's part of the attention: row tiles of `rows`, workgroups, and its part of the workspace.
struct ChunkKernel {
    int rows, rows_above, rows_upto, slots, unit_shift;
    long long grid;
    bool large() const { return rows == kChunkTileRows; }
    int parts_count() const { return large() ? slots : 2 * slots; }
    size_t records_off() const { return round_up(partials_bytes((size_t)parts_count() * rows), kAlign); }
    size_t total_off() const { return records_off() + round_up(slots * sizeof(int4), kAlign); }
    size_t bytes() const { return total_off() + kAlign; }
    ChunkParts parts(uint8_t* ws) const {
        const Partials P = carve(ws, (size_t)parts_count() * rows);
        return ChunkParts{P.m, P.l, P.acc, reinterpret_cast<int4*>(ws + records_off()),
                          large() ? reinterpret_cast<int*>(ws + total_off()) : nullptr, rows, parts_count()};
    }
    int merge_wgs() const { return slots * 4 * (rows / chunk_merge_rows(rows)); }
};
ChunkKernel chunk_kernel(int B, int T, int Hq, int Hkv, long long Lcap, int rows, int above, int upto, int per_cu) {
    ChunkKernel k{rows, above, upto, per_cu * device_cus(), 0, 0};
    const int G = Hq / Hkv;
    // every sequence has at most one tile that is not full
    const long long tiles = ((long long)T * G / rows + std::min(B, T)) * Hkv;
    // (T Hq < 2^28 and B Hkv <= 2^20: below 2^22 workgroups)
    k.grid = k.large() ? std::max((long long)k.slots, k.slots / 2 + tiles) : k.slots;
    while (tiles * (((Lcap + kRound - 1) / kRound >> k.unit_shift) + 1) >= 1LL << 31) ++k.unit_shift;
    return k;
}
// Sequences with up to kFewRows query rows per KV head go to the kernel of few rows, the others to the one of large tiles. One
// kernel takes all where the batch cannot have both kinds (few rows in all, or one sequence, whose rows are taken to be all T), has at
// most two new tokens a sequence, or has little work: rows times tokens of the capacity per CU.
// Two tokens a sequence: a batch that decodes would pay for the second kernel (256 sequences of 2K 366 us, 399 with it), one that hides a
// chunk would win by it (256 tokens on 32K in that batch 1420 us, 554 with it). Nothing but T tells them apart on the host.
// Little work. Large / few, whole calls, tables as long as the sequences, eight KV heads of four in bf16: 32K (256 tokens on 1K) 34.2 /
// 33.4 us; 64K (512 on 1K) 36.8 / 33.9, (128 on 4K) 36.1 / 42.3; 128K (256 on 4K) 41.5 / 58.1, (32 on 32K) 41.2 / 56.0, (512 on 2K) 42.3 /
// 48.7. In 8 bits 32K 35.8 / 24.7; 64K 40.1 / 32.9, 42.5 / 43.0; 128K 52.0 / 62.6, 58.0 / 58.9, 52.2 / 52.7. Long tables count as long
// sequences: three prompts of up to 1K with 20 to 37 new tokens 15 us, with a table for 128K tokens 24.
constexpr int kFewRows = 32;
constexpr long long kLittleWork = 40 << 10;
// Tiles of the kernel of few rows: 32 rows, so that a tile's tokens are read once for them; 16 where the batch has hardly more in a
// sequence, and where that leaves no more than one workgroup of two blocks for each CU. 16 / 32, whole calls, four heads per KV head:
// 8 tokens on 300 11.9 / 15.8 us, 16 on 1K 13.0 / 16.8, 8 on 4K 15.0 / 18.0 (256 such pairs), 16 on 4K 21.9 / 19.2 (512), 8 on 32K
// 53 / 39.
bool may_be_large(int B, int T, int Hq, int Hkv) { return (long long)T * (Hq / Hkv) > kFewRows && T > 2LL * B; }
struct ChunkLaunches {
    bool few, large;
    bool cut;                   // tiles may be cut, and need the merge
    ChunkKernel few_kernel, large_kernel;
    size_t large_off, total;
};
ChunkLaunches chunk_launches(int B, int T, int Hq, int Hkv, long long Lcap, bool i8) {
    ChunkLaunches p;
    const long long rows = (long long)T * (Hq / Hkv);
    p.large = may_be_large(B, T, Hq, Hkv) && rows * Lcap * Hkv > kLittleWork * device_cus();
    p.few = B > 1 || !p.large;
    const long long pairs = (rows + 15LL * std::min(B, T)) / 16 * Hkv * ((Lcap + 2 * kRound - 1) / (2 * kRound));
    p.cut = p.large || Lcap > kWholeBlocks * kRound;
    const int tile = rows <= 16LL * B || p.large || pairs <= device_cus() ? 16 : 32;
    p.few_kernel = chunk_kernel(B, T, Hq, Hkv, Lcap, tile, 0, p.large ? kFewRows : INT32_MAX, tile == 16 && i8 ? 3 : 2);
    p.large_kernel = chunk_kernel(B, T, Hq, Hkv, Lcap, kChunkTileRows, p.few ? kFewRows : 0, INT32_MAX, 1);
    p.large_off = p.few ? p.few_kernel.bytes() : 0;
    p.total = p.large_off + (p.large ? p.large_kernel.bytes() : 0);
    return p;
}
// Enough for any capacity and form of the cache.
size_t chunk_workspace(int B, int T, int Hq, int Hkv) {
    const size_t few = std::max(chunk_kernel(B, T, Hq, Hkv, 0, 16, 0, 0, 3).bytes(), chunk_kernel(B, T, Hq, Hkv, 0, 32, 0, 0, 2).bytes());
    return few + (may_be_large(B, T, Hq, Hkv) ? chunk_kernel(B, T, Hq, Hkv, 0, kChunkTileRows, 0, 0, 1).bytes() : 0);
}

template <int CT, bool I8>
void launch_rows_ruled(bool ruled, dim3 grid, hipStream_t stream, const ChunkAttendArgs& a) {
    if (ruled) hipLaunchKernelGGL((chunk_rows_kernel<CT, I8, true>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((chunk_rows_kernel<CT, I8, false>), grid, dim3(kThreads), 0, stream, a);
}
void launch_rows(int rows, bool i8, bool ruled, dim3 grid, hipStream_t stream, const ChunkAttendArgs& a) {
    if (rows == 16 && i8) launch_rows_ruled<1, true>(ruled, grid, stream, a);
    else if (rows == 16) launch_rows_ruled<1, false>(ruled, grid, stream, a);
    else if (i8) launch_rows_ruled<2, true>(ruled, grid, stream, a);
    else launch_rows_ruled<2, false>(ruled, grid, stream, a);
}

// Query rows of a sequence up to which the weights' workgroups take equal shares, three to a CU; above, a unit each, in which the
// rows that may see it differ, with two places for rows in LDS. Shares / units, eight KV heads of four: 128 rows on 32K 26.1 / 40.4 us,
// 256 45.3 / 51.5, on 4 x 8K 53.3 / 52.4, 512 on 32K 78.2 / 80.1, 2K on 8 x 2K 221 / 115 with tables as long as the sequences. By the mean
// of the batch, so one chunk of 512 tokens beside 15 that decode, on 8K, takes shares (791 us, units 165); and units are of the
// capacity: eight whole prompts of 2K 399 us, with a table for 128K tokens 445.
constexpr int kFewWeightRows = 256;
template <bool MANY>
void launch_weights(bool i8, bool ruled, hipStream_t stream, const ChunkWeightsArgs& a) {
    const dim3 grid((unsigned)a.slots), block(kThreads);
    if (i8 && ruled) hipLaunchKernelGGL((chunk_weights_kernel<true, true, MANY>), grid, block, 0, stream, a);
    else if (i8) hipLaunchKernelGGL((chunk_weights_kernel<true, false, MANY>), grid, block, 0, stream, a);
    else if (ruled) hipLaunchKernelGGL((chunk_weights_kernel<false, true, MANY>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((chunk_weights_kernel<false, false, MANY>), grid, block, 0, stream, a);
}

int check_strides(const int64_t* s) { return s && (s[0] < 0 || s[0] % 8 || s[1] < 0 || s[1] % 8) ? FFD_ERR_INVALID_ARGUMENT : FFD_OK; }

}  // namespace

extern "C" {

int ffd_write_paged(const void* q, const void* k, const void* v, const int64_t* q_strides, const int64_t* k_strides,
                    const int64_t* v_strides, void* q_out, const ffd_rotation* rotation, const ffd_paged* cache,
                    const int32_t* q_start, const int32_t* seq_lens, int B, int T, int Hq, int Hkv, int D,
                    hipStream_t stream) {
    int st = check_heads(Hq, Hkv, D);
    if (st == FFD_OK) st = check_batch(B, T, Hq + 2 * Hkv);
    if (st != FFD_OK) return st;
    if (check_strides(q_strides) || check_strides(k_strides) || check_strides(v_strides)) return FFD_ERR_INVALID_ARGUMENT;
    static const ffd_rotation none{};
    const ffd_rotation& r = rotation ? *rotation : none;
    if (!(r.eps >= 0.f) || std::isinf(r.eps)) return FFD_ERR_INVALID_ARGUMENT;
    if (r.table) {
        if (r.rows <= 0 || r.dims <= 0 || r.dims % 2 || r.dims > D) return FFD_ERR_INVALID_ARGUMENT;
        if (r.dims % 32) return FFD_ERR_UNSUPPORTED;
    }
    if (B == 0 || T == 0) return FFD_OK;
    bool i8;
    if ((st = check_paged(cache, &i8)) != FFD_OK) return st;
    if (!k || !v || !q_start || !seq_lens || !q != !q_out) return FFD_ERR_INVALID_ARGUMENT;
    for (const void* p : {q, k, v, (const void*)q_out, r.q_weight, r.k_weight, (const void*)r.table})
        if (!aligned16(p)) return FFD_ERR_INVALID_ARGUMENT;
    if (!aligned4(q_start) || !aligned4(seq_lens) || !aligned4(r.positions)) return FFD_ERR_INVALID_ARGUMENT;
    WritePagedArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.q_weight = static_cast<const uint16_t*>(r.q_weight);
    a.k_weight = static_cast<const uint16_t*>(r.k_weight);
    a.rope = r.table;
    a.positions = r.positions;
    a.pages = paged_of(*cache);
    a.q_start = q_start;
    a.seq_lens = seq_lens;
    const int64_t cq[2] = {(int64_t)Hq * D, D}, ckv[2] = {(int64_t)Hkv * D, D};
    for (int i = 0; i < 2; ++i) {
        a.qs[i] = (q_strides ? q_strides : cq)[i];
        a.ks[i] = (k_strides ? k_strides : ckv)[i];
        a.vs[i] = (v_strides ? v_strides : ckv)[i];
    }
    a.B = B, a.T = T, a.Hq = Hq, a.Hkv = Hkv;
    a.rope_rows = r.rows, a.rope_dims = r.table ? r.dims : 0;
    a.eps = r.eps;
    // one vector a group of lanes while that leaves CUs idle, else up to twelve, so that the table's row is loaded less often
    const int vectors = (q ? Hq : 0) + 2 * Hkv, groups = (vectors + 3) / 4;
    const long long wanted = 16LL * device_cus();
    const int waves = (int)std::min<long long>(groups, std::max<long long>((groups + 11) / 12, wanted / T));
    a.parts = 4 * waves;
    const dim3 grid((unsigned)(((long long)T * waves + kWaves - 1) / kWaves));
    const bool inter = r.table && r.interleaved;
    if (i8 && inter) hipLaunchKernelGGL((write_paged_kernel<true, true>), grid, dim3(kThreads), 0, stream, a);
    else if (i8) hipLaunchKernelGGL((write_paged_kernel<true, false>), grid, dim3(kThreads), 0, stream, a);
    else if (inter) hipLaunchKernelGGL((write_paged_kernel<false, true>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((write_paged_kernel<false, false>), grid, dim3(kThreads), 0, stream, a);
    return launch_status();
}

size_t ffd_paged_workspace_bytes(int B, int T, int Hq, int Hkv, int D) {
    CallScope scope;
    if (check_heads(Hq, Hkv, D) != FFD_OK || check_batch(B, T, Hq) != FFD_OK || B == 0 || T == 0) return 0;
    return pairs_fit(B, Hkv) ? chunk_workspace(B, T, Hq, Hkv) : 0;
}

int ffd_paged_attention(const void* q, const ffd_paged* cache, const int32_t* q_start, const int32_t* seq_lens,
                        const ffd_score_rules* rules, int B, int T, int Hq, int Hkv, int D, float softmax_scale, void* out,
                        float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    CallScope scope;
    int st = check_heads(Hq, Hkv, D);
    if (st == FFD_OK) st = check_batch(B, T, Hq);
    if (st != FFD_OK) return st;
    if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale)) return FFD_ERR_INVALID_ARGUMENT;
    if ((st = check_rules(rules)) != FFD_OK || B == 0 || T == 0) return st;
    bool i8;
    if ((st = check_paged(cache, &i8)) != FFD_OK) return st;
    if (!q || !q_start || !seq_lens || !out || !workspace) return FFD_ERR_INVALID_ARGUMENT;
    if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) || !aligned4(q_start) || !aligned4(seq_lens) || !aligned4(lse))
        return FFD_ERR_INVALID_ARGUMENT;
    if (!pairs_fit(B, Hkv)) return FFD_ERR_UNSUPPORTED;
    const ChunkLaunches plan = chunk_launches(B, T, Hq, Hkv, (long long)cache->max_pages * cache->page, i8);
    if (workspace_bytes < chunk_workspace(B, T, Hq, Hkv)) return FFD_ERR_WORKSPACE_TOO_SMALL;
    ChunkAttendArgs a{};
    static_cast<ChunkArgs&>(a) = chunk_args(q, *cache, q_start, seq_lens, rules, B, T, Hq, Hkv, softmax_scale);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    const bool ruled = rules && (rules->softcap > 0.f || rules->slopes);
    ChunkMergeArgs m{{}, 0, a.out, lse, Hq, Hkv, Hq / Hkv};
    int sets = 0, wgs = 0;
    auto prepare = [&](const ChunkKernel& k, uint8_t* ws) {
        a.parts = k.parts(ws);
        a.rows_above = k.rows_above, a.rows_upto = k.rows_upto, a.slots = k.slots, a.unit_shift = k.unit_shift;
        m.parts[sets++] = a.parts;
        if (sets == 1) m.wgs = k.merge_wgs();
        wgs += k.merge_wgs();
    };
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (plan.large) {
        const ChunkKernel& k = plan.large_kernel;
        prepare(k, ws + plan.large_off);
        const dim3 grid((unsigned)k.grid), block(kChunkTileThreads);
        if (i8 && ruled) hipLaunchKernelGGL((chunk_tile8_kernel<true>), grid, block, 0, stream, a);
        else if (i8) hipLaunchKernelGGL((chunk_tile8_kernel<false>), grid, block, 0, stream, a);
        else if (ruled) hipLaunchKernelGGL((chunk_tile_kernel<true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((chunk_tile_kernel<false>), grid, block, 0, stream, a);
        if ((st = launch_status()) != FFD_OK) return st;
    }
    if (plan.few) {
        prepare(plan.few_kernel, ws);
        launch_rows(plan.few_kernel.rows, i8, ruled, dim3((unsigned)plan.few_kernel.grid), stream, a);
        if ((st = launch_status()) != FFD_OK) return st;
    }
    if (!plan.cut) return FFD_OK;
    hipLaunchKernelGGL(chunk_merge_kernel, dim3((unsigned)wgs), dim3(kThreads), 0, stream, m);
    return launch_status();
}

int ffd_paged_attention_weights(const void* q, const ffd_paged* cache, const int32_t* q_start, const int32_t* seq_lens,
                                const ffd_score_rules* rules, const float* lse, int B, int T, int Hq, int Hkv, int D,
                                float softmax_scale, int last, const float* previous, float* weights, hipStream_t stream) {
    CallScope scope;
    int st = check_heads(Hq, Hkv, D);
    if (st == FFD_OK) st = check_batch(B, T, Hq);
    if (st != FFD_OK) return st;
    if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale) || last < 0) return FFD_ERR_INVALID_ARGUMENT;
    if ((st = check_rules(rules)) != FFD_OK || B == 0) return st;
    bool i8;
    if ((st = check_paged(cache, &i8)) != FFD_OK) return st;
    if (!q_start || !seq_lens || !weights || (T > 0 && (!q || !lse))) return FFD_ERR_INVALID_ARGUMENT;
    if (!pairs_fit(B, Hkv)) return FFD_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(weights) || !aligned16(previous) || !aligned4(lse) || !aligned4(q_start) || !aligned4(seq_lens))
        return FFD_ERR_INVALID_ARGUMENT;
    ChunkWeightsArgs a{};
    static_cast<ChunkArgs&>(a) = chunk_args(q, *cache, q_start, seq_lens, rules, B, T, Hq, Hkv, softmax_scale);
    a.lse = lse;
    a.previous = previous;
    a.weights = weights;
    a.last = last;
    const bool ruled = rules && (rules->softcap > 0.f || rules->slopes);
    long long units = 0;
    while (units == 0 || units >= 1LL << 23) units = (long long)B * Hkv * ((a.Lcap + (kRound << a.unit_shift) - 1) / (kRound << a.unit_shift)), ++a.unit_shift;
    --a.unit_shift;
    const long long rows = std::min<long long>(T, last > 0 ? (long long)last * B : T) * a.G;
    const bool many = rows > kFewWeightRows * (long long)B;
    a.slots = (int)(many ? units : std::min<long long>(units, 3LL * device_cus()));
    if (many) launch_weights<true>(i8, ruled, stream, a);
    else launch_weights<false>(i8, ruled, stream, a);
    return launch_status();
}

int ffd_evict_paged(const ffd_paged* cache, const int32_t* new_table, int new_max_pages, const int32_t* seq_lens,
                    const float* weights, int B, int Hkv, int D, int budget, int recent, int32_t* new_lens, int32_t* kept,
                    float* new_weights, hipStream_t stream) {
    int st = check_heads(Hkv, Hkv, D);
    if (st == FFD_OK) st = check_batch(B, 0, 0);
    if (st != FFD_OK) return st;
    if (new_max_pages <= 0 || budget <= 0 || recent < 0 || recent > budget) return FFD_ERR_INVALID_ARGUMENT;
    if (B == 0) return FFD_OK;
    bool i8;
    if ((st = check_paged(cache, &i8)) != FFD_OK) return st;
    if ((long long)new_max_pages * cache->page > kMaxCapacity) return FFD_ERR_UNSUPPORTED;
    if (budget > new_max_pages * cache->page) return FFD_ERR_INVALID_ARGUMENT;
    if (!new_table || !seq_lens || !weights || !new_lens || !kept) return FFD_ERR_INVALID_ARGUMENT;
    if (!aligned16(weights) || !aligned4(new_table) || !aligned4(seq_lens) || !aligned4(new_lens) || !aligned4(kept) || !aligned4(new_weights))
        return FFD_ERR_INVALID_ARGUMENT;
    const long long moves = 2LL * ((budget + kEvictMoveRows - 1) / kEvictMoveRows);
    if (!pairs_fit(B, Hkv) || moves * B * Hkv * kThreads >= 1LL << 31) return FFD_ERR_UNSUPPORTED;
    const size_t pairs = (size_t)B * Hkv * cache->page, at = reinterpret_cast<uintptr_t>(weights), new_at = reinterpret_cast<uintptr_t>(new_weights);
    if (new_table == cache->page_table) return FFD_ERR_INVALID_ARGUMENT;
    if (new_weights && new_at < at + pairs * cache->max_pages * sizeof(float) && at < new_at + pairs * new_max_pages * sizeof(float)) return FFD_ERR_INVALID_ARGUMENT;
    const EvictArgs a{paged_of(*cache), new_table, seq_lens, weights, new_lens, kept, new_weights, Hkv, new_max_pages, budget, recent};
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)Hkv, (unsigned)B), dim3(kEvictThreads), 0, stream, a);
    if ((st = launch_status()) != FFD_OK) return st;
    const dim3 grid((unsigned)moves, (unsigned)Hkv, (unsigned)B);
    if (i8) hipLaunchKernelGGL(evict_move_kernel<true>, grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL(evict_move_kernel<false>, grid, dim3(kThreads), 0, stream, a);
    return launch_status();
}

}  // extern "C"
