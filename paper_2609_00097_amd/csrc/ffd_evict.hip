// Eviction from a paged cache by accumulated attention weight: of a sequence's tokens each KV head keeps its latest ones and
// the heaviest of the others, `budget` in all, moved together in their order into other pages.
//
// evict_select_kernel, one workgroup per (sequence, KV head): the order-preserving integer image of the weights, kept tokens
// being those above a threshold and, of those equal to it, the first ones. The threshold is found by counting digits from
// the highest on (11, 11 and 10 bits), each digit's counts in LDS; a last pass counts the kept tokens of each wave's part of the
// sequence and then writes the list in the tokens' order. Up to 32K keys lie in LDS, those behind are made anew in each pass.
// evict_move_kernel copies rows by the list. New pages are others than the old ones, so that rows can be copied in any order. It
// also leaves the new lengths, which may take the old ones' place: the selection's workgroups, which all read those, are done.
//
// Bound: the selection by its chain of passes, keys in LDS (four sequences of 32K, eight heads: 31 us, of which 11 bring the keys
// and count the first digit, 10 the two others, 10 count and write the list; 1K tokens 8 us), the move by HBM (8K of each of them: 57 us,
// 4.7 TB/s). Workgroups of 256 threads are no faster for 1K tokens (11.9 and 12.2 us both kernels) and slower from 2K on.
#include "ffd_paged.h"

namespace ffd {

namespace {

constexpr int kEvictWaves = kEvictThreads / 64;
constexpr int kPerThread = 4;
constexpr int kEvictStep = kEvictThreads * kPerThread;          // tokens a round
constexpr int kHeld = 32768;                    // keys in LDS
constexpr int kDigits = 2048;
static_assert(kHeld % kEvictStep == 0);

// Larger weight, larger key; +0 and -0 alike, NaN above infinity. 0 is no weight's key, and ~0 neither.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kLatest = 0xffffffffu;

struct EvictLds {
    alignas(16) uint32_t keys[kHeld];
    int hist[3][kDigits];                       // of each pass
    int sums[3][kEvictWaves];
    int digit[3], above[3];
};

// hist[digit] += 1 for the active lanes, those of one digit by one atomic where the first lane's digit is common.
__device__ __forceinline__ void count_digit(int* hist, int digit, bool active, int lane) {
    const uint64_t act = __ballot(active);
    if (act == 0) return;
    const int first = __builtin_amdgcn_readlane(digit, (int)__builtin_ctzll(act));
    const uint64_t same = __ballot(active && digit == first);
    if (lane == (int)__builtin_ctzll(act)) atomicAdd(&hist[first], (int)__popcll(same));
    if (active && digit != first) atomicAdd(&hist[digit], 1);
}

}  // namespace

__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(EvictArgs a) {
    __shared__ EvictLds lds;
    const int tid = threadIdx.x, lane = tid & 63;
    const int kvh = blockIdx.x, b = blockIdx.y;
    const int cap = a.from.max_pages << a.from.page_shift;
    const int L = min(max(a.seq_lens[b], 0), cap);
    const size_t pair = (size_t)b * gridDim.x + kvh;
    const float* weights = a.weights + pair * cap;
    const int latest = L - min(a.recent, L);
    // Keys of tokens j .. j + 3; 0: no token, or none of its page. 16 tokens of a page, of 16 or more, belong together.
    const int last4 = max(L - 1, 0) & ~(kPerThread - 1);
    auto keys_of = [&](int j, const float4& w, int entry) {
        const float x[kPerThread] = {w.x, w.y, w.z, w.w};
        const bool there = page_there(a.from, entry);
        uint32_t key[kPerThread];
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            const uint32_t k = j + e >= latest ? kLatest : weight_key(x[e]);
            key[e] = there & (j + e < L) ? k : 0u;
        }
        return make_uint4(key[0], key[1], key[2], key[3]);
    };
    auto weights_at = [&](int j) { return *reinterpret_cast<const float4*>(weights + min(j, last4)); };
    auto keys_at = [&](int j) {
        return j < kHeld ? *reinterpret_cast<const uint4*>(&lds.keys[j]) : keys_of(j, weights_at(j), page_entry(a.from, b, min(j, last4)));
    };
    const int rounds = (L + kEvictStep - 1) / kEvictStep;
    // The digits of the first pass are counted as the keys are made.
    for (int i = tid; i < 3 * kDigits; i += kEvictThreads) lds.hist[0][i] = 0;
    __syncthreads();
    auto count_keys = [&](const uint4& k4, int pass, int shift, int bits, uint32_t prefix) {
        const uint32_t key[kPerThread] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            const bool active = key[e] != 0 && (pass == 0 || key[e] >> (shift + bits) == prefix);
            count_digit(lds.hist[pass], (int)(key[e] >> shift) & ((1 << bits) - 1), active, lane);
        }
    };
    // rounds of tokens, four asked for together while the four before are counted
    constexpr int U = 4;
    float4 w[U];
    int entry[U];
    auto ask = [&](int i0) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = (i0 + i) * kEvictStep + kPerThread * tid;
            w[i] = weights_at(j);
            entry[i] = page_entry(a.from, b, min(j, last4));
        }
    };
    const int held = min(rounds, kHeld / kEvictStep);
    ask(0);
    for (int i0 = 0; i0 < held; i0 += U) {
        uint4 k4[U];
#pragma unroll
        for (int i = 0; i < U; ++i) k4[i] = keys_of((i0 + i) * kEvictStep + kPerThread * tid, w[i], entry[i]);
        if (i0 + U < held) {                    // uniform
            ask(i0 + U);
            asm volatile("" ::: "memory");      // here, not where they are used
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (i0 + i >= held) break;          // uniform
            *reinterpret_cast<uint4*>(&lds.keys[(i0 + i) * kEvictStep + kPerThread * tid]) = k4[i];
            count_keys(k4[i], 0, 21, 11, 0);
        }
    }
    // tokens above the threshold and equal to it: what is still to be found is the wanted-th largest of the keys with this prefix
    uint32_t prefix = 0;
    int wanted = a.budget, there = 0;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = pass == 0 ? kHeld / kEvictStep : 0; i < rounds; ++i) count_keys(keys_at(i * kEvictStep + kPerThread * tid), pass, shift, bits, prefix);
        __syncthreads();
        // counts from the highest digit down: thread t has digits 2047 - 2 t and 2046 - 2 t
        const int high = lds.hist[pass][kDigits - 1 - 2 * tid], low = lds.hist[pass][kDigits - 2 - 2 * tid];
        int total;
        const int before = wg_exclusive_scan<kEvictWaves>(high + low, lds.sums[pass], &total);
        if (pass == 0) there = total;
        if (there <= a.budget) break;           // uniform: all are kept
        if (before < wanted && wanted <= before + high) {
            lds.digit[pass] = kDigits - 1 - 2 * tid;
            lds.above[pass] = before;
        } else if (before + high < wanted && wanted <= before + high + low) {
            lds.digit[pass] = kDigits - 2 - 2 * tid;
            lds.above[pass] = before + high;
        }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)lds.digit[pass];
        wanted -= lds.above[pass];
    }
    const int count = min(there, a.budget);
    const uint32_t threshold = there <= a.budget ? 0 : prefix;
    const int ties = there <= a.budget ? 0 : wanted;            // of the tokens equal to the threshold
    int32_t* kept = a.kept + pair * a.budget;
    const int new_cap = a.to_pages << a.from.page_shift;
    float* new_weights = a.new_weights ? a.new_weights + pair * new_cap : nullptr;
    // Each wave takes a part of the sequence: first its tokens above the threshold and equal to it are counted, then they are written.
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = (L + kEvictWaves * 256 - 1) / (kEvictWaves * 256) * 256, begin = min(wave * part, L), end = min(begin + part, L);
    int above = 0, equal = 0;
    auto of_thread = [&](const uint4& k, int& above, int& equal) {
        above = (k.x > threshold) + (k.y > threshold) + (k.z > threshold) + (k.w > threshold);
        equal = threshold == 0 ? 0 : (k.x == threshold) + (k.y == threshold) + (k.z == threshold) + (k.w == threshold);
    };
    for (int j = begin + kPerThread * lane; j < end; j += 64 * kPerThread) {
        int x, y;
        of_thread(keys_at(j), x, y);
        above += x;
        equal += y;
    }
    above = wave_sum_dpp(above);
    equal = wave_sum_dpp(equal);
    __syncthreads();
    if (lane == 0) {
        lds.sums[0][wave] = above;
        lds.sums[1][wave] = equal;
    }
    __syncthreads();
    int equals = 0, to_wave = 0;                // before this wave's part: equal ones, kept ones
    for (int w = 0; w < wave; ++w) {
        to_wave += lds.sums[0][w];
        equals += lds.sums[1][w];
    }
    to_wave += min(equals, ties);
    float4 next = weights_at(begin + kPerThread * lane);        // a round early
    for (int j0 = begin; j0 < end; j0 += 64 * kPerThread) {
        const int j = j0 + kPerThread * lane;
        const uint4 k4 = keys_at(min(j, last4));
        const uint32_t key[kPerThread] = {k4.x, k4.y, k4.z, k4.w};
        const float4 w4 = next;
        next = weights_at(j + 64 * kPerThread);
        asm volatile("" ::: "memory");          // here, not where it is used
        const float w[kPerThread] = {w4.x, w4.y, w4.z, w4.w};
        int x = 0, y = 0;
        if (j < end) of_thread(k4, x, y);
        const int both = x | y << 16, incl = wave_inclusive_scan(both), before = incl - both, all = __builtin_amdgcn_readlane(incl, 63);
        int equal_here = equals + (before >> 16);
        int to = to_wave + (before & 0xffff) + min(equal_here, ties) - min(equals, ties);
        if (j < end) {
#pragma unroll
            for (int e = 0; e < kPerThread; ++e) {
                const bool is_equal = threshold != 0 && key[e] == threshold;
                if (key[e] > threshold || (is_equal && equal_here < ties)) {
                    kept[to] = j + e;
                    if (new_weights) new_weights[to] = w[e];
                    ++to;
                }
                equal_here += is_equal;
            }
        }
        to_wave += (all & 0xffff) + min(equals + (all >> 16), ties) - min(equals, ties);
        equals += all >> 16;
    }
    for (int r = count + tid; r < a.budget; r += kEvictThreads) kept[r] = -1;
}

// 128 places of a (sequence, KV head), keys or values: 16 lanes a bf16 row, eight an 8-bit one. Everything passes once.
template <bool I8>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(EvictArgs a) {
    constexpr int kLanes = I8 ? 8 : 16, kRows = kThreads / kLanes, kSteps = kEvictMoveRows / kRows;
    const bool values = blockIdx.x & 1;
    const int kvh = blockIdx.y, b = blockIdx.z, c = threadIdx.x % kLanes, r0 = (int)(blockIdx.x >> 1) * kEvictMoveRows + (int)threadIdx.x / kLanes;
    const int32_t* kept = a.kept + ((size_t)b * a.Hkv + kvh) * a.budget;
    const PagedKv to{a.from.kv, a.to_table, a.from.num_pages, a.from.page_shift, a.to_pages};
    const bool counts = !values && kvh == 0;    // uniform: these workgroups leave the new length
    int j[kSteps], to_entry[kSteps], after[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const int r = min(r0 + u * kRows, a.budget - 1);
        j[u] = kept[r];
        to_entry[u] = page_entry(to, b, r);
    }
    if (counts) {
#pragma unroll
        for (int u = 0; u < kSteps; ++u) after[u] = kept[min(r0 + u * kRows + 1, a.budget - 1)];
    }
    size_t src[kSteps], dst[kSteps];
    bool move[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const int from_entry = page_entry(a.from, b, max(j[u], 0));
        move[u] = r0 + u * kRows < a.budget && j[u] >= 0 && page_there(a.from, from_entry) && page_there(to, to_entry[u]);
        src[u] = move[u] ? page_row(a.from, a.Hkv, kvh, from_entry, j[u]) : 0;
        dst[u] = move[u] ? page_row(to, a.Hkv, kvh, to_entry[u], r0 + u * kRows) : 0;
    }
    v4i* tokens = reinterpret_cast<v4i*>(const_cast<uint8_t*>(values ? a.from.kv.v : a.from.kv.k));
    uint16_t* absmax = const_cast<uint16_t*>(values ? a.from.kv.v_absmax : a.from.kv.k_absmax);
    v4i x[kSteps];
    uint16_t m[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        x[u] = __builtin_nontemporal_load(tokens + src[u] * kLanes + c);
        if constexpr (I8) m[u] = absmax[src[u]];
    }
    if (counts && c == 0) {                     // of the list's last place in use, or of its first where there is none
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int r = r0 + u * kRows;
            if (r < a.budget && (j[u] >= 0 ? after[u] < 0 || r + 1 == a.budget : r == 0)) a.new_lens[b] = j[u] >= 0 ? r + 1 : 0;
        }
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        if (!move[u]) continue;
        __builtin_nontemporal_store(x[u], tokens + dst[u] * kLanes + c);
        if constexpr (I8) {
            if (c == 0) absmax[dst[u]] = m[u];
        }
    }
}

template __global__ void evict_move_kernel<false>(EvictArgs);
template __global__ void evict_move_kernel<true>(EvictArgs);

}  // namespace ffd
