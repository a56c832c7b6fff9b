// Eviction from a paged cache by accumulated attention weight: of a sequence's tokens each KV head keeps its latest ones and
// the heaviest of the others, `budget` in all, moved together in their order into other pages.
//
// evict_select_kernel, one workgroup per (sequence, KV head): the order-preserving integer image of the weights, kept tokens
// being those above a threshold and, of those equal to it, the first ones. The threshold is found by counting digits from
// the highest on (11, 11 and 10 bits), each digit's counts in LDS, then a last pass in the tokens' order writes the list.
// evict_move_kernel copies rows by the list. New pages are others than the old ones, so that rows can be copied in any order.
//
// Bound: the selection by its chain of passes over 4 bytes a token (out of L2 after the first), the move by HBM.
#include "ffd_paged.h"

namespace ffd {

namespace {

constexpr int kEvictWaves = kEvictThreads / 64;
constexpr int kPerThread = 4;
constexpr int kEvictStep = kEvictThreads * kPerThread;          // tokens a round
constexpr int kDigits = 2048;

// Larger weight, larger key; +0 and -0 alike, NaN above infinity. 0 is no weight's key, and ~0 neither.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kLatest = 0xffffffffu;

struct EvictLds {
    int hist[kDigits];
    int sums[2][kEvictWaves];
    int digit, above;
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
    // keys of tokens 4 i .. 4 i + 3; 0: no token, or none of its page
    auto keys_at = [&](int j, uint32_t (&key)[kPerThread], float (&w)[kPerThread]) {
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) key[e] = 0, w[e] = 0.f;
        if (j >= L || !page_there(a.from, page_entry(a.from, b, j))) return;
        const float4 x = *reinterpret_cast<const float4*>(weights + j);         // 16 tokens of a page, of 16 or more, belong together
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) key[e] = j + e >= L ? 0u : j + e >= latest ? kLatest : weight_key(w[e]);
    };
    // tokens above the threshold and equal to it: what is still to be found is the wanted-th largest of the keys with this prefix
    uint32_t prefix = 0;
    int wanted = a.budget, there = 0;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < kDigits; i += kEvictThreads) lds.hist[i] = 0;
        __syncthreads();
        for (int j0 = 0; j0 < L; j0 += kEvictStep) {
            uint32_t key[kPerThread];
            float w[kPerThread];
            keys_at(j0 + kPerThread * tid, key, w);
#pragma unroll
            for (int e = 0; e < kPerThread; ++e) {
                const bool active = key[e] != 0 && (pass == 0 || key[e] >> (shift + bits) == prefix);
                count_digit(lds.hist, (int)(key[e] >> shift) & ((1 << bits) - 1), active, lane);
            }
        }
        __syncthreads();
        // counts from the highest digit down: thread t has digits 2047 - 2 t and 2046 - 2 t
        const int high = lds.hist[kDigits - 1 - 2 * tid], low = lds.hist[kDigits - 2 - 2 * tid];
        int total;
        const int before = wg_exclusive_scan<kEvictWaves>(high + low, lds.sums[pass & 1], &total);
        if (pass == 0) there = total;
        if (there <= a.budget) break;           // uniform: all are kept
        if (before < wanted && wanted <= before + high) {
            lds.digit = kDigits - 1 - 2 * tid;
            lds.above = before;
        } else if (before + high < wanted && wanted <= before + high + low) {
            lds.digit = kDigits - 2 - 2 * tid;
            lds.above = before + high;
        }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)lds.digit;
        wanted -= lds.above;
        __syncthreads();
    }
    const int count = min(there, a.budget);
    const uint32_t threshold = there <= a.budget ? 0 : prefix;
    const int ties = there <= a.budget ? 0 : wanted;            // of the tokens equal to the threshold
    int32_t* kept = a.kept + pair * a.budget;
    const int new_cap = a.to_pages << a.from.page_shift;
    float* new_weights = a.new_weights ? a.new_weights + pair * new_cap : nullptr;
    __syncthreads();
    int at = 0, equal = 0;
    int turn = 0;
    for (int j0 = 0; j0 < L; j0 += kEvictStep, turn ^= 1) {
        uint32_t key[kPerThread];
        float w[kPerThread];
        const int j = j0 + kPerThread * tid;
        keys_at(j, key, w);
        int mine = 0;                           // above in the low half, equal in the high one
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) mine += (key[e] > threshold ? 1 : 0) + (key[e] != 0 && key[e] == threshold ? 1 << 16 : 0);
        int total;
        const int before = wg_exclusive_scan<kEvictWaves>(mine, lds.sums[turn], &total);
        int above_here = before & 0xffff, equal_here = equal + (before >> 16);
        // kept before this thread: those above, and the equal ones up to `ties`
        int to = at + above_here + min(equal_here, ties) - min(equal, ties);
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            const bool is_equal = key[e] != 0 && key[e] == threshold;
            if (key[e] > threshold || (is_equal && equal_here < ties)) {
                kept[to] = j + e;
                if (new_weights) new_weights[to] = w[e];
                ++to;
            }
            equal_here += is_equal;
        }
        at += (total & 0xffff) + min(equal + (total >> 16), ties) - min(equal, ties);
        equal += total >> 16;
    }
    for (int r = count + tid; r < a.budget; r += kEvictThreads) kept[r] = -1;
    if (kvh == 0 && tid == 0) a.new_lens[b] = count;
}

// 64 places of a (sequence, KV head), keys and values: 16 lanes a bf16 row, eight an 8-bit one.
template <bool I8>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(EvictArgs a) {
    constexpr int kLanes = I8 ? 8 : 16, kRows = kThreads / kLanes, kSteps = kEvictMoveRows / kRows;
    const int kvh = blockIdx.y, b = blockIdx.z, c = threadIdx.x % kLanes;
    const int32_t* kept = a.kept + ((size_t)b * a.Hkv + kvh) * a.budget;
    const PagedKv to{a.from.kv, a.to_table, a.from.num_pages, a.from.page_shift, a.to_pages};
    size_t src[kSteps], dst[kSteps];
    bool move[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const int r = (int)blockIdx.x * kEvictMoveRows + u * kRows + (int)threadIdx.x / kLanes;
        const int j = r < a.budget ? kept[r] : -1;
        const int from_entry = page_entry(a.from, b, max(j, 0)), to_entry = page_entry(to, b, min(r, a.budget - 1));
        move[u] = j >= 0 && page_there(a.from, from_entry) && page_there(to, to_entry);
        src[u] = move[u] ? page_row(a.from, a.Hkv, kvh, from_entry, j) : 0;
        dst[u] = move[u] ? page_row(to, a.Hkv, kvh, to_entry, r) : 0;
    }
    uint4* k = reinterpret_cast<uint4*>(const_cast<uint8_t*>(a.from.kv.k));
    uint4* v = reinterpret_cast<uint4*>(const_cast<uint8_t*>(a.from.kv.v));
    uint4 x[2][kSteps];
    uint16_t m[2][kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        x[0][u] = k[src[u] * kLanes + c];
        x[1][u] = v[src[u] * kLanes + c];
        if constexpr (I8) {
            m[0][u] = a.from.kv.k_absmax[src[u]];
            m[1][u] = a.from.kv.v_absmax[src[u]];
        }
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        if (!move[u]) continue;
        k[dst[u] * kLanes + c] = x[0][u];
        v[dst[u] * kLanes + c] = x[1][u];
        if constexpr (I8) {
            if (c == 0) {
                const_cast<uint16_t*>(a.from.kv.k_absmax)[dst[u]] = m[0][u];
                const_cast<uint16_t*>(a.from.kv.v_absmax)[dst[u]] = m[1][u];
            }
        }
    }
}

template __global__ void evict_move_kernel<false>(EvictArgs);
template __global__ void evict_move_kernel<true>(EvictArgs);

}  // namespace ffd
