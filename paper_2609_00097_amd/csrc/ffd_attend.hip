// Attention of few query rows per KV head (ffd_attend.h has the mathematics and the mapping).
#include "ffd_attend.h"

namespace ffd {

template <bool I8, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void own_decode_kernel(OwnArgs a) {
    __shared__ JoinLds<1> lds;
    own_decode<I8, WHOLE>(a, lds, blockIdx.x);
}

// The batch over its shared prefix, and in the workgroups behind those over the sequences' own caches: one launch. Without
// LDS in the loop every wave loads, converts and sorts its tokens for at most 32 rows: 64K tokens in bf16, eight KV heads,
// 16 rows 48 to 50 us (5.5 TB/s), 32 rows 52 (5.2), 64 rows in two tiles 62; 128K in 8 bits, 16 rows 48 to 50 (5.6), 32
// rows 62 (4.4, the vector instructions). Three waves per SIMD for 16 rows: with two, four sequences on 64K tokens with 16K of their own take 106 us, not 98.
template <int CT, bool I8, bool OWN8>
__global__ __launch_bounds__(kThreads, CT == 1 ? 3 : 2) void prefix_kernel(PrefixArgs a, OwnArgs own) {
    __shared__ union {
        JoinLds<CT> lds;
        JoinLds<1> own_lds;
    } sm;
    if ((int)blockIdx.x >= a.wgs) {
        own_decode<OWN8>(own, sm.own_lds, blockIdx.x - a.wgs);
        return;
    }
    JoinLds<CT>& lds = sm.lds;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int g = lane >> 4, n = lane & 15;
    // Workgroups of one run but different tiles read the same tokens: they are eight apart, on one XCD (consecutive
    // workgroups go to the eight XCDs in turn).
    const int tile = (int)(blockIdx.x >> 3) % a.tiles;
    const int pair = (int)(blockIdx.x >> 3) / a.tiles * 8 + (int)(blockIdx.x & 7);
    if (pair >= a.Hkv * a.S) return;
    const int kvh = pair / a.S, run = pair % a.S;
    const int rows = a.B * a.G;
    const int gs = __builtin_ctz(a.G);
    v8bf q[CT][4];
    int len[CT], lim[CT], longest = 0, shortest = INT32_MAX;
#pragma unroll
    for (int c = 0; c < CT; ++c) {                      // queries and lengths, asked for together
        const int r = (tile * CT + c) * 16 + n, b = min(r >> gs, a.B - 1);
        load_query<I8>(q[c], a.q + ((size_t)b * a.Hq + kvh * a.G + (r & (a.G - 1))) * kD, g);
        len[c] = a.prefix_lens[b];
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const bool live = (tile * CT + c) * 16 + n < rows;
        lim[c] = live ? min(max(len[c], 0), a.Pcap) : INT32_MAX;
        longest = max(longest, live ? lim[c] : 0);
        shortest = min(shortest, lim[c]);
    }
#pragma unroll
    for (int x = 8; x; x >>= 1) {
        longest = max(longest, __shfl_xor(longest, x));
        shortest = min(shortest, __shfl_xor(shortest, x));
    }
    longest = __builtin_amdgcn_readfirstlane(longest);
    shortest = __builtin_amdgcn_readfirstlane(shortest);
    // equal runs of whole rounds, the first ones one longer
    const int units = (longest + kRound - 1) / kRound, each = units / a.S, more = units - each * a.S;
    const int begin = (each * run + min(run, more)) * kRound;
    const int end = min(begin + (each + (run < more)) * kRound, longest);
    const size_t row0 = (size_t)kvh * a.Pcap, bytes = I8 ? kD : 2 * kD;
    const KvSource kv{a.kv.k + row0 * bytes, a.kv.v + row0 * bytes, I8 ? a.kv.k_absmax + row0 : nullptr,
                      I8 ? a.kv.v_absmax + row0 : nullptr};
    RowState<CT> st;
    st.clear();
    const float zscale = a.scale * kLog2e / (I8 ? 127.f : 1.f);
    attend<CT, I8, kTwoParts>(st, q, kv, begin, end, longest, lim, shortest, zscale, wave, n, g);
    if (!I8 && __ballot(!st.all_finite()) != 0) {
        st.clear();
        attend<CT, I8, kTwoPartsFinite>(st, q, kv, begin, end, longest, lim, shortest, zscale, wave, n, g);
    }
    join_waves(lds, st, wave, n, g);
    const size_t out0 = ((size_t)pair * a.tiles + tile) * (16 * CT);
    const int live = min(16 * CT, rows - tile * 16 * CT);
    for (int i = tid; i < live * (kD / 4); i += kThreads) {
        const int r = i >> 5, d4 = i & 31;
        const float4 x = *reinterpret_cast<const float4*>(&lds.acc[0][r][4 * d4]);
        const float4 y = *reinterpret_cast<const float4*>(&lds.acc[1][r][4 * d4]);
        *reinterpret_cast<float4*>(a.part_acc + (out0 + r) * kD + 4 * d4) = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
        if (d4 == 0) {
            float m, l;
            joined_ml(lds, r, m, l);
            a.part_m[out0 + r] = m;
            a.part_l[out0 + r] = l;
        }
    }
}

template __global__ void own_decode_kernel<false, false>(OwnArgs);
template __global__ void own_decode_kernel<true, false>(OwnArgs);
template __global__ void own_decode_kernel<true, true>(OwnArgs);
template __global__ void prefix_kernel<1, false, false>(PrefixArgs, OwnArgs);
template __global__ void prefix_kernel<1, false, true>(PrefixArgs, OwnArgs);
template __global__ void prefix_kernel<1, true, false>(PrefixArgs, OwnArgs);
template __global__ void prefix_kernel<1, true, true>(PrefixArgs, OwnArgs);
template __global__ void prefix_kernel<2, false, false>(PrefixArgs, OwnArgs);
template __global__ void prefix_kernel<2, false, true>(PrefixArgs, OwnArgs);
template __global__ void prefix_kernel<2, true, false>(PrefixArgs, OwnArgs);
template __global__ void prefix_kernel<2, true, true>(PrefixArgs, OwnArgs);

}  // namespace ffd
