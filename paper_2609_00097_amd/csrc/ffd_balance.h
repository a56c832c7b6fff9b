// Workgroups of a ragged batch in proportion to its sequences' blocks, for the decode kernels over whole caches
// (DenseArgs, Kv8Args).
#pragma once

#include "ffd_device.h"

namespace ffd {

// Balanced mode: this workgroup's (sequence, KV head) and run of blocks, computed by every wave
// alone from the sequence lengths (lane l: sequences 4l .. 4l + 3). Returns false for a workgroup
// past the last one used.
template <class Args>
__device__ __forceinline__ bool balanced_share(const Args& a, int wg, int lane, int& b, int& kvh, int& jb,
                                               int& je) {
    int nb[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int bi = 4 * lane + k;
        const int L = bi < a.B ? min(max(a.seq_lens[bi], 0), a.Lcap) : 0;
        nb[k] = (L + kBlock - 1) / kBlock;
        sum += nb[k];
    }
    const int incl = wave_inclusive_scan(sum);
    const long long N = (long long)__builtin_amdgcn_readlane(incl, 63) * a.Hkv;
    const long long W = (long long)a.S * a.B * a.Hkv;
    const long long Weff = N > 0 ? min(W, N) : 1;
    int wb[4], span = 0;                            // workgroups per KV head of each sequence
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int bi = 4 * lane + k;
        wb[k] = bi < a.B ? (nb[k] > 0 ? (int)(((long long)nb[k] * Weff + N - 1) / N) : 1) : 0;
        span += wb[k] * a.Hkv;
    }
    const int sincl = wave_inclusive_scan(span);
    int q0 = sincl - span, hit = -1;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (hit < 0 && wg >= q0 && wg < q0 + wb[k] * a.Hkv) hit = k;
        if (hit < 0) q0 += wb[k] * a.Hkv;
    }
    const uint64_t hb = __ballot(hit >= 0);
    if (hb == 0) return false;                      // uniform: past the last sequence's workgroups
    const int src = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hb));
    const int kk = __builtin_amdgcn_readlane(hit, src);
    int wsel = wb[0], nsel = nb[0];
#pragma unroll
    for (int k = 1; k < 4; ++k) if (kk == k) { wsel = wb[k]; nsel = nb[k]; }
    const int Wb = __builtin_amdgcn_readlane(wsel, src), n = __builtin_amdgcn_readlane(nsel, src);
    const int Qb = __builtin_amdgcn_readlane(q0, src);
    b = 4 * src + kk;
    kvh = (wg - Qb) / Wb;
    const int p = (wg - Qb) % Wb;
    jb = (int)((long long)p * n / Wb);
    je = (int)((long long)(p + 1) * n / Wb);
    if (p == 0 && lane == 0 && threadIdx.x == 0)
        a.table[(size_t)b * a.Hkv + kvh] = make_int2(Qb + kvh * Wb, Qb + kvh * Wb + Wb - 1);
    return true;
}

}  // namespace ffd
