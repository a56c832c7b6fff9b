// Workgroups of a ragged batch in proportion to its sequences' blocks, for the decode kernels over whole caches
// (DenseArgs, OwnArgs).
#pragma once

#include "ffd_device.h"

namespace ffd {

// floor(x / n) of non-negative integers below 2^52, rn = 1.0 / n: the product is off by less than one.
__device__ __forceinline__ long long floor_div(long long x, long long n, double rn) {
    long long q = (long long)((double)x * rn);
    const long long r = x - q * n;
    if (r < 0) --q;
    else if (r >= n) ++q;
    return q;
}

// Balanced mode: this workgroup's (sequence, KV head), the sequence's length and the run of blocks, computed by every
// wave alone from the sequence lengths (lane l: sequences 4l .. 4l + 3). Returns false for a workgroup past the last
// one used.
template <class Args>
__device__ __forceinline__ bool balanced_share(const Args& a, int wg, int lane, int& b, int& kvh, int& L, int& jb,
                                               int& je) {
    int len[4], nb[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) len[k] = a.seq_lens[min(4 * lane + k, a.B - 1)];        // asked for together
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        len[k] = 4 * lane + k < a.B ? min(max(len[k], 0), a.Lcap) : 0;
        nb[k] = (len[k] + kBlock - 1) / kBlock;
        sum += nb[k];
    }
    const int incl = wave_inclusive_scan(sum);
    const long long N = (long long)__builtin_amdgcn_readlane(incl, 63) * a.Hkv;
    const long long W = (long long)a.S * a.B * a.Hkv;
    const long long Weff = N > 0 ? min(W, N) : 1;
    const double rN = 1.0 / (double)max(N, 1LL);
    int wb[4], span = 0;                            // workgroups per KV head of each sequence
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        wb[k] = 4 * lane + k < a.B ? (nb[k] > 0 ? (int)floor_div((long long)nb[k] * Weff + N - 1, N, rN) : 1) : 0;
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
    int wsel = wb[0], lsel = len[0];
#pragma unroll
    for (int k = 1; k < 4; ++k) if (kk == k) { wsel = wb[k]; lsel = len[k]; }
    const int Wb = __builtin_amdgcn_readlane(wsel, src);
    L = __builtin_amdgcn_readlane(lsel, src);
    const int n = (L + kBlock - 1) / kBlock;
    const int Qb = __builtin_amdgcn_readlane(q0, src);
    b = 4 * src + kk;
    kvh = (wg - Qb) / Wb;
    const int p = (wg - Qb) % Wb;
    const double rW = 1.0 / (double)Wb;
    jb = (int)floor_div((long long)p * n, Wb, rW);
    je = (int)floor_div((long long)(p + 1) * n, Wb, rW);
    if (p == 0 && lane == 0 && threadIdx.x == 0)
        a.table[(size_t)b * a.Hkv + kvh] = make_int2(Qb + kvh * Wb, Qb + kvh * Wb + Wb - 1);
    return true;
}

}  // namespace ffd
