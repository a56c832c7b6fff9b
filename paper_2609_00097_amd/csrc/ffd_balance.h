// Workgroups of a ragged batch in proportion to its sequences' blocks, for the decode kernels over whole caches
// (DenseArgs, OwnArgs).
#pragma once

#include "ffd_device.h"

namespace ffd {

// 1 / n to 2^-44: the hardware's estimate (2^-22 or better) and one step of Newton's method.
__device__ __forceinline__ double reciprocal(double n) {
    const double r = __builtin_amdgcn_rcp(n);
    return fma(fma(-n, r, 1.0), r, r);
}

// floor(x / n) of non-negative integers, quotient below 2^40, x below 2^52, rn = reciprocal(n): the product is off by
// less than one.
__device__ __forceinline__ long long floor_div(long long x, long long n, double rn) {
    long long q = (long long)((double)x * rn);
    const long long r = x - q * n;
    if (r < 0) --q;
    else if (r >= n) ++q;
    return q;
}

// Balanced mode: this workgroup's (sequence, KV head), the sequence's length and the run of blocks, computed by every
// wave alone from the sequence lengths, 64 sequences at a time (B <= 256). Returns false for a workgroup past the last
// one used.
template <class Args>
__device__ __forceinline__ bool balanced_share(const Args& a, int wg, int lane, int& b, int& kvh, int& L, int& jb,
                                               int& je) {
    int len[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) len[k] = a.seq_lens[min(lane + 64 * k, a.B - 1)];       // asked for together
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        len[k] = lane + 64 * k < a.B ? min(max(len[k], 0), a.Lcap) : 0;
        sum += (len[k] + kBlock - 1) / kBlock;
    }
    const long long N = (long long)__builtin_amdgcn_readlane(wave_inclusive_scan(sum), 63) * a.Hkv;
    const long long W = (long long)a.S * a.B * a.Hkv;
    const long long Weff = N > 0 ? min(W, N) : 1;
    const double rN = reciprocal((double)max(N, 1LL));
    int Wb = 0, Qb = 0;                             // workgroups per KV head of the sequence, the first of them
#pragma unroll
    for (int k = 0, before = 0; k < 4; ++k) {
        if (64 * k >= a.B) return false;            // uniform, as the next
        const int nb = (len[k] + kBlock - 1) / kBlock;
        const int wb = lane + 64 * k < a.B ? (nb > 0 ? (int)floor_div((long long)nb * Weff + N - 1, N, rN) : 1) : 0;
        const int span = wb * a.Hkv, incl = wave_inclusive_scan(span), q0 = before + incl - span;
        const uint64_t hit = __ballot(wg >= q0 && wg < q0 + span);
        if (hit != 0) {
            const int src = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hit));
            Wb = __builtin_amdgcn_readlane(wb, src);
            Qb = __builtin_amdgcn_readlane(q0, src);
            L = __builtin_amdgcn_readlane(len[k], src);
            b = 64 * k + src;
            break;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    if (Wb == 0) return false;
    const int n = (L + kBlock - 1) / kBlock;
    kvh = (wg - Qb) / Wb;
    const int p = wg - Qb - kvh * Wb;
    const double rW = reciprocal((double)Wb);
    jb = (int)floor_div((long long)p * n, Wb, rW);
    je = (int)floor_div((long long)(p + 1) * n, Wb, rW);
    if (p == 0 && threadIdx.x == 0)
        a.table[(size_t)b * a.Hkv + kvh] = make_int2(Qb + kvh * Wb, Qb + kvh * Wb + Wb - 1);
    return true;
}

}  // namespace ffd
