// Log-sum-exp merge of split partials (the flash-decoding reduction, Sec. 2): for each (sequence,
// query head), M* = max_s m_s, l* = sum_s e^{m_s - M*} l_s, out = sum_s e^{m_s - M*} acc_s / l*,
// lse = M* + ln l*. Splits that kept nothing carry m = -inf and are skipped (their l and acc may hold
// anything); a head with no split gets out = 0 and lse = -inf.
//
// Partial rows of head bh = b * Hq + h: i * G + bh % G for i = first .. last, (first, last) = table[bh / G]
// (last < first: none), or, without a table, the S rows from S * (bh / G) on.
//
// Bound: latency (a table load, the rows, two reductions, the store), and with very many heads the number
// of waves. One workgroup of NW waves per head and quarter of its dims, so that few heads still spread over
// the CUs; thread (r, d4) takes rows r, r + 8 NW, ... of dims 4 d4 .. 4 d4 + 3, all of a batch's rows
// requested at once (16 NW rows, or 64 NW where there are more), their common maximum first and then one
// rescaling per row. Against one workgroup per head that folded the rows one after the other: 4 heads of
// 256 rows 6.4 -> 3.9 us (NW = 4), the step at 1 x 256K 25.7 -> 23.9 us;
// 1024, 2048 and 4096 heads of 2 to 4 rows 5.2, 9.3 and 16.0 -> 4.0, 5.0 and 8.0 us (NW = 1; 6.3, 10.8 and
// 18.8 us with four waves).
#include "ffd_device.h"
#include "ffd_kernels.h"

namespace ffd {

namespace {

constexpr int kSliceDims = kD / kMergeSlices;  // 8 lanes of 4 dims

struct State {
    float m, l;
    float a[4];
};

__device__ __forceinline__ float rescale(float m, float M) { return m == -INFINITY ? 0.f : __expf(m - M); }

// Places of partial rows: `count` of them from `first` on.
struct Rows {
    size_t first, stride;
    int count;
};

// Rows s0 + LANES u (u < U) below rows.count: loaded, and folded into a state. The row index is clamped, so that the
// loads are unconditional.
template <int U, int LANES>
struct Batch {
    float m[U], l[U];
    float4 a[U];
    __device__ __forceinline__ void load(const float* __restrict__ part_m, const float* __restrict__ part_l,
                                         const float* __restrict__ part_acc, const Rows& rows, int s0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * LANES;
            const size_t row = rows.first + (size_t)min(s, rows.count - 1) * rows.stride;
            m[u] = part_m[row];
            l[u] = part_l[row];
            a[u] = *reinterpret_cast<const float4*>(part_acc + row * kD);
            if (s >= rows.count) m[u] = -INFINITY;
        }
    }
    __device__ __forceinline__ void fold(State& st) const {
        float M = st.m;
#pragma unroll
        for (int u = 0; u < U; ++u) M = fmaxf(M, m[u]);
        const float c = rescale(st.m, M);
        st.m = M;
        st.l *= c;
#pragma unroll
        for (int e = 0; e < 4; ++e) st.a[e] *= c;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float w = rescale(m[u], M);
            const bool any = m[u] != -INFINITY;         // else l and a may be NaN
            st.l = fmaf(w, any ? l[u] : 0.f, st.l);
            st.a[0] = fmaf(w, any ? a[u].x : 0.f, st.a[0]);
            st.a[1] = fmaf(w, any ? a[u].y : 0.f, st.a[1]);
            st.a[2] = fmaf(w, any ? a[u].z : 0.f, st.a[2]);
            st.a[3] = fmaf(w, any ? a[u].w : 0.f, st.a[3]);
        }
    }
};
template <int U, int LANES>
__device__ __forceinline__ void fold_rows(State& st, const float* __restrict__ part_m, const float* __restrict__ part_l,
                                          const float* __restrict__ part_acc, const Rows& rows, int s0) {
    Batch<U, LANES> x;
    x.load(part_m, part_l, part_acc, rows, s0);
    x.fold(st);
}

// max and sum over the lanes that differ in bits 3, 4 and 5 (the rows of a wave)
__device__ __forceinline__ float rows_max(float x) {
    x = fmaxf(x, dpp_f<kDppRor8>(x));
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
    x += dpp_f<kDppRor8>(x);
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Joins the states of NW waves, tid a thread's number among them, and writes head blockIdx.x's dims of a slice.
template <int NW>
__device__ __forceinline__ void finish(State st, float (&part)[NW][8][8], int tid, int slice, uint16_t* __restrict__ out,
                                       float* __restrict__ lse) {
    const int d4 = tid & 7, wave = tid >> 6, lane = tid & 63;
    const float M = rows_max(st.m);
    const float c = rescale(st.m, M);
    const float l = rows_sum(st.l * c);
    float a[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = rows_sum(st.a[e] * c);
    if (lane < 8) {
        *reinterpret_cast<float4*>(&part[wave][d4][0]) = make_float4(a[0], a[1], a[2], a[3]);
        *reinterpret_cast<float2*>(&part[wave][d4][4]) = make_float2(M, l);
    }
    if constexpr (NW > 1) __syncthreads();
    else wave_lds_fence();
    if (tid >= 8) return;
    float Mw[NW], Mx = -INFINITY, lx = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        Mw[w] = part[w][d4][4];
        Mx = fmaxf(Mx, Mw[w]);
    }
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float cw = rescale(Mw[w], Mx);
        const float4 aw = *reinterpret_cast<const float4*>(&part[w][d4][0]);
        lx = fmaf(cw, part[w][d4][5], lx);
        o.x = fmaf(cw, aw.x, o.x);
        o.y = fmaf(cw, aw.y, o.y);
        o.z = fmaf(cw, aw.z, o.z);
        o.w = fmaf(cw, aw.w, o.w);
    }
    const bool any = Mx != -INFINITY;
    const float inv = any ? 1.f / lx : 0.f;
    uint2 packed;
    packed.x = (uint32_t)f32_to_bf16(o.x * inv) | ((uint32_t)f32_to_bf16(o.y * inv) << 16);
    packed.y = (uint32_t)f32_to_bf16(o.z * inv) | ((uint32_t)f32_to_bf16(o.w * inv) << 16);
    *reinterpret_cast<uint2*>(out + (size_t)blockIdx.x * kD + slice * kSliceDims + 4 * d4) = packed;
    if (lse && slice == 0 && d4 == 0) lse[blockIdx.x] = any ? Mx + logf(lx) : -INFINITY;
}

}  // namespace

// Grid (B * Hq, kMergeSlices).
template <int NW>
__global__ __launch_bounds__(64 * NW) void lse_merge_kernel(const float* __restrict__ part_m,
                                                             const float* __restrict__ part_l,
                                                             const float* __restrict__ part_acc, int S,
                                                             const int2* __restrict__ table, int G,
                                                             uint16_t* __restrict__ out, float* __restrict__ lse) {
    constexpr int kRowLanes = 8 * NW;               // rows in parallel
    alignas(16) __shared__ float part[NW][8][8];    // each wave's state per d4
    const int tid = threadIdx.x, d4 = tid & 7, r = tid >> 3;
    const size_t x = blockIdx.x / G;                        // blockIdx.x = b * Hq + h
    size_t first = x * S;
    if (table) {
        const int2 fl = table[x];
        first = fl.x;
        S = fl.y - fl.x + 1;
    }
    const Rows rows{first * G + blockIdx.x % G, (size_t)G, S};
    const float* acc = part_acc + blockIdx.y * kSliceDims + 4 * d4;
    State st{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    if (S > 2 * kRowLanes) {                                // uniform
        for (int s0 = 0; s0 < S; s0 += 8 * kRowLanes) fold_rows<8, kRowLanes>(st, part_m, part_l, acc, rows, s0 + r);
    } else if (S > 0) {
        fold_rows<2, kRowLanes>(st, part_m, part_l, acc, rows, r);
    }
    finish<NW>(st, part, tid, blockIdx.y, out, lse);
}

template __global__ void lse_merge_kernel<1>(const float*, const float*, const float*, int, const int2*, int, uint16_t*, float*);
template __global__ void lse_merge_kernel<4>(const float*, const float*, const float*, int, const int2*, int, uint16_t*, float*);


// The same over the rows of two attentions: the head's rows of the shared prefix, one of each workgroup of its tile, and
// the own cache's, all rows of one array. NW waves per slice as above; with one the workgroup's four waves take the four
// slices, so that there are fewer workgroups to dispatch (4096 heads of 18 rows: 14.5 us with a workgroup per slice, 12.1
// so; 1024 of 34 5.9).
template <int NW>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedMergeArgs a) {
    constexpr int kRowLanes = 8 * NW;
    alignas(16) __shared__ float part[4 / NW][NW][8][8];
    const int unit = threadIdx.x / (64 * NW), tid = threadIdx.x % (64 * NW), d4 = tid & 7, r = tid >> 3;
    const int slice = NW == 1 ? unit : blockIdx.y;
    const int b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, kvh = h / a.G;
    const size_t x = (size_t)b * a.Hkv + kvh;
    const float* acc = a.acc + slice * kSliceDims + 4 * d4;
    int2 fl = make_int2(0, -1);
    PrefixPlace p{0, a.tiles, a.S_prefix, b};
    if (a.table) fl = a.table[x];                           // both asked for before either is used
    if (a.places) p = a.places[b];
    const int q_row = p.place * a.G + h % a.G;
    if (!a.places) p.first = q_row / a.tile_rows;
    const Rows prefix{((size_t)kvh * a.S_prefix * a.tiles + p.first) * a.tile_rows + q_row % a.tile_rows,
                      (size_t)p.stride * a.tile_rows, p.count};
    // the prefix's first rows under way before the own ones are located (any row where there is none: nothing is
    // folded); those lie side by side without a table, with one with those of the group's other heads
    constexpr int U = NW == 1 ? 4 : 2;
    Batch<U, kRowLanes> x0;
    Batch<1, kRowLanes> y0;
    x0.load(a.m, a.l, acc, prefix.count > 0 ? prefix : Rows{0, 0, 1}, r);
    const Rows own{a.prefix_rows + (a.table ? (size_t)fl.x * a.G + h % a.G : (size_t)blockIdx.x * a.S_own),
                   a.table ? (size_t)a.G : 1, a.table ? fl.y - fl.x + 1 : a.S_own};
    y0.load(a.m, a.l, acc, own, r);
    State st{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    if (prefix.count > 0) x0.fold(st);                      // uniform
    y0.fold(st);
    for (int s0 = U * kRowLanes; s0 < prefix.count; s0 += U * kRowLanes) fold_rows<U, kRowLanes>(st, a.m, a.l, acc, prefix, s0 + r);
    for (int s0 = kRowLanes; s0 < own.count; s0 += 2 * kRowLanes) fold_rows<2, kRowLanes>(st, a.m, a.l, acc, own, s0 + r);
    finish<NW>(st, part[unit], tid, slice, a.out, a.lse);
}

template __global__ void shared_merge_kernel<1>(SharedMergeArgs);
template __global__ void shared_merge_kernel<4>(SharedMergeArgs);

}  // namespace ffd
