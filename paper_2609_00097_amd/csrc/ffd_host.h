// Host helpers of the C ABI's sources: the device's compute units, argument checks, launch status, workspace parts.
#pragma once

#include <atomic>
#include <cstddef>
#include <cstdint>

#include "ffd.h"
#include "ffd_device.h"
#include "ffd_kernels.h"

namespace ffd {

// Compute units of the current device, queried once per device and cached (with the no-alloc
// entry point's per-device scratch address, the only state the library keeps). kFallbackCus
// (an MI355X's count) is used if the query fails.
constexpr int kFallbackCus = 256;
constexpr int kMaxDevices = 64;
inline std::atomic<int> g_cus[kMaxDevices];

inline int lookup_cus() {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return kFallbackCus;
    int n = g_cus[dev].load(std::memory_order_relaxed);
    if (n > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
        n = kFallbackCus;
    g_cus[dev].store(n, std::memory_order_relaxed);
    return n;
}

// The count, looked up once per call of an entry point (a call's sizes ask for it a dozen times, and the
// current device can change between calls only).
inline thread_local int t_call_cus = 0;
struct CallScope {
    const int outer = t_call_cus;
    CallScope() { if (outer == 0) t_call_cus = lookup_cus(); }
    ~CallScope() { t_call_cus = outer; }
};
inline int device_cus() { return t_call_cus != 0 ? t_call_cus : lookup_cus(); }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int launch_status() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FFD_OK : FFD_ERR_HIP;
}

// Partial states of `rows` heads, at the start of a workspace: acc [rows, D], then m [rows], l [rows] (fp32). acc
// comes first because the merge reads it four floats at a time: after an odd number of m and l (one query head
// per KV head, odd counts) its rows would lie on 8 bytes only.
struct Partials {
    float* m;
    float* l;
    float* acc;
};

constexpr size_t kAlign = 256;
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline size_t partials_bytes(size_t rows) { return rows * (kD + 2) * sizeof(float); }

inline Partials carve(void* ws, size_t rows) {
    static_assert(kD * sizeof(float) % 16 == 0, "rows of acc on 16 bytes, like the workspace");
    float* acc = static_cast<float*>(ws);
    return Partials{acc + rows * kD, acc + rows * (kD + 1), acc};
}

// Pointers of a cache argument: all there and aligned; *bits is 8 or 16. An 8-bit one is required where only8.
inline int check_kv(const ffd_kv* c, bool only8, int* bits) {
    if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return FFD_ERR_INVALID_ARGUMENT;
    if (!c->k_absmax != !c->v_absmax || (only8 && !c->k_absmax)) return FFD_ERR_INVALID_ARGUMENT;
    if (c->k_absmax && (!aligned16(c->k_absmax) || !aligned16(c->v_absmax))) return FFD_ERR_INVALID_ARGUMENT;
    *bits = c->k_absmax ? 8 : 16;
    return FFD_OK;
}

inline KvSource source_of(const ffd_kv& c) {
    return KvSource{static_cast<const uint8_t*>(c.k), static_cast<const uint8_t*>(c.v),
                    static_cast<const uint16_t*>(c.k_absmax), static_cast<const uint16_t*>(c.v_absmax)};
}

}  // namespace ffd
