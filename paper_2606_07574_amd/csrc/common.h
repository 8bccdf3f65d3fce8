// common.h -- what the kernels' sources share: vector types, bf16 conversions, 16-byte chunks of
// a stream's row, and the host side's checks and launches.
#ifndef BIRKHOFF_COMMON_H
#define BIRKHOFF_COMMON_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <tuple>

#include "birkhoff4.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ float rcp(float x) { return __builtin_amdgcn_rcpf(x); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two values rounded to nearest even bf16 in one word (the hardware conversion).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

template <int DX>
struct MixChunk {  // channels in one 16-byte chunk of a row
    static constexpr int E = (DX == BIRKHOFF4_BF16) ? 8 : 4;
};

template <int DX>
__device__ __forceinline__ void unpack_chunk(const v4u w, float v[MixChunk<DX>::E]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (DX == BIRKHOFF4_BF16) {
            v[2 * k + 0] = __uint_as_float(u[k] << 16);
            v[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
        } else {
            v[k] = __uint_as_float(u[k]);
        }
    }
}

// bf16 outputs are rounded to nearest even (the hardware conversion).
template <int DX>
__device__ __forceinline__ v4u pack_chunk(const float v[MixChunk<DX>::E]) {
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (DX == BIRKHOFF4_BF16)
            u[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
        else
            u[k] = __float_as_uint(v[k]);
    }
    return v4u{u[0], u[1], u[2], u[3]};
}

// Sum over the four lanes of a quad, in the association ((x0 + x1) + (x2 + x3)); all four
// lanes receive the same value. Contraction is off here: fused into a product computed by the
// caller, the first add would become fma(own factors, partner's rounded product), which
// differs between partner lanes, and the quad's replicated step control would split.
__device__ __forceinline__ float qsum(float x) {
#pragma clang fp contract(off)
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, true));  // (1,0,3,2)
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, true));  // (2,3,0,1)
    return x;
}

// Sum over the two lanes of a pair (2k, 2k + 1); both receive the same value (the add
// commutes, and contraction is off so that it is not fused into the caller's product).
__device__ __forceinline__ float psum(float x) {
#pragma clang fp contract(off)
    return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, true));
}

// Sum over a group of G lanes, the same value in all of them (contraction off as in qsum):
// partners (1,0,3,2), then (2,3,0,1), then, with eight lanes, the other quad by a mirror.
template <int G>
__device__ __forceinline__ float gsum_lanes(float x) {
#pragma clang fp contract(off)
    if constexpr (G == 2) return psum(x);
    x = qsum(x);
    if constexpr (G == 8)
        x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xF, 0xF, true));  // row_half_mirror
    return x;
}

// Sums over lanes by halving exchanges: a step adds, for each pair of values, the two halves
// of the lanes that differ in bit M, and leaves one value of the pair in each half, so 2 n
// values become n. Between the halves of the wave and of 32 lanes that is a register swap and
// an add; within 16 lanes a DPP move (half-mirror for the partner across 4: lanes i and 7 - i,
// whose lower bits the later steps sum over).
template <int M>
__device__ __forceinline__ float halve_pair(float a, float b, int lane) {
    if constexpr (M == 32 || M == 16) {
        const auto r = M == 32 ? __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false)
                               : __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        constexpr int kCtrl = M == 8 ? 0x128 : M == 4 ? 0x141 : M == 2 ? 0x4E : 0xB1;  // row_ror:8, half-mirror, quad_perm
        const bool hi = (lane & M) != 0;
        const float keep = hi ? b : a, send = hi ? a : b;
        return keep + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(send), kCtrl, 0xF, 0xF, true));
    }
}

// The values v[0 .. NV) summed over the 2 M lanes that share the bits above M: lane c of them
// keeps the sums of values NV / (2 M) c onwards (NV / (2 M) of them), or, where NV < 2 M, the
// one of value c NV / (2 M), its lowest bits still to be summed over.
template <int M, int NV>
__device__ __forceinline__ void lane_sums(const float (&v)[NV], float (&out)[NV / (2 * M) > 0 ? NV / (2 * M) : 1],
                                          int lane) {
    if constexpr (M == 0 || NV == 1) {
#pragma unroll
        for (int k = 0; k < NV; ++k) out[k] = v[k];
    } else {
        float h[NV / 2];
#pragma unroll
        for (int k = 0; k < NV / 2; ++k) h[k] = halve_pair<M>(v[k], v[k + NV / 2], lane);
        if constexpr (M == 1) {
#pragma unroll
            for (int k = 0; k < NV / 2; ++k) out[k] = h[k];
        } else {
            lane_sums<M / 2, NV / 2>(h, out, lane);
        }
    }
}

// Sum over the 64 / N lanes that lane_sums leaves of one of N values, in all of them.
template <int N>
__device__ __forceinline__ float rest_sum(float x) {
    x = gsum_lanes<8>(x);
    if constexpr (N == 4)
        x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xF, 0xF, true));  // row_ror:8
    return x;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int kMaxDevices = 64;
int g_cus[kMaxDevices];  // cached compute-unit counts (0 = not queried yet)

// Compute units of the device that `stream` belongs to (the null stream: the current device).
int device_cus(hipStream_t stream, int* cus, int* dev_out = nullptr) {
    hipDevice_t dev = 0;
    if (hipStreamGetDevice(stream, &dev) != hipSuccess || dev < 0 || dev >= kMaxDevices)
        return BIRKHOFF4_ERR_DEVICE;
    if (g_cus[dev] == 0) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
            return BIRKHOFF4_ERR_DEVICE;
        g_cus[dev] = n;
    }
    *cus = g_cus[dev];
    if (dev_out) *dev_out = dev;
    return BIRKHOFF4_OK;
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

struct Span {
    const void* p;
    size_t bytes;
};

// No output overlaps another output or an input.
bool disjoint(const Span* outs, int no, const Span* ins, int ni) {
    for (int a = 0; a < no; ++a) {
        for (int b = a + 1; b < no; ++b)
            if (overlaps(outs[a].p, outs[a].bytes, outs[b].p, outs[b].bytes)) return false;
        for (int b = 0; b < ni; ++b)
            if (overlaps(outs[a].p, outs[a].bytes, ins[b].p, ins[b].bytes)) return false;
    }
    return true;
}

size_t dtype_bytes(int dt) { return dt == BIRKHOFF4_BF16 ? 2 : 4; }
bool dtype_ok(int dt) { return dt == BIRKHOFF4_F32 || dt == BIRKHOFF4_BF16; }

// Status of the launches made by this thread since the last call: taken from each launch's
// own return value, so an error left pending by someone else's earlier launch is neither
// reported as ours nor cleared.
thread_local int t_launch = BIRKHOFF4_OK;

template <typename... KArgs, typename... Args>
void launch_kernel(void (*kern)(KArgs...), dim3 grid, dim3 block, unsigned lds, hipStream_t stream, Args... args) {
    static_assert(sizeof...(KArgs) == sizeof...(Args), "kernel argument count");
    std::tuple<KArgs...> vals(args...);
    void* ptrs[sizeof...(KArgs)];
    std::apply([&](auto&... v) {
        int k = 0;
        ((ptrs[k++] = static_cast<void*>(&v)), ...);
    }, vals);
    if (hipLaunchKernel(reinterpret_cast<const void*>(kern), grid, block, ptrs, lds, stream) != hipSuccess &&
        t_launch == BIRKHOFF4_OK)
        t_launch = BIRKHOFF4_ERR_LAUNCH;
}

int launch_status() {
    const int r = t_launch;
    t_launch = BIRKHOFF4_OK;
    return r;
}

}  // namespace

#endif  // BIRKHOFF_COMMON_H
