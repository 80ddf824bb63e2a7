// Activations held in 8 bits (include/pp_act8.h).
#include <hip/hip_runtime.h>

#include "adapter_rules.hpp"
#include "pieces.hpp"
#include "pp_act8.h"

namespace ppc {

struct Act8Args {
    const void* x;              // [rows][n]
    int8_t* q;                  // [rows][pitch]
    uint8_t* scale;             // [blocks][scale_pitch]
    int64_t pitch, scale_pitch, units;      // units: rows * blocks
    int32_t rows, n, blocks;
};

// Sixteen lanes take a row's block of 128 values, eight to a lane.  Magnitudes are compared as whole numbers, which orders them and puts
// infinities and NaN on top.  Bound by memory: every value is read once and a byte of it written.
template <typename T> __global__ __launch_bounds__(256) void act8_pack(const Act8Args a) {
    constexpr uint32_t kInfBits = 0x7f800000u;
    const int part = (int)(threadIdx.x & 15u);
    for (int64_t unit = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); unit < a.units; unit += (int64_t)gridDim.x * 16) {
        const int row = (int)(unit / a.blocks), b = (int)(unit - (int64_t)row * a.blocks);
        const int t = b * kAct8Block + part * 8;
        const k8_any<T, 8> v = k8_load<T, 8>(static_cast<const T*>(a.x) + (int64_t)row * a.n + t, a.n - t);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = __builtin_bit_cast(uint32_t, (float)v[i]) & 0x7fffffffu;
            top = bits > top ? bits : top;
        }
#pragma unroll
        for (int x = 1; x < 16; x *= 2) {
            const uint32_t o = (uint32_t)__shfl_xor((int)top, x);
            top = o > top ? o : top;
        }
        // amax = 1.m * 2^E: e = E - 6 if 1.m <= 127 / 64, else E - 5
        int e = (int)(top >> 23) - 127 - ((top & 0x7fffffu) <= 0x7e0000u ? 6 : 5);
        e = e < -126 ? -126 : e;
        const bool bad = top >= kInfBits;
        const float inv = __builtin_bit_cast(float, (uint32_t)(127 - (bad ? 0 : e)) << 23);
        uint32_t word[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float f = (float)v[i];
            int q = bad ? 0 : (int)__builtin_rintf(f * inv);
            if (q == 0) q = f < 0.0f ? -1 : (f == 0.0f ? 0 : 1);
            word[i >> 2] |= ((uint32_t)q & 0xffu) << (8 * (i & 3));
        }
        *reinterpret_cast<uint2*>(a.q + (int64_t)row * a.pitch + t) = uint2{word[0], word[1]};
        if (part == 0) a.scale[(int64_t)b * a.scale_pitch + row] = (uint8_t)(bad ? 255 : e + 127);
    }
}

template <typename T> __global__ __launch_bounds__(256) void act8_unpack(const Act8Args a) {
    const int part = (int)(threadIdx.x & 15u);
    for (int64_t unit = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); unit < a.units; unit += (int64_t)gridDim.x * 16) {
        const int row = (int)(unit / a.blocks), b = (int)(unit - (int64_t)row * a.blocks);
        const int t = b * kAct8Block + part * 8;
        const uint2 q = *reinterpret_cast<const uint2*>(a.q + (int64_t)row * a.pitch + t);
        const uint32_t s = a.scale[(int64_t)b * a.scale_pitch + row];
        const float factor = __builtin_bit_cast(float, s == 255u ? 0x7fc00000u : s << 23);
        k8_any<T, 8> v;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f = (float)(int8_t)((i < 4 ? q.x : q.y) >> (8 * (i & 3))) * factor;
            if (sizeof(T) == 2) f = f > 65504.0f ? 65504.0f : (f < -65504.0f ? -65504.0f : f);
            v[i] = (T)f;
        }
        k8_store<T, 8>(const_cast<T*>(static_cast<const T*>(a.x)) + (int64_t)row * a.n + t, a.n - t, v);
    }
}

}  // namespace ppc

namespace {

using namespace ppc;

pp_status_t act8_check(const void* x_dev, int32_t rows, int32_t n, int32_t dtype, const void* held_dev) {
    if (!x_dev || !held_dev) return PP_ERR_NULL;
    if (rows < 1 || n < 1 || (int64_t)rows * n >= ((int64_t)1 << 31)) return PP_ERR_SHAPE;
    if (dtype != PP_F16 && dtype != PP_F32) return PP_ERR_UNSUPPORTED;
    const uintptr_t xa = reinterpret_cast<uintptr_t>(x_dev), ha = reinterpret_cast<uintptr_t>(held_dev);
    if ((xa | ha) & 15u) return PP_ERR_ALIGN;
    const uintptr_t xe = xa + (uintptr_t)((int64_t)rows * n * (dtype == PP_F16 ? 2 : 4)), he = ha + (uintptr_t)act8_bytes(rows, n);
    return xa < he && ha < xe ? PP_ERR_ALIGN : PP_OK;
}

Act8Args act8_args(const void* x_dev, int32_t rows, int32_t n, void* held_dev) {
    Act8Args a;
    a.x = x_dev, a.q = static_cast<int8_t*>(held_dev);
    a.rows = rows, a.n = n, a.blocks = (n + kAct8Block - 1) / kAct8Block;
    a.pitch = act8_pitch(n), a.scale_pitch = act8_scale_pitch(rows);
    a.scale = static_cast<uint8_t*>(held_dev) + rows * a.pitch;
    a.units = (int64_t)rows * a.blocks;
    return a;
}

unsigned act8_grid(const Act8Args& a) {
    const int64_t wgs = (a.units + 15) / 16;
    return (unsigned)(wgs < (1 << 20) ? wgs : (1 << 20));
}

}  // namespace

extern "C" {

int64_t pp_act8_bytes(int32_t rows, int32_t n) {
    if (rows < 1 || n < 1 || (int64_t)rows * n >= ((int64_t)1 << 31)) return 0;
    return act8_bytes(rows, n);
}

pp_status_t pp_act8_pack(const void* x_dev, int32_t rows, int32_t n, int32_t dtype, void* held_dev, void* hip_stream) {
    const pp_status_t st = act8_check(x_dev, rows, n, dtype, held_dev);
    if (st != PP_OK) return st;
    const Act8Args a = act8_args(x_dev, rows, n, held_dev);
    (void)hipGetLastError();
    if (dtype == PP_F16) hipLaunchKernelGGL(act8_pack<_Float16>, dim3(act8_grid(a)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    else hipLaunchKernelGGL(act8_pack<float>, dim3(act8_grid(a)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_DEVICE;
}

pp_status_t pp_act8_unpack(const void* held_dev, int32_t rows, int32_t n, int32_t dtype, void* x_dev, void* hip_stream) {
    const pp_status_t st = act8_check(x_dev, rows, n, dtype, held_dev);
    if (st != PP_OK) return st;
    const Act8Args a = act8_args(x_dev, rows, n, const_cast<void*>(held_dev));
    (void)hipGetLastError();
    if (dtype == PP_F16) hipLaunchKernelGGL(act8_unpack<_Float16>, dim3(act8_grid(a)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    else hipLaunchKernelGGL(act8_unpack<float>, dim3(act8_grid(a)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_DEVICE;
}

}  // extern "C"
