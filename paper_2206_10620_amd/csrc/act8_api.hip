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
    int64_t pitch, scale_pitch, units;      // units: rows * runs
    int32_t rows, n, blocks, runs;          // runs of kAct8Ahead blocks
};

// Sixteen lanes take a row's blocks of 128 values, eight to a lane, kAct8Ahead blocks at a time: the loads of all are on their way before
// the first is looked at.  Magnitudes are compared as whole numbers, which orders them and puts infinities and NaN on top.  Bound by memory:
// a value is read once and a byte of it written.
constexpr int kAct8Ahead = 4;

// The largest magnitude of a lane's eight values, as binary32's bits
__device__ __forceinline__ uint32_t act8_top(const k8_any<_Float16, 8>& v) {
    typedef uint16_t u8 __attribute__((ext_vector_type(8)));
    typedef uint16_t u2 __attribute__((ext_vector_type(2)));
    const u8 m = __builtin_bit_cast(u8, v) & (uint16_t)0x7fff;
    const u2 t = __builtin_elementwise_max(__builtin_elementwise_max(m.s01, m.s23), __builtin_elementwise_max(m.s45, m.s67));
    return __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, t.x > t.y ? t.x : t.y));
}
__device__ __forceinline__ uint32_t act8_top(const k8_any<float, 8>& v) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float f = v[i];                    // (a bit cast of an element itself would take the first one's)
        const uint32_t bits = __builtin_bit_cast(uint32_t, f) & 0x7fffffffu;
        top = bits > top ? bits : top;
    }
    return top;
}
// and of sixteen lanes: neighbours, pairs, then mirrored halves
__device__ __forceinline__ uint32_t act8_row_max(uint32_t v) {
    auto with = [&](uint32_t o) { v = o > v ? o : v; };
    with((uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true));
    with((uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true));
    with((uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));
    with((uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));
    return v;
}

template <typename T> __global__ __launch_bounds__(256) void act8_pack(const Act8Args a) {
    constexpr uint32_t kInfBits = 0x7f800000u;
    const int part = (int)(threadIdx.x & 15u);
    for (int64_t unit = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); unit < a.units; unit += (int64_t)gridDim.x * 16) {
        const int row = (int)(unit / a.runs), b0 = (int)(unit - (int64_t)row * a.runs) * kAct8Ahead;
        const T* src = static_cast<const T*>(a.x) + (int64_t)row * a.n;
        k8_any<T, 8> v[kAct8Ahead];
#pragma unroll
        for (int u = 0; u < kAct8Ahead; ++u) {
            const int64_t t = (int64_t)(b0 + u) * kAct8Block + part * 8;         // behind the last block it may pass 31 bits
            v[u] = k8_load<T, 8>(src + t, t < a.n ? a.n - (int)t : 0);
        }
#pragma unroll
        for (int u = 0; u < kAct8Ahead; ++u) {
            const int b = b0 + u;
            if (b >= a.blocks) break;
            const uint32_t top = act8_row_max(act8_top(v[u]));
            // amax = 1.m * 2^E: e = E - 6 if 1.m <= 127 / 64, else E - 5
            int e = (int)(top >> 23) - 127 - ((top & 0x7fffffu) <= 0x7e0000u ? 6 : 5);
            e = e < -126 ? -126 : e;
            const bool bad = top >= kInfBits;
            const float inv = __builtin_bit_cast(float, (uint32_t)(127 - (bad ? 0 : e)) << 23);
            uint32_t q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float f = (float)v[u][i];
                // what is not 0 stays so: 0.75 becomes 1.  1.5 * 2^23 added rounds to a whole number, ties to even, and leaves it in the low bits
                const float m = __builtin_copysignf(__builtin_fmaxf(__builtin_fabsf(f * inv), 0.75f), f);
                q[i] = __builtin_bit_cast(uint32_t, (f != 0.0f ? m : 0.0f) + 12582912.0f);
            }
            if (__builtin_amdgcn_ballot_w64(bad) != 0) {         // rare
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float f = (float)v[u][i];
                    if (bad) q[i] = f < 0.0f ? 0xffu : (f == 0.0f ? 0u : 1u);
                }
            }
            uint32_t word[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                word[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x0c0c0400u), __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400u), 0x05040100u);
            *reinterpret_cast<uint2*>(a.q + (int64_t)row * a.pitch + (int64_t)b * kAct8Block + part * 8) = uint2{word[0], word[1]};
            if (part == 0) a.scale[(int64_t)b * a.scale_pitch + row] = (uint8_t)(bad ? 255 : e + 127);
        }
    }
}

template <typename T> __global__ __launch_bounds__(256) void act8_unpack(const Act8Args a) {
    const int part = (int)(threadIdx.x & 15u);
    for (int64_t unit = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); unit < a.units; unit += (int64_t)gridDim.x * 16) {
        const int row = (int)(unit / a.runs), b0 = (int)(unit - (int64_t)row * a.runs) * kAct8Ahead;
        uint2 q[kAct8Ahead];
        uint32_t s[kAct8Ahead];
#pragma unroll
        for (int u = 0; u < kAct8Ahead; ++u) {
            const int b = b0 + u < a.blocks ? b0 + u : a.blocks - 1;
            q[u] = *reinterpret_cast<const uint2*>(a.q + (int64_t)row * a.pitch + (int64_t)b * kAct8Block + part * 8);
            s[u] = a.scale[(int64_t)b * a.scale_pitch + row];
        }
        T* dst = const_cast<T*>(static_cast<const T*>(a.x)) + (int64_t)row * a.n;
#pragma unroll
        for (int u = 0; u < kAct8Ahead; ++u) {
            const int64_t t = (int64_t)(b0 + u) * kAct8Block + part * 8;
            const float factor = __builtin_bit_cast(float, s[u] == 255u ? 0x7fc00000u : s[u] << 23);
            k8_any<T, 8> v;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float f = (float)(int8_t)((i < 4 ? q[u].x : q[u].y) >> (8 * (i & 3))) * factor;
                constexpr float most = sizeof(T) == 2 ? 65504.0f : 3.4028235e38f;
                f = f > most ? most : (f < -most ? -most : f);   // (a NaN stays one)
                v[i] = (T)f;
            }
            k8_store<T, 8>(dst + t, t < a.n ? a.n - (int)t : 0, v);
        }
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

Act8Args act8_args(const Act8Shape& sh, const void* x_dev, int32_t rows, int32_t n, void* held_dev) {
    Act8Args a;
    a.x = x_dev, a.q = static_cast<int8_t*>(held_dev);
    a.rows = rows, a.n = n, a.blocks = sh.blocks, a.runs = sh.runs, a.units = sh.units;
    a.pitch = act8_pitch(n), a.scale_pitch = act8_scale_pitch(rows);
    a.scale = static_cast<uint8_t*>(held_dev) + rows * a.pitch;
    return a;
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
    const Act8Shape sh = act8_shape(rows, n, kAct8Ahead);
    const Act8Args a = act8_args(sh, x_dev, rows, n, held_dev);
    (void)hipGetLastError();
    if (dtype == PP_F16) hipLaunchKernelGGL(act8_pack<_Float16>, dim3(sh.wgs), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    else hipLaunchKernelGGL(act8_pack<float>, dim3(sh.wgs), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_DEVICE;
}

pp_status_t pp_act8_unpack(const void* held_dev, int32_t rows, int32_t n, int32_t dtype, void* x_dev, void* hip_stream) {
    const pp_status_t st = act8_check(x_dev, rows, n, dtype, held_dev);
    if (st != PP_OK) return st;
    const Act8Shape sh = act8_shape(rows, n, kAct8Ahead);
    const Act8Args a = act8_args(sh, x_dev, rows, n, const_cast<void*>(held_dev));
    (void)hipGetLastError();
    if (dtype == PP_F16) hipLaunchKernelGGL(act8_unpack<_Float16>, dim3(sh.wgs), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    else hipLaunchKernelGGL(act8_unpack<float>, dim3(sh.wgs), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_DEVICE;
}

}  // extern "C"
