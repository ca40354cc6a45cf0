// Shared by the training kernels: 16-bit element access, the 8-bit block form, activations, and the
// host-side checks of their arguments.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "pg_training.h"

namespace pgt {

constexpr int kBlock8 = 32;        // values that share a scale in the 8-bit form
constexpr int kSMs = 148;          // streaming multiprocessors of a B200
constexpr int64_t kMaxDim = 1 << 30;

// ------------------------------------------------------------------ 16-bit elements
template <typename H> struct Elem;
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kLeastScale = 1;          // 2^-126, the smallest normal number
    __device__ static float up(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
    __device__ static uint16_t down(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
    __device__ static uint32_t down2(float lo, float hi) {
        __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&p);
    }
};
template <> struct Elem<__half> {
    static constexpr int kLeastScale = 127 - 24;   // 2^-24, the step of fp16's subnormal numbers
    __device__ static float up(uint16_t b) { return __half2float(__ushort_as_half(b)); }
    __device__ static uint16_t down(float v) { return __half_as_ushort(__float2half_rn(v)); }
    __device__ static uint32_t down2(float lo, float hi) {
        __half2 p = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&p);
    }
};

// V neighbouring 16-bit elements in one access, as they lie in memory (two to a word).  V = 8 and 2 need
// 16- and 4-byte addresses.  Loading is kept apart from widening so that all loads of a row are on their
// way before the first one is needed.
template <int V> struct Raw { uint32_t w[(V + 1) / 2]; };

template <int V>
__device__ __forceinline__ Raw<V> load_raw(const void* base, int64_t at) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    Raw<V> r;
    if constexpr (V == 8) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        r.w[0] = u.x;
        r.w[1] = u.y;
        r.w[2] = u.z;
        r.w[3] = u.w;
    } else if constexpr (V == 2) {
        r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        r.w[0] = *p;
    }
    return r;
}
// The first n < V of them (the end of a row); the rest are zero.
template <int V>
__device__ __forceinline__ Raw<V> load_raw_end(const void* base, int64_t at, int n) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    Raw<V> r = {};
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < n) r.w[i / 2] |= static_cast<uint32_t>(p[i]) << (16 * (i & 1));
    return r;
}
template <typename H, int V>
__device__ __forceinline__ void widen(const Raw<V>& r, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = Elem<H>::up(static_cast<uint16_t>(i & 1 ? r.w[i / 2] >> 16 : r.w[i / 2] & 0xffffu));
}
template <typename H, int V>
__device__ __forceinline__ void store16(void* base, int64_t at, const float (&v)[V]) {
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    if constexpr (V == 8) {
        uint4 w;
        w.x = Elem<H>::down2(v[0], v[1]);
        w.y = Elem<H>::down2(v[2], v[3]);
        w.z = Elem<H>::down2(v[4], v[5]);
        w.w = Elem<H>::down2(v[6], v[7]);
        *reinterpret_cast<uint4*>(p) = w;
    } else if constexpr (V == 2) {
        *reinterpret_cast<uint32_t*>(p) = Elem<H>::down2(v[0], v[1]);
    } else {
        *p = Elem<H>::down(v[0]);
    }
}
template <typename H, int V>
__device__ __forceinline__ void store16n(void* base, int64_t at, int n, const float (&v)[V]) {
    if (n >= V) {
        store16<H, V>(base, at, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < n) static_cast<uint16_t*>(base)[at + i] = Elem<H>::down(v[i]);
}

// ------------------------------------------------------------------ the 8-bit form
// Scale byte of a block from the largest |v| in it, given as the bits of an fp32 number: those order
// like the numbers, with infinities and NaN above all of them.
template <typename H>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits) {
    const int e = static_cast<int>(top_bits >> 23);
    return e >= 255 ? 255u : static_cast<uint32_t>(max(e - 6, Elem<H>::kLeastScale));
}
// 2^-(scale - 127); a block marked 255 gets a factor that keeps its values away from the clamp's edge cases.
__device__ __forceinline__ float scale_inverse(uint32_t s) { return __uint_as_float((254u - (s < 254u ? s : 253u)) << 23); }
__device__ __forceinline__ float scale_value(uint32_t s) { return __uint_as_float(s == 255u ? 0x7fc00000u : s << 23); }
// Adding 1.5 * 2^23 rounds a number below 2^22 to an integer, ties to even, and leaves that integer in
// the sum's low bits: one fused multiply-add instead of two conversions, which run at a quarter of the rate.
// The clamp acts on the sum; a NaN comes out as some valid byte and is marked by its block's scale.
constexpr float kRound = 12582912.0f;
struct Q8 {
    float t;                                           // kRound + q
    __device__ float value(float scale) const { return (t - kRound) * scale; }
    __device__ uint32_t bits() const { return __float_as_uint(t); }   // q in the low byte
};
__device__ __forceinline__ Q8 to8(float v, float inverse) {
    return Q8{fminf(fmaxf(fmaf(v, inverse, kRound), kRound - 127.0f), kRound + 127.0f)};
}

// Largest bits among the lanes that share a block when every lane holds V neighbouring values.
template <int V>
__device__ __forceinline__ uint32_t block_top(uint32_t top) {
#pragma unroll
    for (int o = kBlock8 / V / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    return top;
}
template <int V>
__device__ __forceinline__ void store8n(int8_t* p, int n, const Q8 (&q)[V]) {
    if (V == 8 && n >= V) {
        uint2 w;
        w.x = __byte_perm(__byte_perm(q[0].bits(), q[1 % V].bits(), 0x0040), __byte_perm(q[2 % V].bits(), q[3 % V].bits(), 0x0040), 0x5410);
        w.y = __byte_perm(__byte_perm(q[4 % V].bits(), q[5 % V].bits(), 0x0040), __byte_perm(q[6 % V].bits(), q[7 % V].bits(), 0x0040), 0x5410);
        *reinterpret_cast<uint2*>(p) = w;
    } else if (V == 2 && n >= V) {
        *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(__byte_perm(q[0].bits(), q[1 % V].bits(), 0x0040));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = static_cast<int8_t>(q[i].bits() & 255u);
    }
}

// V neighbouring 8-bit values as they lie in memory, and their numbers.
template <int V> struct Raw8 { uint32_t w[(V + 3) / 4]; };
template <int V>
__device__ __forceinline__ Raw8<V> load_raw8(const int8_t* p) {
    Raw8<V> r;
    if constexpr (V == 8) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        r.w[0] = u.x;
        r.w[1] = u.y;
    } else if constexpr (V == 2) {
        r.w[0] = *reinterpret_cast<const uint16_t*>(p);
    } else {
        r.w[0] = static_cast<uint8_t>(*p);
    }
    return r;
}
template <int V>
__device__ __forceinline__ Raw8<V> load_raw8_end(const int8_t* p, int n) {
    Raw8<V> r = {};
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < n) r.w[i / 4] |= static_cast<uint32_t>(static_cast<uint8_t>(p[i])) << (8 * (i & 3));
    return r;
}
// A byte with its sign bit flipped (q + 128) under the exponent of 2^23 reads 2^23 + 128 + q.
template <int V>
__device__ __forceinline__ void widen8(const Raw8<V>& r, float scale, float (&v)[V]) {
    uint32_t w[(V + 3) / 4];
#pragma unroll
    for (int i = 0; i < (V + 3) / 4; ++i) w[i] = r.w[i] ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (__uint_as_float(__byte_perm(w[i / 4], 0x4b000000u, 0x7650 + (i & 3))) - 8388736.0f) * scale;
}

// ------------------------------------------------------------------ activations
// s(v) = 1 / (1 + 2^(-v log2 e)); both approximations are good to two units in the last place, 2^x overflows to
// infinity and 1 / infinity is 0, so the ends are exact.
__device__ __forceinline__ float sigmoid(float v) {
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
    return s;
}
constexpr float kGelu0 = 1.5957691216057308f;             // 2 sqrt(2/pi)
constexpr float kGelu1 = 0.044715f * 1.5957691216057308f;

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == PG_ACT_RELU) return z > 0.0f ? z : (z <= 0.0f ? 0.0f : z);   // NaN stays NaN
    if constexpr (ACT == PG_ACT_GELU) return z * sigmoid(z * fmaf(kGelu1, z * z, kGelu0));
    if constexpr (ACT == PG_ACT_SILU) return z * sigmoid(z);
    return z;
}
template <int ACT>
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == PG_ACT_RELU) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    if constexpr (ACT == PG_ACT_GELU) {
        // z^2 is kept from overflowing; far from zero s (1 - s) is 0 and stays so
        const float z2 = fminf(z * z, 300.0f);
        const float s = sigmoid(z * fmaf(kGelu1, z2, kGelu0));
        return fmaf(s * (1.0f - s) * z, fmaf(3.0f * kGelu1, z2, kGelu0), s);
    }
    if constexpr (ACT == PG_ACT_SILU) {
        const float s = sigmoid(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    return 1.0f;
}

// ------------------------------------------------------------------ host-side checks
inline bool device_pointer(const void* p, uintptr_t align, int device) {
    if (!p || reinterpret_cast<uintptr_t>(p) % align != 0) return false;
    cudaPointerAttributes a;
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return (a.type == cudaMemoryTypeDevice || a.type == cudaMemoryTypeManaged) && a.device == device;
}
// A batch of rows x cols matrices of elements of `size` bytes.  Outputs must keep workers apart.
inline bool matrix_ok(const pg_matrix& m, int64_t batch, int64_t rows, int64_t cols, int size, bool output, int device) {
    if (m.ld < cols || m.ld > (int64_t{1} << 40) || m.stride < 0 || m.stride > (int64_t{1} << 44)) return false;
    if (output && batch > 1 && rows > 0 && m.stride < (rows - 1) * m.ld + cols) return false;
    return batch == 0 || rows == 0 || device_pointer(m.data, size, device);
}
inline bool matrix8_ok(const pg_matrix8& m, int64_t batch, int64_t rows, int64_t cols, bool output, int device) {
    const int64_t blocks = (cols + kBlock8 - 1) / kBlock8;
    if (m.ld < cols || m.ld % 16 != 0 || m.stride % 16 != 0 || m.scale_ld < blocks) return false;
    if (m.stride < 0 || m.scale_stride < 0 || m.ld > (int64_t{1} << 40) || m.scale_ld > (int64_t{1} << 40) ||
        m.stride > (int64_t{1} << 44) || m.scale_stride > (int64_t{1} << 44))
        return false;
    if (output && batch > 1 && rows > 0 &&
        (m.stride < (rows - 1) * m.ld + cols || m.scale_stride < (rows - 1) * m.scale_ld + blocks))
        return false;
    return batch == 0 || rows == 0 || (device_pointer(m.values, 16, device) && device_pointer(m.scales, 1, device));
}
inline bool vector_ok(const void* p, int64_t stride, int64_t batch, int64_t n, bool output, int device) {
    if (stride < 0 || stride > (int64_t{1} << 44) || (output && batch > 1 && stride < n)) return false;
    return batch == 0 || device_pointer(p, 4, device);
}
inline bool sizes_ok(int64_t dtype, int64_t batch, int64_t tokens, int64_t a, int64_t b) {
    return (dtype == PG_BF16 || dtype == PG_F16) && batch >= 0 && batch <= 65535 && tokens >= 0 && tokens <= kMaxDim && a >= 1 &&
           a <= kMaxDim && b >= 1 && b <= kMaxDim;
}
// Elements that one access may take so that all rows of all these matrices are aligned for it.
inline int access_width(std::initializer_list<const pg_matrix*> ms, int64_t batch) {
    uint64_t bits = 0;
    for (const pg_matrix* m : ms)
        if (m->data) {
            bits |= reinterpret_cast<uintptr_t>(m->data) | static_cast<uint64_t>(m->ld) * 2;
            if (batch > 1) bits |= static_cast<uint64_t>(m->stride) * 2;
        }
    return bits % 16 == 0 ? 8 : bits % 4 == 0 ? 2 : 1;
}
inline int launch_status() { return cudaGetLastError() == cudaSuccess ? PG_OK : PG_ERR_CUDA; }

}  // namespace pgt
