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

// ------------------------------------------------------------------ bounds-checked build
// With -DPG_BOUNDS_CHECK every access that a kernel makes by an address of its own is looked up in the operands of its call
// first: a read has to touch one (16- and 4-byte pieces may reach past its ends), a write has to lie in an output.  Another one is
// skipped and reported by pg_training_status (PG_ERR_BOUNDS).  Copies by TMA are bounded by their tensor maps.  That build takes one
// call at a time on a device.
#ifdef PG_BOUNDS_CHECK
constexpr bool kChecked = true;
#else
constexpr bool kChecked = false;
#endif
constexpr int kMaxSpans = 16;
struct Span { uintptr_t lo, hi; };
struct Spans {
    Span at[kMaxSpans];
    int count, outputs;        // the outputs come first
};
constexpr unsigned kTimedOut = 1, kOutside = 2;        // bits of the error words
#ifdef PG_BOUNDS_CHECK
static __device__ Spans g_spans;
static __device__ unsigned g_outside;
static __device__ __noinline__ bool may_access(const void* p, int bytes, bool write) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p), hi = lo + bytes;
    for (int i = 0; i < (write ? g_spans.outputs : g_spans.count); ++i)
        if (write ? lo >= g_spans.at[i].lo && hi <= g_spans.at[i].hi : lo < g_spans.at[i].hi && hi > g_spans.at[i].lo) return true;
    atomicOr(&g_outside, kOutside);
    return false;
}
#define PGT_READ(p, bytes) may_access(p, bytes, false)
#define PGT_WRITE(p, bytes) may_access(p, bytes, true)
#else
#define PGT_READ(p, bytes) ((void)sizeof(p), true)       // names its operand, evaluates nothing
#define PGT_WRITE(p, bytes) ((void)sizeof(p), true)
#endif
#define PGT_LOAD(ref) (PGT_READ(&(ref), sizeof(ref)) ? (ref) : decltype((ref) + 0)(0))
#define PGT_STORE(ref, value) do { if (PGT_WRITE(&(ref), sizeof(ref))) (ref) = (value); } while (0)

// ------------------------------------------------------------------ pairs of fp32
// Two fp32 numbers in one 64-bit register pair: add, multiply and fused multiply-add take both at once.
struct F2 { unsigned long long u; };
__device__ __forceinline__ F2 pair(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.u) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ F2 both(float v) { return pair(v, v); }
__device__ __forceinline__ void split(F2 p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p.u)); }
__device__ __forceinline__ F2 add(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
    return r;
}
__device__ __forceinline__ F2 mul(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
    return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(c.u));
    return r;
}
__device__ __forceinline__ float sum2(F2 a) {
    float lo, hi;
    split(a, lo, hi);
    return lo + hi;
}

// ------------------------------------------------------------------ 16-bit elements
template <typename H> struct Elem;
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kLeastScale = 1;          // 2^-126, the smallest normal number
    __device__ static float up(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
    __device__ static F2 up2(uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    __device__ static uint16_t down(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
    __device__ static uint32_t down2(F2 v) {
        float lo, hi;
        split(v, lo, hi);
        __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&p);
    }
};
template <> struct Elem<__half> {
    static constexpr int kLeastScale = 127 - 24;   // 2^-24, the step of fp16's subnormal numbers
    __device__ static float up(uint16_t b) { return __half2float(__ushort_as_half(b)); }
    __device__ static F2 up2(uint32_t w) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        return pair(f.x, f.y);
    }
    __device__ static uint16_t down(float v) { return __half_as_ushort(__float2half_rn(v)); }
    __device__ static uint32_t down2(F2 v) {
        float lo, hi;
        split(v, lo, hi);
        __half2 p = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&p);
    }
};

// An octet: eight neighbouring elements of a row, what a lane holds.  W = 8: all rows of the call start on 16-byte
// boundaries.  W = 1: they may start anywhere, and an octet is cut out of the two 16-byte pieces of memory that hold it.
// A piece is only read if it holds an element of the row, so it lies in the row's own allocation, and what it holds
// besides is masked out.  Loading is
// kept apart from widening, and free of branches, so that all loads of a row are on their way before the first one
// is needed.
struct Oct { uint32_t w[4]; };
template <int W> struct Piece { uint4 a, b; };
template <> struct Piece<8> { uint4 a; };
template <int W>
__device__ __forceinline__ Piece<W> load_oct(const uint16_t* row, int col, int cols) {
    Piece<W> r = {};
    if constexpr (W == 8) {
        if (col < cols && PGT_READ(row + col, 16)) r.a = *reinterpret_cast<const uint4*>(row + col);
    } else {
        const int off = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / 2;         // the same for all lanes of a row
        const uint4* p = reinterpret_cast<const uint4*>(row + col - off);
        if (col < cols && PGT_READ(p, 16)) r.a = p[0];
        if (col + 8 - off < cols && off > 0 && PGT_READ(p + 1, 16)) r.b = p[1];
    }
    return r;
}
// The eight elements that start `off` elements into the 32 bytes a, b.
__device__ __forceinline__ Oct cut(const uint4& a, const uint4& b, int off) {
    Oct r;
    uint32_t v[7] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z};
#pragma unroll
    for (int i = 0; i < 6; ++i) v[i] = off & 2 ? v[i + 1] : v[i];
    v[6] = off & 2 ? b.w : v[6];
#pragma unroll
    for (int i = 0; i < 5; ++i) v[i] = off & 4 ? v[i + 2] : v[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = __funnelshift_r(v[i], v[i + 1], (off & 1) * 16);
    return r;
}
template <int W>
__device__ __forceinline__ Oct octet(const Piece<W>& p, const uint16_t* row, int col, int cols) {
    Oct r;
    if constexpr (W == 8) r = Oct{{p.a.x, p.a.y, p.a.z, p.a.w}};
    else r = cut(p.a, p.b, static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / 2);
    if (col + 8 > cols) {                          // what follows the row's end is another row's, or padding
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = col + 2 * i + 1 < cols ? r.w[i] : col + 2 * i < cols ? r.w[i] & 0xffffu : 0u;
    }
    return r;
}
// All octets c T + t of a row: loaded, and later taken out.
template <int W, int C, int T>
__device__ __forceinline__ void load_row(const uint16_t* row, int cols, int t, Piece<W> (&r)[C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) r[c] = load_oct<W>(row, (c * T + t) * 8, cols);
}
template <typename H>
__device__ __forceinline__ void widen(const Oct& r, F2 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = Elem<H>::up2(r.w[i]);
}
template <typename H, int W>
__device__ __forceinline__ void store_oct(uint16_t* row, int col, int cols, const F2 (&v)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = Elem<H>::down2(v[i]);
    if (W == 8 && col + 8 <= cols) {
        PGT_STORE(*reinterpret_cast<uint4*>(row + col), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) PGT_STORE(row[col + i], static_cast<uint16_t>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu));
    }
}

// ------------------------------------------------------------------ the 8-bit form
// Largest |v| of an octet, as the bits of an fp32 number: those order like the numbers, with infinities and NaN
// (which the maximum passes on) above all of them.
__device__ __forceinline__ float top3(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t top_bits(const F2 (&v)[4]) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) split(v[i], e[2 * i], e[2 * i + 1]);
    return __float_as_uint(top3(top3(top3(e[0], e[1], e[2]), e[3], e[4]), top3(e[5], e[6], e[7]), 0.0f));
}
// The largest of the four lanes whose octets make a block.
__device__ __forceinline__ uint32_t block_top(uint32_t top) {
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    return max(top, __shfl_xor_sync(0xffffffffu, top, 2));
}
// Scale byte of a block from the largest |v| in it.
template <typename H>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const int e = static_cast<int>(top >> 23);
    return e >= 255 ? 255u : static_cast<uint32_t>(max(e - 6, Elem<H>::kLeastScale));
}
// 2^-(scale - 127); a block marked 255 gets some finite factor.
__device__ __forceinline__ float scale_inverse(uint32_t s) { return __uint_as_float((254u - (s < 254u ? s : 253u)) << 23); }
__device__ __forceinline__ float scale_value(uint32_t s) { return __uint_as_float(s == 255u ? 0x7fc00000u : s << 23); }
// Adding 1.5 * 2^23 rounds a number below 2^22 to an integer, ties to even, and leaves that integer in
// the sum's low bits: one fused multiply-add instead of two conversions, which run at a quarter of the rate.
// The clamp acts on the sum; a NaN comes out as some valid byte and is marked by its block's scale.
constexpr float kRound = 12582912.0f;
__device__ __forceinline__ float clamp8(float t) { return fminf(fmaxf(t, kRound - 127.0f), kRound + 127.0f); }
__device__ __forceinline__ F2 to8(F2 v, F2 inverse) {          // kRound + q
    float lo, hi;
    split(fma(v, inverse, both(kRound)), lo, hi);
    return pair(clamp8(lo), clamp8(hi));
}
__device__ __forceinline__ F2 value8(F2 t, F2 scale) { return mul(add(t, both(-kRound)), scale); }

struct Oct8 { uint32_t w[2]; };
__device__ __forceinline__ Oct8 pack8(const F2 (&t)[4]) {      // the low bytes of kRound + q
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        split(t[i], lo, hi);
        h[i] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x0040);
    }
    return Oct8{{__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[2], h[3], 0x5410)}};
}
__device__ __forceinline__ void store_oct8(int8_t* row, int col, int cols, Oct8 o) {
    if (col + 8 <= cols) {
        PGT_STORE(*reinterpret_cast<uint2*>(row + col), make_uint2(o.w[0], o.w[1]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) PGT_STORE(row[col + i], static_cast<int8_t>(o.w[i / 4] >> (8 * (i & 3)) & 255u));
    }
}
// An octet of an 8-bit row (rows start on 16-byte boundaries); what it holds past the row's end is not masked.
__device__ __forceinline__ Oct8 load_oct8(const int8_t* row, int col, int cols) {
    Oct8 r = {};
    if (col < cols && PGT_READ(row + col, 8)) {
        const uint2 u = *reinterpret_cast<const uint2*>(row + col);
        r.w[0] = u.x;
        r.w[1] = u.y;
    }
    return r;
}
// A byte with its sign bit flipped (q + 128) under the exponent of 2^23 reads 2^23 + 128 + q.
__device__ __forceinline__ void widen8(const Oct8& r, float scale, F2 (&v)[4]) {
    const uint32_t w[2] = {r.w[0] ^ 0x80808080u, r.w[1] ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 f = pair(__uint_as_float(__byte_perm(w[i / 2], 0x4b000000u, 0x7650 + (2 * i & 3))),
                          __uint_as_float(__byte_perm(w[i / 2], 0x4b000000u, 0x7650 + (2 * i + 1 & 3))));
        v[i] = mul(add(f, both(-8388736.0f)), both(scale));
    }
}

// ------------------------------------------------------------------ activations
// s(v) = 1 / (1 + 2^(-v log2 e)); both approximations are good to two units in the last place, 2^x overflows to
// infinity and 1 / infinity is 0, so the ends are exact.  Given v (-log2 e).
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ F2 sigmoid_of(F2 v) {
    float a, b;
    split(v, a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    split(add(pair(a, b), both(1.0f)), a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return pair(a, b);
}
constexpr double kGelu0 = 1.5957691216057308;                  // 2 sqrt(2/pi)
constexpr double kGelu1 = 0.044715 * kGelu0;
__device__ __forceinline__ float relu(float z) { return z > 0.0f ? z : (z <= 0.0f ? 0.0f : z); }      // NaN stays NaN
__device__ __forceinline__ float step(float z) { return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z); }

template <int ACT>
__device__ __forceinline__ F2 activate(F2 z) {
    if constexpr (ACT == PG_ACT_RELU) {
        float a, b;
        split(z, a, b);
        return pair(relu(a), relu(b));
    } else if constexpr (ACT == PG_ACT_GELU) {
        const F2 g = fma(mul(z, z), both(static_cast<float>(-kGelu1 * kLog2e)), both(static_cast<float>(-kGelu0 * kLog2e)));
        return mul(z, sigmoid_of(mul(z, g)));
    } else if constexpr (ACT == PG_ACT_SILU) {
        return mul(z, sigmoid_of(mul(z, both(-kLog2e))));
    }
    return z;
}
// |z| < 2^63, so that z^2 is finite.
template <int ACT>
__device__ __forceinline__ F2 slope(F2 z) {
    if constexpr (ACT == PG_ACT_RELU) {
        float a, b;
        split(z, a, b);
        return pair(step(a), step(b));
    } else if constexpr (ACT == PG_ACT_GELU) {
        // far from zero s (1 - s) = s - s^2 is 0 and stays so
        const F2 z2 = mul(z, z);
        const F2 s = sigmoid_of(mul(z, fma(z2, both(static_cast<float>(-kGelu1 * kLog2e)), both(static_cast<float>(-kGelu0 * kLog2e)))));
        const F2 w = mul(fma(s, mul(s, both(-1.0f)), s), z);
        return fma(w, fma(z2, both(static_cast<float>(3.0 * kGelu1)), both(static_cast<float>(kGelu0))), s);
    } else if constexpr (ACT == PG_ACT_SILU) {
        const F2 s = sigmoid_of(mul(z, both(-kLog2e)));
        return fma(fma(s, mul(s, both(-1.0f)), s), z, s);
    }
    return both(1.0f);
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
// 8 if all rows of all these matrices start on 16-byte boundaries, else 1.
inline int access_width(std::initializer_list<const pg_matrix*> ms, int64_t batch) {
    uint64_t bits = 0;
    for (const pg_matrix* m : ms)
        if (m->data) {
            bits |= reinterpret_cast<uintptr_t>(m->data) | static_cast<uint64_t>(m->ld) * 2;
            if (batch > 1) bits |= static_cast<uint64_t>(m->stride) * 2;
        }
    return bits % 16 == 0 ? 8 : 1;
}
// The operands of a call, for the bounds-checked build (elsewhere nothing is kept): all outputs first.
class Operands {
public:
    Operands& output(const pg_matrix& m, int64_t batch, int64_t rows, int64_t cols, int size) {
        if (kChecked && m.data && batch > 0 && rows > 0) add(m.data, ((batch - 1) * m.stride + (rows - 1) * m.ld + cols) * size);
        if (kChecked) spans_.outputs = spans_.count;
        return *this;
    }
    Operands& output(const pg_matrix8& m, int64_t batch, int64_t rows, int64_t cols) {
        output(pg_matrix{m.values, m.ld, m.stride}, batch, rows, cols, 1);
        return output(pg_matrix{m.values ? m.scales : nullptr, m.scale_ld, m.scale_stride}, batch, rows, (cols + kBlock8 - 1) / kBlock8, 1);
    }
    Operands& output(const void* p, int64_t stride, int64_t batch, int64_t n) { return output(pg_matrix{const_cast<void*>(p), n, stride}, batch, 1, n, 4); }
    template <typename... A> Operands& input(const A&... a) {
        const int outputs = spans_.outputs;
        output(a...);
        spans_.outputs = outputs;
        return *this;
    }
    int publish(cudaStream_t st) const {
#ifdef PG_BOUNDS_CHECK
        if (cudaMemcpyToSymbolAsync(g_spans, &spans_, sizeof spans_, 0, cudaMemcpyHostToDevice, st) != cudaSuccess) return PG_ERR_CUDA;
#else
        static_cast<void>(st);
#endif
        return PG_OK;
    }

private:
    void add(const void* p, int64_t bytes) {
        if (spans_.count < kMaxSpans) spans_.at[spans_.count++] = Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes};
    }
    Spans spans_ = {};
};
// Waits for `st`, reads a word of device memory and clears it.
inline int take_word(unsigned* word, unsigned& value, cudaStream_t st) {
    const unsigned none = 0;
    if (cudaMemcpyAsync(&value, word, sizeof value, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return PG_ERR_CUDA;
    if (value != 0 && (cudaMemcpyAsync(word, &none, sizeof none, cudaMemcpyHostToDevice, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess))
        return PG_ERR_CUDA;
    return PG_OK;
}
int take_row_errors(unsigned& value, cudaStream_t st);     // of the row kernels (pg_train_rows.cu)
inline int launch_status() { return cudaGetLastError() == cudaSuccess ? PG_OK : PG_ERR_CUDA; }

}  // namespace pgt
