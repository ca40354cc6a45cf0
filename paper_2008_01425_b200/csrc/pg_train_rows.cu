// Row-wise training operators: the norm and its gradient, the activation's gradient, the 8-bit form.
// All of them are bound by memory: every element is read once, held in registers as fp32, and
// written once.
#include <cooperative_groups.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "pg_train_device.h"

namespace pgt {
namespace {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------- rows in registers
// A group of T threads holds one row in registers: chunk c of a thread is the V neighbouring
// elements at (c T + t) V, so a warp reads consecutive addresses whatever V is, and a block of the
// 8-bit form lies in 32 / V neighbouring lanes.
template <int T>
__device__ __forceinline__ float group_sum(float v, float* s_part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (T > 32) {        // one group per block
        __syncthreads();
        if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < T / 32; ++w) v += s_part[w];
    }
    return v;
}
// All loads of a row, with no branch between them; only a row whose end cuts a chunk short takes a second look.
template <int V, int C, int T>
__device__ __forceinline__ void read_row(const void* base, int64_t at, int cols, int t, Raw<V> (&r)[C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * T + t) * V;
        r[c] = Raw<V>{};
        if (col + V <= cols) r[c] = load_raw<V>(base, at + col);
    }
    if (V > 1 && cols % V != 0) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * T + t) * V;
            if (col < cols && col + V > cols) r[c] = load_raw_end<V>(base, at + col, cols - col);
        }
    }
}
template <typename H, int V, int C, int T>
__device__ __forceinline__ void write_row(void* base, int64_t at, int cols, int t, const float (&v)[C][V]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * T + t) * V;
        if (col < cols) store16n<H, V>(base, at + col, cols - col, v[c]);
    }
}
// A worker's gains for a thread's columns; `wide`: V = 8 and 16-byte addresses.
template <int V>
__device__ __forceinline__ void read_gain(const float* gain, bool wide, int col, int cols, float (&g)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = 1.0f;
    if (!gain) return;
    if (V == 8 && wide) {
        if (col + V <= cols) {
            const float4 lo = *reinterpret_cast<const float4*>(gain + col), hi = *reinterpret_cast<const float4*>(gain + col + 4);
            const float u[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = u[i];
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (col + i < cols) g[i] = gain[col + i];
}
__device__ __forceinline__ bool wide_gain(const float* gain) { return reinterpret_cast<uintptr_t>(gain) % 16 == 0; }
// The 8-bit form of a row held in registers, and back in v the values it stands for.
template <typename H, int V, int C, int T>
__device__ __forceinline__ void row_to_8(float (&v)[C][V], int cols, int t, int8_t* values, uint8_t* scales) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * T + t) * V;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(v[c][i]) & 0x7fffffffu);
        top = block_top<V>(top);
        const uint32_t s = scale_byte<H>(top);
        const float inverse = scale_inverse(s), value = scale_value(s);
        Q8 q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            q[i] = to8(v[c][i], inverse);
            v[c][i] = q[i].value(value);
        }
        if (col < cols) {
            store8n<V>(values + col, cols - col, q);
            if (col % kBlock8 == 0) scales[col / kBlock8] = static_cast<uint8_t>(s);
        }
    }
}

// ---------------------------------------------------------------- norm
// Block: kGroups rows of one worker.  The row is read once; the sum of squares comes from the registers.
template <typename H, int V, int C, int T>
__global__ void __launch_bounds__(T > 32 ? T : 256)
norm_kernel(const pg_norm_args a) {
    __shared__ float s_part[32];
    const int t = T > 32 ? threadIdx.x : threadIdx.x & 31;
    const int64_t b = blockIdx.y;
    const int tok = T > 32 ? blockIdx.x : blockIdx.x * 8 + (threadIdx.x >> 5);
    if (tok >= a.tokens) return;                       // the whole group
    float v[C][V];
    {
        Raw<V> x[C], r[C];
        read_row<V, C, T>(a.x.data, b * a.x.stride + tok * a.x.ld, a.cols, t, x);
        if (a.residual.data) read_row<V, C, T>(a.residual.data, b * a.residual.stride + tok * a.residual.ld, a.cols, t, r);
#pragma unroll
        for (int c = 0; c < C; ++c) widen<H, V>(x[c], v[c]);
        if (a.residual.data) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float w[V];
                widen<H, V>(r[c], w);
#pragma unroll
                for (int i = 0; i < V; ++i) v[c][i] += w[i];
            }
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) sum = fmaf(v[c][i], v[c][i], sum);
    sum = group_sum<T>(sum, s_part);
    const float rstd = rsqrtf(sum / a.cols + a.eps);
    if (a.rstd && t == 0) a.rstd[b * a.tokens + tok] = rstd;
    if (a.h.data) write_row<H, V, C, T>(a.h.data, b * a.h.stride + tok * a.h.ld, a.cols, t, v);
    if (a.h8.values) {
        float w[C][V];
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) w[c][i] = v[c][i];
        row_to_8<H, V, C, T>(w, a.cols, t, a.h8.values + b * a.h8.stride + tok * a.h8.ld,
                             a.h8.scales + b * a.h8.scale_stride + tok * a.h8.scale_ld);
    }
    if (!a.y.data && !a.y8.values) return;
    const float* gain = a.gain ? a.gain + b * a.gain_stride : nullptr;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float g[V];
        read_gain<V>(gain, wide_gain(gain), (c * T + t) * V, a.cols, g);
#pragma unroll
        for (int i = 0; i < V; ++i) v[c][i] *= rstd * g[i];
    }
    if (a.y8.values)
        row_to_8<H, V, C, T>(v, a.cols, t, a.y8.values + b * a.y8.stride + tok * a.y8.ld,
                             a.y8.scales + b * a.y8.scale_stride + tok * a.y8.scale_ld);
    if (a.y.data) write_row<H, V, C, T>(a.y.data, b * a.y.stride + tok * a.y.ld, a.cols, t, v);
}

// ---------------------------------------------------------------- norm gradient
// Rows as above, R of them at a time so that one exchange serves R dot products and R rows are on their way
// together; every group also keeps the sum of dy u over its rows of one worker in registers.  What was
// read stays packed and is widened again for the second use: dx needs the row's dot product first.
// partial[b][k][cols]: what block k of worker b added up; summed in that order by the second kernel.
constexpr int kGradBlock = 128;
template <typename H, int V, int C, int T, int R, bool EIGHT>
__global__ void __launch_bounds__(T > 32 ? T : kGradBlock)
norm_grad_kernel(const pg_norm_grad_args a, float* __restrict__ partial, int rows_per_group) {
    extern __shared__ float s_sum[];                   // warps x cols, T == 32 only
    __shared__ float s_part[2][R][32];
    constexpr int kGroups = T > 32 ? 1 : kGradBlock / T;
    const int t = T > 32 ? threadIdx.x : threadIdx.x & 31;
    const int64_t b = blockIdx.y;
    const int group = blockIdx.x * kGroups + (T > 32 ? 0 : threadIdx.x >> 5);
    const int64_t r0 = static_cast<int64_t>(group) * rows_per_group;
    const int64_t r1 = min(static_cast<int64_t>(a.tokens), r0 + rows_per_group);
    const float* gain = a.gain ? a.gain + b * a.gain_stride : nullptr;
    float sum_dg[C][V], g[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        read_gain<V>(gain, wide_gain(gain), (c * T + t) * V, a.cols, g[c]);
#pragma unroll
        for (int i = 0; i < V; ++i) sum_dg[c][i] = 0.0f;
    }
    int flip = 0;
    for (int64_t r = r0; r < r1; r += R, flip ^= 1) {
        Raw<V> dy_raw[R][C], h_raw[R][C], dh_raw[R][C];
        Raw8<V> q_raw[R][C];
        uint32_t q_scale[R][C];
        float rstd[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {                  // a row past the last one reads the last one again, and counts for nothing
            const int64_t row = min(r + k, r1 - 1);
            read_row<V, C, T>(a.dy.data, b * a.dy.stride + row * a.dy.ld, a.cols, t, dy_raw[k]);
            if constexpr (EIGHT) {
                const int8_t* q = a.h8.values + b * a.h8.stride + row * a.h8.ld;
                const uint8_t* s = a.h8.scales + b * a.h8.scale_stride + row * a.h8.scale_ld;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int col = (c * T + t) * V;
                    q_raw[k][c] = Raw8<V>{};
                    q_scale[k][c] = 0;
                    if (col + V <= a.cols) q_raw[k][c] = load_raw8<V>(q + col);
                    if (col < a.cols) q_scale[k][c] = s[col / kBlock8];
                }
                if (V > 1 && a.cols % V != 0) {
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        const int col = (c * T + t) * V;
                        if (col < a.cols && col + V > a.cols) q_raw[k][c] = load_raw8_end<V>(q + col, a.cols - col);
                    }
                }
            } else {
                read_row<V, C, T>(a.h.data, b * a.h.stride + row * a.h.ld, a.cols, t, h_raw[k]);
            }
            if (a.dh.data) read_row<V, C, T>(a.dh.data, b * a.dh.stride + row * a.dh.ld, a.cols, t, dh_raw[k]);
            rstd[k] = a.rstd[b * a.tokens + row];
        }
        // u of a chunk; past the end of the row it is zero, as dy is
        auto unit = [&](int k, int c, float (&u)[V]) {
            if constexpr (EIGHT) widen8<V>(q_raw[k][c], scale_value(q_scale[k][c]), u);
            else widen<H, V>(h_raw[k][c], u);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                u[i] *= rstd[k];
                if (EIGHT && (c * T + t) * V + i >= a.cols) u[i] = 0.0f;     // not NaN, where the last block's scale says so
            }
        };
        float dot[R];
#pragma unroll
        for (int k = 0; k < R; ++k) dot[k] = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                float dy[V], u[V];
                widen<H, V>(dy_raw[k][c], dy);
                unit(k, c, u);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float w = dy[i] * u[i];
                    if (r + k < r1) sum_dg[c][i] += w;
                    dot[k] = fmaf(w, g[c][i], dot[k]);
                }
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < R; ++k) dot[k] += __shfl_xor_sync(0xffffffffu, dot[k], o);
        if constexpr (T > 32) {        // (the other half of s_part is still being read by slower warps)
            if ((threadIdx.x & 31) == 0)
#pragma unroll
                for (int k = 0; k < R; ++k) s_part[flip][k][threadIdx.x >> 5] = dot[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < R; ++k) {
                dot[k] = 0.0f;
#pragma unroll
                for (int w = 0; w < T / 32; ++w) dot[k] += s_part[flip][k][w];
            }
        }
#pragma unroll
        for (int k = 0; k < R; ++k) dot[k] /= a.cols;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * T + t) * V;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                float dy[V], u[V], dx[V];
                widen<H, V>(dy_raw[k][c], dy);
                unit(k, c, u);
#pragma unroll
                for (int i = 0; i < V; ++i) dx[i] = 0.0f;
                if (a.dh.data) widen<H, V>(dh_raw[k][c], dx);
#pragma unroll
                for (int i = 0; i < V; ++i) dx[i] += rstd[k] * (dy[i] * g[c][i] - u[i] * dot[k]);
                if (col < a.cols && r + k < r1)
                    store16n<H, V>(a.dx.data, b * a.dx.stride + (r + k) * a.dx.ld + col, a.cols - col, dx);
            }
        }
    }
    if (!a.dgain) return;
    float* out = partial + (b * gridDim.x + blockIdx.x) * a.cols;
    float* mine = T > 32 ? out : s_sum + (threadIdx.x >> 5) * a.cols;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int col = (c * T + t) * V + i;
            if (col < a.cols) mine[col] = sum_dg[c][i];
        }
    if constexpr (T == 32) {
        __syncthreads();
        for (int col = threadIdx.x; col < a.cols; col += kGradBlock) {
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kGroups; ++w) v += s_sum[w * a.cols + col];
            out[col] = v;
        }
    }
}

__global__ void __launch_bounds__(256)
sum_partials_kernel(const float* __restrict__ partial, int parts, int cols, float* __restrict__ out, int64_t out_stride, int accumulate) {
    __shared__ float s_sum[8][32];
    const int64_t b = blockIdx.y;
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    float sum = 0.0f;
    if (col < cols)
#pragma unroll 4
        for (int k = w; k < parts; k += 8) sum += partial[(b * parts + k) * cols + col];
    s_sum[w][threadIdx.x & 31] = sum;
    __syncthreads();
    if (w == 0 && col < cols) {
        float* o = out + b * out_stride + col;
        sum = accumulate ? *o : 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += s_sum[k][threadIdx.x];
        *o = sum;
    }
}

// ---------------------------------------------------------------- activation gradient
// A block takes a strip of 32 V columns and a share of a worker's tokens; 8 rows at a time, one per
// warp, four times that in flight.  Column sums stay in registers, are joined over the warps in shared
// memory and over the blocks of a cluster (the shares of one strip) through distributed shared memory, in
// a fixed order.
template <typename H, int V, int ACT>
__global__ void __launch_bounds__(256, 3)
activation_grad_kernel(const pg_activation_grad_args a, int rows_per_block) {
    __shared__ float s_sum[8][32 * V];
    const int64_t b = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int splits = gridDim.z, split = blockIdx.z;
    const int col = (blockIdx.x * 32 + lane) * V;
    const int64_t r0 = static_cast<int64_t>(split) * rows_per_block;
    const int r1 = static_cast<int>(min(static_cast<int64_t>(a.tokens), r0 + rows_per_block));
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.0f;
    const void* dy_at = static_cast<const uint16_t*>(a.dy.data) + b * a.dy.stride + col;
    void* dz_at = a.dz.data ? static_cast<uint16_t*>(a.dz.data) + b * a.dz.stride + col : nullptr;
    const int8_t* q_at = a.z8.values ? a.z8.values + b * a.z8.stride + col : nullptr;
    const uint8_t* s_at = a.z8.values ? a.z8.scales + b * a.z8.scale_stride + col / kBlock8 : nullptr;
    auto one = [&](const Raw<V>& dy_raw, const Raw8<V>& q_raw, uint32_t scale, float (&dy)[V]) {
        widen<H, V>(dy_raw, dy);
        if (q_at) {
            float z[V];
            widen8<V>(q_raw, scale_value(scale), z);
#pragma unroll
            for (int i = 0; i < V; ++i) dy[i] *= slope<ACT>(z[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += dy[i];
    };
    if (col + V <= a.cols) {
        for (int64_t r = r0 + warp; r < r1; r += 32) {      // rows past the end read as zeros
            Raw<V> d[4] = {};
            Raw8<V> q[4] = {};
            uint32_t s[4] = {};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (r + 8 * k < r1) d[k] = load_raw<V>(dy_at, (r + 8 * k) * a.dy.ld);
            if (q_at) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (r + 8 * k < r1) {
                        q[k] = load_raw8<V>(q_at + (r + 8 * k) * a.z8.ld);
                        s[k] = s_at[(r + 8 * k) * a.z8.scale_ld];
                    }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float dy[V];
                one(d[k], q[k], s[k], dy);
                if (dz_at && r + 8 * k < r1) store16<H, V>(dz_at, (r + 8 * k) * a.dz.ld, dy);
            }
        }
    } else if (col < a.cols) {             // the lane that the row's end cuts short
        const int n = a.cols - col;
        for (int64_t r = r0 + warp; r < r1; r += 8) {
            float dy[V];
            const Raw8<V> q = q_at ? load_raw8_end<V>(q_at + r * a.z8.ld, n) : Raw8<V>{};
            one(load_raw_end<V>(dy_at, r * a.dy.ld, n), q, q_at ? s_at[r * a.z8.scale_ld] : 0u, dy);
            if (dz_at) store16n<H, V>(dz_at, r * a.dz.ld, n, dy);
        }
    }
    if (!a.dbias) return;
#pragma unroll
    for (int i = 0; i < V; ++i) s_sum[warp][lane * V + i] = sum[i];
    __syncthreads();
    float mine = 0.0f;
    const int at = threadIdx.x;
    if (at < 32 * V) {
#pragma unroll
        for (int w = 0; w < 8; ++w) mine += s_sum[w][at];
    }
    cg::cluster_group cluster = cg::this_cluster();
    if (splits > 1) {
        __syncthreads();
        if (at < 32 * V) s_sum[0][at] = mine;
        cluster.sync();
        if (split == 0 && at < 32 * V) {
            for (int k = 1; k < splits; ++k) mine += cluster.map_shared_rank(&s_sum[0][0], k)[at];
        }
        cluster.sync();
    }
    const int out_col = blockIdx.x * 32 * V + at;
    if (split == 0 && at < 32 * V && out_col < a.cols) {
        float* o = a.dbias + b * a.dbias_stride + out_col;
        *o = a.accumulate ? *o + mine : mine;
    }
}

// ---------------------------------------------------------------- checkpoints
template <typename H, int V, bool WRITE>
__global__ void __launch_bounds__(256)
checkpoint_kernel(const pg_checkpoint_args a, int64_t rows, int chunks) {
    // one thread per V elements of a row; the lanes of a block of 32 values are neighbours because a
    // row takes a whole number of blocks (chunks is a multiple of 32 / V)
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t r = at / chunks;
    const int col = static_cast<int>(at - r * chunks) * V;
    const bool live = r < rows && col < a.cols;
    const int64_t b = live ? r / a.tokens : 0, tok = live ? r - b * a.tokens : 0;
    const int n = a.cols - col;
    int8_t* values = a.x8.values + b * a.x8.stride + tok * a.x8.ld + col;
    uint8_t* scale = a.x8.scales + b * a.x8.scale_stride + tok * a.x8.scale_ld + col / kBlock8;
    float v[V];
    if constexpr (WRITE) {
        Q8 q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.0f;
        if (live) {
            const int64_t from = b * a.x.stride + tok * a.x.ld + col;
            widen<H, V>(n >= V ? load_raw<V>(a.x.data, from) : load_raw_end<V>(a.x.data, from, n), v);
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
        top = block_top<V>(top);
        const uint32_t s = scale_byte<H>(top);
        const float inverse = scale_inverse(s);
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] = to8(v[i], inverse);
        if (live) {
            store8n<V>(values, n, q);
            if (col % kBlock8 == 0) *scale = static_cast<uint8_t>(s);
        }
    } else if (live) {
        widen8<V>(n >= V ? load_raw8<V>(values) : load_raw8_end<V>(values, n), scale_value(*scale), v);
        store16n<H, V>(a.x.data, b * a.x.stride + tok * a.x.ld + col, n, v);
    }
}

int current_device() {
    int d = 0;
    return cudaGetDevice(&d) == cudaSuccess ? d : -1;
}

// Calls f with a compile-time element type and access width.
template <typename F>
void with_type(int dtype, int width, F&& f) {
    auto w = [&](auto h) {
        using H = decltype(h);
        if (width == 8) f(H{}, std::integral_constant<int, 8>{});
        else if (width == 2) f(H{}, std::integral_constant<int, 2>{});
        else f(H{}, std::integral_constant<int, 1>{});
    };
    if (dtype == PG_BF16) w(__nv_bfloat16{});
    else w(__half{});
}
// Calls f with the number of elements a thread holds and the threads that share a row: a warp to
// 1024 columns, then 16 elements a thread and up to 1024 threads.
template <typename F>
void with_row(int cols, F&& f) {
    using std::integral_constant;
    if (cols <= 256) f(integral_constant<int, 8>{}, integral_constant<int, 32>{});
    else if (cols <= 512) f(integral_constant<int, 16>{}, integral_constant<int, 32>{});
    else if (cols <= 768) f(integral_constant<int, 24>{}, integral_constant<int, 32>{});
    else if (cols <= 1024) f(integral_constant<int, 32>{}, integral_constant<int, 32>{});
    else if (cols <= 2048) f(integral_constant<int, 16>{}, integral_constant<int, 128>{});
    else if (cols <= 4096) f(integral_constant<int, 16>{}, integral_constant<int, 256>{});
    else if (cols <= 8192) f(integral_constant<int, 16>{}, integral_constant<int, 512>{});
    else f(integral_constant<int, 16>{}, integral_constant<int, 1024>{});
}
constexpr int kMaxNormCols = 16384;

// The gradient holds three packed rows, the gains and a sum per column: 8 elements a thread, or 16 where that saves
// the exchange between warps or there is no room for more threads.  `blocks`: resident per SM.
struct GradRow { int elements, threads, rows, blocks; };
constexpr GradRow kGradRows[] = {{8, 32, 2, 4}, {16, 32, 2, 3}, {8, 128, 2, 5}, {8, 256, 2, 2}, {8, 512, 2, 1}, {16, 512, 2, 1}, {16, 1024, 1, 1}};
int grad_row(int cols) {
    int k = 0;
    while (kGradRows[k].elements * kGradRows[k].threads < cols) ++k;
    return k;
}
template <typename F>
void with_grad_row(int cols, F&& f) {
    using std::integral_constant;
    switch (grad_row(cols)) {
        case 0: f(integral_constant<int, 0>{}); break;
        case 1: f(integral_constant<int, 1>{}); break;
        case 2: f(integral_constant<int, 2>{}); break;
        case 3: f(integral_constant<int, 3>{}); break;
        case 4: f(integral_constant<int, 4>{}); break;
        case 5: f(integral_constant<int, 5>{}); break;
        default: f(integral_constant<int, 6>{});
    }
}

// Blocks that share the rows of one worker in the gradient: as many as are resident at once, with two steps of R
// rows a group at least.
int norm_grad_blocks(const pg_norm_grad_args& a) {
    const GradRow g = kGradRows[grad_row(a.cols)];
    const int groups = g.threads > 32 ? 1 : kGradBlock / 32;
    int64_t n = a.batch > 0 ? int64_t{kSMs} * g.blocks / a.batch : 1;
    n = std::min<int64_t>(n, (a.tokens + 2 * g.rows * groups - 1) / (2 * g.rows * groups));
    return static_cast<int>(std::max<int64_t>(n, 1));
}

}  // namespace
}  // namespace pgt

using namespace pgt;

extern "C" {

int pg_add_rms_norm(const pg_norm_args* args, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_norm_args& a = *args;
    const int dev = current_device();
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.cols, 1) || !(a.eps >= 0.0f) || a.eps > 3e38f) return PG_ERR_INVALID;
    if (!matrix_ok(a.x, a.batch, a.tokens, a.cols, 2, false, dev)) return PG_ERR_INVALID;
    if (a.residual.data && !matrix_ok(a.residual, a.batch, a.tokens, a.cols, 2, false, dev)) return PG_ERR_INVALID;
    if (a.h.data && !matrix_ok(a.h, a.batch, a.tokens, a.cols, 2, true, dev)) return PG_ERR_INVALID;
    if (a.y.data && !matrix_ok(a.y, a.batch, a.tokens, a.cols, 2, true, dev)) return PG_ERR_INVALID;
    if ((a.y8.values || a.y8.scales) && !matrix8_ok(a.y8, a.batch, a.tokens, a.cols, true, dev)) return PG_ERR_INVALID;
    if ((a.h8.values || a.h8.scales) && !matrix8_ok(a.h8, a.batch, a.tokens, a.cols, true, dev)) return PG_ERR_INVALID;
    if (a.gain && !vector_ok(a.gain, a.gain_stride, a.batch, a.cols, false, dev)) return PG_ERR_INVALID;
    if (a.rstd && !vector_ok(a.rstd, a.tokens, a.batch, a.tokens, true, dev)) return PG_ERR_INVALID;
    if (a.cols > kMaxNormCols) return PG_ERR_TOO_LARGE;
    if (a.batch == 0 || a.tokens == 0) return PG_OK;
    const int width = access_width({&a.x, &a.residual, &a.h, &a.y}, a.batch);
    with_type(a.dtype, width, [&](auto h, auto v) {
        using H = decltype(h);
        constexpr int V = decltype(v)::value;
        with_row(a.cols, [&](auto e, auto threads) {
            constexpr int T = decltype(threads)::value, C = decltype(e)::value / V;
            const dim3 grid(T > 32 ? a.tokens : (a.tokens + 7) / 8, a.batch);
            norm_kernel<H, V, C, T><<<grid, T > 32 ? T : 256, 0, static_cast<cudaStream_t>(stream)>>>(a);
        });
    });
    return launch_status();
}

int pg_add_rms_norm_grad_workspace_bytes(const pg_norm_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->cols, 1)) return PG_ERR_INVALID;
    *bytes_out = args->dgain ? sizeof(float) * norm_grad_blocks(*args) * static_cast<size_t>(args->batch) * args->cols : 0;
    return PG_OK;
}

int pg_add_rms_norm_grad(const pg_norm_grad_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_norm_grad_args& a = *args;
    const int dev = current_device();
    const bool eight = a.h8.values != nullptr;
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.cols, 1)) return PG_ERR_INVALID;
    if (eight == (a.h.data != nullptr) && int64_t{a.batch} * a.tokens > 0) return PG_ERR_INVALID;
    if (!matrix_ok(a.dy, a.batch, a.tokens, a.cols, 2, false, dev)) return PG_ERR_INVALID;
    if (eight ? !matrix8_ok(a.h8, a.batch, a.tokens, a.cols, false, dev)
              : !matrix_ok(a.h, a.batch, a.tokens, a.cols, 2, false, dev))
        return PG_ERR_INVALID;
    if (a.tokens > 0 && !vector_ok(a.rstd, a.tokens, a.batch, a.tokens, false, dev)) return PG_ERR_INVALID;
    if (a.gain && !vector_ok(a.gain, a.gain_stride, a.batch, a.cols, false, dev)) return PG_ERR_INVALID;
    if (a.dh.data && !matrix_ok(a.dh, a.batch, a.tokens, a.cols, 2, false, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.dx, a.batch, a.tokens, a.cols, 2, true, dev)) return PG_ERR_INVALID;
    if (a.dgain && !vector_ok(a.dgain, a.dgain_stride, a.batch, a.cols, true, dev)) return PG_ERR_INVALID;
    if (a.cols > kMaxNormCols) return PG_ERR_TOO_LARGE;
    size_t need = 0;
    pg_add_rms_norm_grad_workspace_bytes(args, &need);
    if (need > 0 && (workspace_bytes < need || !device_pointer(workspace, 16, dev))) return PG_ERR_WORKSPACE;
    if (a.batch == 0) return PG_OK;
    const int blocks = norm_grad_blocks(a);
    float* partial = static_cast<float*>(workspace);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.tokens > 0 || a.dgain) {
        const int width = access_width({&a.dy, &a.h, &a.dh, &a.dx}, a.batch);
        with_type(a.dtype, width, [&](auto h, auto v) {
            using H = decltype(h);
            constexpr int V = decltype(v)::value;
            with_grad_row(a.cols, [&](auto shape) {
                constexpr GradRow g = kGradRows[decltype(shape)::value];
                constexpr int T = g.threads, C = g.elements / V, kGroups = T > 32 ? 1 : kGradBlock / 32;
                const int per = (a.tokens + blocks * kGroups - 1) / (blocks * kGroups);
                const dim3 grid(blocks, a.batch);
                const size_t smem = T > 32 ? 0 : sizeof(float) * kGroups * a.cols;
                if (eight) norm_grad_kernel<H, V, C, T, g.rows, true><<<grid, T > 32 ? T : kGradBlock, smem, st>>>(a, partial, per);
                else norm_grad_kernel<H, V, C, T, g.rows, false><<<grid, T > 32 ? T : kGradBlock, smem, st>>>(a, partial, per);
            });
        });
        if (a.dgain)
            sum_partials_kernel<<<dim3((a.cols + 31) / 32, a.batch), 256, 0, st>>>(partial, blocks, a.cols, a.dgain, a.dgain_stride,
                                                                                  a.accumulate);
    }
    return launch_status();
}

int pg_activation_grad(const pg_activation_grad_args* args, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_activation_grad_args& a = *args;
    const int dev = current_device();
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.cols, 1) || a.activation < PG_ACT_NONE || a.activation > PG_ACT_SILU) return PG_ERR_INVALID;
    if (!matrix_ok(a.dy, a.batch, a.tokens, a.cols, 2, false, dev)) return PG_ERR_INVALID;
    if (a.z8.values ? !matrix8_ok(a.z8, a.batch, a.tokens, a.cols, false, dev)
                    : (a.activation != PG_ACT_NONE && int64_t{a.batch} * a.tokens > 0))
        return PG_ERR_INVALID;
    if (a.dz.data && !matrix_ok(a.dz, a.batch, a.tokens, a.cols, 2, true, dev)) return PG_ERR_INVALID;
    if (a.dbias && !vector_ok(a.dbias, a.dbias_stride, a.batch, a.cols, true, dev)) return PG_ERR_INVALID;
    if (a.batch == 0 || (a.tokens == 0 && !a.dbias)) return PG_OK;
    const int width = access_width({&a.dy, &a.dz}, a.batch);
    const int strips = (a.cols + 32 * width - 1) / (32 * width);
    // Shares of a strip's tokens: until the GPU has about 16 blocks per SM (five waves, so that the last one weighs
    // little), eight at most (the portable cluster size), no share under 32 tokens.
    int splits = 1;
    while (splits < 8 && int64_t{strips} * a.batch * splits < kSMs * 16 && a.tokens >= 64 * splits) splits *= 2;
    const int per = (a.tokens + splits - 1) / splits;
    int rc = PG_OK;
    with_type(a.dtype, width, [&](auto h, auto v) {
        using H = decltype(h);
        constexpr int V = decltype(v)::value;
        auto launch = [&](auto kernel) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(strips, a.batch, splits);
            cfg.blockDim = dim3(256);
            cfg.stream = static_cast<cudaStream_t>(stream);
            cudaLaunchAttribute at[1];
            at[0].id = cudaLaunchAttributeClusterDimension;
            at[0].val.clusterDim.x = at[0].val.clusterDim.y = 1;
            at[0].val.clusterDim.z = splits;
            cfg.attrs = at;
            cfg.numAttrs = 1;
            if (cudaLaunchKernelEx(&cfg, kernel, a, per) != cudaSuccess) {
                cudaGetLastError();
                rc = PG_ERR_CUDA;
            }
        };
        if (a.activation == PG_ACT_RELU) launch(activation_grad_kernel<H, V, PG_ACT_RELU>);
        else if (a.activation == PG_ACT_GELU) launch(activation_grad_kernel<H, V, PG_ACT_GELU>);
        else if (a.activation == PG_ACT_SILU) launch(activation_grad_kernel<H, V, PG_ACT_SILU>);
        else launch(activation_grad_kernel<H, V, PG_ACT_NONE>);
    });
    return rc;
}

static int checkpoint(const pg_checkpoint_args* args, bool write, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_checkpoint_args& a = *args;
    const int dev = current_device();
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.cols, 1)) return PG_ERR_INVALID;
    if (!matrix_ok(a.x, a.batch, a.tokens, a.cols, 2, !write, dev)) return PG_ERR_INVALID;
    if (!matrix8_ok(a.x8, a.batch, a.tokens, a.cols, write, dev)) return PG_ERR_INVALID;
    const int64_t rows = int64_t{a.batch} * a.tokens;
    if (rows == 0) return PG_OK;
    const int width = access_width({&a.x}, a.batch);
    const int chunks = (a.cols + kBlock8 - 1) / kBlock8 * (kBlock8 / width);
    const int64_t blocks = (rows * chunks + 255) / 256;
    if (blocks > 0x7fffffff) return PG_ERR_TOO_LARGE;
    with_type(a.dtype, width, [&](auto h, auto v) {
        using H = decltype(h);
        constexpr int V = decltype(v)::value;
        if (write) checkpoint_kernel<H, V, true><<<static_cast<unsigned>(blocks), 256, 0, static_cast<cudaStream_t>(stream)>>>(a, rows, chunks);
        else checkpoint_kernel<H, V, false><<<static_cast<unsigned>(blocks), 256, 0, static_cast<cudaStream_t>(stream)>>>(a, rows, chunks);
    });
    return launch_status();
}
int pg_checkpoint_write(const pg_checkpoint_args* args, void* stream) { return checkpoint(args, true, stream); }
int pg_checkpoint_read(const pg_checkpoint_args* args, void* stream) { return checkpoint(args, false, stream); }

}  // extern "C"
