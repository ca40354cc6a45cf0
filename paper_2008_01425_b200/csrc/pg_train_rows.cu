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

// ---------------------------------------------------------------- norm
// A group of T threads holds one row in registers: chunk c of a thread is the V neighbouring
// elements at (c T + t) V, so a warp reads consecutive addresses whatever V is, and a block of the
// 8-bit form lies in 32 / V neighbouring lanes.  The row is read once; the sum of squares comes
// from the registers.
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
        int q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            q[i] = to8(v[c][i], inverse);
            v[c][i] = q[i] * value;
        }
        if (col < cols) {
            store8n<V>(values + col, cols - col, q);
            if (col % kBlock8 == 0) scales[col / kBlock8] = static_cast<uint8_t>(s);
        }
    }
}

template <typename H, int V, int C, int T>
__global__ void __launch_bounds__(T > 32 ? T : 256)
norm_kernel(const pg_norm_args a, int64_t rows, int64_t rows_per_group) {
    __shared__ float s_part[32];
    constexpr int kGroups = T > 32 ? 1 : 256 / T;
    const int t = T > 32 ? threadIdx.x : threadIdx.x & 31;
    const int64_t group = static_cast<int64_t>(blockIdx.x) * kGroups + (T > 32 ? 0 : threadIdx.x >> 5);
    const int64_t r0 = group * rows_per_group;
    const int64_t r1 = min(rows, r0 + rows_per_group);
    constexpr bool kKeep = T <= 256;   // registers left for the gain of the rows' worker
    int64_t held = -1;             // worker whose gain is in registers
    float gain[C][V];
    for (int64_t r = r0; r < r1; ++r) {
        const int64_t b = r / a.tokens, tok = r - b * a.tokens;
        float v[C][V];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * T + t) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] = 0.0f;
            if (col < a.cols) load16n<H, V>(a.x.data, b * a.x.stride + tok * a.x.ld + col, a.cols - col, v[c]);
        }
        if (a.residual.data) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * T + t) * V;
                float w[V];
                if (col < a.cols) {
                    load16n<H, V>(a.residual.data, b * a.residual.stride + tok * a.residual.ld + col, a.cols - col, w);
#pragma unroll
                    for (int i = 0; i < V; ++i) v[c][i] += w[i];
                }
            }
        }
        if (kKeep && b != held) {
            held = b;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int col = (c * T + t) * V + i;
                    gain[c][i] = !a.gain ? 1.0f : col < a.cols ? a.gain[b * a.gain_stride + col] : 0.0f;
                }
        }
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) sum = fmaf(v[c][i], v[c][i], sum);
        sum = group_sum<T>(sum, s_part);
        const float rstd = rsqrtf(sum / a.cols + a.eps);
        if (a.rstd && t == 0) a.rstd[r] = rstd;
        if (a.h.data) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * T + t) * V;
                if (col < a.cols) store16n<H, V>(a.h.data, b * a.h.stride + tok * a.h.ld + col, a.cols - col, v[c]);
            }
        }
        if (a.h8.values) {
            float w[C][V];
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < V; ++i) w[c][i] = v[c][i];
            row_to_8<H, V, C, T>(w, a.cols, t, a.h8.values + b * a.h8.stride + tok * a.h8.ld,
                                 a.h8.scales + b * a.h8.scale_stride + tok * a.h8.scale_ld);
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int col = (c * T + t) * V + i;
                if constexpr (!kKeep) gain[c][i] = a.gain && col < a.cols ? a.gain[b * a.gain_stride + col] : 1.0f;
                v[c][i] *= rstd * gain[c][i];
            }
        if (a.y8.values)
            row_to_8<H, V, C, T>(v, a.cols, t, a.y8.values + b * a.y8.stride + tok * a.y8.ld,
                                 a.y8.scales + b * a.y8.scale_stride + tok * a.y8.scale_ld);
        if (a.y.data) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * T + t) * V;
                if (col < a.cols) store16n<H, V>(a.y.data, b * a.y.stride + tok * a.y.ld + col, a.cols - col, v[c]);
            }
        }
    }
}

// ---------------------------------------------------------------- norm gradient
// Rows as above; every group also keeps the sum of dy u over its rows of one worker in registers.
// partial[b][k][cols]: what group k of worker b added up; summed in that order by the second kernel.
template <typename H, int V, int C, int T, bool EIGHT>
__global__ void __launch_bounds__(T > 32 ? T : 256)
norm_grad_kernel(const pg_norm_grad_args a, float* __restrict__ partial, int groups, int rows_per_group) {
    __shared__ float s_part[32];
    constexpr int kGroups = T > 32 ? 1 : 256 / T;
    const int t = T > 32 ? threadIdx.x : threadIdx.x & 31;
    const int64_t b = blockIdx.y;
    const int group = blockIdx.x * kGroups + (T > 32 ? 0 : threadIdx.x >> 5);
    if (group >= groups) return;                       // T > 32: the whole block; T == 32: the whole warp
    const int r0 = group * rows_per_group;
    const int r1 = min(a.tokens, r0 + rows_per_group);
    float gain[C][V], sum_dg[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int col = (c * T + t) * V + i;
            if constexpr (T <= 256) gain[c][i] = !a.gain ? 1.0f : col < a.cols ? a.gain[b * a.gain_stride + col] : 0.0f;
            sum_dg[c][i] = 0.0f;
        }
    for (int r = r0; r < r1; ++r) {
        float dy[C][V], u[C][V];
        const float rstd = a.rstd[b * a.tokens + r];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * T + t) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) dy[c][i] = u[c][i] = 0.0f;
            if (col < a.cols) {
                load16n<H, V>(a.dy.data, b * a.dy.stride + r * a.dy.ld + col, a.cols - col, dy[c]);
                if constexpr (EIGHT) {
                    int q[V];
                    load8n<V>(a.h8.values + b * a.h8.stride + r * a.h8.ld + col, a.cols - col, q);
                    const float s = scale_value(a.h8.scales[b * a.h8.scale_stride + r * a.h8.scale_ld + col / kBlock8]);
#pragma unroll
                    for (int i = 0; i < V; ++i) u[c][i] = i < a.cols - col ? q[i] * s : 0.0f;
                } else {
                    load16n<H, V>(a.h.data, b * a.h.stride + r * a.h.ld + col, a.cols - col, u[c]);
                }
            }
        }
        float dot = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                u[c][i] *= rstd;
                sum_dg[c][i] = fmaf(dy[c][i], u[c][i], sum_dg[c][i]);
                if constexpr (T > 256) {
                    const int col = (c * T + t) * V + i;
                    gain[c][i] = a.gain && col < a.cols ? a.gain[b * a.gain_stride + col] : 1.0f;
                }
                dy[c][i] *= gain[c][i];
                dot = fmaf(dy[c][i], u[c][i], dot);
            }
        dot = group_sum<T>(dot, s_part) / a.cols;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * T + t) * V;
            if (col < a.cols) {
                float dx[V];
#pragma unroll
                for (int i = 0; i < V; ++i) dx[i] = 0.0f;
                if (a.dh.data) load16n<H, V>(a.dh.data, b * a.dh.stride + r * a.dh.ld + col, a.cols - col, dx);
#pragma unroll
                for (int i = 0; i < V; ++i) dx[i] += rstd * (dy[c][i] - u[c][i] * dot);
                store16n<H, V>(a.dx.data, b * a.dx.stride + r * a.dx.ld + col, a.cols - col, dx);
            }
        }
    }
    if (a.dgain) {
        float* out = partial + (b * groups + group) * a.cols;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int col = (c * T + t) * V + i;
                if (col < a.cols) out[col] = sum_dg[c][i];
            }
    }
}

__global__ void __launch_bounds__(256)
sum_partials_kernel(const float* __restrict__ partial, int groups, int cols, float* __restrict__ out, int64_t out_stride, int accumulate) {
    __shared__ float s_sum[8][32];
    const int64_t b = blockIdx.y;
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    float sum = 0.0f;
    if (col < cols)
        for (int k = w; k < groups; k += 8) sum += partial[(b * groups + k) * cols + col];
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
// warp.  Column sums stay in registers, are joined over the warps in shared memory and over the
// blocks of a cluster (the shares of one strip) through distributed shared memory, in a fixed order.
template <typename H, int V, int ACT>
__global__ void __launch_bounds__(256)
activation_grad_kernel(const pg_activation_grad_args a, int rows_per_block) {
    __shared__ float s_sum[8][32 * V];
    const int64_t b = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int splits = gridDim.z, split = blockIdx.z;
    const int col = (blockIdx.x * 32 + lane) * V;
    const int r1 = min(a.tokens, (split + 1) * rows_per_block);
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.0f;
    if (col < a.cols) {
        const int n = a.cols - col;
#pragma unroll 4
        for (int r = split * rows_per_block + warp; r < r1; r += 8) {
            float dy[V], z[V];
            load16n<H, V>(a.dy.data, b * a.dy.stride + r * a.dy.ld + col, n, dy);
            if (a.z8.values) {
                int q[V];
                load8n<V>(a.z8.values + b * a.z8.stride + r * a.z8.ld + col, n, q);
                const float s = scale_value(a.z8.scales[b * a.z8.scale_stride + r * a.z8.scale_ld + col / kBlock8]);
#pragma unroll
                for (int i = 0; i < V; ++i) z[i] = q[i] * s;
#pragma unroll
                for (int i = 0; i < V; ++i) dy[i] *= slope<ACT>(z[i]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += dy[i];
            if (a.dz.data) store16n<H, V>(a.dz.data, b * a.dz.stride + r * a.dz.ld + col, n, dy);
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
    int q[V];
    if constexpr (WRITE) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.0f;
        if (live) load16n<H, V>(a.x.data, b * a.x.stride + tok * a.x.ld + col, n, v);
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
        load8n<V>(values, n, q);
        const float s = scale_value(*scale);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = q[i] * s;
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

int row_threads(int cols) { return cols <= 1024 ? 32 : cols <= 2048 ? 128 : cols <= 4096 ? 256 : cols <= 8192 ? 512 : 1024; }

// Groups that share the rows of one worker in the gradient: about two waves of warps on the GPU, each
// with four rows at least.
int norm_grad_groups(const pg_norm_grad_args& a) {
    const int64_t per_gpu = int64_t{kSMs} * 2048 / 2 / row_threads(a.cols);
    int64_t g = a.batch > 0 ? (per_gpu + a.batch - 1) / a.batch : 1;
    g = std::min<int64_t>(g, (a.tokens + 3) / 4);
    return static_cast<int>(std::max<int64_t>(g, 1));
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
    const int64_t rows = int64_t{a.batch} * a.tokens;
    if (rows == 0) return PG_OK;
    const int width = access_width({&a.x, &a.residual, &a.h, &a.y}, a.batch);
    with_type(a.dtype, width, [&](auto h, auto v) {
        using H = decltype(h);
        constexpr int V = decltype(v)::value;
        with_row(a.cols, [&](auto e, auto threads) {
            constexpr int T = decltype(threads)::value, C = decltype(e)::value / V;
            constexpr int kGroups = T > 32 ? 1 : 8, kBlock = T > 32 ? T : 256;
            const int64_t most = int64_t{kSMs} * 8 * (2048 / 8 / kBlock > 0 ? 2048 / 8 / kBlock : 1) * kGroups;
            const int64_t per = std::max<int64_t>(1, (rows + most - 1) / most);
            const int64_t groups = (rows + per - 1) / per;
            norm_kernel<H, V, C, T><<<static_cast<unsigned>((groups + kGroups - 1) / kGroups), kBlock, 0,
                                      static_cast<cudaStream_t>(stream)>>>(a, rows, per);
        });
    });
    return launch_status();
}

int pg_add_rms_norm_grad_workspace_bytes(const pg_norm_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->cols, 1)) return PG_ERR_INVALID;
    *bytes_out = args->dgain ? sizeof(float) * norm_grad_groups(*args) * static_cast<size_t>(args->batch) * args->cols : 0;
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
    const int groups = norm_grad_groups(a);
    const int per = (a.tokens + groups - 1) / groups;
    float* partial = static_cast<float*>(workspace);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.tokens > 0 || a.dgain) {
        const int width = access_width({&a.dy, &a.h, &a.dh, &a.dx}, a.batch);
        with_type(a.dtype, width, [&](auto h, auto v) {
            using H = decltype(h);
            constexpr int V = decltype(v)::value;
            with_row(a.cols, [&](auto e, auto threads) {
                constexpr int T = decltype(threads)::value, C = decltype(e)::value / V;
                constexpr int kGroups = T > 32 ? 1 : 8, kBlock = T > 32 ? T : 256;
                const dim3 grid((groups + kGroups - 1) / kGroups, a.batch);
                if (eight) norm_grad_kernel<H, V, C, T, true><<<grid, kBlock, 0, st>>>(a, partial, groups, per);
                else norm_grad_kernel<H, V, C, T, false><<<grid, kBlock, 0, st>>>(a, partial, groups, per);
            });
        });
        if (a.dgain)
            sum_partials_kernel<<<dim3((a.cols + 31) / 32, a.batch), 256, 0, st>>>(partial, groups, a.cols, a.dgain, a.dgain_stride,
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
    // Shares of a strip's tokens: until the GPU has about four blocks per SM, eight at most (the portable
    // cluster size), no share under 32 tokens.
    int splits = 1;
    while (splits < 8 && int64_t{strips} * a.batch * splits < kSMs * 4 && a.tokens >= 64 * splits) splits *= 2;
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
