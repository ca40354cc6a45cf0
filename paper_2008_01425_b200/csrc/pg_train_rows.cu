// Row-wise training operators: the norm and its gradient, the activation's gradient, the 8-bit form.
// All of them are bound by memory: every element is read once, held in registers as fp32, and
// written once.  A lane holds octets (eight neighbouring elements), so four lanes make a block of the 8-bit form
// whatever the alignment of the rows is; only the width of the accesses goes by that.
#include <cooperative_groups.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "pg_train_device.h"

namespace pgt {
namespace {

namespace cg = cooperative_groups;

// A worker's gains for an octet (of global memory, or where a block has copied them to); `wide`: 16-byte addresses.
template <bool SHARED = false>
__device__ __forceinline__ void load_gain(const float* gain, bool wide, int col, int cols, F2 (&g)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = both(1.0f);
    if (!gain) return;
    if (wide && col + 8 <= cols && (SHARED || (PGT_READ(gain + col, 16) && PGT_READ(gain + col + 4, 16)))) {
        const float4 lo = *reinterpret_cast<const float4*>(gain + col), hi = *reinterpret_cast<const float4*>(gain + col + 4);
        g[0] = pair(lo.x, lo.y);
        g[1] = pair(lo.z, lo.w);
        g[2] = pair(hi.x, hi.y);
        g[3] = pair(hi.z, hi.w);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            g[i] = pair(col + 2 * i < cols ? PGT_LOAD(gain[col + 2 * i]) : 0.0f, col + 2 * i + 1 < cols ? PGT_LOAD(gain[col + 2 * i + 1]) : 0.0f);
    }
}
__device__ __forceinline__ bool wide_gain(const float* gain) { return reinterpret_cast<uintptr_t>(gain) % 16 == 0; }

// The 8-bit form of an octet, stored, and back in v the values it stands for.  All lanes of a warp take part.
template <typename H>
__device__ __forceinline__ void octet_to_8(F2 (&v)[4], int8_t* row, uint8_t* scales, int col, int cols) {
    const uint32_t s = scale_byte<H>(block_top(top_bits(v)));
    const F2 inverse = both(scale_inverse(s)), value = both(scale_value(s));
    F2 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t[i] = to8(v[i], inverse);
        v[i] = value8(t[i], value);
    }
    if (col < cols) {
        store_oct8(row, col, cols, pack8(t));
        if (col % kBlock8 == 0) PGT_STORE(scales[col / kBlock8], static_cast<uint8_t>(s));
    }
}

// ---------------------------------------------------------------- norm
// T threads hold one row, C octets each; a block has 256 / T rows of one worker, at least one.  The row is read
// once; the sum of squares comes from the registers.
template <typename H, int W, int WO, int C, int T>
__global__ void __launch_bounds__(T > 32 ? T : 256)
norm_kernel(const pg_norm_args a) {
    __shared__ float s_part[32];
    __shared__ __align__(16) float s_gain[T > 32 ? 4 : C * 256];
    const int t = T > 32 ? threadIdx.x : threadIdx.x & 31;
    const int64_t b = blockIdx.y;
    const int tok = T > 32 ? blockIdx.x : blockIdx.x * 8 + (threadIdx.x >> 5);
    const float* gain = a.gain ? a.gain + b * a.gain_stride : nullptr;
    if constexpr (T == 32) {                           // eight rows share the gains
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = c * 256 + threadIdx.x;
            s_gain[col] = gain && col < a.cols ? PGT_LOAD(gain[col]) : 1.0f;
        }
        __syncthreads();
    }
    if (tok >= a.tokens) return;                       // the whole group
    F2 v[C][4];
    {
        const uint16_t* x_row = static_cast<const uint16_t*>(a.x.data) + b * a.x.stride + tok * a.x.ld;
        const uint16_t* r_row = static_cast<const uint16_t*>(a.residual.data) + b * a.residual.stride + tok * a.residual.ld;
        Piece<W> x[C], r[C];
        load_row<W, C, T>(x_row, a.cols, t, x);
        if (a.residual.data) load_row<W, C, T>(r_row, a.cols, t, r);
#pragma unroll
        for (int c = 0; c < C; ++c) widen<H>(octet<W>(x[c], x_row, (c * T + t) * 8, a.cols), v[c]);
        if (a.residual.data) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                F2 w[4];
                widen<H>(octet<W>(r[c], r_row, (c * T + t) * 8, a.cols), w);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[c][i] = add(v[c][i], w[i]);
            }
        }
    }
    auto sum_of_row = [&](F2 sums) {
        float sum = sum2(sums);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if constexpr (T > 32) {
            if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = sum;
            __syncthreads();
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < T / 32; ++w) sum += s_part[w];
        }
        return sum;
    };
    F2 sums = both(0.0f);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums = fma(v[c][i], v[c][i], sums);
    float sum = sum_of_row(sums), scale = 1.0f, eps = a.eps;
    // bf16 reaches to 2^128 and fp32 squares do not: where the sum leaves fp32's range, at the upper end or (with an eps too small
    // to matter there) at the lower one, it is taken once more of the row times a power of two.  The same for the whole row.
    if (!(sum <= 3.4028235e38f) || (sum < 8.2718061e-25f && eps < 7.8886091e-31f)) {       // 2^-80, 2^-100
        scale = sum < 1.0f ? 7.9228163e28f : 1.2621774e-29f;                               // 2^96, 2^-96
        eps = eps * scale * scale;
        sums = both(0.0f);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const F2 w = mul(v[c][i], both(scale));
                sums = fma(w, w, sums);
            }
        if constexpr (T > 32) __syncthreads();         // (the shares of the first sum have been read)
        sum = sum_of_row(sums);
    }
    const float rstd = rsqrtf(sum / a.cols + eps);     // of the scaled row
    if (a.rstd && t == 0) PGT_STORE(a.rstd[b * a.tokens + tok], rstd * scale);
    if (a.h.data) {
        uint16_t* h = static_cast<uint16_t*>(a.h.data) + b * a.h.stride + tok * a.h.ld;
#pragma unroll
        for (int c = 0; c < C; ++c)
            if ((c * T + t) * 8 < a.cols) store_oct<H, WO>(h, (c * T + t) * 8, a.cols, v[c]);
    }
    if (a.h8.values) {
        int8_t* q = a.h8.values + b * a.h8.stride + tok * a.h8.ld;
        uint8_t* s = a.h8.scales + b * a.h8.scale_stride + tok * a.h8.scale_ld;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            F2 w[4];                                       // of h as it is stored, in 16 bits
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = Elem<H>::up2(Elem<H>::down2(v[c][i]));
            octet_to_8<H>(w, q, s, (c * T + t) * 8, a.cols);
        }
    }
    if (!a.y.data && !a.y8.values) return;
    if (scale != 1.0f) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[c][i] = mul(v[c][i], both(scale));
    }
    const bool wide = wide_gain(gain);
    uint16_t* y = a.y.data ? static_cast<uint16_t*>(a.y.data) + b * a.y.stride + tok * a.y.ld : nullptr;
    int8_t* q = a.y8.values + b * a.y8.stride + tok * a.y8.ld;
    uint8_t* s = a.y8.scales + b * a.y8.scale_stride + tok * a.y8.scale_ld;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * T + t) * 8;
        F2 g[4];
        if constexpr (T == 32) load_gain<true>(s_gain, true, col, C * 256, g);
        else load_gain(gain, wide, col, a.cols, g);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[c][i] = mul(v[c][i], mul(both(rstd), g[i]));
        if (a.y8.values) octet_to_8<H>(v[c], q, s, col, a.cols);
        if (y && col < a.cols) store_oct<H, WO>(y, col, a.cols, v[c]);
    }
}

// ---------------------------------------------------------------- norm gradient
// Rows as above, R of them at a time so that one exchange serves R dot products and R rows are on their way
// together; every group also keeps the sum of dy u over its rows of one worker in registers.  What was
// read stays packed and is widened again for the second use: dx needs the row's dot product first.
// partial[b][k][cols]: what block k of worker b added up; summed in that order by the second kernel.
constexpr int kGradBlock = 128;
template <typename H, int W, int WO, int C, int T, int R, int BLOCKS, bool EIGHT>
__global__ void __launch_bounds__(T > 32 ? T : kGradBlock, BLOCKS)
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
    F2 sum_dg[C][4], g[C][4];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        load_gain(gain, wide_gain(gain), (c * T + t) * 8, a.cols, g[c]);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum_dg[c][i] = both(0.0f);
    }
    int flip = 0;
    for (int64_t r = r0; r < r1; r += R, flip ^= 1) {
        Oct dy_raw[R][C], h_raw[R][C], dh_raw[R][C];
        Oct8 q_raw[R][C];
        uint32_t q_scale[R][C];
        float rstd[R];
        Piece<W> dy_piece[R][C], h_piece[R][C], dh_piece[R][C];
        auto row_of = [&](const pg_matrix& m, int k) {         // a row past the last one reads the last one again, and counts for nothing
            return static_cast<const uint16_t*>(m.data) + b * m.stride + min(r + k, r1 - 1) * m.ld;
        };
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t row = min(r + k, r1 - 1);
            load_row<W, C, T>(row_of(a.dy, k), a.cols, t, dy_piece[k]);
            if constexpr (EIGHT) {
                const int8_t* q = a.h8.values + b * a.h8.stride + row * a.h8.ld;
                const uint8_t* s = a.h8.scales + b * a.h8.scale_stride + row * a.h8.scale_ld;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int col = (c * T + t) * 8;
                    q_raw[k][c] = load_oct8(q, col, a.cols);
                    q_scale[k][c] = col < a.cols ? PGT_LOAD(s[col / kBlock8]) : 0;
                }
            } else {
                load_row<W, C, T>(row_of(a.h, k), a.cols, t, h_piece[k]);
            }
            if (a.dh.data) load_row<W, C, T>(row_of(a.dh, k), a.cols, t, dh_piece[k]);
            rstd[k] = PGT_LOAD(a.rstd[b * a.tokens + row]);
        }
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * T + t) * 8;
                dy_raw[k][c] = octet<W>(dy_piece[k][c], row_of(a.dy, k), col, a.cols);
                if constexpr (!EIGHT) h_raw[k][c] = octet<W>(h_piece[k][c], row_of(a.h, k), col, a.cols);
                if (a.dh.data) dh_raw[k][c] = octet<W>(dh_piece[k][c], row_of(a.dh, k), col, a.cols);
            }
        auto unit = [&](int k, int c, F2 (&u)[4]) {
            if constexpr (EIGHT) widen8(q_raw[k][c], scale_value(q_scale[k][c]), u);
            else widen<H>(h_raw[k][c], u);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = mul(u[i], both(rstd[k]));
        };
        float dot[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            F2 d = both(0.0f);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                F2 dy[4], u[4];
                widen<H>(dy_raw[k][c], dy);
                unit(k, c, u);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    F2 w = mul(dy[i], u[i]);
                    if (EIGHT && (c * T + t) * 8 + 2 * i + 1 >= a.cols) {       // values past the row's end are not the block's NaN
                        float lo, hi;
                        split(w, lo, hi);
                        w = pair((c * T + t) * 8 + 2 * i < a.cols ? lo : 0.0f, 0.0f);
                    }
                    if (r + k < r1) sum_dg[c][i] = add(sum_dg[c][i], w);
                    d = fma(w, g[c][i], d);
                }
            }
            dot[k] = sum2(d);
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
        for (int k = 0; k < R; ++k) {
            const F2 minus = both(-dot[k] / a.cols), by = both(rstd[k]);
            uint16_t* out = static_cast<uint16_t*>(a.dx.data) + b * a.dx.stride + (r + k) * a.dx.ld;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * T + t) * 8;
                F2 dy[4], u[4], dx[4];
                widen<H>(dy_raw[k][c], dy);
                unit(k, c, u);
#pragma unroll
                for (int i = 0; i < 4; ++i) dx[i] = both(0.0f);
                if (a.dh.data) widen<H>(dh_raw[k][c], dx);
#pragma unroll
                for (int i = 0; i < 4; ++i) dx[i] = fma(by, fma(u[i], minus, mul(dy[i], g[c][i])), dx[i]);
                if (col < a.cols && r + k < r1) store_oct<H, WO>(out, col, a.cols, dx);
            }
        }
    }
    if (!a.dgain) return;
    float* out = partial + (b * gridDim.x + blockIdx.x) * a.cols;
    float* mine = T > 32 ? out : s_sum + (threadIdx.x >> 5) * a.cols;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = (c * T + t) * 8 + 2 * i;
            float lo, hi;
            split(sum_dg[c][i], lo, hi);
            if (col < a.cols && (T == 32 || PGT_WRITE(mine + col, 4))) mine[col] = lo;
            if (col + 1 < a.cols && (T == 32 || PGT_WRITE(mine + col + 1, 4))) mine[col + 1] = hi;
        }
    if constexpr (T == 32) {
        __syncthreads();
        for (int col = threadIdx.x; col < a.cols; col += kGradBlock) {
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kGroups; ++w) v += s_sum[w * a.cols + col];
            PGT_STORE(out[col], v);
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
        for (int k = w; k < parts; k += 8) sum += PGT_LOAD(partial[(b * parts + k) * cols + col]);
    s_sum[w][threadIdx.x & 31] = sum;
    __syncthreads();
    if (w == 0 && col < cols) {
        float* o = out + b * out_stride + col;
        sum = accumulate ? PGT_LOAD(*o) : 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += s_sum[k][threadIdx.x];
        PGT_STORE(*o, sum);
    }
}

// ---------------------------------------------------------------- activation gradient
// A block takes a strip of 256 columns and a share of a worker's tokens; 8 rows at a time, one per
// warp, four times that in flight.  Column sums stay in registers, are joined over the warps in shared
// memory and over the blocks of a cluster (the shares of one strip) through distributed shared memory, in
// a fixed order.  (Three blocks per SM with four rows in flight: 76 us for 700 tokens x 2600 columns of 32 workers; two blocks with
// more registers 97 us, four with two rows 86 us.  At its 80 registers the form for rows that start anywhere spills 28 to 76 bytes.)
constexpr int kStrip = 256, kStripRows = 4;
template <typename H, int W, int WO, int ACT>
__global__ void __launch_bounds__(256, 3)
activation_grad_kernel(const pg_activation_grad_args a, int rows_per_block) {
    __shared__ float s_sum[8][kStrip];
    const int64_t b = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int splits = gridDim.z, split_at = blockIdx.z;
    const int col = blockIdx.x * kStrip + lane * 8;
    const int64_t r0 = static_cast<int64_t>(split_at) * rows_per_block;
    const int64_t r1 = min(static_cast<int64_t>(a.tokens), r0 + rows_per_block);
    F2 sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = both(0.0f);
    if (col < a.cols) {
        const bool eight = a.z8.values != nullptr;
        const uint16_t* dy_at = static_cast<const uint16_t*>(a.dy.data) + b * a.dy.stride + (r0 + warp) * a.dy.ld;
        uint16_t* dz_at = a.dz.data ? static_cast<uint16_t*>(a.dz.data) + b * a.dz.stride + (r0 + warp) * a.dz.ld : nullptr;
        const int8_t* q_at = a.z8.values + b * a.z8.stride + (r0 + warp) * a.z8.ld;
        const uint8_t* s_at = a.z8.scales + b * a.z8.scale_stride + (r0 + warp) * a.z8.scale_ld + col / kBlock8;
        for (int64_t r = r0 + warp; r < r1; r += 8 * kStripRows) {              // rows past the end read as zeros
            Piece<W> d[kStripRows] = {};
            Oct8 q[kStripRows] = {};
            uint32_t s[kStripRows] = {};
#pragma unroll
            for (int k = 0; k < kStripRows; ++k)
                if (r + 8 * k < r1) {
                    d[k] = load_oct<W>(dy_at + 8 * k * a.dy.ld, col, a.cols);
                    if (eight) {
                        q[k] = load_oct8(q_at + 8 * k * a.z8.ld, col, a.cols);
                        s[k] = PGT_LOAD(s_at[8 * k * a.z8.scale_ld]);
                    }
                }
#pragma unroll
            for (int k = 0; k < kStripRows; ++k) {
                F2 dy[4];
                widen<H>(octet<W>(d[k], dy_at + 8 * k * a.dy.ld, col, r + 8 * k < r1 ? a.cols : 0), dy);
                if (eight) {
                    F2 z[4];
                    widen8(q[k], scale_value(s[k] == 255u ? 255u : min(s[k], 183u)), z);      // 127 * 2^56 is as far from zero as any
#pragma unroll
                    for (int i = 0; i < 4; ++i) dy[i] = mul(dy[i], slope<ACT>(z[i]));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = add(sum[i], dy[i]);
                if (dz_at && r + 8 * k < r1) store_oct<H, WO>(dz_at + 8 * k * a.dz.ld, col, a.cols, dy);
            }
            dy_at += 8 * kStripRows * a.dy.ld;
            if (dz_at) dz_at += 8 * kStripRows * a.dz.ld;
            q_at += 8 * kStripRows * a.z8.ld;
            s_at += 8 * kStripRows * a.z8.scale_ld;
        }
    }
    if (!a.dbias) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) split(sum[i], s_sum[warp][lane * 8 + 2 * i], s_sum[warp][lane * 8 + 2 * i + 1]);
    __syncthreads();
    const int at = threadIdx.x;
    float mine = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) mine += s_sum[w][at];
    if (splits > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        __syncthreads();
        s_sum[0][at] = mine;
        cluster.sync();
        if (split_at == 0)
            for (int k = 1; k < splits; ++k) mine += cluster.map_shared_rank(&s_sum[0][0], k)[at];
        cluster.sync();
    }
    const int out_col = blockIdx.x * kStrip + at;
    if (split_at == 0 && out_col < a.cols) {
        float* o = a.dbias + b * a.dbias_stride + out_col;
        PGT_STORE(*o, a.accumulate ? PGT_LOAD(*o) + mine : mine);
    }
}

// ---------------------------------------------------------------- checkpoints
// A block takes kRowsPerThread * 256 / G rows, G octets of them side by side (G a power of two that divides 256, four at least,
// so that the four lanes of a block of 32 values are neighbours); all loads of a thread are issued together.
constexpr int kRowsPerThread = 4;
template <typename H, int W, int WO, bool WRITE>
__global__ void __launch_bounds__(256)
checkpoint_kernel(const pg_checkpoint_args a, int log_g) {
    const int64_t b = blockIdx.z;
    const int col = ((blockIdx.y << log_g) + (threadIdx.x & ((1 << log_g) - 1))) * 8;
    const int rows_at_once = 256 >> log_g;
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * kRowsPerThread * rows_at_once + (threadIdx.x >> log_g);
    uint16_t* x = static_cast<uint16_t*>(a.x.data) + b * a.x.stride;
    int8_t* q = a.x8.values + b * a.x8.stride;
    uint8_t* s = a.x8.scales + b * a.x8.scale_stride;
    auto row = [&](int k) { return r0 + k * rows_at_once; };
    auto cols = [&](int k) { return row(k) < a.tokens ? a.cols : 0; };
    if constexpr (WRITE) {
        Piece<W> p[kRowsPerThread];
#pragma unroll
        for (int k = 0; k < kRowsPerThread; ++k) p[k] = load_oct<W>(x + row(k) * a.x.ld, col, cols(k));
#pragma unroll
        for (int k = 0; k < kRowsPerThread; ++k) {
            F2 v[4];
            widen<H>(octet<W>(p[k], x + row(k) * a.x.ld, col, cols(k)), v);
            octet_to_8<H>(v, q + row(k) * a.x8.ld, s + row(k) * a.x8.scale_ld, col, cols(k));
        }
    } else {
        Oct8 p[kRowsPerThread];
        uint32_t scale[kRowsPerThread];
#pragma unroll
        for (int k = 0; k < kRowsPerThread; ++k) {
            p[k] = load_oct8(q + row(k) * a.x8.ld, col, cols(k));
            scale[k] = col < cols(k) ? PGT_LOAD(s[row(k) * a.x8.scale_ld + col / kBlock8]) : 0u;
        }
#pragma unroll
        for (int k = 0; k < kRowsPerThread; ++k) {
            F2 v[4];
            widen8(p[k], scale_value(scale[k]), v);
            if (col < cols(k)) store_oct<H, WO>(x + row(k) * a.x.ld, col, a.cols, v);
        }
    }
}

int current_device() {
    int d = 0;
    return cudaGetDevice(&d) == cudaSuccess ? d : -1;
}

// Calls f with a compile-time element type, the width of read accesses and that of written ones.
template <typename F>
void with_type(int dtype, int in, int out, F&& f) {
    using std::integral_constant;
    auto w = [&](auto h) {
        using H = decltype(h);
        if (out < 8) f(H{}, integral_constant<int, 1>{}, integral_constant<int, 1>{});
        else if (in == 8) f(H{}, integral_constant<int, 8>{}, integral_constant<int, 8>{});
        else f(H{}, integral_constant<int, 1>{}, integral_constant<int, 8>{});
    };
    if (dtype == PG_BF16) w(__nv_bfloat16{});
    else w(__half{});
}
// Calls f with the number of octets a thread holds and the threads that share a row: a warp to 1024 columns, then two
// octets a thread and up to 1024 threads.
template <typename F>
void with_row(int cols, F&& f) {
    using std::integral_constant;
    if (cols <= 256) f(integral_constant<int, 1>{}, integral_constant<int, 32>{});
    else if (cols <= 512) f(integral_constant<int, 2>{}, integral_constant<int, 32>{});
    else if (cols <= 768) f(integral_constant<int, 3>{}, integral_constant<int, 32>{});
    else if (cols <= 1024) f(integral_constant<int, 4>{}, integral_constant<int, 32>{});
    else if (cols <= 2048) f(integral_constant<int, 2>{}, integral_constant<int, 128>{});
    else if (cols <= 4096) f(integral_constant<int, 2>{}, integral_constant<int, 256>{});
    else if (cols <= 8192) f(integral_constant<int, 2>{}, integral_constant<int, 512>{});
    else f(integral_constant<int, 2>{}, integral_constant<int, 1024>{});
}
constexpr int kMaxNormCols = 16384;

// The gradient holds three packed rows, the gains and a sum per column: one octet a thread, or two where that saves
// the exchange between warps or there is no room for more threads.  `blocks`: resident per SM.  The last one holds kMaxNormCols.
// 134 MB matrices of 64 workers, 1024 to 16384 columns by powers of two: 94, 114, 128, 109 and 174 us (4.3, 3.5, 3.1, 3.7 and 2.3
// TB/s).  Above 4096 columns the registers of 512 and 1024 threads do not hold it all and 112 to 560 bytes a thread are spilled.
struct GradRow { int octets, threads, rows, blocks; };
constexpr int kGradShapes = 7;
constexpr GradRow kGradRows[kGradShapes] = {{1, 32, 2, 4}, {2, 32, 2, 3}, {1, 128, 2, 5}, {1, 256, 2, 2}, {1, 512, 2, 1}, {2, 512, 2, 1}, {2, 1024, 1, 1}};
static_assert(kGradRows[kGradShapes - 1].octets * 8 * kGradRows[kGradShapes - 1].threads == kMaxNormCols, "the widest rows");
int grad_row(int cols) {
    int k = 0;
    while (k + 1 < kGradShapes && kGradRows[k].octets * 8 * kGradRows[k].threads < cols) ++k;
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

// Shares of a strip's tokens in the activation's gradient, eight at most (the portable cluster size): the number whose
// blocks (three per SM at once) take the fewest steps of eight rows, a block's start and end counted as six.  Workers x tokens x
// columns by 1, 2, 4 and 8 shares, and by the rule: 32 x 700 x 2600 80, 75, 86 and 95 us (75); 64 x 1024 x 1024 92.5, 92.8, 86.8 and
// 92.7 (92.6); 16 x 300 x 4096 32.6, 32.9, 37.6 and 49.6 (32.9); 8 x 2000 x 512 129, 69, 38 and 25 (25); 1 x 4096 x 2048 254, 131, 70
// and 39 (38); 64 x 2048 x 256 142, 78, 51 and 56 (55).
int strip_splits(int64_t strips, int64_t tokens) {
    int best = 1;
    double least = 0.0;
    for (int s = 1; s <= 8; s *= 2) {
        const double waves = std::max(1.0, strips * s / (3.0 * kSMs));
        const double cost = waves * ((tokens + s - 1) / s / 8.0 + 6.0);
        if (s == 1 || cost < least) {
            best = s;
            least = cost;
        }
    }
    return best;
}

}  // namespace

int take_row_errors(unsigned& value, cudaStream_t st) {
    value = 0;
#ifdef PG_BOUNDS_CHECK
    void* word = nullptr;
    if (cudaGetSymbolAddress(&word, g_outside) != cudaSuccess) return PG_ERR_CUDA;
    return take_word(static_cast<unsigned*>(word), value, st);
#else
    static_cast<void>(st);
    return PG_OK;
#endif
}

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
    Operands operands;
    operands.output(a.h, a.batch, a.tokens, a.cols, 2).output(a.y, a.batch, a.tokens, a.cols, 2).output(a.y8, a.batch, a.tokens, a.cols);
    operands.output(a.h8, a.batch, a.tokens, a.cols).output(a.rstd, a.tokens, a.batch, a.tokens);
    operands.input(a.x, a.batch, a.tokens, a.cols, 2).input(a.residual, a.batch, a.tokens, a.cols, 2).input(a.gain, a.gain_stride, a.batch, a.cols);
    if (operands.publish(static_cast<cudaStream_t>(stream)) != PG_OK) return PG_ERR_CUDA;
    with_type(a.dtype, access_width({&a.x, &a.residual}, a.batch), access_width({&a.h, &a.y}, a.batch), [&](auto h, auto in, auto out) {
        using H = decltype(h);
        constexpr int W = decltype(in)::value, WO = decltype(out)::value;
        with_row(a.cols, [&](auto octets, auto threads) {
            constexpr int T = decltype(threads)::value, C = decltype(octets)::value;
            const dim3 grid(T > 32 ? a.tokens : (a.tokens + 7) / 8, a.batch);
            norm_kernel<H, W, WO, C, T><<<grid, T > 32 ? T : 256, 0, static_cast<cudaStream_t>(stream)>>>(a);
        });
    });
    return launch_status();
}

int pg_add_rms_norm_grad_workspace_bytes(const pg_norm_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->cols, 1)) return PG_ERR_INVALID;
    if (args->cols > kMaxNormCols) return PG_ERR_TOO_LARGE;
    *bytes_out = args->dgain ? sizeof(float) * norm_grad_blocks(*args) * static_cast<size_t>(args->batch) * args->cols : 0;
    return PG_OK;
}

int pg_add_rms_norm_grad(const pg_norm_grad_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_norm_grad_args& a = *args;
    const int dev = current_device();
    const bool eight = a.h8.values != nullptr;
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.cols, 1)) return PG_ERR_INVALID;
    const bool any = int64_t{a.batch} * a.tokens > 0;              // without tokens there is no h to be had
    if (any && eight == (a.h.data != nullptr)) return PG_ERR_INVALID;
    if (!matrix_ok(a.dy, a.batch, a.tokens, a.cols, 2, false, dev)) return PG_ERR_INVALID;
    if (any && (eight ? !matrix8_ok(a.h8, a.batch, a.tokens, a.cols, false, dev)
              : !matrix_ok(a.h, a.batch, a.tokens, a.cols, 2, false, dev)))
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
    Operands operands;
    operands.output(a.dx, a.batch, a.tokens, a.cols, 2).output(a.dgain, a.dgain_stride, a.batch, a.cols).output(need > 0 ? workspace : nullptr, 0, 1, need / 4);
    operands.input(a.dy, a.batch, a.tokens, a.cols, 2).input(a.dh, a.batch, a.tokens, a.cols, 2).input(a.h, a.batch, a.tokens, a.cols, 2);
    operands.input(a.h8, a.batch, a.tokens, a.cols).input(a.rstd, a.tokens, a.batch, a.tokens).input(a.gain, a.gain_stride, a.batch, a.cols);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    if (a.tokens > 0 || a.dgain) {
        with_type(a.dtype, access_width({&a.dy, &a.h, &a.dh}, a.batch), access_width({&a.dx}, a.batch), [&](auto h, auto in, auto out) {
            using H = decltype(h);
            constexpr int W = decltype(in)::value, WO = decltype(out)::value;
            with_grad_row(a.cols, [&](auto shape) {
                constexpr GradRow g = kGradRows[decltype(shape)::value];
                constexpr int T = g.threads, C = g.octets, kGroups = T > 32 ? 1 : kGradBlock / 32;
                const int per = (a.tokens + blocks * kGroups - 1) / (blocks * kGroups);
                const dim3 grid(blocks, a.batch);
                const size_t smem = T > 32 ? 0 : sizeof(float) * kGroups * a.cols;
                if (eight) norm_grad_kernel<H, W, WO, C, T, g.rows, g.blocks, true><<<grid, T > 32 ? T : kGradBlock, smem, st>>>(a, partial, per);
                else norm_grad_kernel<H, W, WO, C, T, g.rows, g.blocks, false><<<grid, T > 32 ? T : kGradBlock, smem, st>>>(a, partial, per);
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
    const int strips = (a.cols + kStrip - 1) / kStrip;
    const int splits = strip_splits(int64_t{strips} * a.batch, a.tokens);
    const int per = (a.tokens + splits - 1) / splits;
    Operands operands;
    operands.output(a.dz, a.batch, a.tokens, a.cols, 2).output(a.dbias, a.dbias_stride, a.batch, a.cols);
    operands.input(a.dy, a.batch, a.tokens, a.cols, 2).input(a.z8, a.batch, a.tokens, a.cols);
    if (operands.publish(static_cast<cudaStream_t>(stream)) != PG_OK) return PG_ERR_CUDA;
    int rc = PG_OK;
    with_type(a.dtype, access_width({&a.dy}, a.batch), access_width({&a.dz}, a.batch), [&](auto h, auto in, auto out) {
        using H = decltype(h);
        constexpr int W = decltype(in)::value, WO = decltype(out)::value;
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
        if (a.activation == PG_ACT_RELU) launch(activation_grad_kernel<H, W, WO, PG_ACT_RELU>);
        else if (a.activation == PG_ACT_GELU) launch(activation_grad_kernel<H, W, WO, PG_ACT_GELU>);
        else if (a.activation == PG_ACT_SILU) launch(activation_grad_kernel<H, W, WO, PG_ACT_SILU>);
        else launch(activation_grad_kernel<H, W, WO, PG_ACT_NONE>);
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
    if (a.batch == 0 || a.tokens == 0) return PG_OK;
    const int width = access_width({&a.x}, a.batch);
    const int octets = (a.cols + kBlock8 - 1) / kBlock8 * (kBlock8 / 8);
    int log_g = 2;
    while (log_g < 8 && (1 << log_g) < octets) ++log_g;
    while (log_g > 5 && (octets & ((1 << log_g) - 1)) != 0 && (1 << log_g) - (octets & ((1 << log_g) - 1)) > (octets >> 3)) --log_g;   // idle lanes: an eighth at most
    const int64_t per_block = kRowsPerThread * (256 >> log_g);
    const dim3 grid(static_cast<unsigned>((a.tokens + per_block - 1) / per_block), static_cast<unsigned>((octets + (1 << log_g) - 1) >> log_g), a.batch);
    if (grid.y > 65535) return PG_ERR_TOO_LARGE;
    Operands operands;
    if (write) operands.output(a.x8, a.batch, a.tokens, a.cols).input(a.x, a.batch, a.tokens, a.cols, 2);
    else operands.output(a.x, a.batch, a.tokens, a.cols, 2).input(a.x8, a.batch, a.tokens, a.cols);
    if (operands.publish(static_cast<cudaStream_t>(stream)) != PG_OK) return PG_ERR_CUDA;
    with_type(a.dtype, write ? width : 8, write ? 8 : width, [&](auto h, auto in, auto out) {
        using H = decltype(h);
        constexpr int W = decltype(in)::value, WO = decltype(out)::value;
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        if (write) checkpoint_kernel<H, W, WO, true><<<grid, 256, 0, st>>>(a, log_g);
        else checkpoint_kernel<H, W, WO, false><<<grid, 256, 0, st>>>(a, log_g);
    });
    return launch_status();
}
int pg_checkpoint_write(const pg_checkpoint_args* args, void* stream) { return checkpoint(args, true, stream); }
int pg_checkpoint_read(const pg_checkpoint_args* args, void* stream) { return checkpoint(args, false, stream); }

}  // extern "C"
