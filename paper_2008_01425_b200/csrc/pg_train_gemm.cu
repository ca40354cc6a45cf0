// The batched linear layer and its gradients.
//
// All three products are computed as D[m][n] = sum_k A[m][k] B[n][k] with m the output's contiguous
// dimension, so that neighbouring lanes always store neighbouring addresses:
//     y  = x W^T     m = out feature  n = token        k = in feature
//     dx = dz W      m = in feature   n = token        k = out feature
//     dW = dz^T x    m = in feature   n = out feature  k = token
#include <initializer_list>

#include "pg_train_device.h"

namespace pgt {
namespace {

// What happens to D: stored as fp32 (dW), or passed through bias, activation and residual to 16 bits.
struct Epilogue {
    int32_t fp32, accumulate, activation;
    pg_matrix out;             // n rows of m elements
    pg_matrix residual;
    const float* bias;
    int64_t bias_stride;
    pg_matrix8 z8;
};
struct Operand {               // element (row, k) of worker b at data + b stride + row ld + k step
    const void* data;
    int64_t ld, step, stride;
    const uint8_t* scales;     // set for an 8-bit operand; its blocks run along the rows index (m)
    int64_t scale_ld, scale_stride;
};

constexpr int kTile = 64, kDepth = 16;

template <typename H>
__global__ void __launch_bounds__(256)
product_kernel(Operand A, Operand B, Epilogue ep, int M, int N, int K) {
    __shared__ float s_a[kDepth][kTile + 1], s_b[kDepth][kTile + 1];
    __shared__ float s_d[kTile][kTile + 1];
    const int64_t b = blockIdx.z;
    const int m0 = blockIdx.x * kTile, n0 = blockIdx.y * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += kDepth) {
        __syncthreads();
        for (int t = threadIdx.x; t < kTile * kDepth; t += 256) {
            const int r = t / kDepth, k = t % kDepth;
            float va = 0.0f, vb = 0.0f;
            if (m0 + r < M && k0 + k < K) {
                const int64_t at = b * A.stride + (m0 + r) * A.ld + (k0 + k) * A.step;
                if (A.scales)
                    va = static_cast<const int8_t*>(A.data)[at] *
                         scale_value(A.scales[b * A.scale_stride + (k0 + k) * A.scale_ld + (m0 + r) / kBlock8]);
                else
                    va = Elem<H>::up(static_cast<const uint16_t*>(A.data)[at]);
            }
            if (n0 + r < N && k0 + k < K)
                vb = Elem<H>::up(static_cast<const uint16_t*>(B.data)[b * B.stride + (n0 + r) * B.ld + (k0 + k) * B.step]);
            s_a[k][r] = va;
            s_b[k][r] = vb;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDepth; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(s_a[k][tx * 4 + i], s_b[k][ty * 4 + j], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s_d[ty * 4 + j][tx * 4 + i] = acc[i][j];
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int m = m0 + (warp & 1) * 32 + lane;
    const float bias = ep.bias && m < M ? ep.bias[b * ep.bias_stride + m] : 0.0f;
    for (int j = warp >> 1; j < kTile && n0 + j < N; j += 4) {
        float v = s_d[j][(warp & 1) * 32 + lane];
        const int64_t n = n0 + j;
        if (ep.fp32) {
            if (m < M) {
                float* o = static_cast<float*>(ep.out.data) + b * ep.out.stride + n * ep.out.ld + m;
                *o = ep.accumulate ? *o + v : v;
            }
            continue;
        }
        v += bias;
        if (ep.z8.values) {
            const uint32_t s = scale_byte<H>(block_top<1>(m < M ? __float_as_uint(v) & 0x7fffffffu : 0u));
            if (m < M) {
                ep.z8.values[b * ep.z8.stride + n * ep.z8.ld + m] = static_cast<int8_t>(to8(v, scale_inverse(s)));
                if (lane == 0) ep.z8.scales[b * ep.z8.scale_stride + n * ep.z8.scale_ld + m / kBlock8] = static_cast<uint8_t>(s);
            }
        }
        if (ep.activation == PG_ACT_RELU) v = activate<PG_ACT_RELU>(v);
        if (ep.activation == PG_ACT_GELU) v = activate<PG_ACT_GELU>(v);
        if (ep.activation == PG_ACT_SILU) v = activate<PG_ACT_SILU>(v);
        if (m < M) {
            if (ep.residual.data)
                v += Elem<H>::up(static_cast<const uint16_t*>(ep.residual.data)[b * ep.residual.stride + n * ep.residual.ld + m]);
            static_cast<uint16_t*>(ep.out.data)[b * ep.out.stride + n * ep.out.ld + m] = Elem<H>::down(v);
        }
    }
}

int run_product(int dtype, int batch, int64_t M, int64_t N, int64_t K, const Operand& A, const Operand& B, const Epilogue& ep, void* stream) {
    const dim3 grid((M + kTile - 1) / kTile, (N + kTile - 1) / kTile, batch);
    if (grid.y > 65535) return PG_ERR_TOO_LARGE;
    if (dtype == PG_BF16) product_kernel<__nv_bfloat16><<<grid, 256, 0, static_cast<cudaStream_t>(stream)>>>(A, B, ep, M, N, K);
    else product_kernel<__half><<<grid, 256, 0, static_cast<cudaStream_t>(stream)>>>(A, B, ep, M, N, K);
    return launch_status();
}

int current_device() {
    int d = 0;
    return cudaGetDevice(&d) == cudaSuccess ? d : -1;
}

}  // namespace
}  // namespace pgt

using namespace pgt;

extern "C" {

int pg_linear_workspace_bytes(const pg_linear_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->in_features, args->out_features)) return PG_ERR_INVALID;
    *bytes_out = 0;
    return PG_OK;
}
int pg_linear(const pg_linear_args* args, void*, size_t, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_linear_args& a = *args;
    const int dev = current_device();
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.in_features, a.out_features) || a.activation < PG_ACT_NONE || a.activation > PG_ACT_SILU)
        return PG_ERR_INVALID;
    if (!matrix_ok(a.x, a.batch, a.tokens, a.in_features, 2, false, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.weight, a.batch, a.out_features, a.in_features, 2, false, dev)) return PG_ERR_INVALID;
    if (a.bias && !vector_ok(a.bias, a.bias_stride, a.batch, a.out_features, false, dev)) return PG_ERR_INVALID;
    if (a.residual.data && !matrix_ok(a.residual, a.batch, a.tokens, a.out_features, 2, false, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.y, a.batch, a.tokens, a.out_features, 2, true, dev)) return PG_ERR_INVALID;
    if ((a.z8.values || a.z8.scales) && !matrix8_ok(a.z8, a.batch, a.tokens, a.out_features, true, dev)) return PG_ERR_INVALID;
    if (a.batch == 0 || a.tokens == 0) return PG_OK;
    const Operand A{a.weight.data, a.weight.ld, 1, a.weight.stride, nullptr, 0, 0};
    const Operand B{a.x.data, a.x.ld, 1, a.x.stride, nullptr, 0, 0};
    const Epilogue ep{0, 0, a.activation, a.y, a.residual, a.bias, a.bias_stride, a.z8};
    return run_product(a.dtype, a.batch, a.out_features, a.tokens, a.in_features, A, B, ep, stream);
}

int pg_linear_input_grad_workspace_bytes(const pg_input_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->in_features, args->out_features)) return PG_ERR_INVALID;
    *bytes_out = 0;
    return PG_OK;
}
int pg_linear_input_grad(const pg_input_grad_args* args, void*, size_t, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_input_grad_args& a = *args;
    const int dev = current_device();
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.in_features, a.out_features)) return PG_ERR_INVALID;
    if (!matrix_ok(a.dz, a.batch, a.tokens, a.out_features, 2, false, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.weight, a.batch, a.out_features, a.in_features, 2, false, dev)) return PG_ERR_INVALID;
    if (a.residual.data && !matrix_ok(a.residual, a.batch, a.tokens, a.in_features, 2, false, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.dx, a.batch, a.tokens, a.in_features, 2, true, dev)) return PG_ERR_INVALID;
    if (a.batch == 0 || a.tokens == 0) return PG_OK;
    const Operand A{a.weight.data, 1, a.weight.ld, a.weight.stride, nullptr, 0, 0};
    const Operand B{a.dz.data, a.dz.ld, 1, a.dz.stride, nullptr, 0, 0};
    const Epilogue ep{0, 0, PG_ACT_NONE, a.dx, a.residual, nullptr, 0, {}};
    return run_product(a.dtype, a.batch, a.in_features, a.tokens, a.out_features, A, B, ep, stream);
}

int pg_linear_weight_grad_workspace_bytes(const pg_weight_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->in_features, args->out_features)) return PG_ERR_INVALID;
    *bytes_out = 0;
    return PG_OK;
}
int pg_linear_weight_grad(const pg_weight_grad_args* args, void*, size_t, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_weight_grad_args& a = *args;
    const int dev = current_device();
    const bool eight = a.x8.values != nullptr;
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.in_features, a.out_features)) return PG_ERR_INVALID;
    if (eight == (a.x.data != nullptr) && int64_t{a.batch} * a.tokens > 0) return PG_ERR_INVALID;
    if (!matrix_ok(a.dz, a.batch, a.tokens, a.out_features, 2, false, dev)) return PG_ERR_INVALID;
    if (eight ? !matrix8_ok(a.x8, a.batch, a.tokens, a.in_features, false, dev)
              : !matrix_ok(a.x, a.batch, a.tokens, a.in_features, 2, false, dev))
        return PG_ERR_INVALID;
    if (!matrix_ok(a.dweight, a.batch, a.out_features, a.in_features, 4, true, dev)) return PG_ERR_INVALID;
    if (a.batch == 0) return PG_OK;
    const Operand A = eight ? Operand{a.x8.values, 1, a.x8.ld, a.x8.stride, a.x8.scales, a.x8.scale_ld, a.x8.scale_stride}
                            : Operand{a.x.data, 1, a.x.ld, a.x.stride, nullptr, 0, 0};
    const Operand B{a.dz.data, 1, a.dz.ld, a.dz.stride, nullptr, 0, 0};
    const Epilogue ep{1, a.accumulate, PG_ACT_NONE, a.dweight, {}, nullptr, 0, {}};
    return run_product(a.dtype, a.batch, a.in_features, a.out_features, a.tokens, A, B, ep, stream);
}

int pg_training_status(void* stream) {
    return cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) == cudaSuccess ? PG_OK : PG_ERR_CUDA;
}

}  // extern "C"
