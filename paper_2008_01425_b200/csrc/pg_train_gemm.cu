// The batched linear layer and its gradients on the fifth-generation tensor cores.
//
// All products are D[m][n] = sum_k A[m][k] B[n][k]; m is the accumulator's lane.
//   few tokens, m = the output's contiguous dimension:
//     y  = x W^T     m = out feature  n = token        k = in feature     A rows of W, B rows of x
//     dx = dz W      m = in feature   n = token        k = out feature    A columns of W, B rows of dz
//   many tokens, m = token:
//     y  = x W^T     m = token        n = out feature  k = in feature     A rows of x, B rows of W
//     dx = dz W      m = token        n = in feature   k = out feature    A rows of dz, B columns of W
//   always m = the output's contiguous dimension:
//     dW = dz^T x    m = in feature   n = out feature  k = token          A columns of x, B columns of dz
// With features as lanes a single token costs a 16-column tile, not a 128-row one, and 32 lanes store 32 neighbouring
// elements.  With tokens as lanes a thread holds 32 neighbouring elements of one row: one block of the 8-bit form,
// packed conversions, and 16-byte pieces that leave through shared memory and TMA.
//
// A block computes 128 x BN tiles (BN up to 256), 64 deep stages: one thread feeds shared memory by TMA, one issues
// tcgen05.mma, eight warps empty the accumulator of one tile while the next one is summed in the other half of tensor
// memory.
#include <cooperative_groups.h>
#include <cuda.h>

#include <algorithm>
#include <initializer_list>
#include <mutex>

#include "pg_train_device.h"
#include "pg_train_ranges.h"

namespace pgt {
namespace {

constexpr int kBM = 128;              // lanes of an accumulator
constexpr int kBK = 64;               // elements of k in a stage: one 128-byte swizzled row
constexpr int kMaxStages = 12;
constexpr int kSmemBytes = 232448;    // what a block may have,
constexpr int kStaticBytes = 2304;    // what of it is left to Shared and the compiler (Shared takes less than 600 bytes),
constexpr int kRingBytes = kSmemBytes - kStaticBytes - 1024;     // and the rest, less what aligning it to 1024 bytes may cost
constexpr int kABytes = kBM * kBK * 2;
constexpr int kRawBytes = kBM * kBK;          // a stage of an 8-bit A before it is widened
constexpr int kScaleStages = 8;               // stages whose scales are fetched at once, 4 bytes for each of their k
constexpr int kScaleBytes = 2 * kScaleStages * kBK * 4;
constexpr int kMaxRaw = 8, kMinRaw = 4;       // such stages: a ring of their own, since they are needed before A and B are
// Blocks of k that tensor memory sums in one go for a weight gradient.  The tensor cores cut a sum off where fp32 arithmetic
// would round it, so the error grows with the length of the sum and, unlike a rounded one's, does not average out; the more bits
// the products have the sooner.  Longer sums are added up, rounding, from parts of this length.  Error of a gradient relative to
// its size for tokens of different sizes, by blocks in a part (an fp32 product's over 768 tokens: 0.25e-6 bf16, 0.49e-6 fp16):
//   bf16         8: 0.55e-6   12: 0.83e-6   16: 1.12e-6           fp16         8: 0.65e-6   12: 0.95e-6   16: 1.25e-6
//   bf16, x8    12: 0.26e-6   16: 0.38e-6   32: 0.87e-6           fp16, x8    12: 0.74e-6   16: 1.0e-6    32: 2.1e-6
// and time over 2048 tokens for 64 workers of 1024 x 1024: 523, 336, 298, 264 and 233 us for 4, 8, 12, 16 and 32 (x8: 572, 387, 358,
// 331 and 305 us; 20 workers x 1500 tokens of 656 x 1000 from 8 bits, one part 69 us, two 98).  Chosen: the longest parts that stay
// under 1e-6, and for bf16 from 8 bits half of that, about twice an fp32 product's error instead of five times.
// Sums of products that all have one sign lose more: 1.5e-6 (bf16), 4.4e-6 (fp16), 0.75e-6 and 1.2e-6 (x8).
constexpr int max_chunk(bool eight, int dtype) { return eight && dtype == PG_BF16 ? 1024 / kBK : 768 / kBK; }
constexpr int kMaxSplits = 8;         // blocks of a cluster that share the k of one tile
constexpr long long kWaitNs = 2000000000;   // a wait longer than this gives up

enum Mode { kForward, kInputGrad, kForwardRows, kInputGradRows, kWeightGrad, kWeightGrad8 };
template <Mode M> constexpr bool kWeightGrads = M == kWeightGrad || M == kWeightGrad8;
template <Mode M> constexpr bool kTokenRows = M == kForwardRows || M == kInputGradRows;
template <Mode M> constexpr bool kAMnMajor = M == kInputGrad || kWeightGrads<M>;
template <Mode M> constexpr bool kBMnMajor = M == kInputGradRows || kWeightGrads<M>;
constexpr int kRowWarps = 12;         // epilogue warps where lanes are tokens
constexpr int kShares = kRowWarps / 4;
constexpr int kOutBytes = 2048;       // 32 rows x 32 elements of one of them on their way out,
constexpr int kHeldBytes = 32 * 80;   // and five 16-byte pieces of residuals for each of the rows
constexpr int kBiasBytes = 512;       // and the biases of its groups;
constexpr int kOut8Bytes = 1024;      // the 8-bit form of a group on its way out, where there is one
constexpr int kOutWarp = kOutBytes + kHeldBytes + kBiasBytes;    // (a multiple of 512, the period of the swizzle)
static_assert((256 / 32 + kShares - 1) / kShares * 128 <= kBiasBytes && kOutWarp % 512 == 0, "a warp's share");
template <Mode M> constexpr int kEpilogueWarps = kTokenRows<M> ? kRowWarps : 8;
template <Mode M> constexpr int kThreads = 128 + 32 * kEpilogueWarps<M> + (M == kWeightGrad8 ? 256 : 0);

// What happens to D: stored as fp32 (dW), or passed through bias, activation and residual to 16 bits.
struct Epilogue {
    int32_t accumulate, activation;
    pg_matrix out;             // n rows of m elements
    pg_matrix residual;
    const float* bias;
    int64_t bias_stride;
    pg_matrix8 z8;
};
struct Problem {
    Epilogue ep;
    int M, N, K;
    int BN, m_tiles, n_tiles, stages, raw_stages, k_blocks, splits;
    int out_warp;              // bytes of an epilogue warp's share
    int part_at;               // split k: where in shared memory a block's part is
    int chunk;                 // blocks of k that are summed in tensor memory before they are added to the rest
    int64_t tiles;
    int a_shared, b_shared;    // operand is the same for every worker
    int residual_aligned;      // its rows start on 16-byte boundaries
    const uint8_t* scales;     // of an 8-bit A
    int64_t scale_ld, scale_stride;
};

__device__ unsigned g_training_error;   // a bounded wait gave up; read and cleared by pg_training_status

// ------------------------------------------------------------------ PTX
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
    return ok != 0;
}
// Waits for the phase; false when the block gave up (this wait ran out, or another thread's did).  The time is looked at
// after a few thousand tries only.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* gave_up, long long limit = kWaitNs) {
#pragma unroll 1
    for (int i = 0; i < 4096; ++i)
        if (bar_try(b, parity)) return true;
    long long t0, t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 1024; ++i)
            if (bar_try(b, parity)) return true;
        if (*gave_up) return false;
        asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
        if (t - t0 > limit) {
            *gave_up = 1;
            atomicOr(&g_training_error, kTimedOut);
            return false;
        }
    }
}
// After a wait that gave up: the last copies that were issued to a ring of `n` stages, `issued` in all, land (or a limit is reached).
__device__ __noinline__ void await_copies(uint64_t* bars, int n, int64_t issued) {
    for (int64_t i = issued > n ? issued - n : 0; i < issued; ++i)
        for (int t = 0; t < 100000 && !bar_try(&bars[i % n], static_cast<uint32_t>(i / n) & 1); ++t) {}
}
// The same where they cannot be waited for: a hundred times what a copy takes.
__device__ __noinline__ void pause() {
    long long t0, t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
    do asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    while (t - t0 < 200000);
}
__device__ __forceinline__ void tma_load(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}
// The same with a barrier of the pair's first block.
__device__ __forceinline__ void tma_load_pair(void* dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
// The address of one of this block's barriers in the first block of its pair.
__device__ __forceinline__ uint32_t first_of_pair(uint64_t* b) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(b)));
    return r;
}
// Arrivals, there and in this block, that say no more than that an accumulator has been read (tcgen05.wait::ld and the fence before them see to that).
__device__ __forceinline__ void bar_arrive_read_at(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive_read(uint64_t* b) {
    asm volatile("mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, const void* src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(smem_u32(src)), "r"(x), "r"(y),
                 "r"(z)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// PAIR: two blocks on neighbouring SMs multiply together, each with its 128 rows of A and half of B's rows in its own
// shared memory; the first of them issues, and its commits reach the same barrier of both.
template <bool PAIR>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    if constexpr (PAIR)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"(add)
                     : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"(add)
                     : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                     "h"(static_cast<uint16_t>(3))
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// One lane of a converged warp.  The loops that feed the tensor cores run in whole warps and choose a lane only to issue:
// then descriptors, coordinates and barriers stay in uniform registers (one lane's own loop fell behind the tensor cores).
__device__ __forceinline__ bool elected() {
    uint32_t yes;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(yes));
    return yes != 0;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
        "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
// Shared-memory operand descriptors, 128-byte swizzle.  K-major: rows of 64 k, 8-row groups 1024 bytes
// apart.  MN-major: rows of 64 m (one per k), 8-k groups 1024 bytes apart, the next 64 m 8192 bytes on.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn_major) {
    const uint64_t lead = mn_major ? 8192 >> 4 : 1, group = 1024 >> 4;
    return static_cast<uint64_t>((addr & 0x3ffff) >> 4) | lead << 16 | group << 32 | uint64_t{1} << 46 | uint64_t{2} << 61;
}

// ------------------------------------------------------------------ epilogue
__device__ __forceinline__ uint32_t byte8(float v, float inverse) { return __float_as_uint(clamp8(fmaf(v, inverse, kRound))) & 255u; }

// Columns n .. n + count - 1 (16 at most) of lane m.
template <typename H, int ACT, bool FP32>
__device__ __forceinline__ void emit(const Epilogue& ep, float (&v)[16], int64_t b, int64_t n, int count, int m, bool live, float bias, bool more = false) {
    if constexpr (FP32) {
        float* o = static_cast<float*>(ep.out.data) + b * ep.out.stride + n * ep.out.ld + m;
        if (!live) return;
        if (ep.accumulate || more) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < count) v[i] += PGT_LOAD(o[i * ep.out.ld]);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < count) PGT_STORE(o[i * ep.out.ld], v[i]);
    } else {
        uint16_t res[16];
        const bool residual = ep.residual.data != nullptr;
        if (residual && live) {
            const uint16_t* r = static_cast<const uint16_t*>(ep.residual.data) + b * ep.residual.stride + n * ep.residual.ld + m;
#pragma unroll
            for (int i = 0; i < 16; ++i) res[i] = i < count ? PGT_LOAD(r[i * ep.residual.ld]) : 0;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] += bias;
        if (ep.z8.values) {        // the warp's 32 lanes are one block
            int8_t* q = ep.z8.values + b * ep.z8.stride + n * ep.z8.ld + m;
            uint8_t* s = ep.z8.scales + b * ep.z8.scale_stride + n * ep.z8.scale_ld + m / kBlock8;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t sb = scale_byte<H>(__reduce_max_sync(0xffffffffu, live ? __float_as_uint(v[i]) & 0x7fffffffu : 0u));
                if (live && i < count) {
                    PGT_STORE(q[i * ep.z8.ld], static_cast<int8_t>(byte8(v[i], scale_inverse(sb))));
                    if (m % kBlock8 == 0) PGT_STORE(s[i * ep.z8.scale_ld], static_cast<uint8_t>(sb));
                }
            }
        }
        if (!live) return;
        uint16_t* o = static_cast<uint16_t*>(ep.out.data) + b * ep.out.stride + n * ep.out.ld + m;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            F2 y = activate<ACT>(pair(v[i], v[i + 1]));
            if (residual) y = add(y, pair(Elem<H>::up(res[i]), Elem<H>::up(res[i + 1])));
            const uint32_t w = Elem<H>::down2(y);
            if (i < count) PGT_STORE(o[i * ep.out.ld], static_cast<uint16_t>(w & 0xffffu));
            if (i + 1 < count) PGT_STORE(o[(i + 1) * ep.out.ld], static_cast<uint16_t>(w >> 16));
        }
    }
}

struct Shared {
    uint64_t raw[kMaxRaw], raw_empty[kMaxRaw], scaled[2], scales_empty[2], loaded[kMaxStages], widened[kMaxStages], empty[kMaxStages], summed[2], drained[2], last;
    uint32_t tmem;
    int gave_up;
};
static_assert(sizeof(Shared) <= 600, "Shared");

// Lanes are tokens: a warp takes every third group of 32 columns of its 32 rows.  The residuals of the next group are on
// their way to shared memory while one group is computed, and while the first one's accumulator is waited for: neighbouring
// lanes copy neighbouring 16-byte pieces, four of a row or five where it starts between two (a lane that fetches its own row
// touches 32 lines per load).  The result goes through shared memory too, in the
// 64-byte swizzle of the output's tensor map, and leaves by TMA, which also cuts off what lies outside the matrix.
struct Residuals {             // of a tile: where a lane's five pieces start, from the tile's first column on
    const char* base;
    uint32_t at[5];            // bytes from the first of the warp's 32 rows
    uint32_t wanted;           // bit i: the row is inside and has such a piece
    uint32_t low;              // the first row's own start, in bytes from its first piece's
    int off;                   // elements from the first piece's start to this lane's own row

    __device__ __forceinline__ void start(const Epilogue& ep, int64_t b, int row0, int rows, int n0, int lane) {
        const int64_t first = b * ep.residual.stride + static_cast<int64_t>(row0) * ep.residual.ld + n0;
        const uintptr_t from = reinterpret_cast<uintptr_t>(ep.residual.data) + first * 2;
        base = reinterpret_cast<const char*>(from & ~uintptr_t{15});
        low = from & 15;
        const uint32_t ld = static_cast<uint32_t>(ep.residual.ld) * 2;
        wanted = 0;
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const uint32_t k = lane + 32 * i, r = k / 5, c = k - r * 5, start_at = low + r * ld;
            at[i] = (start_at & ~15u) + c * 16;
            if (row0 + static_cast<int>(r) < rows && (c < 4 || (start_at & 15) != 0)) wanted |= 1u << i;
        }
        off = static_cast<int>(low + lane * ld & 15) / 2;
    }
    // Copies the pieces of the 32 columns from n0 + j on; `left`: columns from there to the matrix's end.  Where they are fewer
    // than all pieces may hold, only those that hold one of them.
    __device__ __forceinline__ void fetch(const Epilogue& ep, uint8_t* held, int j, int left, int lane) const {
        const char* from = base + 2 * j;
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const uint32_t k = lane + 32 * i, r = k / 5, c = k - r * 5;
            bool in = wanted >> i & 1;
            if (left < 40) in = in && static_cast<int>(8 * c) - static_cast<int>(low + r * static_cast<uint32_t>(ep.residual.ld) * 2 & 15) / 2 < left;
            if (in && PGT_READ(from + at[i], 16)) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(held) + k * 16), "l"(from + at[i]) : "memory");
        }
    }
};
template <typename H, int ACT>
__device__ __forceinline__ void empty_rows(const Problem& p, const CUtensorMap* map_out, const CUtensorMap* map_out8, uint32_t tmem, uint8_t* out, int64_t b, int m0,
                                           int n0, int share, int quarter, int lane, const Residuals& residuals) {
    const Epilogue& ep = p.ep;
    uint8_t* held = out + kOutBytes;
    const float* s_bias = reinterpret_cast<const float*>(held + kHeldBytes);
    const int row = m0 + quarter * 32 + lane;
    const bool live = row < p.M;
    const int end = min(p.BN, p.N - n0);
    const bool add_residual = ep.residual.data != nullptr;
    for (int j = share * 32; j < end; j += kShares * 32, s_bias += 32) {
        const int n = n0 + j;
        uint4 piece[5];
        if (add_residual) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 5; ++i) piece[i] = *reinterpret_cast<const uint4*>(held + (lane * 5 + i) * 16);
            if (!p.residual_aligned) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Oct o = cut(piece[i], piece[i + 1], residuals.off);
                    piece[i] = make_uint4(o.w[0], o.w[1], o.w[2], o.w[3]);
                }
            }
        }
        __syncwarp();
        const int next = j + kShares * 32;
        if (add_residual && next < end) residuals.fetch(ep, held, next, p.N - n0 - next, lane);
        const uint32_t from = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + j;
        if (ep.z8.values) {
            F2 v[4][4];
            float acc[32];
            tmem_load32(from, acc);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 f = reinterpret_cast<const float4*>(s_bias)[i];
                v[i / 2][2 * (i & 1)] = add(pair(acc[4 * i], acc[4 * i + 1]), pair(f.x, f.y));
                v[i / 2][2 * (i & 1) + 1] = add(pair(acc[4 * i + 2], acc[4 * i + 3]), pair(f.z, f.w));
            }
            const uint32_t s = scale_byte<H>(max(max(top_bits(v[0]), top_bits(v[1])), max(top_bits(v[2]), top_bits(v[3]))));
            const F2 inverse = both(scale_inverse(s));
            Oct8 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                F2 t[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) t[k] = to8(v[i][k], inverse);
                q[i] = pack8(t);
            }
            if (live) PGT_STORE(ep.z8.scales[b * ep.z8.scale_stride + row * ep.z8.scale_ld + n / kBlock8], static_cast<uint8_t>(s));
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");      // the last group's copies have been read
            __syncwarp();
            uint4* to = reinterpret_cast<uint4*>(out + kOutWarp + lane * 32);
            to[0] = make_uint4(q[0].w[0], q[0].w[1], q[1].w[0], q[1].w[1]);
            to[1] = make_uint4(q[2].w[0], q[2].w[1], q[3].w[0], q[3].w[1]);
        }
        // (the accumulator is read again: tensor memory is faster than registers are plenty)
        uint32_t w[16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float acc[16];
            tmem_load16(from + 16 * h, acc);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 f = reinterpret_cast<const float4*>(s_bias)[4 * h + i];
                F2 lo = activate<ACT>(add(pair(acc[4 * i], acc[4 * i + 1]), pair(f.x, f.y)));
                F2 hi = activate<ACT>(add(pair(acc[4 * i + 2], acc[4 * i + 3]), pair(f.z, f.w)));
                if (add_residual) {
                    const int k = 2 * h + i / 2;
                    lo = add(lo, Elem<H>::up2(i & 1 ? piece[k].z : piece[k].x));
                    hi = add(hi, Elem<H>::up2(i & 1 ? piece[k].w : piece[k].y));
                }
                w[8 * h + 2 * i] = Elem<H>::down2(lo);
                w[8 * h + 2 * i + 1] = Elem<H>::down2(hi);
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");      // the last group's copy has been read
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(out + lane * 64 + ((i ^ (lane >> 1 & 3)) << 4)) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0 && m0 + quarter * 32 < p.M) {
            if (ep.z8.values) tma_store(map_out8, out + kOutWarp, n, m0 + quarter * 32, static_cast<int>(b));
            tma_store(map_out, out, n, m0 + quarter * 32, static_cast<int>(b));
        }
    }
}

// 16 whole columns for a warp whose lanes are all inside: no predicates, residuals fetched beforehand.
// Addresses are a base that is the same for the warp and a lane's 32-bit offset.
template <typename H, int ACT>
__device__ __forceinline__ void emit_full(const Epilogue& ep, float (&v)[16], const uint16_t (&res)[16], char* out, int8_t* q, uint8_t* s,
                                          uint32_t lane_out, uint32_t lane_q, bool first, float bias) {
    F2 y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = add(pair(v[2 * i], v[2 * i + 1]), both(bias));
    if (q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float lo, hi;
            split(y[i], lo, hi);
            const uint32_t s0 = scale_byte<H>(__reduce_max_sync(0xffffffffu, __float_as_uint(lo) & 0x7fffffffu));
            const uint32_t s1 = scale_byte<H>(__reduce_max_sync(0xffffffffu, __float_as_uint(hi) & 0x7fffffffu));
            PGT_STORE((q + 2 * i * ep.z8.ld)[lane_q], static_cast<int8_t>(byte8(lo, scale_inverse(s0))));
            PGT_STORE((q + (2 * i + 1) * ep.z8.ld)[lane_q], static_cast<int8_t>(byte8(hi, scale_inverse(s1))));
            if (first) {
                PGT_STORE(s[2 * i * ep.z8.scale_ld], static_cast<uint8_t>(s0));
                PGT_STORE(s[(2 * i + 1) * ep.z8.scale_ld], static_cast<uint8_t>(s1));
            }
        }
    }
    const bool residual = ep.residual.data != nullptr;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = activate<ACT>(y[i]);
        if (residual) y[i] = add(y[i], pair(Elem<H>::up(res[2 * i]), Elem<H>::up(res[2 * i + 1])));
        const uint32_t w = Elem<H>::down2(y[i]);
        PGT_STORE(*reinterpret_cast<uint16_t*>(out + 2 * i * ep.out.ld * 2 + lane_out), static_cast<uint16_t>(w & 0xffffu));
        PGT_STORE(*reinterpret_cast<uint16_t*>(out + (2 * i + 1) * ep.out.ld * 2 + lane_out), static_cast<uint16_t>(w >> 16));
    }
}

// One tile's accumulator to the output, or (split k) to this block's part in shared memory.  The two warps of a
// quarter take every other 16 columns.
template <typename H, int ACT, bool FP32>
__device__ __forceinline__ void empty_tile(const Problem& p, uint32_t tmem, float* part, bool more, int64_t b, int m0, int n0, int half, int quarter, int lane) {
    const Epilogue& ep = p.ep;
    const int m = m0 + quarter * 32 + lane;
    const bool live = m < p.M;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    const int end = part ? p.BN : min(p.BN, p.N - n0);
    const float bias = !FP32 && ep.bias && live ? PGT_LOAD(ep.bias[b * ep.bias_stride + m]) : 0.0f;
    float v[16];
    if (part || p.K == 0) {
        for (int j = half * 16; j < end; j += 32) {
            if (p.K > 0) tmem_load16(lanes + j, v);
            else {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = 0.0f;
            }
            if (part) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float* at = part + (j + i) * kBM + quarter * 32 + lane;
                    *at = more ? *at + v[i] : v[i];
                }
            } else {
                emit<H, ACT, FP32>(ep, v, b, n0 + j, min(16, end - j), m, live, bias);
            }
        }
        return;
    }
    int j = half * 16;
    if (m0 + quarter * 32 + 32 <= p.M) {
        if constexpr (FP32) {
            float* o = static_cast<float*>(ep.out.data) + b * ep.out.stride + static_cast<int64_t>(n0 + j) * ep.out.ld + m;
            const bool add = ep.accumulate || more;
            for (; j + 16 <= end; j += 32, o += 32 * ep.out.ld) {
                float old[16];
                if (add) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) old[i] = PGT_LOAD(o[i * ep.out.ld]);
                }
                tmem_load16(lanes + j, v);
                if (add) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] += old[i];
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) PGT_STORE(o[i * ep.out.ld], v[i]);
            }
        } else {
            const int64_t n = n0 + j;
            char* out = static_cast<char*>(ep.out.data) + (b * ep.out.stride + n * ep.out.ld) * 2;
            const char* in = static_cast<const char*>(ep.residual.data) + (b * ep.residual.stride + n * ep.residual.ld) * 2;
            int8_t* q = ep.z8.values ? ep.z8.values + b * ep.z8.stride + n * ep.z8.ld : nullptr;
            uint8_t* s = ep.z8.values ? ep.z8.scales + b * ep.z8.scale_stride + n * ep.z8.scale_ld + (m0 + quarter * 32) / kBlock8 : nullptr;
            const uint32_t lane_m = static_cast<uint32_t>(m);
            const bool add = ep.residual.data != nullptr;
            uint16_t res[16], next[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) next[i] = 0;
            auto fetch = [&](int at) {
                if (add && at + 16 <= end) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) next[i] = PGT_LOAD(*reinterpret_cast<const uint16_t*>(in + i * ep.residual.ld * 2 + lane_m * 2));
                }
                in += 64 * ep.residual.ld;
            };
            fetch(j);
            for (; j + 16 <= end; j += 32) {
#pragma unroll
                for (int i = 0; i < 16; ++i) res[i] = next[i];
                fetch(j + 32);
                tmem_load16(lanes + j, v);
                emit_full<H, ACT>(ep, v, res, out, q, s, lane_m * 2, lane_m, lane == 0, bias);
                out += 64 * ep.out.ld;
                if (q) {
                    q += 32 * ep.z8.ld;
                    s += 32 * ep.z8.scale_ld;
                }
            }
        }
    }
    for (; j < end; j += 32) {             // the last columns, or lanes past the last row
        tmem_load16(lanes + j, v);
        emit<H, ACT, FP32>(ep, v, b, n0 + j, min(16, end - j), m, live, bias, more);
    }
}
// Split k: this block adds up all parts of its share of the columns, in the order of the blocks.
template <typename H, int ACT, bool FP32>
__device__ __forceinline__ void join_parts(const Problem& p, float* part, int64_t b, int m0, int n0, int rank, int half, int quarter, int lane) {
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    const int m = m0 + quarter * 32 + lane;
    const bool live = m < p.M;
    const float bias = !FP32 && p.ep.bias && live ? PGT_LOAD(p.ep.bias[b * p.ep.bias_stride + m]) : 0.0f;
    const int per = p.BN / p.splits, each = per / 2;       // BN is a multiple of 16 and splits at most 8
    const int j0 = rank * per + half * each;
    for (int j = j0; j < j0 + each && n0 + j < p.N; j += 16) {
        const int count = min(min(16, j0 + each - j), p.N - n0 - j);
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = 0.0f;
        for (int r = 0; r < p.splits; ++r) {
            const float* far = cluster.map_shared_rank(part, r) + j * kBM + quarter * 32 + lane;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < count) v[i] += far[i * kBM];
        }
        emit<H, ACT, FP32>(p.ep, v, b, n0 + j, count, m, live, bias);
    }
}
template <typename H, Mode MODE, typename F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
    if constexpr (MODE == kForward || MODE == kForwardRows) {
        if (act == PG_ACT_GELU) f(std::integral_constant<int, PG_ACT_GELU>{});
        else if (act == PG_ACT_SILU) f(std::integral_constant<int, PG_ACT_SILU>{});
        else if (act == PG_ACT_RELU) f(std::integral_constant<int, PG_ACT_RELU>{});
        else f(std::integral_constant<int, PG_ACT_NONE>{});
    } else {
        f(std::integral_constant<int, PG_ACT_NONE>{});
    }
}

// ------------------------------------------------------------------ 8-bit operand
// Four 8-bit values to two pairs of 16-bit ones times a power of two, exactly: with bit 7 set aside, a
// byte's low bits L under the exponent of 128 (bf16) or 1024 (fp16) read 128 + L, the sign bit alone
// 128 or 256, and their difference is L - 128 sign, the byte's value.
template <typename H>
__device__ __forceinline__ void widen4(uint32_t w, uint32_t scale2, uint32_t& lo, uint32_t& hi) {
    constexpr uint32_t kOne = std::is_same<H, __half>::value ? 0x64006400u : 0x43004300u;
    using H2 = typename std::conditional<std::is_same<H, __half>::value, __half2, __nv_bfloat162>::type;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t t = __byte_perm(w, 0, i ? 0x4342 : 0x4140);
        uint32_t a = (t & 0x007f007fu) | kOne, s = (t & 0x00800080u) | kOne;
        H2 d = __hmul2(__hsub2(*reinterpret_cast<H2*>(&a), *reinterpret_cast<H2*>(&s)), *reinterpret_cast<H2*>(&scale2));
        (i ? hi : lo) = *reinterpret_cast<uint32_t*>(&d);
    }
}
template <typename H>
__device__ __forceinline__ uint32_t scale_pair(uint32_t s) {
    return Elem<H>::down2(both(scale_value(s)));
}

// ------------------------------------------------------------------ the kernel
// Warps: 0 loads, 1 multiplies, 2 owns the tensor memory, 2 and 3 load an 8-bit A and its scales, 4 - 11 (with tokens as lanes 15)
// empty accumulators, 12 - 19 widen it.  Every wait ends: it is for work that has already been started, and a wait that takes
// two seconds makes the whole block give up, see g_training_error.
template <typename H, Mode MODE, bool PAIR>
__global__ void __launch_bounds__(kThreads<MODE>, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out,
               const __grid_constant__ CUtensorMap map_out8, const __grid_constant__ Problem p) {
    extern __shared__ uint8_t s_raw[];
    __shared__ Shared sh;
    constexpr bool kAMn = kAMnMajor<MODE>, kBMn = kBMnMajor<MODE>, kFp32 = kWeightGrads<MODE>, kEight = MODE == kWeightGrad8;
    constexpr int kBlocks = PAIR ? 2 : 1;
    static_assert(!PAIR || !kEight, "see pg_linear_weight_grad");
    uint8_t* ring = s_raw + ((1024 - (smem_u32(s_raw) & 1023)) & 1023);
    const int b_rows = p.BN / kBlocks;                  // of B in this block's shared memory
    const int b_bytes = (kBMn ? (b_rows + 63) / 64 * 64 : b_rows) * kBK * 2;
    const int stage_bytes = kABytes + b_bytes;
    [[maybe_unused]] uint8_t* raw_ring = ring + p.stages * stage_bytes;
    [[maybe_unused]] float* part = reinterpret_cast<float*>(ring + p.part_at);
    [[maybe_unused]] uint32_t* scale_ring = reinterpret_cast<uint32_t*>(raw_ring + p.raw_stages * kRawBytes);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // uniform, and known to be
    const int tmem_cols = p.BN <= 16 ? 32 : p.BN <= 32 ? 64 : p.BN <= 64 ? 128 : p.BN <= 128 ? 256 : 512;
    const int in_pair = PAIR ? blockIdx.x & 1 : 0;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            bar_init(&sh.loaded[s], 1);
            bar_init(&sh.widened[s], 8);
            bar_init(&sh.empty[s], 1);
        }
        for (int s = 0; s < kMaxRaw; ++s) {
            bar_init(&sh.raw[s], 1);
            bar_init(&sh.raw_empty[s], 8);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&sh.scaled[i], 1);
            bar_init(&sh.scales_empty[i], 8);
            bar_init(&sh.summed[i], 1);
            bar_init(&sh.drained[i], kEpilogueWarps<MODE> * kBlocks);
        }
        bar_init(&sh.last, 1);
        sh.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async;" ::: "memory");
    }
    if (warp == 2) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (PAIR) cluster_barrier();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh.tmem;
    volatile int* gave_up = &sh.gave_up;

    // the tiles of a block (or pair): every so many, or with split k the one of its cluster
    const int rank = !PAIR && p.splits > 1 ? blockIdx.x % p.splits : 0;
    const int64_t first = PAIR ? blockIdx.x >> 1 : p.splits > 1 ? blockIdx.x / p.splits : blockIdx.x;
    const int64_t step = PAIR ? gridDim.x >> 1 : p.splits > 1 ? p.tiles : gridDim.x;
    const int kb0 = PAIR ? 0 : p.k_blocks * rank / p.splits, kb1 = PAIR ? p.k_blocks : p.k_blocks * (rank + 1) / p.splits;
    const int64_t per_worker = int64_t{p.m_tiles} * p.n_tiles;
    // worker, this block's first row, the tile's first column
    auto place = [&](int64_t tile, int64_t& b, int& m0, int& n0) {
        b = tile / per_worker;
        const int64_t in = tile - b * per_worker;
        n0 = static_cast<int>(in / p.m_tiles) * p.BN;
        m0 = (static_cast<int>(in % p.m_tiles) * kBlocks + in_pair) * kBM;
    };

    if (warp == 0) {
        int s = 0, turn = 0;
        int64_t issued = 0;
        bool ok = true;
        for (int64_t tile = first; ok && tile < p.tiles; tile += step) {
            int64_t b;
            int m0, n0;
            place(tile, b, m0, n0);
            n0 += in_pair * b_rows;
            const int ba = p.a_shared ? 0 : static_cast<int>(b), bb = p.b_shared ? 0 : static_cast<int>(b);
            for (int kb = kb0; kb < kb1; ++kb) {
                if (turn > 0 && !(ok = bar_wait(&sh.empty[s], (turn - 1) & 1, gave_up))) break;
                if (elected()) {
                    uint8_t* a = ring + s * stage_bytes;
                    uint8_t* bt = a + kABytes;
                    const int k0 = kb * kBK;
                    // the pair's first block is told of the bytes of both
                    if (in_pair == 0) bar_expect(&sh.loaded[s], ((kEight ? 0 : kABytes) + b_bytes) * kBlocks);
                    const uint32_t at = PAIR ? first_of_pair(&sh.loaded[s]) : 0;
                    auto load = [&](void* dst, const CUtensorMap* map, int x, int y, int z) {
                        if constexpr (PAIR) tma_load_pair(dst, map, x, y, z, at);
                        else tma_load(dst, map, x, y, z, &sh.loaded[s]);
                    };
                    if constexpr (kEight) {            // A comes from the widening warps
                    } else if constexpr (kAMn) {
                        load(a, &map_a, m0, k0, ba);
                        load(a + 8192, &map_a, m0 + 64, k0, ba);
                    } else {
                        load(a, &map_a, k0, m0, ba);
                    }
                    if constexpr (kBMn) {
                        for (int j = 0; j < b_rows; j += 64) load(bt + j * 128, &map_b, n0 + j, k0, bb);
                    } else {
                        load(bt, &map_b, k0, n0, bb);
                    }
                }
                __syncwarp();
                ++issued;
                if (++s == p.stages) {
                    s = 0;
                    ++turn;
                }
            }
        }
        // copies still on their way must land before the block ends
        if (!ok && in_pair == 0) await_copies(sh.loaded, p.stages, issued);
        if (!ok && in_pair != 0) pause();                  // a second block's are reported to the first
    } else if (warp == 1 && in_pair == 0) {
        constexpr uint32_t fmt = std::is_same<H, __half>::value ? 0 : 1;
        const uint32_t idesc = 1u << 4 | fmt << 7 | fmt << 10 | (kAMn ? 1u : 0u) << 15 | (kBMn ? 1u : 0u) << 16 |
                               static_cast<uint32_t>(p.BN >> 3) << 17 | static_cast<uint32_t>(kBM * kBlocks >> 4) << 24;
        constexpr int kStepA = (kAMn ? 2048 : 32) >> 4, kStepB = (kBMn ? 2048 : 32) >> 4;     // 16 of k in a descriptor
        const uint64_t ring_a = operand_desc(smem_u32(ring), kAMn), ring_b = operand_desc(smem_u32(ring) + kABytes, kBMn);
        const int last_steps = (p.K - (p.k_blocks - 1) * kBK + 15) / 16;        // of the last block of k; the others have four
        int s = 0, parity = 0, done = 0;
        bool ok = true;
        for (int64_t tile = first; ok && tile < p.tiles; tile += step) {
            int kb = kb0;
            do {                                       // chunks of k; without any k there is one of none
                const uint32_t d = tmem + (done & 1) * p.BN;
                const int from = kb, to = min(kb1, kb + p.chunk);
                if (done >= 2 && !(ok = bar_wait(&sh.drained[done & 1], (done / 2 - 1) & 1, gave_up))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (; kb < to; ++kb) {
                    if (!(ok = bar_wait(&sh.loaded[s], parity, gave_up))) break;
                    if (kEight && !(ok = bar_wait(&sh.widened[s], parity, gave_up))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t a = ring_a + (s * stage_bytes >> 4), bd = ring_b + (s * stage_bytes >> 4);
                    if (elected()) {
                        mma_f16<PAIR>(d, a, bd, idesc, kb > from);
                        if (kb + 1 < p.k_blocks) {
#pragma unroll
                            for (int k = 1; k < 4; ++k) mma_f16<PAIR>(d, a + k * kStepA, bd + k * kStepB, idesc, 1);
                        } else {
                            for (int k = 1; k < last_steps; ++k) mma_f16<PAIR>(d, a + k * kStepA, bd + k * kStepB, idesc, 1);
                        }
                        mma_commit<PAIR>(&sh.empty[s]);
                        if (kb + 1 == to) mma_commit<PAIR>(&sh.summed[done & 1]);
                    }
                    __syncwarp();
                    if (++s == p.stages) {
                        s = 0;
                        parity ^= 1;
                    }
                }
                if (!ok) break;
                if (from == to && elected()) mma_commit<PAIR>(&sh.summed[done & 1]);
                __syncwarp();
                ++done;
            } while (kb < kb1);
        }
        if (!ok) {
            if (elected()) mma_commit<PAIR>(&sh.last);
            for (int t = 0; t < 100000 && !bar_try(&sh.last, 0); ++t) {}
        }
    } else if (warp >= 4 && warp < 4 + kEpilogueWarps<MODE>) {
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t drained[2] = {PAIR ? first_of_pair(&sh.drained[0]) : 0u, PAIR ? first_of_pair(&sh.drained[1]) : 0u};
        // the body for every combination that the epilogue is compiled for
        with_activation<H, MODE>(p.ep.activation, [&](auto act) {
            [[maybe_unused]] uint8_t* out = ring + p.stages * stage_bytes + (warp - 4) * p.out_warp;
            int done = 0, kb = kb0;
            for (int64_t tile = first; tile < p.tiles; ++done) {
                const int acc = done & 1;
                [[maybe_unused]] const bool more = kb > kb0;            // what comes is added to an earlier chunk
                int64_t b;
                int m0, n0;
                place(tile, b, m0, n0);
                [[maybe_unused]] Residuals residuals;
                if constexpr (kTokenRows<MODE>) {
                    const int j = half * 32;
                    if (p.ep.residual.data) residuals.start(p.ep, b, m0 + quarter * 32, p.M, n0, lane);
                    if (p.ep.residual.data && j < min(p.BN, p.N - n0)) residuals.fetch(p.ep, out + kOutBytes, j, p.N - n0 - j, lane);
                    // the biases of its groups; not one by one in the groups, whose fences would wait for the load
                    float bias[(8 + kShares - 1) / kShares];
#pragma unroll
                    for (int g = 0; g < (8 + kShares - 1) / kShares; ++g) {
                        const int n = n0 + j + g * kShares * 32 + lane;
                        bias[g] = p.ep.bias && n < p.N ? PGT_LOAD(p.ep.bias[b * p.ep.bias_stride + n]) : 0.0f;
                    }
                    __syncwarp();
#pragma unroll
                    for (int g = 0; g < (8 + kShares - 1) / kShares; ++g) reinterpret_cast<float*>(out + kOutBytes + kHeldBytes)[g * 32 + lane] = bias[g];
                    __syncwarp();
                }
                if (!bar_wait(&sh.summed[acc], (done / 2) & 1, gave_up)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                __syncwarp();
                if constexpr (kTokenRows<MODE>)
                    empty_rows<H, decltype(act)::value>(p, &map_out, &map_out8, tmem + acc * p.BN, out, b, m0, n0, half, quarter, lane, residuals);
                else
                    empty_tile<H, decltype(act)::value, kFp32>(p, tmem + acc * p.BN, !PAIR && p.splits > 1 ? part : nullptr, more, b, m0, n0, half, quarter,
                                                               lane);
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) bar_arrive_read_at(drained[acc]);
                    else bar_arrive_read(&sh.drained[acc]);
                }
                kb += p.chunk;
                if (kb >= kb1) {
                    kb = kb0;
                    tile += step;
                }
            }
        });
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (kTokenRows<MODE> && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (kEight && warp == 2) {
        int q = 0, turn = 0;
        int64_t issued = 0;
        bool ok = true;
        for (int64_t tile = first; ok && tile < p.tiles; tile += step) {
            int64_t b;
            int m0, n0;
            place(tile, b, m0, n0);
            for (int kb = kb0; kb < kb1; ++kb) {
                if (turn > 0 && !(ok = bar_wait(&sh.raw_empty[q], (turn - 1) & 1, gave_up))) break;
                if (elected()) {
                    bar_expect(&sh.raw[q], kRawBytes);
                    tma_load(raw_ring + q * kRawBytes, &map_a, m0, kb * kBK, p.a_shared ? 0 : static_cast<int>(b), &sh.raw[q]);
                }
                __syncwarp();
                ++issued;
                if (++q == p.raw_stages) {
                    q = 0;
                    ++turn;
                }
            }
        }
        if (!ok) await_copies(sh.raw, p.raw_stages, issued);
    } else if (kEight && warp == 3) {
        // The scales of an 8-bit A, for eight stages at a time, so that no load is outstanding when they are handed over:
        // an arrival on a barrier (and a fence) waits for the thread's earlier loads, and one per stage would wait for memory.
        int half = 0, turn = 0;
        bool ok = true;
        for (int64_t tile = first; ok && tile < p.tiles; tile += step) {
            int64_t b;
            int m0, n0;
            place(tile, b, m0, n0);
            const uint8_t* at = p.scales + b * p.scale_stride + m0 / kBlock8;
            const int count = scales_of_tile(p.M, m0);
            for (int kb = kb0; kb < kb1; kb += kScaleStages) {
                if (turn > 0 && !(ok = bar_wait(&sh.scales_empty[half], (turn - 1) & 1, gave_up))) break;
                const int64_t k0 = static_cast<int64_t>(kb) * kBK, k1 = min(static_cast<int64_t>(p.K), k0 + kScaleStages * kBK);
                uint32_t* to = scale_ring + half * kScaleStages * kBK;
                // a row's four bytes, cut out of the one or two words that hold them (no others are read); all rows' on their way together
                constexpr int kRows = kScaleStages * kBK / 32;
                uint32_t lo[kRows], hi[kRows];
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    const int64_t k = k0 + lane + 32 * u;
                    const uintptr_t from = reinterpret_cast<uintptr_t>(at + k * p.scale_ld);
                    const uint32_t* word = reinterpret_cast<const uint32_t*>(from & ~uintptr_t{3});
                    const int words = k < k1 ? words_of_scales(from, count) : 0;
                    lo[u] = hi[u] = 0;
                    if (words > 0) lo[u] = PGT_LOAD(word[0]);
                    if (words > 1) hi[u] = PGT_LOAD(word[1]);
                }
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    const uint32_t shift = (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(at)) + static_cast<uint32_t>(k0 + lane + 32 * u) * static_cast<uint32_t>(p.scale_ld) & 3) * 8;
                    to[lane + 32 * u] = __funnelshift_r(lo[u], hi[u], shift);
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.scaled[half]);
                half ^= 1;
                if (half == 0) ++turn;
            }
        }
    } else if (kEight && warp >= 12) {
        // Eight lanes take the 128 values of a row (one k) of the stage, 16 each, and a thread two rows.
        const int c = lane & 7, r0 = (warp - 12) * 4 + (lane >> 3);    // rows r0 and r0 + 32
        const int64_t left = kb1 > kb0 && p.tiles > first ? (p.tiles - first + step - 1) / step * (kb1 - kb0) : 0;
        int s = 0, turn = 0, q = 0, raw_parity = 0, kb = kb0, half = 0, scale_parity = 0;
        for (int64_t i = 0; i < left; ++i) {
            const int in_chunk = (kb - kb0) & (kScaleStages - 1);
            if (in_chunk == 0 && !bar_wait(&sh.scaled[half], scale_parity, gave_up)) break;
            if (!bar_wait(&sh.raw[q], raw_parity, gave_up)) break;
            const uint8_t* raw = raw_ring + q * kRawBytes;
            const uint8_t* scales = reinterpret_cast<const uint8_t*>(scale_ring + (half * kScaleStages + in_chunk) * kBK);
            uint4 v[2];
            uint32_t f[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                v[j] = *reinterpret_cast<const uint4*>(raw + (r0 + 32 * j) * 128 + c * 16);
                f[j] = scales[(r0 + 32 * j) * 4 + (c >> 1)];
            }
            uint4 o[2][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f[j] = scale_pair<H>(f[j]);
                widen4<H>(v[j].x, f[j], o[j][0].x, o[j][0].y);
                widen4<H>(v[j].y, f[j], o[j][0].z, o[j][0].w);
                widen4<H>(v[j].z, f[j], o[j][1].x, o[j][1].y);
                widen4<H>(v[j].w, f[j], o[j][1].z, o[j][1].w);
            }
            __syncwarp();
            const bool chunk_done = in_chunk == kScaleStages - 1 || kb + 1 == kb1;
            if (lane == 0) {
                bar_arrive(&sh.raw_empty[q]);
                if (chunk_done) bar_arrive(&sh.scales_empty[half]);
            }
            if (++q == p.raw_stages) {
                q = 0;
                raw_parity ^= 1;
            }
            if (chunk_done) {
                half ^= 1;
                if (half == 0) scale_parity ^= 1;
            }
            if (++kb == kb1) kb = kb0;
            if (turn > 0 && !bar_wait(&sh.empty[s], (turn - 1) & 1, gave_up)) break;
            uint8_t* a = ring + s * stage_bytes + (c >> 2) * 8192;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = r0 + 32 * j;
                // the lanes of the upper 64 values take their two pieces the other way round: eight lanes, eight banks
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int w = e ^ (c >> 2);
                    *reinterpret_cast<uint4*>(a + r * 128 + (((2 * (c & 3) + w) ^ (r & 7)) << 4)) = w ? o[j][1] : o[j][0];
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.widened[s]);
            if (++s == p.stages) {
                s = 0;
                ++turn;
            }
        }
    }

    __syncwarp();
    if (!PAIR && !kTokenRows<MODE> && p.splits > 1) {
        cluster_barrier();
        if (warp >= 4 && warp < 12 && !*gave_up) {
            int64_t b;
            int m0, n0;
            place(first, b, m0, n0);
            with_activation<H, MODE>(p.ep.activation, [&](auto act) {
                join_parts<H, decltype(act)::value, kFp32>(p, part, b, m0, n0, rank, (warp - 4) >> 2, warp & 3, lane);
            });
        }
        __syncwarp();
        cluster_barrier();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (PAIR) cluster_barrier();             // neither block goes while the other's copies, products or arrivals may reach it
    if (warp == 2) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));
    }
}

// ------------------------------------------------------------------ few tokens
// y for one to four tokens: the weights are read once, which is all the time there is, so they go from memory to registers
// and are multiplied as fp32 pairs.  A block computes 32 features (one block of the 8-bit form), a warp four of them at a time
// over all of k; which lane has which k does not matter to a sum, so a lane takes as many neighbours (8, 2 or 1) as the
// rows' alignment lets it read at once.  The tokens wait in shared memory as they are stored.
constexpr int kFewTokens = 4, kFewBytes = 40 * 1024;
// W neighbouring elements as pairs; the second of a pair may lie past the row's end (`valid` elements are inside).
template <typename H, int W> struct Few {
    static constexpr int kPairs = W == 1 ? 1 : W / 2, kUnroll = W == 8 ? 2 : 6;
    uint32_t w[kPairs];
    template <bool SHARED> __device__ __forceinline__ void load(const uint16_t* row, int e, int valid) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) w[i] = 0;
        if (valid <= 0 || !(SHARED || PGT_READ(row + e, 2 * W))) return;
        if constexpr (W == 8) {
            const uint4 u = *reinterpret_cast<const uint4*>(row + e);
            w[0] = u.x;
            w[1] = u.y;
            w[2] = u.z;
            w[3] = u.w;
        } else if constexpr (W == 2) {
            w[0] = *reinterpret_cast<const uint32_t*>(row + e);
        } else {
            w[0] = row[e];
        }
    }
    __device__ __forceinline__ void mask(int valid) {
        if (W > 1 && valid < W) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) w[i] = 2 * i + 1 < valid ? w[i] : 2 * i < valid ? w[i] & 0xffffu : 0u;
        }
    }
};
template <typename H, int W, int T, int ACT>
__global__ void __launch_bounds__(256)
few_tokens_kernel(const pg_linear_args a) {
    extern __shared__ uint4 s_x[];                     // T rows of octets
    __shared__ float s_z[T][32];
    using F = Few<H, W>;
    const int64_t b = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int K = a.in_features, octets = (K + 7) / 8;
    for (int i = threadIdx.x; i < T * octets; i += 256) {
        const int t = i / octets, col = (i - t * octets) * 8;
        const uint16_t* x = static_cast<const uint16_t*>(a.x.data) + b * a.x.stride + t * a.x.ld;
        const Oct o = octet<1>(load_oct<1>(x, col, K), x, col, K);
        s_x[i] = make_uint4(o.w[0], o.w[1], o.w[2], o.w[3]);
    }
    const uint16_t* x16 = reinterpret_cast<const uint16_t*>(s_x);
    const int n0 = blockIdx.x * 32 + warp * 4;
    const uint16_t* row[4];
#pragma unroll
    for (int r = 0; r < 4; ++r)                        // a feature past the last one is computed again and not used
        row[r] = static_cast<const uint16_t*>(a.weight.data) + b * a.weight.stride + min(n0 + r, a.out_features - 1) * a.weight.ld;
    F2 acc[4][T];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[r][t] = both(0.0f);
    bool first = true;
    for (int k = 0; k < K; k += 32 * W * F::kUnroll) {
        F w[F::kUnroll][4];
#pragma unroll
        for (int u = 0; u < F::kUnroll; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int e = k + (u * 32 + lane) * W;
                w[u][r].template load<false>(row[r], e, K - e);
            }
        if (first) __syncthreads();                    // the tokens; the first weights are on their way meanwhile
        first = false;
#pragma unroll
        for (int u = 0; u < F::kUnroll; ++u) {
            const int e = k + (u * 32 + lane) * W;
            if (e >= K) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) w[u][r].mask(K - e);
#pragma unroll
            for (int t = 0; t < T; ++t) {
                F x;
                x.template load<true>(x16 + t * octets * 8, e, W);
#pragma unroll
                for (int i = 0; i < F::kPairs; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[r][t] = fma(Elem<H>::up2(w[u][r].w[i]), Elem<H>::up2(x.w[i]), acc[r][t]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) {
            float v = sum2(acc[r][t]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == 0) s_z[t][warp * 4 + r] = v;
        }
    __syncthreads();
    if (warp < T) {
        const Epilogue ep{0, ACT, a.y, a.residual, a.bias, a.bias_stride, a.z8};
        const int m = blockIdx.x * 32 + lane;
        const bool live = m < a.out_features;
        float v[16] = {s_z[warp][lane]};
        emit<H, ACT, false>(ep, v, b, warp, 1, m, live, a.bias && live ? PGT_LOAD(a.bias[b * a.bias_stride + m]) : 0.0f);
    }
}
template <typename H, int W, int T>
int few_tokens(const pg_linear_args& a, cudaStream_t st) {
    const dim3 grid((a.out_features + 31) / 32, a.batch);
    const size_t smem = static_cast<size_t>(T) * ((a.in_features + 7) / 8) * 16;
    if (a.activation == PG_ACT_GELU) few_tokens_kernel<H, W, T, PG_ACT_GELU><<<grid, 256, smem, st>>>(a);
    else if (a.activation == PG_ACT_SILU) few_tokens_kernel<H, W, T, PG_ACT_SILU><<<grid, 256, smem, st>>>(a);
    else if (a.activation == PG_ACT_RELU) few_tokens_kernel<H, W, T, PG_ACT_RELU><<<grid, 256, smem, st>>>(a);
    else few_tokens_kernel<H, W, T, PG_ACT_NONE><<<grid, 256, smem, st>>>(a);
    return launch_status();
}
template <typename H>
int few_tokens(const pg_linear_args& a, cudaStream_t st) {
    const uint64_t bits = reinterpret_cast<uintptr_t>(a.weight.data) | static_cast<uint64_t>(a.weight.ld) * 2 |
                          (a.batch > 1 ? static_cast<uint64_t>(a.weight.stride) * 2 : 0);
    auto with = [&](auto tokens) {
        constexpr int T = decltype(tokens)::value;
        return bits % 16 == 0 ? few_tokens<H, 8, T>(a, st) : bits % 4 == 0 ? few_tokens<H, 2, T>(a, st) : few_tokens<H, 1, T>(a, st);
    };
    switch (a.tokens) {
        case 1: return with(std::integral_constant<int, 1>{});
        case 2: return with(std::integral_constant<int, 2>{});
        case 3: return with(std::integral_constant<int, 3>{});
        default: return with(std::integral_constant<int, 4>{});
    }
}
// Rows of 16-bit elements copied to rows that start on 16-byte boundaries, for operands TMA cannot read
// where they are: 8 elements a thread.
__global__ void __launch_bounds__(256)
align_rows_kernel(const uint16_t* __restrict__ src, int64_t src_ld, int64_t src_stride, uint16_t* __restrict__ dst, int64_t dst_ld, int rows, int cols,
                  int64_t total) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (at >= total) return;
    const int chunks = static_cast<int>(dst_ld / 8);
    const int64_t row = at / chunks;
    const int col = static_cast<int>(at - row * chunks) * 8;
    const int64_t b = row / rows, r = row - b * rows;
    const uint16_t* p = src + b * src_stride + r * src_ld;
    const Oct o = octet<1>(load_oct<1>(p, col, cols), p, col, cols);
    PGT_STORE(*reinterpret_cast<uint4*>(dst + row * dst_ld + col), make_uint4(o.w[0], o.w[1], o.w[2], o.w[3]));
}

// The products' wait on a barrier that nothing arrives on, by a whole block and with a limit of a millisecond.
__global__ void __launch_bounds__(64) wait_probe_kernel() {
    __shared__ uint64_t bar;
    __shared__ int gave_up;
    if (threadIdx.x == 0) {
        bar_init(&bar, 1);
        gave_up = 0;
    }
    __syncthreads();
    bar_wait(&bar, 0, &gave_up, 1000000);
}

// Asks the bounds check about a word that is an operand, then about the one behind it; touches neither.
__global__ void bounds_probe_kernel(const char* word) {
    if (!PGT_READ(word, 4) || !PGT_WRITE(word, 4)) atomicOr(&g_training_error, kTimedOut);     // must not happen
    if (PGT_READ(word + 4, 4) && kChecked) atomicOr(&g_training_error, kTimedOut);
}

// ------------------------------------------------------------------ host
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
    static EncodeFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

// A matrix as TMA sees it: `rows` rows of `cols` elements per worker, boxes of box_rows x box_bytes, swizzled over them (8-bit:
// not).
bool make_map(CUtensorMap& map, int dtype, bool eight, const pg_matrix& m, int64_t batch, int64_t rows, int64_t cols, int box_bytes, int box_rows) {
    EncodeFn fn = encoder();
    if (!fn) return false;
    const int64_t size = eight ? 1 : 2, unit = 16 / size;
    const bool shared = batch > 1 && m.stride == 0;
    const int64_t ld = rows > 1 ? m.ld : (cols + unit - 1) / unit * unit;
    const int64_t stride = batch > 1 && !shared ? m.stride : ld * rows;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(shared ? 1 : batch)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld * size), static_cast<cuuint64_t>(stride * size)};
    const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_bytes / size), static_cast<cuuint32_t>(box_rows), 1};
    const cuuint32_t one[3] = {1, 1, 1};
    const CUtensorMapDataType type = eight ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : dtype == PG_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return fn(&map, type, 3, m.data, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              eight ? CU_TENSOR_MAP_SWIZZLE_NONE : box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Can TMA read the operand where it is?
bool aligned(const pg_matrix& m, int64_t batch, int64_t rows) {
    return reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (rows <= 1 || m.ld % 8 == 0) && (batch <= 1 || m.stride % 8 == 0);
}
// Up to four tokens where the product would have to copy the weights' rows first (32 workers x 2600 x 650: 27, 33, 44 and 47 us
// for 1 to 4 tokens, 75 us by copy and product); one where it would not (2600 x 656: 24 us, and 35 for two; the product
// takes 25 for up to 16).
bool few(const pg_linear_args& a) {
    return a.tokens <= (aligned(a.weight, a.batch, a.out_features) ? 1 : kFewTokens) && static_cast<int64_t>(a.tokens) * ((a.in_features + 7) / 8) * 16 <= kFewBytes;
}

size_t copy_bytes(const pg_matrix& m, int64_t batch, int64_t rows, int64_t cols) {
    if (batch == 0 || rows == 0 || aligned(m, batch, rows)) return 0;
    const int64_t workers = m.stride == 0 ? 1 : batch;
    return static_cast<size_t>((workers * rows * ((cols + 7) / 8 * 8) * 2 + 255) / 256 * 256);
}
// The operand, or its copy with aligned rows in the workspace.
int aligned_operand(pg_matrix& m, int64_t batch, int64_t rows, int64_t cols, uint8_t*& workspace, cudaStream_t st) {
    const size_t bytes = copy_bytes(m, batch, rows, cols);
    if (bytes == 0) return PG_OK;
    const int64_t workers = m.stride == 0 ? 1 : batch;
    const int64_t ld = (cols + 7) / 8 * 8, total = workers * rows * (ld / 8);
    if ((total + 255) / 256 > 0x7fffffff) return PG_ERR_TOO_LARGE;
    align_rows_kernel<<<static_cast<unsigned>((total + 255) / 256), 256, 0, st>>>(static_cast<const uint16_t*>(m.data), m.ld, m.stride,
                                                                                  reinterpret_cast<uint16_t*>(workspace), ld, static_cast<int>(rows),
                                                                                  static_cast<int>(cols), total);
    m.data = workspace;
    m.ld = ld;
    m.stride = m.stride == 0 ? 0 : rows * ld;
    workspace += bytes;
    return launch_status();
}

template <typename H, Mode MODE, bool PAIR>
int launch(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, const CUtensorMap& out8, const Problem& p, int smem, cudaStream_t st) {
    static std::once_flag once[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= 64) return PG_ERR_CUDA;
    bool fine = true;
    std::call_once(once[dev], [&] {
        fine = cudaFuncSetAttribute(product_kernel<H, MODE, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes - kStaticBytes) == cudaSuccess;
    });
    if (!fine) return PG_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(PAIR ? 2 * std::min<int64_t>(p.tiles, kSMs / 2) : p.splits > 1 ? p.tiles * p.splits : std::min<int64_t>(p.tiles, kSMs)));
    cfg.blockDim = dim3(kThreads<MODE>);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = PAIR ? 2 : p.splits;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, product_kernel<H, MODE, PAIR>, a, b, out, out8, p) != cudaSuccess) {
        cudaGetLastError();
        return PG_ERR_CUDA;
    }
    return PG_OK;
}

template <Mode MODE, bool PAIR>
int run_product(int dtype, int64_t batch, int64_t M, int64_t N, int64_t K, const pg_matrix& A, const pg_matrix& B, const Epilogue& ep, const pg_matrix8* a8,
                cudaStream_t st) {
    constexpr bool kBMn = kBMnMajor<MODE>, kAMn = kAMnMajor<MODE>, kRows = kTokenRows<MODE>;
    constexpr int kBlocks = PAIR ? 2 : 1;
    Problem p = {};
    p.ep = ep;
    p.M = static_cast<int>(M);
    p.N = static_cast<int>(N);
    p.K = static_cast<int>(K);
    p.m_tiles = static_cast<int>((M + kBM * kBlocks - 1) / (kBM * kBlocks));
    // Widths of a tile: multiples of 16 columns, of 32 where a thread holds blocks of 32, of 64 where TMA loads boxes of
    // 64 columns and every other one is stored.  The one that covers N with the fewest columns, a tile's start and
    // end counted as 64 more; the widest of equals.
    const int unit = kWeightGrads<MODE> ? 64 : kRows ? 32 : 16;
    const int most = max_chunk(MODE == kWeightGrad8, dtype);
    p.k_blocks = static_cast<int>((K + kBK - 1) / kBK);
    auto cover = [&](int widest) {
        int64_t least = 0;
        for (int w = widest; w >= unit && w >= std::min<int64_t>(N, kRows || kWeightGrads<MODE> ? 128 : 16); w -= unit) {
            const int64_t tiles = (N + w - 1) / w, cost = tiles * (w + 64);
            if (least == 0 || cost < least) {
                least = cost;
                p.BN = w;
            }
        }
        p.n_tiles = static_cast<int>((N + p.BN - 1) / p.BN);
        p.tiles = int64_t{p.m_tiles} * p.n_tiles * batch;
        p.splits = 1;
        if (!PAIR)
            // (eight blocks of a cluster have to find room in one GPC: 16 tiles in clusters of eight ran one after the other, 33 us
            // where 24 in clusters of four take 16.5)
            while (p.splits < kMaxSplits && p.tiles * p.splits * 2 <= (p.splits == 4 ? kSMs / 2 : kSMs) && p.k_blocks >= p.splits * 2) p.splits *= 2;
    };
    cover(256);
    // A block's part of a split k that is itself a sum of chunks has to have a place beside the ring: 128 columns at most.  Where the
    // tiles are so few and k is long, narrow ones also share it among more blocks (1536 tokens, 512 x 512: 12.4 us, wide 18.5).
    if (kWeightGrads<MODE> && p.splits > 1 && p.k_blocks > most) cover(128);
    const int b_rows = p.BN / kBlocks;
    const int stage = kABytes + (kBMn ? (b_rows + 63) / 64 * 64 : b_rows) * kBK * 2;
    // The other products sum all of k in tensor memory: their results are rounded to 16 bits, beside which what is cut off is
    // little.  It is most for fp16 products of one sign, 5.6e-9 of the sum for each k: 2.6e-5 at 4608, where half a step of
    // fp16 is 4.9e-4 at most and 2.4e-4 at least (bf16, both signs, 2600: 4e-6 of half a step's 2e-3).
    const int per_split = std::max(1, (p.k_blocks + p.splits - 1) / p.splits), parts = kWeightGrads<MODE> ? (per_split + most - 1) / most : 1;
    p.chunk = (per_split + parts - 1) / parts;
    const int part_bytes = p.splits > 1 && parts > 1 ? kBM * p.BN * 4 : 0;
    p.out_warp = kOutWarp + (ep.z8.values ? kOut8Bytes : 0);
    const int rest = kRows ? kRowWarps * p.out_warp : MODE == kWeightGrad8 ? kMinRaw * kRawBytes + kScaleBytes : 0;
    p.stages = std::min(kMaxStages, (kRingBytes - rest - part_bytes) / stage);
    p.raw_stages = MODE == kWeightGrad8 ? std::min(kMaxRaw, (kRingBytes - kScaleBytes - part_bytes - p.stages * stage) / kRawBytes) : 0;
    p.a_shared = A.stride == 0;
    p.b_shared = B.stride == 0;
    p.residual_aligned = access_width({&ep.residual}, batch) == 8;
    if (a8) {
        p.scales = a8->scales;
        p.scale_ld = a8->scale_ld;
        p.scale_stride = a8->scale_stride;
    }
    CUtensorMap map_a = {}, map_b = {}, map_out = {}, map_out8 = {};
    if (K > 0) {
        const bool fine = make_map(map_a, dtype, MODE == kWeightGrad8, A, batch, kAMn ? K : M, kAMn ? M : K, 128, kAMn ? kBK : kBM) &&
                          make_map(map_b, dtype, false, B, batch, kBMn ? K : N, kBMn ? N : K, 128, kBMn ? kBK : b_rows) &&
                          (!kRows || make_map(map_out, dtype, false, ep.out, batch, M, N, 64, 32)) &&
                          (!kRows || !ep.z8.values || make_map(map_out8, dtype, true, pg_matrix{ep.z8.values, ep.z8.ld, ep.z8.stride}, batch, M, N, 32, 32));
        if (!fine) return PG_ERR_CUDA;
    }
    const int ring = p.stages * stage + (MODE == kWeightGrad8 ? p.raw_stages * kRawBytes + kScaleBytes : rest);
    p.part_at = part_bytes > 0 ? ring : 0;             // a sum of one chunk is only there when the ring is done with
    const int smem = ring + part_bytes + 1024;
    return dtype == PG_BF16 ? launch<__nv_bfloat16, MODE, PAIR>(map_a, map_b, map_out, map_out8, p, smem, st)
                            : launch<__half, MODE, PAIR>(map_a, map_b, map_out, map_out8, p, smem, st);
}

constexpr int64_t kMaxResidualLd = 1 << 25;       // 32 rows of residuals are addressed with 32 bits

// Pairs of blocks multiply 256-row tiles; one row more than a block's 128 has to be there, and tiles for a share of the GPU:
// with fewer, single blocks that share the k of a tile finish earlier.  A quarter of the SMs where lanes are tokens, half for the
// weight gradient.  Pairs / single blocks in us, by 128-row blocks of tiles in pairs (37 and 74 are the limits):
//   layer, 256 tokens, 1024 to 1024      8: 12.4 / 18.6   32: 12.4 / 16.5   64: 12.4 / 16.5   96: 12.5 / 12.5  192: 18.6 / 20.0
//   layer, 1024 tokens, 256 to 256      16:  8.4 / 14.5   48:  8.4 / 14.4   96:  8.6 /  9.2  192: 10.4 / 12.5
//   layer, 200 tokens, 2048 to 640      12: 15.5 / 14.5   24: 15.6 / 14.9   48: 16.4 / 16.6   96: 16.5 / 16.5
//   input gradient, 320, 2600 to 656    12: 20.6 / 16.5   24: 20.7 / 16.5   36: 20.6 / 28.9   48: 20.7 / 18.6
//   weight gradient, 256, 1024 x 1024   32:  9.8 / 14.5   64: 10.2 / 13.3   96: 10.4 /  8.6  192: 12.5 / 12.4  768: 30.8 / 30.0
//   weight gradient, 2000, 1024 x 328   16: 20.6 / 12.4   64: 21.7 / 18.6   96: 21.9 / 18.5  128: 22.5 / 30.9
//   weight gradient, 512, 512 x 512     16: 10.4 / 14.4   64: 10.4 / 14.4   96: 10.4 / 10.4  192: 14.5 / 15.0
// Long k and few tiles are for single blocks, short k for pairs at once; the limits are where pairs lose little at either.
bool enough_for_pairs(int64_t batch, int64_t M, int64_t N, int sms) {
    return M > kBM && batch * ((M + 2 * kBM - 1) / (2 * kBM)) * ((N + 255) / 256) * 2 >= sms;
}

int current_device() {
    int d = 0;
    return cudaGetDevice(&d) == cudaSuccess ? d : -1;
}
bool workspace_ok(size_t need, const void* workspace, size_t bytes, int dev) {
    return need == 0 || (bytes >= need && device_pointer(workspace, 16, dev));
}

}  // namespace
}  // namespace pgt

using namespace pgt;

extern "C" {

int pg_linear_workspace_bytes(const pg_linear_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->in_features, args->out_features)) return PG_ERR_INVALID;
    *bytes_out = few(*args) ? 0
                            : copy_bytes(args->x, args->batch, args->tokens, args->in_features) +
                                  copy_bytes(args->weight, args->batch, args->out_features, args->in_features);
    return PG_OK;
}
int pg_linear(const pg_linear_args* args, void* workspace, size_t workspace_bytes, void* stream) {
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
    size_t need = 0;
    pg_linear_workspace_bytes(args, &need);
    if (!workspace_ok(need, workspace, workspace_bytes, dev)) return PG_ERR_WORKSPACE;
    if (a.batch == 0 || a.tokens == 0) return PG_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Operands operands;
    operands.output(a.y, a.batch, a.tokens, a.out_features, 2).output(a.z8, a.batch, a.tokens, a.out_features).output(need > 0 ? workspace : nullptr, 0, 1, need / 4);
    operands.input(a.x, a.batch, a.tokens, a.in_features, 2).input(a.weight, a.batch, a.out_features, a.in_features, 2);
    operands.input(a.bias, a.bias_stride, a.batch, a.out_features).input(a.residual, a.batch, a.tokens, a.out_features, 2);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    if (few(a)) return a.dtype == PG_BF16 ? few_tokens<__nv_bfloat16>(a, st) : few_tokens<__half>(a, st);
    uint8_t* at = static_cast<uint8_t*>(workspace);
    pg_matrix x = a.x, w = a.weight;
    int rc = aligned_operand(x, a.batch, a.tokens, a.in_features, at, st);
    if (rc == PG_OK) rc = aligned_operand(w, a.batch, a.out_features, a.in_features, at, st);
    const Epilogue ep{0, a.activation, a.y, a.residual, a.bias, a.bias_stride, a.z8};
    if (rc != PG_OK) return rc;
    if (enough_for_pairs(a.batch, a.tokens, a.out_features, kSMs / 4) && aligned(a.y, a.batch, a.tokens) && a.residual.ld < kMaxResidualLd)
        return run_product<kForwardRows, true>(a.dtype, a.batch, a.tokens, a.out_features, a.in_features, x, w, ep, nullptr, st);
    return run_product<kForward, false>(a.dtype, a.batch, a.out_features, a.tokens, a.in_features, w, x, ep, nullptr, st);
}

int pg_linear_input_grad_workspace_bytes(const pg_input_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->in_features, args->out_features)) return PG_ERR_INVALID;
    *bytes_out = copy_bytes(args->dz, args->batch, args->tokens, args->out_features) +
                 copy_bytes(args->weight, args->batch, args->tokens ? args->out_features : 0, args->in_features);
    return PG_OK;
}
int pg_linear_input_grad(const pg_input_grad_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_input_grad_args& a = *args;
    const int dev = current_device();
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.in_features, a.out_features)) return PG_ERR_INVALID;
    if (!matrix_ok(a.dz, a.batch, a.tokens, a.out_features, 2, false, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.weight, a.batch, a.out_features, a.in_features, 2, false, dev)) return PG_ERR_INVALID;
    if (a.residual.data && !matrix_ok(a.residual, a.batch, a.tokens, a.in_features, 2, false, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.dx, a.batch, a.tokens, a.in_features, 2, true, dev)) return PG_ERR_INVALID;
    size_t need = 0;
    pg_linear_input_grad_workspace_bytes(args, &need);
    if (!workspace_ok(need, workspace, workspace_bytes, dev)) return PG_ERR_WORKSPACE;
    if (a.batch == 0 || a.tokens == 0) return PG_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Operands operands;
    operands.output(a.dx, a.batch, a.tokens, a.in_features, 2).output(need > 0 ? workspace : nullptr, 0, 1, need / 4);
    operands.input(a.dz, a.batch, a.tokens, a.out_features, 2).input(a.weight, a.batch, a.out_features, a.in_features, 2);
    operands.input(a.residual, a.batch, a.tokens, a.in_features, 2);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    uint8_t* at = static_cast<uint8_t*>(workspace);
    pg_matrix dz = a.dz, w = a.weight;
    int rc = aligned_operand(dz, a.batch, a.tokens, a.out_features, at, st);
    if (rc == PG_OK) rc = aligned_operand(w, a.batch, a.out_features, a.in_features, at, st);
    const Epilogue ep{0, PG_ACT_NONE, a.dx, a.residual, nullptr, 0, {}};
    if (rc != PG_OK) return rc;
    if (enough_for_pairs(a.batch, a.tokens, a.in_features, kSMs / 4) && aligned(a.dx, a.batch, a.tokens) && a.residual.ld < kMaxResidualLd)
        return run_product<kInputGradRows, true>(a.dtype, a.batch, a.tokens, a.in_features, a.out_features, dz, w, ep, nullptr, st);
    return run_product<kInputGrad, false>(a.dtype, a.batch, a.in_features, a.tokens, a.out_features, w, dz, ep, nullptr, st);
}

int pg_linear_weight_grad_workspace_bytes(const pg_weight_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out || !sizes_ok(args->dtype, args->batch, args->tokens, args->in_features, args->out_features)) return PG_ERR_INVALID;
    *bytes_out = copy_bytes(args->dz, args->batch, args->tokens, args->out_features) +
                 (args->x8.values ? 0 : copy_bytes(args->x, args->batch, args->tokens, args->in_features));
    return PG_OK;
}
int pg_linear_weight_grad(const pg_weight_grad_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_weight_grad_args& a = *args;
    const int dev = current_device();
    const bool eight = a.x8.values != nullptr;
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.in_features, a.out_features)) return PG_ERR_INVALID;
    const bool any = int64_t{a.batch} * a.tokens > 0;              // without tokens there is no x to be had
    if (any && eight == (a.x.data != nullptr)) return PG_ERR_INVALID;
    if (!matrix_ok(a.dz, a.batch, a.tokens, a.out_features, 2, false, dev)) return PG_ERR_INVALID;
    if (any && (eight ? !matrix8_ok(a.x8, a.batch, a.tokens, a.in_features, false, dev)
                      : !matrix_ok(a.x, a.batch, a.tokens, a.in_features, 2, false, dev)))
        return PG_ERR_INVALID;
    if (!matrix_ok(a.dweight, a.batch, a.out_features, a.in_features, 4, true, dev)) return PG_ERR_INVALID;
    size_t need = 0;
    pg_linear_weight_grad_workspace_bytes(args, &need);
    if (!workspace_ok(need, workspace, workspace_bytes, dev)) return PG_ERR_WORKSPACE;
    if (a.batch == 0) return PG_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Operands operands;
    operands.output(a.dweight, a.batch, a.out_features, a.in_features, 4).output(need > 0 ? workspace : nullptr, 0, 1, need / 4);
    operands.input(a.dz, a.batch, a.tokens, a.out_features, 2).input(a.x, a.batch, a.tokens, a.in_features, 2).input(a.x8, a.batch, a.tokens, a.in_features);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    uint8_t* at = static_cast<uint8_t*>(workspace);
    const Epilogue ep{a.accumulate, PG_ACT_NONE, a.dweight, {}, nullptr, 0, {}};
    pg_matrix dz = a.dz, x = a.x;
    int rc = a.tokens > 0 ? aligned_operand(dz, a.batch, a.tokens, a.out_features, at, st) : PG_OK;
    if (rc != PG_OK) return rc;
    if (eight) {
        x = pg_matrix{a.x8.values, a.x8.ld, a.x8.stride};
        // Single blocks only.  In a pair the first block's thread issues products that read what the second block's warps have
        // widened, and the release to the cluster that this takes costs what a pair saves, three stages at a time (one at a time, 544
        // us where single blocks take 322; pairs and single blocks: 64 workers x 2048 tokens, 1024 x 1024 322 and 322 us, 32 x 700,
        // 650 x 2600 134 and 130, 64 x 512, 512 x 512 39 and 34, 10 x 256, 1024 x 1024 20.6 and 18.5).
        return run_product<kWeightGrad8, false>(a.dtype, a.batch, a.in_features, a.out_features, a.tokens, x, dz, ep, &a.x8, st);
    }
    if (a.tokens > 0) rc = aligned_operand(x, a.batch, a.tokens, a.in_features, at, st);
    if (rc != PG_OK) return rc;
    return enough_for_pairs(a.batch, a.in_features, a.out_features, kSMs / 2)
               ? run_product<kWeightGrad, true>(a.dtype, a.batch, a.in_features, a.out_features, a.tokens, x, dz, ep, nullptr, st)
               : run_product<kWeightGrad, false>(a.dtype, a.batch, a.in_features, a.out_features, a.tokens, x, dz, ep, nullptr, st);
}

int pg_selftest_training_timeout(void* stream) {
    wait_probe_kernel<<<1, 64, 0, static_cast<cudaStream_t>(stream)>>>();
    return launch_status() == PG_OK ? pg_training_status(stream) : PG_ERR_CUDA;
}
int pg_selftest_training_bounds(void* stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_training_error) != cudaSuccess) return PG_ERR_CUDA;
    Operands operands;
    operands.output(p, 0, 1, 1);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    bounds_probe_kernel<<<1, 1, 0, st>>>(static_cast<const char*>(p));
    return launch_status() == PG_OK ? pg_training_status(stream) : PG_ERR_CUDA;
}
int pg_training_status(void* stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    unsigned word = 0, rows = 0, loss = 0, sequence = 0, outside = 0;
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_training_error) != cudaSuccess || take_word(static_cast<unsigned*>(p), word, st) != PG_OK ||
        take_row_errors(rows, st) != PG_OK || take_loss_errors(loss, st) != PG_OK || take_sequence_errors(sequence, st) != PG_OK)
        return PG_ERR_CUDA;
#ifdef PG_BOUNDS_CHECK
    if (cudaGetSymbolAddress(&p, g_outside) != cudaSuccess || take_word(static_cast<unsigned*>(p), outside, st) != PG_OK) return PG_ERR_CUDA;
#endif
    return word & kTimedOut ? PG_ERR_TIMEOUT : (rows | loss | sequence | outside) & kOutside ? PG_ERR_BOUNDS : PG_OK;
}

}  // extern "C"
