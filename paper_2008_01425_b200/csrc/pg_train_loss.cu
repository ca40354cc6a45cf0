// The distillation loss (pg_distillation_loss): softmax statistics of every row of logits and what a teacher's top
// logits and a label make of them, forward, backward, and both with one read of the logits.
//
// One block has one row.  With k = log2(e) / tau a logit x counts 2^(k x - r), r a whole number, the row's largest k x
// rounded up: k x - r is then one fused multiply-add, and a thread whose r grows corrects its sums by an
// exact power of two.  Where tau is 1, 2 or 4 the exponentials at temperature 1 are powers of these; elsewhere there
// are two per logit.  With the gradient the row stays in shared memory as it was read, so the logits are read once.
// Memory bounds all of it: 2 bytes a logit for the loss, 4 with the gradient.
#include <algorithm>
#include <type_traits>

#include "pg_train_device.h"

namespace pgt {
namespace {

constexpr int kMaxTop = 1024;                          // entries of a teacher's list
constexpr float kNoLogit = -1e30f;                     // r before the first logit; 2^(kNoLogit - r) is 0
constexpr size_t kMaxRowBytes = 200 * 1024;            // of a block's shared memory

__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ F2 ex2(F2 v) {
    float a, b;
    split(v, a, b);
    return pair(ex2(a), ex2(b));
}

// What a block knows of its row.  Logits lie in 16-byte pieces of memory: piece j holds elements 8 j - off to 8 j - off + 7.
struct Row {
    const uint16_t* x;
    int off, classes, pieces;
    __device__ Row(const pg_matrix& m, int64_t b, int64_t t, int n) {
        x = static_cast<const uint16_t*>(m.data) + b * m.stride + t * m.ld;
        off = static_cast<int>(reinterpret_cast<uintptr_t>(x) & 15) / 2;
        classes = n;
        pieces = (off + n + 7) / 8;
    }
    __device__ uint4 piece(int j) const {              // (every piece holds an element of the row)
        const uint4* p = reinterpret_cast<const uint4*>(x - off) + j;
        return PGT_READ(p, 16) ? *p : make_uint4(0, 0, 0, 0);
    }
};

// fp32 values of an octet whose first element has index `at`; -inf where there is no element.
template <typename H>
__device__ __forceinline__ void logits_of(const uint4& p, int at, int classes, F2 (&v)[4]) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = Elem<H>::up2(w[i]);
    if (at < 0 || at + 8 > classes) {
        const float none = __int_as_float(0xff800000);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b;
            split(v[i], a, b);
            v[i] = pair(at + 2 * i >= 0 && at + 2 * i < classes ? a : none, at + 2 * i + 1 >= 0 && at + 2 * i + 1 < classes ? b : none);
        }
    }
}

// POWER: exponentials at temperature 1 are those at tau to this power (1, 2, 4); 0: they are computed on their own.
// With one of the two terms only, POWER is 1 and k belongs to that term.
struct Sums {
    float r, s;        // at k
    float r1, s1;      // at temperature 1, where POWER != 1
};
template <int POWER>
__device__ __forceinline__ F2 power(F2 e) {
    if constexpr (POWER == 1) return e;
    else if constexpr (POWER == 2) return mul(e, e);
    else return mul(mul(e, e), mul(e, e));
}
template <int POWER>
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
    Sums c;
    c.r = fmaxf(a.r, b.r);
    const float fa = ex2(a.r - c.r), fb = ex2(b.r - c.r);
    c.s = a.s * fa + b.s * fb;
    if constexpr (POWER == 0) {
        c.r1 = fmaxf(a.r1, b.r1);
        c.s1 = a.s1 * ex2(a.r1 - c.r1) + b.s1 * ex2(b.r1 - c.r1);
    } else {
        c.r1 = POWER * c.r;
        c.s1 = POWER == 1 ? c.s : a.s1 * ex2(POWER * (a.r - c.r)) + b.s1 * ex2(POWER * (b.r - c.r));
    }
    return c;
}
template <int POWER, int T>
__device__ __forceinline__ Sums join_block(Sums m, Sums* shared) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Sums other;
        other.r = __shfl_xor_sync(0xffffffffu, m.r, o);
        other.s = __shfl_xor_sync(0xffffffffu, m.s, o);
        other.r1 = POWER == 0 ? __shfl_xor_sync(0xffffffffu, m.r1, o) : 0.0f;
        other.s1 = POWER == 1 ? 0.0f : __shfl_xor_sync(0xffffffffu, m.s1, o);
        m = join<POWER>(m, other);
    }
    if constexpr (T > 32) {
        if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = m;
        __syncthreads();
        m = shared[0];
#pragma unroll
        for (int w = 1; w < T / 32; ++w) m = join<POWER>(m, shared[w]);
    }
    return m;
}
// An octet is counted in: its largest value first, then its exponentials.
template <int POWER>
__device__ __forceinline__ void count(Sums& m, F2& s, F2& s1, const F2 (&v)[4], float k) {
    float top = __int_as_float(0xff800000);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        split(v[i], a, b);
        top = fmaxf(top, fmaxf(a, b));
    }
    const float r = ceilf(top * k);
    if (r > m.r) {
        const float f = ex2(m.r - r);
        s = mul(s, both(f));
        if constexpr (POWER > 1) s1 = mul(s1, power<POWER>(both(f)));
        m.r = r;
    }
    if constexpr (POWER == 0) {
        const float r1 = ceilf(top * kLog2e);
        if (r1 > m.r1) {
            s1 = mul(s1, both(ex2(m.r1 - r1)));
            m.r1 = r1;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 e = ex2(fma(v[i], both(k), both(-m.r)));
        s = add(s, e);
        if constexpr (POWER > 1) s1 = add(s1, power<POWER>(e));
        if constexpr (POWER == 0) s1 = add(s1, ex2(fma(v[i], both(kLog2e), both(-m.r1))));
    }
}

// The teacher's list of a row in shared memory: class (-1: none), probability, its logarithm (base 2), the student's logit.
struct List {
    int* id;
    float *p, *log_p, *x;
};
// By the first warp.  Returns whether the list has an entry that counts: its id is a class and its logit not -inf.
template <typename H>
__device__ __forceinline__ bool read_list(const pg_distillation_args& a, const Row& row, int64_t b, int64_t t, const List& list, float k) {
    const float none = __int_as_float(0xff800000);
    const int lane = threadIdx.x & 31;
    const int32_t* ids = static_cast<const int32_t*>(a.ids.data) + b * a.ids.stride + t * a.ids.ld;
    const uint16_t* teacher = static_cast<const uint16_t*>(a.teacher.data) + b * a.teacher.stride + t * a.teacher.ld;
    float top = none;
    for (int i = lane; i < a.top; i += 32) {
        const int id = PGT_LOAD(ids[i]);
        const bool is = id >= 0 && id < a.classes;
        const float v = is ? Elem<H>::up(PGT_LOAD(teacher[i])) : none;
        list.id[i] = is ? id : -1;
        list.log_p[i] = v;
        list.x[i] = is ? Elem<H>::up(PGT_LOAD(row.x[id])) : 0.0f;
        top = fmaxf(top, v);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float r = fmaxf(ceilf(top * k), kNoLogit);
    float sum = 0.0f;
    for (int i = lane; i < a.top; i += 32) {
        const float v = fmaf(list.log_p[i], k, -r), e = ex2(v);
        list.log_p[i] = v;
        list.p[i] = e;
        sum += e;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const bool any = sum != 0.0f;                      // (NaN is something, too)
    const float inverse = any ? 1.0f / sum : 0.0f, log_sum = any ? log2f(sum) : 0.0f;
    for (int i = lane; i < a.top; i += 32) {
        list.p[i] *= inverse;
        list.log_p[i] -= log_sum;
    }
    return any;
}

// FORWARD: loss and lse.  BOTH: the gradient too, from the row as it was kept in shared memory; AGAIN: the same for rows
// that shared memory does not hold, which are read twice.  BACKWARD: the gradient from lse, a row by gridDim.z blocks.
enum { FORWARD, BOTH, AGAIN, BACKWARD };
template <typename H, int POWER, int T, int MODE>
__global__ void __launch_bounds__(T, T == 512 ? 3 : 1)
distillation_kernel(const pg_distillation_args a, float k, float soft, float hard) {
    extern __shared__ __align__(16) uint4 s_row[];     // the row's pieces (BOTH), then the list
    __shared__ Sums s_sums[T / 32];
    __shared__ bool s_any;
    const int64_t b = blockIdx.y, t = blockIdx.x, at_row = b * a.tokens + t;
    const Row row(a.logits, b, t, a.classes);
    float* words = reinterpret_cast<float*>(s_row + (MODE == BOTH ? (a.classes + 14) / 8 : 0));
    const List list = {reinterpret_cast<int*>(words), words + a.top, words + 2 * a.top, words + 3 * a.top};
    const int label = a.labels ? PGT_LOAD(a.labels[at_row]) : -1;
    const bool labelled = hard != 0.0f && label >= 0 && label < a.classes;
    const float x_label = labelled ? Elem<H>::up(PGT_LOAD(row.x[label])) : 0.0f;
    if (soft != 0.0f && threadIdx.x < 32) {
        const bool any = read_list<H>(a, row, b, t, list, k);
        if (threadIdx.x == 0) s_any = any;
    }
    const float g = a.dloss ? PGT_LOAD(a.dloss[at_row]) : 1.0f;
    Sums m = {kNoLogit, 0.0f, kNoLogit, 0.0f};
    if constexpr (MODE != BACKWARD) {
        F2 s = both(0.0f), s1 = both(0.0f);
        constexpr int U = 4;                           // pieces on their way at once
        for (int j0 = threadIdx.x; j0 < row.pieces; j0 += U * T) {
            uint4 p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) p[u] = j0 + u * T < row.pieces ? row.piece(j0 + u * T) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * T;
                if (j >= row.pieces) break;
                if constexpr (MODE == BOTH) s_row[j] = p[u];
                F2 v[4];
                logits_of<H>(p[u], 8 * j - row.off, a.classes, v);
                count<POWER>(m, s, s1, v, k);
            }
        }
        m.s = sum2(s);
        m.s1 = POWER == 1 ? 0.0f : sum2(s1);
        m = join_block<POWER, T>(m, s_sums);
        if constexpr (POWER == 1) m.s1 = m.s;
        if constexpr (POWER != 0) m.r1 = POWER * m.r;
        if (threadIdx.x < 32) {
            const float log_s = log2f(m.s), log_s1 = POWER == 1 ? log_s : log2f(m.s1), k1 = POWER == 0 ? kLog2e : POWER * k;
            float loss = 0.0f;                         // in bits
            if (soft != 0.0f) {
                __syncwarp();
                for (int i = threadIdx.x; i < a.top; i += 32) {
                    const float p = list.p[i];
                    if (p != 0.0f) loss += p * (list.log_p[i] - (fmaf(list.x[i], k, -m.r) - log_s));
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
                loss *= soft * (kLog2e / k) * (kLog2e / k);
            }
            if (labelled) loss += hard * (log_s1 - fmaf(x_label, k1, -m.r1));
            if (threadIdx.x == 0) {
                if (a.loss) PGT_STORE(a.loss[at_row], loss * kLn2);
                if (a.lse) {
                    PGT_STORE(a.lse[2 * at_row], hard != 0.0f ? (m.r1 + log_s1) * kLn2 : 0.0f);
                    PGT_STORE(a.lse[2 * at_row + 1], soft != 0.0f ? (m.r + log_s) * kLn2 : 0.0f);
                }
            }
        }
        if constexpr (MODE == FORWARD) return;
    } else {
        // 2^(k x - r) is the softmax at k as it is; of its power at temperature 1, 1 / s1 is
        const float lse1 = a.lse ? PGT_LOAD(a.lse[2 * at_row]) * kLog2e : 0.0f, lse = a.lse ? PGT_LOAD(a.lse[2 * at_row + 1]) * kLog2e : 0.0f;
        m.r = soft != 0.0f ? lse : lse1;
        m.r1 = POWER == 0 ? lse1 : POWER * m.r;
        m.s = 1.0f;
        m.s1 = POWER == 0 ? 1.0f : ex2(lse1 - m.r1);
    }
    if constexpr (MODE == BACKWARD) __syncthreads();                   // the list
    const float to_soft = soft != 0.0f && s_any ? g * soft * (kLog2e / k) : 0.0f, to_hard = labelled ? g * hard : 0.0f;
    const float by = to_soft / m.s, by1 = to_hard / m.s1;
    uint16_t* out = static_cast<uint16_t*>(a.dlogits.data) + b * a.dlogits.stride + t * a.dlogits.ld;
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(out) & 15) / 2, pieces = (off + a.classes + 7) / 8;
    const int share = (pieces + gridDim.z - 1) / gridDim.z, first = blockIdx.z * share, last = min(pieces, first + share);
    auto exponential = [&](F2 x) { return ex2(fma(x, both(k), both(-m.r))); };
    auto exponential1 = [&](F2 x, F2 e) {
        if constexpr (POWER == 0) return ex2(fma(x, both(kLog2e), both(-m.r1)));
        else return power<POWER>(e);
    };
    auto read = [&](int j) {
        if (j < 0 || j >= row.pieces) return make_uint4(0, 0, 0, 0);
        if constexpr (MODE == BOTH) return s_row[j];
        else return row.piece(j);
    };
    auto gradient = [&](uint4 p, int j) {
        F2 v[4];
        const int at = 8 * j - off;
        logits_of<H>(p, at, a.classes, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F2 e = exponential(v[i]);
            if constexpr (POWER == 1) v[i] = mul(e, both(by + by1));
            else if constexpr (POWER == 2) v[i] = mul(e, fma(e, both(by1), both(by)));
            else v[i] = fma(exponential1(v[i], e), both(by1), mul(e, both(by)));
        }
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = Elem<H>::down2(v[i]);
        if (at >= 0 && at + 8 <= a.classes) {
            PGT_STORE(*reinterpret_cast<uint4*>(out + at), make_uint4(w[0], w[1], w[2], w[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at + i >= 0 && at + i < a.classes) PGT_STORE(out[at + i], static_cast<uint16_t>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu));
        }
    };
    const int shift = row.off - off;                   // elements from an input's piece to the output's
    if (shift == 0) {
        constexpr int U = 4;
        for (int j0 = first + threadIdx.x; j0 < last; j0 += U * T) {
            uint4 p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) p[u] = read(j0 + u * T);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j0 + u * T < last) gradient(p[u], j0 + u * T);
        }
    } else {
        for (int j = first + threadIdx.x; j < last; j += T) {
            const int from = shift < 0 ? j - 1 : j;
            const Oct o = cut(read(from), read(from + 1), shift & 7);
            gradient(make_uint4(o.w[0], o.w[1], o.w[2], o.w[3]), j);
        }
    }
    // The classes of the list and the label once more, with what the formula takes off there.  A class that is listed twice is
    // computed twice, from the same sum.
    __syncthreads();
    const int entries = to_soft != 0.0f ? a.top : 0;
    for (int i = threadIdx.x; i <= entries; i += T) {
        if (i == entries && !labelled) break;
        const int id = i < entries ? list.id[i] : label;
        if (id < 0 || id < 8 * first - off || id >= 8 * last - off) continue;
        float p = 0.0f;
        for (int j = 0; j < entries; ++j) p += list.id[j] == id ? list.p[j] : 0.0f;
        const F2 x = both(i < entries ? list.x[i] : x_label), e = exponential(x), e1 = exponential1(x, e);
        float q, q1, same;
        split(e, q, same);
        split(e1, q1, same);
        // (with the label's term only k belongs to that)
        const float v = to_soft * (q / m.s - p) + to_hard * ((soft != 0.0f ? q1 : q) / m.s1 - (labelled && id == label ? 1.0f : 0.0f));
        PGT_STORE(out[id], Elem<H>::down(v));
    }
}

int current_device() {
    int d = 0;
    return cudaGetDevice(&d) == cudaSuccess ? d : -1;
}

// Threads of a row: a warp to 1024 classes, four to 8192, sixteen above.
template <typename F>
void with_threads(int classes, F&& f) {
    using std::integral_constant;
    if (classes <= 1024) f(integral_constant<int, 32>{});
    else if (classes <= 8192) f(integral_constant<int, 128>{});
    else f(integral_constant<int, 512>{});
}

int distillation(const pg_distillation_args* args, bool backward, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_distillation_args& a = *args;
    const int dev = current_device();
    if (!sizes_ok(a.dtype, a.batch, a.tokens, a.classes, 1) || a.top < 0) return PG_ERR_INVALID;
    if (!(a.temperature > 0.0f) || a.temperature > 1e30f || a.temperature < 1e-30f || !(a.alpha >= 0.0f && a.alpha <= 1.0f)) return PG_ERR_INVALID;
    if (!matrix_ok(a.logits, a.batch, a.tokens, a.classes, 2, false, dev)) return PG_ERR_INVALID;
    if (a.top > 0 && (!matrix_ok(a.ids, a.batch, a.tokens, a.top, 4, false, dev) || !matrix_ok(a.teacher, a.batch, a.tokens, a.top, 2, false, dev)))
        return PG_ERR_INVALID;
    const bool rows = a.tokens > 0;
    if (rows && a.labels && !vector_ok(a.labels, a.tokens, a.batch, a.tokens, false, dev)) return PG_ERR_INVALID;
    if (rows && a.dloss && !vector_ok(a.dloss, a.tokens, a.batch, a.tokens, false, dev)) return PG_ERR_INVALID;
    if (rows && a.loss && !vector_ok(a.loss, a.tokens, a.batch, a.tokens, true, dev)) return PG_ERR_INVALID;
    if (rows && (a.lse || backward) && !vector_ok(a.lse, 2 * int64_t{a.tokens}, a.batch, 2 * int64_t{a.tokens}, !backward, dev)) return PG_ERR_INVALID;
    if (backward || a.dlogits.data) {
        if (!matrix_ok(a.dlogits, a.batch, a.tokens, a.classes, 2, true, dev)) return PG_ERR_INVALID;
        // in place: the same elements, so that every thread reads what it overwrites itself
        if (a.dlogits.data == a.logits.data && rows && a.batch > 0 && (a.dlogits.ld != a.logits.ld || (a.batch > 1 && a.dlogits.stride != a.logits.stride)))
            return PG_ERR_INVALID;
    }
    if (a.top > kMaxTop) return PG_ERR_TOO_LARGE;
    if (a.batch == 0 || a.tokens == 0) return PG_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Operands operands;
    operands.output(a.dlogits, a.batch, a.tokens, a.classes, 2);
    if (!backward) operands.output(a.loss, a.tokens, a.batch, a.tokens).output(a.lse, 2 * int64_t{a.tokens}, a.batch, 2 * int64_t{a.tokens});
    else operands.input(a.lse, 2 * int64_t{a.tokens}, a.batch, 2 * int64_t{a.tokens});
    operands.input(a.logits, a.batch, a.tokens, a.classes, 2).input(a.labels, a.tokens, a.batch, a.tokens).input(a.dloss, a.tokens, a.batch, a.tokens);
    if (a.top > 0) operands.input(a.ids, a.batch, a.tokens, a.top, 4).input(a.teacher, a.batch, a.tokens, a.top, 2);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;

    const float soft = a.top > 0 ? a.alpha : 0.0f, hard = a.labels ? 1.0f - a.alpha : 0.0f;
    const bool two = soft != 0.0f && hard != 0.0f;
    const float k = static_cast<float>(1.4426950408889634 / (soft != 0.0f ? static_cast<double>(a.temperature) : 1.0));
    const size_t words = soft != 0.0f ? 16 * static_cast<size_t>(a.top) : 0, kept = (static_cast<size_t>(a.classes) + 14) / 8 * 16;
    const int mode = backward ? BACKWARD : !a.dlogits.data ? FORWARD : kept + words <= kMaxRowBytes ? BOTH : AGAIN;
    int rc = PG_OK;
    auto launch = [&](auto h, auto power, auto threads, auto which) {
        using H = decltype(h);
        constexpr int POWER = decltype(power)::value, T = decltype(threads)::value, MODE = decltype(which)::value;
        const auto kernel = distillation_kernel<H, POWER, T, MODE>;
        const size_t smem = words + (MODE == BOTH ? kept : 0);
        if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess) {
            cudaGetLastError();
            rc = PG_ERR_CUDA;
            return;
        }
        int splits = 1;
        if (MODE == BACKWARD) {                        // few rows: as many blocks as there is room for, two steps of all threads each at least
            const int64_t all = int64_t{a.batch} * a.tokens, steps = (int64_t{a.classes} + 8 * T - 1) / (8 * T);
            splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(steps / 2, 4 * kSMs / all)));
        }
        kernel<<<dim3(a.tokens, a.batch, splits), T, smem, st>>>(a, k, soft, hard);
        rc = launch_status();
    };
    auto with_mode = [&](auto h, auto power) {
        with_threads(a.classes, [&](auto threads) {
            using std::integral_constant;
            if (mode == FORWARD) launch(h, power, threads, integral_constant<int, FORWARD>{});
            else if (mode == BOTH) launch(h, power, threads, integral_constant<int, BOTH>{});
            else if (mode == BACKWARD) launch(h, power, threads, integral_constant<int, BACKWARD>{});
            else launch(h, power, integral_constant<int, 512>{}, integral_constant<int, AGAIN>{});
        });
    };
    auto with_power = [&](auto h) {
        using std::integral_constant;
        if (!two || a.temperature == 1.0f) with_mode(h, integral_constant<int, 1>{});
        else if (a.temperature == 2.0f) with_mode(h, integral_constant<int, 2>{});
        else if (a.temperature == 4.0f) with_mode(h, integral_constant<int, 4>{});
        else with_mode(h, integral_constant<int, 0>{});
    };
    if (a.dtype == PG_BF16) with_power(__nv_bfloat16{});
    else with_power(__half{});
    return rc;
}

}  // namespace

int take_loss_errors(unsigned& value, cudaStream_t st) {
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

int pg_distillation_loss(const pg_distillation_args* args, void* stream) { return distillation(args, false, stream); }
int pg_distillation_loss_grad(const pg_distillation_args* args, void* stream) { return distillation(args, true, stream); }

}  // extern "C"
