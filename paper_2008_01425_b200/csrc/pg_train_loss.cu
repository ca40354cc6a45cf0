// The distillation loss (pg_distillation_loss): softmax statistics of every row of logits and what a teacher's top
// logits and a label make of them, forward, backward, and both with one read of the logits.
//
// A logit x counts 2^(k (x - r)), k = log2(e) / tau and r a logit near the largest that a thread has seen: that of its first ones,
// until one is kSlack bits above it (fp32 has room for what is between).  The difference comes first, so that logits of any
// size, a type's lowest number among them, are told apart as well as the type does.  Where tau is 1, 2 or 4 the exponentials at temperature 1
// are powers of these; elsewhere there are two per logit.  With the gradient the row stays in shared memory as it was read, so the
// logits are read once.  Memory bounds it, 2 bytes a logit for the loss and 4 with the gradient, and nearly as much the exponential unit:
// 22400 rows of 28000 classes at tau = 2 take 245 us (0.78 of the copy rate), with the gradient 493 us (0.78), in a steady run under the power cap
// 270 and 558; with two exponentials a logit (tau = 1.7) 365 and 720 us.  Exponentials of the first pass kept in registers for the second
// (512 threads, one block an SM): 1.3 times as long, since a block's phases then wait for one another.
// Fewer blocks are resident where rows are longer, one above 57000 classes: 5600 rows of 50000, 64000, 98000 and 128000 classes take 119, 168, 231
// and 244 us (bytes: 85, 109, 167, 218), with the gradient 262, 410, 558 and, the logits read twice, 679 us; 128000 from lse 469 us.
#include <algorithm>
#include <type_traits>

#include "pg_train_device.h"

namespace pgt {
namespace {

constexpr int kWide = 256;                              // threads of the widest rows
constexpr int kMaxTop = 1024;                          // entries of a teacher's list
constexpr float kNoLogit = -3.4028235e38f;             // r before the first logit, below all that are numbers
constexpr float kSlack = 20.0f;                        // (of the fourth power, 2^80 and a sum of as many as there are)
constexpr size_t kMaxRowBytes = 200 * 1024;            // of a block's shared memory


// What a block knows of its row.  Logits lie in 16-byte pieces of memory: piece j holds elements 8 j - off to 8 j - off + 7.
struct Row {
    const uint16_t* x;
    int off, classes, pieces, first, last;             // first to last - 1: pieces that lie in the row whole
    __device__ Row(const pg_matrix& m, int64_t b, int64_t t, int n) {
        x = static_cast<const uint16_t*>(m.data) + b * m.stride + t * m.ld;
        off = static_cast<int>(reinterpret_cast<uintptr_t>(x) & 15) / 2;
        classes = n;
        pieces = (off + n + 7) / 8;
        first = off > 0;
        last = (off + n) / 8;
    }
    __device__ const uint4* at(int j) const { return reinterpret_cast<const uint4*>(x - off) + j; }
    __device__ uint4 piece(int j) const {              // (every piece holds an element of the row)
        const uint4* p = at(j);
        return PGT_READ(p, 16) ? *p : make_uint4(0, 0, 0, 0);
    }
};

// fp32 values of an octet; -inf in place of those that are not in the row, whose first has index `at` in it.
template <typename H>
__device__ __forceinline__ void logits_of(const uint4& p, F2 (&v)[4]) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = Elem<H>::up2(w[i]);
}
__device__ __forceinline__ void only_row(F2 (&v)[4], int at, int classes) {
    const float none = __int_as_float(0xff800000);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        split(v[i], a, b);
        v[i] = pair(at + 2 * i >= 0 && at + 2 * i < classes ? a : none, at + 2 * i + 1 >= 0 && at + 2 * i + 1 < classes ? b : none);
    }
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// POWER: exponentials at temperature 1 are those at tau to this power (1, 2, 4); 0: they are computed on their own.
// With one of the two terms only, POWER is 1 and k belongs to that term.
struct Sums {
    float r, s;        // at k
    float s1;          // at temperature 1, where POWER != 1
};
template <int POWER>
__device__ __forceinline__ F2 power(F2 e) {
    if constexpr (POWER == 1) return e;
    else if constexpr (POWER == 2) return mul(e, e);
    else return mul(mul(e, e), mul(e, e));
}
// The sums of N neighbouring lanes (of all of them the same), brought to the largest r.
template <int POWER, int N>
__device__ __forceinline__ Sums join(Sums m, float k) {
    auto over = [](float v, auto f) {
#pragma unroll
        for (int o = N / 2; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
        return v;
    };
    auto most = [](float a, float b) { return fmaxf(a, b); };
    auto add = [](float a, float b) { return a + b; };
    const float r = over(m.r, most), d = m.r - r, f = ex2(d * k);
    m.s = over(m.s * f, add);
    if constexpr (POWER == 1) {
        m.s1 = m.s;
    } else {
        float f1 = f;
        if constexpr (POWER == 0) f1 = ex2(d * kLog2e);
        if constexpr (POWER > 1) f1 *= f1;
        if constexpr (POWER > 2) f1 *= f1;
        m.s1 = over(m.s1 * f1, add);
    }
    m.r = r;
    return m;
}
// A warp's sums go to shared memory; after the block's barrier every warp adds them up, in the same order.
template <int POWER>
__device__ __forceinline__ void join_warp(const Sums& m, float k, Sums* shared) {
    const Sums all = join<POWER, 32>(m, k);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = all;
}
template <int POWER, int WARPS>
__device__ __forceinline__ Sums all_sums(const Sums* shared, float k) {
    return join<POWER, WARPS>(shared[threadIdx.x & (WARPS - 1)], k);
}

// An octet is counted in.
template <int POWER>
__device__ __forceinline__ void count(Sums& m, F2& s, F2& s1, const F2 (&v)[4], float k) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) split(v[i], e[2 * i], e[2 * i + 1]);
    const float top = max3(max3(max3(e[0], e[1], e[2]), e[3], e[4]), max3(e[5], e[6], e[7]), e[0]);
    if ((top - m.r) * k > kSlack) {
        const float d = m.r - top, f = ex2(d * k);
        s = mul(s, both(f));
        if constexpr (POWER > 1) s1 = mul(s1, power<POWER>(both(f)));
        if constexpr (POWER == 0) s1 = mul(s1, both(ex2(d * kLog2e)));
        m.r = top;
    }
    if constexpr (POWER == 0) {                        // (at tau > 1 the exponentials at temperature 1 grow faster)
        if ((top - m.r) * kLog2e > kSlack) {
            const float d = m.r - top;
            s = mul(s, both(ex2(d * k)));
            s1 = mul(s1, both(ex2(d * kLog2e)));
            m.r = top;
        }
    }
    const F2 minus = both(-m.r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 d = add(v[i], minus), x = ex2(mul(d, both(k)));
        s = add(s, x);
        if constexpr (POWER > 1) s1 = add(s1, power<POWER>(x));
        if constexpr (POWER == 0) s1 = add(s1, ex2(mul(d, both(kLog2e))));
    }
}

// The teacher's list of a row in shared memory: class (-1: none), probability, its logarithm, the student's logit.
struct List {
    int* id;
    float *p, *log_p, *x;
};
// By one warp.  Returns whether the list has an entry that counts: its id is a class and its logit not -inf.
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
    const float r = fmaxf(top, kNoLogit);
    float sum = 0.0f;
    for (int i = lane; i < a.top; i += 32) {
        const float v = list.log_p[i] - r, e = ex2(v * k);
        list.log_p[i] = v * (k * kLn2);
        list.p[i] = e;
        sum += e;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const bool any = sum != 0.0f;                      // (NaN is something, too)
    const float inverse = any ? 1.0f / sum : 0.0f, log_sum = any ? log2f(sum) * kLn2 : 0.0f;
    for (int i = lane; i < a.top; i += 32) {
        list.p[i] *= inverse;
        list.log_p[i] -= log_sum;
    }
    return any;
}

// A row's constants on the way back: the gradient of a logit x is
//     by 2^(k (x - r)) + by1 2^(log2(e) (x - r1)),  less what list and label take off at their classes (r1 = r but for POWER = 0 from lse).
template <int POWER>
struct Slope {
    float k, r, r1, by, by1;
    __device__ F2 exponential(F2 x) const { return ex2(mul(add(x, both(-r)), both(k))); }
    __device__ F2 exponential1(F2 x, F2 e) const {
        if constexpr (POWER == 0) return ex2(mul(add(x, both(-r1)), both(kLog2e)));
        else return power<POWER>(e);
    }
    template <typename H>
    __device__ void apply(F2 (&v)[4], uint32_t (&w)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F2 e = exponential(v[i]);
            if constexpr (POWER == 1) v[i] = mul(e, both(by + by1));
            else if constexpr (POWER == 2) v[i] = mul(e, fma(e, both(by1), both(by)));
            else v[i] = fma(exponential1(v[i], e), both(by1), mul(e, both(by)));
            w[i] = Elem<H>::down2(v[i]);
        }
    }
};
struct Out {                                           // a row of the gradient, in pieces as Row's
    uint16_t* x;
    int off, classes, pieces, first, last;
    __device__ Out(const pg_matrix& m, int64_t b, int64_t t, int n) {
        x = static_cast<uint16_t*>(m.data) + b * m.stride + t * m.ld;
        off = static_cast<int>(reinterpret_cast<uintptr_t>(x) & 15) / 2;
        classes = n;
        pieces = (off + n + 7) / 8;
        first = off > 0;
        last = (off + n) / 8;
    }
    __device__ void store(int j, const uint32_t (&w)[4]) const { PGT_STORE(*reinterpret_cast<uint4*>(x + 8 * j - off), make_uint4(w[0], w[1], w[2], w[3])); }
    __device__ void store_part(int j, const uint32_t (&w)[4]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = 8 * j - off + i;
            if (at >= 0 && at < classes) PGT_STORE(x[at], static_cast<uint16_t>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu));
        }
    }
};
// Piece j of the output, from the input's pieces (read(i): its i-th, zeros outside), whose rows start `shift` elements later in theirs.
template <typename F>
__device__ __forceinline__ uint4 moved(F&& read, int j, int shift) {
    if (shift == 0) return read(j);
    const int from = shift < 0 ? j - 1 : j;
    const Oct o = cut(read(from), read(from + 1), shift & 7);
    return make_uint4(o.w[0], o.w[1], o.w[2], o.w[3]);
}

// The label and what it weighs.
template <typename H>
struct Label {
    int at;
    bool is;
    float x;
    __device__ Label(const pg_distillation_args& a, const Row& row, int64_t at_row, float hard) {
        at = a.labels ? PGT_LOAD(a.labels[at_row]) : -1;
        is = hard != 0.0f && at >= 0 && at < a.classes;
        x = is ? Elem<H>::up(PGT_LOAD(row.x[at])) : 0.0f;
    }
};

// The classes of the list and the label once more, with what the formula takes off there, by threads `at`, at + step, ..; classes from
// `from` to `to` - 1 only.  A class that is listed twice is computed twice, from the same sum.  The work goes with the square of the list's length; a
// warp beside the row's hides it to some 32 entries: 22400 rows of 28000 classes with gradient take 493 us with 32 entries, 559 with 64, 710
// with 128, 1840 with 300 and 20900 with 1024.
template <typename H, int POWER>
__device__ __forceinline__ void take_off(const Out& out, const List& list, int top, const Label<H>& label, const Slope<POWER>& slope, const Sums& m, bool soft,
                                         float to_soft, float to_hard, int at, int step, int from, int to) {
    const int entries = to_soft != 0.0f ? top : 0;
    for (int i = at; i <= entries; i += step) {
        if (i == entries && !label.is) break;
        const int id = i < entries ? list.id[i] : label.at;
        if (id < 0 || id < from || id >= to) continue;
        float p = 0.0f;
        for (int j = 0; j < entries; ++j) p += list.id[j] == id ? list.p[j] : 0.0f;
        const F2 x = both(i < entries ? list.x[i] : label.x), e = slope.exponential(x), e1 = slope.exponential1(x, e);
        float q, q1, same;
        split(e, q, same);
        split(e1, q1, same);
        // (with the label's term only k belongs to that)
        const float v = to_soft * (q / m.s - p) + to_hard * ((soft ? q1 : q) / m.s1 - (label.is && id == label.at ? 1.0f : 0.0f));
        PGT_STORE(out.x[id], Elem<H>::down(v));
    }
}

// Loss and log-sum-exps of a row, by one warp, from the row's sums.
template <typename H, int POWER>
__device__ __forceinline__ void store_loss(const pg_distillation_args& a, int64_t at_row, const List& list, const Label<H>& label, const Sums& m, float k, float soft,
                                           float hard) {
    const int lane = threadIdx.x & 31;
    const float log_s = log2f(m.s) * kLn2, log_s1 = POWER == 1 ? log_s : log2f(m.s1) * kLn2;
    float loss = 0.0f;
    if (soft != 0.0f) {                                // tau^2 sum p (log p + log s) - tau sum p (x - r): the logits' part in the logits' own range
        float logs = 0.0f, logits = 0.0f;
        for (int i = lane; i < a.top; i += 32) {
            const float p = list.p[i];
            if (p != 0.0f) {
                logs += p * (list.log_p[i] + log_s);
                logits += p * (list.x[i] - m.r);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            logs += __shfl_xor_sync(0xffffffffu, logs, o);
            logits += __shfl_xor_sync(0xffffffffu, logits, o);
        }
        const float tau = kLog2e / k;
        loss = soft * tau * (tau * logs - logits);
    }
    if (label.is) loss += hard * (log_s1 - (label.x - m.r));
    if (lane == 0) {
        if (a.loss) PGT_STORE(a.loss[at_row], loss);
        if (a.lse) {
            PGT_STORE(a.lse[2 * at_row], hard != 0.0f ? m.r + log_s1 : 0.0f);
            PGT_STORE(a.lse[2 * at_row + 1], soft != 0.0f ? fmaf(m.r, k * kLn2, log_s) : 0.0f);
        }
    }
}
template <int ID>
__device__ __forceinline__ void bar_sync(int threads) { asm volatile("bar.sync %0, %1;" ::"n"(ID), "r"(threads) : "memory"); }
template <int ID>
__device__ __forceinline__ void bar_arrive(int threads) { asm volatile("bar.arrive %0, %1;" ::"n"(ID), "r"(threads) : "memory"); }
__device__ __forceinline__ void copy16(void* shared, const void* global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(shared))), "l"(global) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Rows in steps of `step`, by worker and token, without a division for each.
struct Walk {
    int64_t at, b;
    int t, tokens, step_b, step_t, step;
    __device__ Walk(uint32_t first, uint32_t by, int n) : at(first), b(first / n), t(first % n), tokens(n), step_b(by / n), step_t(by % n), step(by) {}
    __device__ void next() {
        at += step;
        b += step_b;
        t += step_t;
        if (t >= tokens) {
            t -= tokens;
            ++b;
        }
    }
};

// Loss, and with GRAD the gradient too, of rows blockIdx.x, blockIdx.x + gridDim.x, ..  The row lies in shared memory, piece j the
// business of thread j mod T alone: as soon as a thread has used a piece for the last time it asks for the same piece of the block's next row, so
// that memory works while the exponentials do.  One more warp reads the teacher's list of the next row meanwhile (three dependent
// trips to memory), computes the loss and corrects the gradient at the list's classes.
// Per row: every thread's sums are there and the list is (barrier 1, all); the gradient is stored (barrier 2, which the list's warp waits at).
// Sums and lists have two places each, the next row's being written while slower warps still read this one's.
template <typename H, int POWER, int T, bool GRAD>
__global__ void __launch_bounds__(T + 32, T == kWide ? 4 : T == 128 ? 7 : 14)
distillation_kernel(const pg_distillation_args a, float k, float soft, float hard) {
    extern __shared__ __align__(16) uint4 s_row[];     // the row's pieces, then two lists
    __shared__ Sums s_sums[2][T / 32];
    __shared__ bool s_any[2];
    const int64_t rows = int64_t{a.batch} * a.tokens;
    float* words = reinterpret_cast<float*>(s_row + (a.classes + 14) / 8);
    auto list_of = [&](int which) {
        float* w = words + 4 * a.top * which;
        return List{reinterpret_cast<int*>(w), w + a.top, w + 2 * a.top, w + 3 * a.top};
    };
    auto row_of = [&](const Walk& w) { return Row(a.logits, w.b, w.t, a.classes); };
    int flip = 0;
    Walk next(blockIdx.x, gridDim.x, a.tokens);
    if (threadIdx.x >= T) {                            // the list's warp
        auto read = [&](const Walk& at, int which) {
            if (soft == 0.0f || at.at >= rows) return;
            const bool any = read_list<H>(a, row_of(at), at.b, at.t, list_of(which), k);
            if (threadIdx.x == T) s_any[which] = any;
            __syncwarp();
        };
        read(next, 0);
        while (next.at < rows) {
            const Walk at = next;
            next.next();
            const Label<H> label(a, row_of(at), at.at, hard);
            const float g = GRAD && a.dloss ? PGT_LOAD(a.dloss[at.at]) : 1.0f;
            bar_sync<1>(T + 32);
            const Sums m = all_sums<POWER, T / 32>(s_sums[flip], k);
            const List list = list_of(flip);
            store_loss<H, POWER>(a, at.at, list, label, m, k, soft, hard);
            read(next, flip ^ 1);
            if constexpr (GRAD) {
                const float to_soft = soft != 0.0f && s_any[flip] ? g * soft * (kLog2e / k) : 0.0f, to_hard = label.is ? g * hard : 0.0f;
                bar_sync<2>(T + 32);
                const Slope<POWER> slope = {k, m.r, m.r, 0.0f, 0.0f};
                take_off<H, POWER>(Out(a.dlogits, at.b, at.t, a.classes), list, a.top, label, slope, m, soft != 0.0f, to_soft, to_hard, threadIdx.x - T, 32, 0,
                                   a.classes);
            }
            flip ^= 1;
        }
        return;
    }
    const uint4* from = nullptr;                       // piece threadIdx.x of the next row, which has `pieces`
    int pieces = 0;
    auto ask = [&](int j) {
        if (j < pieces && PGT_READ(from + (j - static_cast<int>(threadIdx.x)), 16)) copy16(s_row + j, from + (j - static_cast<int>(threadIdx.x)));
    };
    // This thread's pieces of a row: f(j) for those that are the row's whole, part(j) for the first and the last if they are not.
    auto walk = [&](const auto& row, auto&& f, auto&& part) {
        int j = threadIdx.x;
        if (j < row.first) {
            part(j);
            j += T;
        }
#pragma unroll 2
        for (; j < row.last; j += T) f(j);
        if (j < row.pieces) part(j);
    };
    Row coming = row_of(next);
    from = coming.at(threadIdx.x);
    pieces = coming.pieces;
    for (int j = threadIdx.x; j < pieces; j += T) ask(j);
    for (; next.at < rows; flip ^= 1) {
        const Walk at = next;
        const Row row = coming;
        next.next();
        pieces = 0;
        if (next.at < rows) {
            coming = row_of(next);
            from = coming.at(threadIdx.x);
            pieces = coming.pieces;
        }
        float g = 1.0f;
        int label = -1;
        if constexpr (GRAD) {
            if (a.dloss) g = PGT_LOAD(a.dloss[at.at]);
            if (a.labels && hard != 0.0f) label = PGT_LOAD(a.labels[at.at]);
        }
        Sums m = {kNoLogit, 0.0f, 0.0f};
        F2 s = both(0.0f), s1 = both(0.0f);
        copies_wait();
        walk(
            row,
            [&](int j) {
                F2 v[4];
                logits_of<H>(s_row[j], v);
                count<POWER>(m, s, s1, v, k);
                if constexpr (!GRAD) ask(j);
            },
            [&](int j) {
                F2 v[4];
                logits_of<H>(s_row[j], v);
                only_row(v, 8 * j - row.off, a.classes);
                count<POWER>(m, s, s1, v, k);
                if constexpr (!GRAD) ask(j);
            });
        m.s = sum2(s);
        m.s1 = POWER == 1 ? 0.0f : sum2(s1);
        join_warp<POWER>(m, k, s_sums[flip]);
        bar_sync<1>(T + 32);
        const int rest = row.pieces + (static_cast<int>(threadIdx.x) - row.pieces % T + T) % T;      // this thread's first piece behind the row's
        if constexpr (GRAD) {
            m = all_sums<POWER, T / 32>(s_sums[flip], k);
            const bool listed = soft != 0.0f && s_any[flip], labelled = label >= 0 && label < a.classes;
            const float to_soft = listed ? g * soft * (kLog2e / k) : 0.0f, to_hard = labelled ? g * hard : 0.0f;
            const Slope<POWER> slope = {k, m.r, m.r, to_soft / m.s, to_hard / m.s1};
            const Out out(a.dlogits, at.b, at.t, a.classes);
            const int shift = row.off - out.off;
            if (!listed && !labelled) {                // no term depends on the row: zeros, whatever its logits are
                const uint32_t zeros[4] = {};
                walk(out, [&](int j) { out.store(j, zeros); }, [&](int j) { out.store_part(j, zeros); });
                for (int j = threadIdx.x; j < pieces; j += T) ask(j);
            } else if (shift == 0) {
                walk(
                    row,
                    [&](int j) {
                        F2 v[4];
                        uint32_t w[4];
                        logits_of<H>(s_row[j], v);
                        slope.template apply<H>(v, w);
                        out.store(j, w);
                        ask(j);
                    },
                    [&](int j) {
                        F2 v[4];
                        uint32_t w[4];
                        logits_of<H>(s_row[j], v);
                        slope.template apply<H>(v, w);
                        out.store_part(j, w);
                        ask(j);
                    });
                for (int j = rest; j < pieces; j += T) ask(j);
            } else {
                auto read = [&](int j) { return j < 0 || j >= row.pieces ? make_uint4(0, 0, 0, 0) : s_row[j]; };
                auto piece = [&](int j, uint32_t (&w)[4]) {
                    F2 v[4];
                    logits_of<H>(moved(read, j, shift), v);
                    slope.template apply<H>(v, w);
                };
                walk(
                    out,
                    [&](int j) {
                        uint32_t w[4];
                        piece(j, w);
                        out.store(j, w);
                    },
                    [&](int j) {
                        uint32_t w[4];
                        piece(j, w);
                        out.store_part(j, w);
                    });
                bar_sync<3>(T);                        // others have read this thread's pieces, too
                for (int j = threadIdx.x; j < pieces; j += T) ask(j);
            }
            __threadfence_block();
            bar_arrive<2>(T + 32);
        } else {
            for (int j = rest; j < pieces; j += T) ask(j);
        }
    }
}

// The loss alone where there are rows for every warp: a warp has a row, its lanes' pieces come through a ring of their own in shared memory,
// kAhead steps of two ahead and into the next row, and no warp waits for another.
constexpr int kAhead = 3;
template <int LEFT>
__device__ __forceinline__ void copies_wait_but() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
template <typename H, int POWER>
__global__ void __launch_bounds__(256, 4)
distillation_warp_kernel(const pg_distillation_args a, float k, float soft, float hard) {
    extern __shared__ __align__(16) float s_lists[];
    __shared__ __align__(16) uint4 s_ring[8][kAhead + 1][2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t rows = int64_t{a.batch} * a.tokens;
    float* words = s_lists + 4 * a.top * warp;
    const List list = {reinterpret_cast<int*>(words), words + a.top, words + 2 * a.top, words + 3 * a.top};
    auto row_of = [&](const Walk& w) { return Row(a.logits, w.b, w.t, a.classes); };
    Walk at(blockIdx.x * 8 + warp, gridDim.x * 8, a.tokens);
    if (at.at >= rows) return;
    Walk ahead = at;
    Row coming = row_of(ahead);
    int from = lane, to = 0, slot = 0;                 // the piece that comes next and where it goes; the place of the one to be used
    auto ask = [&] {
        if (ahead.at < rows) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int j = from + 32 * i;
                if (j < coming.pieces && PGT_READ(coming.at(j), 16)) copy16(&s_ring[warp][to][i][lane], coming.at(j));
            }
            from += 64;
            if (from - lane >= coming.pieces) {
                from = lane;
                ahead.next();
                if (ahead.at < rows) coming = row_of(ahead);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        to = to == kAhead ? 0 : to + 1;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ask();
    for (; at.at < rows; at.next()) {
        const Row row = row_of(at);
        Sums m = {kNoLogit, 0.0f, 0.0f};
        F2 s = both(0.0f), s1 = both(0.0f);
        for (int j0 = lane; j0 - lane < row.pieces; j0 += 64) {
            ask();
            copies_wait_but<kAhead>();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int j = j0 + 32 * i;
                if (j < row.pieces) {
                    F2 v[4];
                    logits_of<H>(s_ring[warp][slot][i][lane], v);
                    if (j < row.first || j >= row.last) only_row(v, 8 * j - row.off, a.classes);
                    count<POWER>(m, s, s1, v, k);
                }
            }
            slot = slot == kAhead ? 0 : slot + 1;
        }
        m.s = sum2(s);
        m.s1 = POWER == 1 ? 0.0f : sum2(s1);
        m = join<POWER, 32>(m, k);
        const Label<H> label(a, row, at.at, hard);
        if (soft != 0.0f) read_list<H>(a, row, at.b, at.t, list, k);
        __syncwarp();
        store_loss<H, POWER>(a, at.at, list, label, m, k, soft, hard);
        __syncwarp();
    }
    copies_wait();
}

// Rows that shared memory does not hold: read twice (AGAIN), or with lse known once (BACKWARD), a row then by gridDim.z blocks.
enum { FORWARD, BOTH, AGAIN, BACKWARD };
template <typename H, int POWER, int T, int MODE>
__global__ void __launch_bounds__(T + 32, T == kWide ? 5 : 1)
distillation_stream_kernel(const pg_distillation_args a, float k, float soft, float hard) {
    extern __shared__ __align__(16) float s_list[];
    __shared__ Sums s_sums[T / 32];
    __shared__ bool s_any;
    const int64_t b = blockIdx.y, t = blockIdx.x, at_row = b * a.tokens + t;
    const Row row(a.logits, b, t, a.classes);
    const List list = {reinterpret_cast<int*>(s_list), s_list + a.top, s_list + 2 * a.top, s_list + 3 * a.top};
    const Label<H> label(a, row, at_row, hard);
    const float g = a.dloss ? PGT_LOAD(a.dloss[at_row]) : 1.0f;
    const bool lists = threadIdx.x >= T;
    constexpr int U = 4;                               // pieces on their way at once
    Sums m = {kNoLogit, 0.0f, 0.0f};
    if (lists) {
        if (soft != 0.0f) {
            const bool any = read_list<H>(a, row, b, t, list, k);
            if (threadIdx.x == T) s_any = any;
        }
    } else if constexpr (MODE == AGAIN) {
        F2 s = both(0.0f), s1 = both(0.0f);
        for (int j0 = threadIdx.x; j0 < row.pieces; j0 += U * T) {
            uint4 p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) p[u] = j0 + u * T < row.pieces ? row.piece(j0 + u * T) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * T;
                if (j < row.pieces) {
                    F2 v[4];
                    logits_of<H>(p[u], v);
                    if (j < row.first || j >= row.last) only_row(v, 8 * j - row.off, a.classes);
                    count<POWER>(m, s, s1, v, k);
                }
            }
        }
        m.s = sum2(s);
        m.s1 = POWER == 1 ? 0.0f : sum2(s1);
        join_warp<POWER>(m, k, s_sums);
    }
    __syncthreads();
    float r1;
    if constexpr (MODE == AGAIN) {
        m = all_sums<POWER, T / 32>(s_sums, k);
        if (lists) store_loss<H, POWER>(a, at_row, list, label, m, k, soft, hard);
        if (!a.dlogits.data) return;
        r1 = m.r;
    } else {
        // 2^(k (x - tau lse)) is the softmax at tau as it is; of its power at temperature 1, 1 / s1 is
        const float lse1 = PGT_LOAD(a.lse[2 * at_row]), lse = PGT_LOAD(a.lse[2 * at_row + 1]);
        m.r = soft != 0.0f ? lse * (kLog2e / k) : lse1;
        m.s = 1.0f;
        m.s1 = POWER > 1 ? ex2((lse1 - m.r) * kLog2e) : 1.0f;
        r1 = POWER == 0 ? lse1 : m.r;
    }
    const bool listed = soft != 0.0f && s_any, none = !listed && !label.is;               // none: zeros, whatever logits and lse are
    const float to_soft = listed ? g * soft * (kLog2e / k) : 0.0f, to_hard = label.is ? g * hard : 0.0f;
    const Slope<POWER> slope = {k, m.r, r1, to_soft / m.s, to_hard / m.s1};
    const Out out(a.dlogits, b, t, a.classes);
    const int share = (out.pieces + gridDim.z - 1) / gridDim.z, first = blockIdx.z * share, last = min(out.pieces, first + share);
    const int shift = row.off - out.off;
    auto read = [&](int j) { return j < 0 || j >= row.pieces ? make_uint4(0, 0, 0, 0) : row.piece(j); };
    if (!lists)
        for (int j0 = first + threadIdx.x; j0 < last; j0 += U * T) {
            uint4 p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) p[u] = j0 + u * T < last ? moved(read, j0 + u * T, shift) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * T;
                if (j < last) {
                    F2 v[4];
                    uint32_t w[4] = {};
                    logits_of<H>(p[u], v);
                    if (!none) slope.template apply<H>(v, w);
                    if (j >= out.first && j < out.last) out.store(j, w);
                    else out.store_part(j, w);
                }
            }
        }
    __syncthreads();
    take_off<H, POWER>(out, list, a.top, label, slope, m, soft != 0.0f, to_soft, to_hard, threadIdx.x, T + 32, 8 * first - out.off, 8 * last - out.off);
}

int current_device() {
    int d = 0;
    return cudaGetDevice(&d) == cudaSuccess ? d : -1;
}

// Threads of a row: a warp to 1024 classes, four to 8192, eight above.
template <typename F>
void with_threads(int classes, F&& f) {
    using std::integral_constant;
    if (classes <= 1024) f(integral_constant<int, 32>{});
    else if (classes <= 8192) f(integral_constant<int, 128>{});
    else f(integral_constant<int, kWide>{});
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
    const int mode = backward ? BACKWARD : kept + 2 * words > kMaxRowBytes ? AGAIN : a.dlogits.data ? BOTH : FORWARD;
    const int64_t rows_in_all = int64_t{a.batch} * a.tokens;
    int rc = PG_OK;
    auto launch = [&](auto h, auto power, auto threads, auto which) {
        using H = decltype(h);
        constexpr int POWER = decltype(power)::value, T = decltype(threads)::value, MODE = decltype(which)::value;
        // The loss alone to 8192 classes: a row a warp where that keeps nine tenths of all warps busy to the end.  22400 rows of 300, 1001, 3000,
        // 5000 and 8000 classes: 27, 33, 50, 68 and 95 us, by blocks 33, 44, 66, 73 and 95; of 28000 classes 271 against 245.
        const int64_t warps = int64_t{kSMs} * 32, turns = (rows_in_all + warps - 1) / warps;
        if constexpr (MODE == FORWARD && T <= 128) {
            if (rows_in_all * 10 >= turns * warps * 9 && 8 * words <= 16 * 1024) {
                distillation_warp_kernel<H, POWER><<<kSMs * 4, 256, 8 * words, st>>>(a, k, soft, hard);
                rc = launch_status();
                return;
            }
        }
        if constexpr (MODE == FORWARD || MODE == BOTH) {
            const auto kernel = distillation_kernel<H, POWER, T, MODE == BOTH>;
            const size_t smem = 2 * words + kept;
            static std::atomic<bool> allowed[64];
            if (smem > 48 * 1024 && !allow_shared_memory(reinterpret_cast<const void*>(kernel), kMaxRowBytes, allowed)) {
                rc = PG_ERR_CUDA;
                return;
            }
            // as many blocks as are resident at once (a block takes 1 KB of shared memory and its sums besides)
            const int64_t fit = std::min<int64_t>(T == kWide ? 4 : T == 128 ? 7 : 14, (228 * 1024) / (smem + 1024 + 2 * sizeof(Sums) * T / 32 + 16));
            kernel<<<static_cast<unsigned>(std::min<int64_t>(rows_in_all, kSMs * std::max<int64_t>(fit, 1))), T + 32, smem, st>>>(a, k, soft, hard);
        } else {
            int splits = 1;
            if (MODE == BACKWARD) {                    // few rows: as many blocks as there is room for, two steps of all threads each at least
                const int64_t steps = (int64_t{a.classes} + 8 * T - 1) / (8 * T);
                splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(steps / 2, 4 * kSMs / rows_in_all)));
            }
            distillation_stream_kernel<H, POWER, T, MODE><<<dim3(a.tokens, a.batch, splits), T + 32, words, st>>>(a, k, soft, hard);
        }
        rc = launch_status();
    };
    auto with_mode = [&](auto h, auto power) {
        with_threads(a.classes, [&](auto threads) {
            using std::integral_constant;
            constexpr int T = decltype(threads)::value;
            if (mode == FORWARD) return launch(h, power, threads, integral_constant<int, FORWARD>{});
            if (mode == BACKWARD) return launch(h, power, threads, integral_constant<int, BACKWARD>{});
            if (mode == BOTH) return launch(h, power, threads, integral_constant<int, BOTH>{});
            if constexpr (T == kWide) launch(h, power, threads, integral_constant<int, AGAIN>{});
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
