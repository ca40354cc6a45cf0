// Operators along the tokens of a sequence: the short causal convolution of every channel, the selective scan, and their gradients.
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "pg_train_device.h"

namespace pgt {
namespace {

__device__ __forceinline__ float rcp(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Tokens that are there of sequence s of worker b.
__device__ __forceinline__ int tokens_of(const int32_t* lengths, int64_t b, int sequences, int s, int length) {
    return lengths ? max(0, min(length, PGT_LOAD(lengths[b * sequences + s]))) : length;
}

__device__ __forceinline__ void copy16(void* shared, const void* global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(shared))), "l"(global) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait_but_last() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Rows of CH neighbouring elements of a 16-bit matrix in shared memory, as the 16-byte pieces of memory that hold them: a row starts as far
// into its first piece as it does in memory.
template <int CH>
struct Rows {
    static constexpr int kPieces = CH / 8 + 1;
    const uint16_t* x;                                 // first row's first element
    int64_t ld;
    __device__ Rows() : x(nullptr), ld(0) {}
    __device__ Rows(const pg_matrix& m, int64_t b, int64_t row, int col) : ld(m.ld) {
        x = static_cast<const uint16_t*>(m.data) + b * m.stride + row * m.ld + col;
    }
    __device__ int off(int t) const { return static_cast<int>((reinterpret_cast<uintptr_t>(x) / 2 + static_cast<uint32_t>(t) * static_cast<uint32_t>(ld)) & 7); }
    // Asks for pieces at, at + 8, .. of row t, which has n elements.
    __device__ void ask(uint4* to, int t, int at, int n) const {
        const uint16_t* row = x + t * ld;
        const int o = off(t);
        const uint4* from = reinterpret_cast<const uint4*>(row - o);
#pragma unroll
        for (int i = 0; i < kPieces; i += 8)
            if (i + at < kPieces && 8 * (i + at) < o + n && PGT_READ(from + i + at, 16)) copy16(to + i + at, from + i + at);
    }
    __device__ uint16_t get(const uint4* held, int t, int c) const { return reinterpret_cast<const uint16_t*>(held)[off(t) + c]; }
};

// ---------------------------------------------------------------- convolution
// A warp has 64 neighbouring channels, a lane two of them, and runs along the tokens of (a part of) one sequence, with the inputs of
// the last width - 1 tokens in registers: every input is read once, but for the few before a run.  Inputs come through shared memory in
// 16-byte pieces, whatever the rows' alignment, a tile of tokens ahead.  4 bytes a value (6 in the gradient) have to move; instructions (some
// 60 for two values of a lane) bound it at 0.45 of the copy rate: 32 x 700 tokens x 1300 channels 43 us.  (Eight channels a thread, cut out of
// their pieces in registers: 88 us.  Plain 2- and 4-byte loads: 43 us, but the gradient of odd widths 145 us instead of 60.)
constexpr int kRun = 64;                               // tokens of a run at most
constexpr int kConvThreads = 128;
constexpr int kStrip = 64;                             // channels
constexpr int kConvTile = 8;                           // tokens

// A lane's two channels.  W = 2: the output's rows start on 4-byte boundaries, and they are neighbours.  W = 1: 32 apart, so that
// a warp's 2-byte accesses touch neighbouring elements.
template <int W>
struct Two {
    static constexpr int kApart = W == 2 ? 1 : 32;
    int c;
    bool first, second;
    __device__ explicit Two(int channels) : c((threadIdx.x & 31) * W) {
        first = c < channels;
        second = c + kApart < channels;
    }
    __device__ uint32_t load(const uint16_t* row) const {
        const uint32_t lo = first ? PGT_LOAD(row[c]) : 0, hi = second ? PGT_LOAD(row[c + kApart]) : 0;
        return lo | hi << 16;
    }
    template <int CH>
    __device__ uint32_t get(const Rows<CH>& rows, const uint4* held, int t) const {
        const uint32_t lo = rows.get(held, t, c), hi = rows.get(held, t, c + kApart);
        return lo | hi << 16;
    }
    template <bool PAIRS = W == 2>
    __device__ void store(uint16_t* row, uint32_t w) const {
        if (PAIRS && second) {
            PGT_STORE(*reinterpret_cast<uint32_t*>(row + c), w);
        } else {
            if (first) PGT_STORE(row[c], static_cast<uint16_t>(w & 0xffffu));
            if (second) PGT_STORE(row[c + kApart], static_cast<uint16_t>(w >> 16));
        }
    }
    __device__ F2 numbers(const float* from, int64_t step) const { return pair(first ? PGT_LOAD(from[c * step]) : 0.0f, second ? PGT_LOAD(from[(c + kApart) * step]) : 0.0f); }
};

struct ConvPlace {
    int64_t b, sequence;                               // sequence: of all workers
    int have;                                          // tokens that are there
    int64_t row;                                       // of the first token, in a worker's matrix
    template <typename Args>
    __device__ ConvPlace(const Args& a, int64_t of_all) : sequence(of_all) {
        b = of_all / a.sequences;
        const int s = static_cast<int>(of_all % a.sequences);
        have = tokens_of(a.lengths, b, a.sequences, s, a.length);
        row = static_cast<int64_t>(s) * a.length;
    }
    __device__ uint16_t* at(const pg_matrix& m, int col) const { return static_cast<uint16_t*>(m.data) + b * m.stride + row * m.ld + col; }
};
// Asks for the rows of a tile from token t on, of those before `stop`, eight lanes a row.
__device__ __forceinline__ void ask_tile(const Rows<kStrip>& rows, uint4* to, int t, int stop, int n) {
#pragma unroll
    for (int r = 0; r < kConvTile; r += 4) {
        const int k = r + (threadIdx.x & 31) / 8;
        if (t + k < stop) rows.ask(to + k * Rows<kStrip>::kPieces, t + k, threadIdx.x & 7, n);
    }
}

template <typename H, int W, int TAPS, int ACT>
__global__ void __launch_bounds__(kConvThreads, 8)
conv_kernel(const pg_conv_args a, int run, int runs) {
    __shared__ __align__(16) uint4 s_in[kConvThreads / 32][2][kConvTile * Rows<kStrip>::kPieces];
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5), of_all = item / runs;
    if (of_all >= static_cast<int64_t>(a.batch) * a.sequences) return;
    const int col = blockIdx.y * kStrip, n = min(kStrip, a.channels - col);
    const Two<W> two(n);
    const ConvPlace at(a, of_all);
    const int t0 = static_cast<int>(item % runs) * run, t1 = min(a.length, t0 + run), stop = min(t1, at.have);
    uint4(&ring)[2][kConvTile * Rows<kStrip>::kPieces] = s_in[threadIdx.x >> 5];
    const Rows<kStrip> rows(a.x, at.b, at.row, col);
    ask_tile(rows, ring[0], t0, stop, n);
    copies_end();
    const uint16_t* x = at.at(a.x, col);
    uint16_t* y = at.at(a.y, col) + t0 * a.y.ld;
    const int64_t held = at.sequence * (TAPS - 1) * a.channels + col;
    const uint16_t* state = a.state ? static_cast<const uint16_t*>(a.state) + held : nullptr;
    auto input = [&](int t) { return t >= 0 ? two.load(x + t * a.x.ld) : state ? two.load(state + static_cast<int64_t>(TAPS - 1 + t) * a.channels) : 0u; };
    F2 w[TAPS], o = both(0.0f), before[TAPS - 1];
    const float* weights = static_cast<const float*>(a.weight.data) + at.b * a.weight.stride + col * a.weight.ld;
#pragma unroll
    for (int j = 0; j < TAPS; ++j) w[j] = two.numbers(weights + j, a.weight.ld);
    if (a.bias) o = two.numbers(a.bias + at.b * a.bias_stride + col, 1);
#pragma unroll
    for (int j = 0; j < TAPS - 1; ++j) before[j] = t0 == 0 || t0 < at.have ? Elem<H>::up2(input(t0 - (TAPS - 1) + j)) : both(0.0f);
    if (t0 == 0 && a.state_out) {                      // the last inputs of the sequence; only this lane reads the old ones
        uint16_t* out = static_cast<uint16_t*>(a.state_out) + held;
        uint32_t last[TAPS - 1];
#pragma unroll
        for (int j = 0; j < TAPS - 1; ++j) last[j] = input(at.have - (TAPS - 1) + j);
#pragma unroll
        for (int j = 0; j < TAPS - 1; ++j) two.template store<false>(out + static_cast<int64_t>(j) * a.channels, last[j]);
    }
    for (int t = t0, stage = 0; t < stop; t += kConvTile, stage ^= 1) {
        ask_tile(rows, ring[stage ^ 1], t + kConvTile, stop, n);
        copies_end();
        copies_wait_but_last();
        __syncwarp();
#pragma unroll 4
        for (int u = 0; u < kConvTile; ++u) {
            if (t + u >= stop) break;
            const F2 v = Elem<H>::up2(two.get(rows, ring[stage] + u * Rows<kStrip>::kPieces, t + u));
            F2 z = o;
#pragma unroll
            for (int j = 0; j < TAPS - 1; ++j) z = fma(before[j], w[j], z);
            z = activate<ACT>(fma(v, w[TAPS - 1], z));
#pragma unroll
            for (int j = 0; j + 1 < TAPS - 1; ++j) before[j] = before[j + 1];
            before[TAPS - 2] = v;
            two.store(y, Elem<H>::down2(z));
            y += a.y.ld;
        }
        __syncwarp();
    }
    for (int t = max(t0, stop); t < t1; ++t, y += a.y.ld) two.store(y, 0);
}

// The gradient.  dx of token t needs the pre-activations' gradients up to token t + TAPS - 1: a run recomputes those of the
// tokens behind it, as far as they are there; what a sequence's last tokens get comes after its loop (with zeros for tokens that are not there, in
// the loop, 32 x 700 x 1300 took 90 us instead of 86).  Sums over tokens: a thread's runs, the four warps of the block (shared memory), then the blocks, whose sums
// go to partial[worker][part][TAPS + 1][channels], the bias last.
template <typename H, int W, int TAPS, int ACT>
__global__ void __launch_bounds__(kConvThreads, 5)
conv_grad_kernel(const pg_conv_grad_args a, float* __restrict__ partial, int run, int runs, int parts) {
    __shared__ __align__(16) uint4 s_in[kConvThreads / 32][2][2][kConvTile * Rows<kStrip>::kPieces];
    __shared__ float s_sum[4][TAPS + 1][kStrip];
    const int warp = threadIdx.x >> 5, col = blockIdx.y * kStrip, n = min(kStrip, a.channels - col);
    const int64_t b = blockIdx.x / parts;
    const int part = static_cast<int>(blockIdx.x % parts);
    const int64_t items = static_cast<int64_t>(a.sequences) * runs;      // of a worker
    const Two<W> two(n);
    F2 w[TAPS], o = both(0.0f), dw[TAPS], db = both(0.0f);
    const float* weights = static_cast<const float*>(a.weight.data) + b * a.weight.stride + col * a.weight.ld;
#pragma unroll
    for (int j = 0; j < TAPS; ++j) {
        w[j] = two.numbers(weights + j, a.weight.ld);
        dw[j] = both(0.0f);
    }
    if (a.bias) o = two.numbers(a.bias + b * a.bias_stride + col, 1);
    for (int64_t item = part * 4 + warp; item < items; item += 4 * parts) {
        const ConvPlace at(a, b * a.sequences + item / runs);
        const int t0 = static_cast<int>(item % runs) * run, t1 = min(a.length, t0 + run);
        const int own = min(t1, at.have), end = own + TAPS - 1, stop = min(at.have, end);        // tokens to own have sums here, those to stop count for dx
        uint16_t* dx = at.at(a.dx, col) + t0 * a.dx.ld;
        if (t0 < own) {
            const Rows<kStrip> rx(a.x, at.b, at.row, col), rd(a.dy, at.b, at.row, col);
            ask_tile(rx, s_in[warp][0][0], t0, stop, n);
            ask_tile(rd, s_in[warp][0][1], t0, stop, n);
            copies_end();
            const uint16_t* x = at.at(a.x, col);
            const uint16_t* state = a.state ? static_cast<const uint16_t*>(a.state) + at.sequence * (TAPS - 1) * a.channels + col : nullptr;
            F2 before[TAPS - 1], dz[TAPS - 1];
#pragma unroll
            for (int j = 0; j < TAPS - 1; ++j) {
                const int t = t0 - (TAPS - 1) + j;
                before[j] = Elem<H>::up2(t >= 0 ? two.load(x + t * a.x.ld) : state ? two.load(state + static_cast<int64_t>(TAPS - 1 + t) * a.channels) : 0u);
                dz[j] = both(0.0f);
            }
            for (int t = t0, stage = 0; t < stop; t += kConvTile, stage ^= 1) {
                ask_tile(rx, s_in[warp][stage ^ 1][0], t + kConvTile, stop, n);
                ask_tile(rd, s_in[warp][stage ^ 1][1], t + kConvTile, stop, n);
                copies_end();
                copies_wait_but_last();
                __syncwarp();
#pragma unroll 4
                for (int u = 0; u < kConvTile; ++u) {
                    if (t + u >= stop) break;
                    const F2 v = Elem<H>::up2(two.get(rx, s_in[warp][stage][0] + u * Rows<kStrip>::kPieces, t + u));
                    F2 g = Elem<H>::up2(two.get(rd, s_in[warp][stage][1] + u * Rows<kStrip>::kPieces, t + u));
                    if constexpr (ACT != PG_ACT_NONE) {
                        F2 z = o;
#pragma unroll
                        for (int j = 0; j < TAPS - 1; ++j) z = fma(before[j], w[j], z);
                        g = mul(g, slope<ACT>(fma(v, w[TAPS - 1], z)));
                    }
                    if (t + u < own) {
                        db = add(db, g);
#pragma unroll
                        for (int j = 0; j < TAPS - 1; ++j) dw[j] = fma(g, before[j], dw[j]);
                        dw[TAPS - 1] = fma(g, v, dw[TAPS - 1]);
                    }
                    F2 out = mul(g, w[0]);             // dz holds the gradients of the TAPS - 1 tokens before this one, the oldest first
#pragma unroll
                    for (int j = 0; j < TAPS - 1; ++j) out = fma(dz[j], w[TAPS - 1 - j], out);
#pragma unroll
                    for (int j = 0; j + 1 < TAPS - 1; ++j) {
                        before[j] = before[j + 1];
                        dz[j] = dz[j + 1];
                    }
                    before[TAPS - 2] = v;
                    dz[TAPS - 2] = g;
                    if (t + u - (TAPS - 1) >= t0) {
                        two.store(dx, Elem<H>::down2(out));
                        dx += a.dx.ld;
                    }
                }
                __syncwarp();
            }
#pragma unroll
            for (int i = 0; i < TAPS - 1; ++i) {       // the sequence's last tokens, from what is there behind them
                if (stop + i >= end || stop + i - (TAPS - 1) < t0) continue;
                F2 out = both(0.0f);
#pragma unroll
                for (int j = i; j < TAPS - 1; ++j) out = fma(dz[j], w[TAPS - 1 - j + i], out);
                two.store(dx, Elem<H>::down2(out));
                dx += a.dx.ld;
            }
        }
        for (int t = max(t0, own); t < t1; ++t, dx += a.dx.ld) two.store(dx, 0);
    }
    copies_wait();                                     // (the last, empty group)
#pragma unroll
    for (int j = 0; j <= TAPS; ++j) split(j < TAPS ? dw[j < TAPS ? j : 0] : db, s_sum[warp][j][two.c], s_sum[warp][j][two.c + Two<W>::kApart]);
    __syncthreads();
    float* out = partial + static_cast<int64_t>(blockIdx.x) * (TAPS + 1) * a.channels + col;
    for (int i = threadIdx.x; i < (TAPS + 1) * kStrip; i += kConvThreads) {
        const int j = i / kStrip, c = i % kStrip;
        if (c < n) PGT_STORE(out[static_cast<int64_t>(j) * a.channels + c], (s_sum[0][j][c] + s_sum[1][j][c]) + (s_sum[2][j][c] + s_sum[3][j][c]));
    }
}

// out[worker][row][col] = sum over parts of partial[worker][part][row * row_step + col * col_step], 0 <= row < rows, 0 <= col < cols, in the
// order of the parts: eight shares, one a warp, then those.
__global__ void __launch_bounds__(256)
sum_parts_kernel(const float* __restrict__ partial, int64_t parts, int64_t part_size, int rows, int cols, int64_t row_step, int64_t col_step, bool rows_first,
                 float* __restrict__ out, int64_t ld, int64_t stride, int accumulate) {
    __shared__ float s_sum[8][32];
    const int64_t b = blockIdx.y;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 32 + (threadIdx.x & 31);
    const int w = threadIdx.x >> 5;
    const bool is = at < static_cast<int64_t>(rows) * cols;
    const int row = static_cast<int>(rows_first ? at % rows : at / cols), col = static_cast<int>(rows_first ? at / rows : at % cols);   // neighbours in `partial`
    const float* from = partial + b * parts * part_size + row * row_step + col * col_step;
    float sum = 0.0f;
    if (is)
#pragma unroll 4
        for (int64_t k = w; k < parts; k += 8) sum += PGT_LOAD(from[k * part_size]);
    s_sum[w][threadIdx.x & 31] = sum;
    __syncthreads();
    if (w == 0 && is) {
        float* o = out + b * stride + row * ld + col;
        sum = accumulate ? PGT_LOAD(*o) : 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += s_sum[k][threadIdx.x];
        PGT_STORE(*o, sum);
    }
}

// ---------------------------------------------------------------- scan
// softplus(v) = max(v, 0) + log(1 + e), e = exp(-|v|), with log(1 + e) = 2 artanh(s), s = e / (2 + e) <= 1/3: the series to s^13 is
// good to 2^-26 of it, for small e too, where a logarithm of 1 + e would lose e's digits.
__device__ __forceinline__ F2 softplus(F2 v) {
    float a, b;
    split(v, a, b);
    const F2 e = pair(ex2(-kLog2e * fabsf(a)), ex2(-kLog2e * fabsf(b)));
    float c, d;
    split(add(e, both(2.0f)), c, d);
    const F2 s = mul(e, pair(rcp(c), rcp(d))), q = mul(s, s);
    F2 p = both(2.0f / 13.0f);
    p = fma(p, q, both(2.0f / 11.0f));
    p = fma(p, q, both(2.0f / 9.0f));
    p = fma(p, q, both(2.0f / 7.0f));
    p = fma(p, q, both(2.0f / 5.0f));
    p = fma(p, q, both(2.0f / 3.0f));
    p = fma(p, q, both(2.0f));
    return fma(s, p, pair(fmaxf(a, 0.0f), fmaxf(b, 0.0f)));
}

// A channel's states lie in LANES neighbouring threads, P each, in pairs.  A block takes CH channels of one sequence at a time, or of a
// chunk of it (an item), in tiles of kScanTile tokens; the next tile is on its way while one is worked on.  Items are numbered by
// worker, channels, sequence and chunk, and a block has neighbours of them, so that it keeps its channels' rates as long as possible.
// The exponential unit is its floor: 16 states and the softplus and the gate take 20 exponentials or reciprocals per token and channel, 145 us
// for 32 x 700 tokens x 1300 channels at 1.9 GHz, where it takes 244 us (issue slots 55 % and the unit 58 % busy, the rest is waiting with 24 warps an SM;
// without tiles ahead 431 us).  Without states carried: 170 us with 4 and 8 states, 236 with 16, 526 with 32, 1197 with 64.  B and C of the tile
// on its way take 4 registers a thread at 16 states and 16 at 64; of the 80 that six blocks leave, 16 to 26 bytes are spilled to 16 states, 198
// to 32 and 280 to 64.
// A polynomial on the multiply-add pipes for an eighth of the exponentials: 3 % slower.  4 to 7 blocks an SM, two or four tokens
// side by side: within 10 % of one another.
constexpr int kScanThreads = 128;
constexpr int kScanTile = 16;                          // tokens; an eighth of the threads
constexpr int kScanBlocks = 6;                       // resident per SM

struct Item {
    int64_t b, sequence;                               // sequence: of all workers
    int s, d0, t0, t1, stop, chunk;                    // tokens t0 to t1, there to stop
    __device__ Item(uint32_t at, uint32_t sequences, int length, int chunk_size, uint32_t chunks, uint32_t tiles, int ch, const int32_t* lengths) {
        chunk = static_cast<int>(at % chunks);
        at /= chunks;
        s = static_cast<int>(at % sequences);
        at /= sequences;
        d0 = static_cast<int>(at % tiles) * ch;
        b = at / tiles;
        sequence = b * sequences + s;
        t0 = chunk * chunk_size;
        t1 = min(length, t0 + chunk_size);
        stop = max(t0, min(t1, tokens_of(lengths, b, static_cast<int>(sequences), s, length)));
    }
};

// A rate a as a power of two's exponent for a step of 1.  The least finite number stands for -inf, whose product with the step 0 (of tokens that only
// fill a tile) would be NaN.
__device__ __forceinline__ float exponent_of(float rate) {
    const float e = rate * kLog2e;
    return e == __int_as_float(0xff800000) ? -3.4028235e38f : e;
}
__device__ __forceinline__ F2 exponent_of(F2 rate) {
    float a, b;
    split(rate, a, b);
    return pair(exponent_of(a), exponent_of(b));
}

// P neighbouring fp32 numbers, `there` of them, in pairs.
template <int P>
__device__ __forceinline__ void load_states(const float* from, int there, bool wide, F2 (&v)[P / 2]) {
#pragma unroll
    for (int p = 0; p < P / 2; ++p) v[p] = both(0.0f);
    if (wide && there >= P) {
#pragma unroll
        for (int p = 0; p < P / 4; ++p) {
            float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (PGT_READ(from + 4 * p, 16)) f = *reinterpret_cast<const float4*>(from + 4 * p);
            v[2 * p] = pair(f.x, f.y);
            v[2 * p + 1] = pair(f.z, f.w);
        }
    } else {
#pragma unroll
        for (int p = 0; p < P / 2; ++p) v[p] = pair(2 * p < there ? PGT_LOAD(from[2 * p]) : 0.0f, 2 * p + 1 < there ? PGT_LOAD(from[2 * p + 1]) : 0.0f);
    }
}
template <int P>
__device__ __forceinline__ void store_states(float* to, int there, bool wide, const F2 (&v)[P / 2]) {
    float e[P];
#pragma unroll
    for (int p = 0; p < P / 2; ++p) split(v[p], e[2 * p], e[2 * p + 1]);
    if (wide && there >= P) {
#pragma unroll
        for (int p = 0; p < P / 4; ++p) PGT_STORE(*reinterpret_cast<float4*>(to + 4 * p), make_float4(e[4 * p], e[4 * p + 1], e[4 * p + 2], e[4 * p + 3]));
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (p < there) PGT_STORE(to[p], e[p]);
    }
}

// LOCAL: a chunk's own part: its last state from a zero one, and the sum of its steps.  Otherwise the chunk's results, from the
// state before it.
template <typename H, int P, int LANES, bool LOCAL>
__global__ void __launch_bounds__(kScanThreads, kScanBlocks)
scan_kernel(const pg_scan_args a, float* __restrict__ states, float* __restrict__ sums, int chunk, int chunks, int tiles, uint32_t items) {
    constexpr int N = P * LANES, CH = kScanThreads / LANES, A = LOCAL ? 2 : 3, kPieces = Rows<CH>::kPieces, kEach = kScanTile * N / kScanThreads;
    __shared__ __align__(16) uint4 s_in[2][A][kScanTile][kPieces];
    __shared__ __align__(16) float s_b[2][kScanTile][N], s_c[LOCAL ? 1 : 2][LOCAL ? 1 : kScanTile][LOCAL ? 1 : N];
    const int c = threadIdx.x / LANES, n0 = threadIdx.x % LANES * P, there = min(max(a.states - n0, 0), P);
    const uint32_t each = (items - 1) / gridDim.x + 1, begin = blockIdx.x * each, end = min(items, begin + each);      // (items + a block's are below 2^32)
    if (begin >= end) return;
    auto item_at = [&](uint32_t at) { return Item(at, a.sequences, a.length, chunk, chunks, tiles, CH, a.lengths); };
    // What is on its way: the tile at `tile` of the item `next`.
    uint32_t ahead = begin;
    Item next = item_at(begin);
    int tile = next.t0, buffer = 0;
    uint16_t rb[kEach], rc[LOCAL ? 1 : kEach];
    auto ask = [&](int to) {
        const int64_t first = static_cast<int64_t>(next.s) * a.length;
        const int count = min(kScanTile, next.stop - tile), n = min(CH, a.channels - next.d0);
        const Rows<CH> in[3] = {Rows<CH>(a.u, next.b, first + tile, next.d0), Rows<CH>(a.delta, next.b, first + tile, next.d0),
                                LOCAL || !a.z.data ? Rows<CH>() : Rows<CH>(a.z, next.b, first + tile, next.d0)};
#pragma unroll
        for (int k = 0; k < A; ++k) {
            if (k == 2 && !a.z.data) break;
            const int row = threadIdx.x / 8;           // eight threads a row
            if (row < count) in[k].ask(&s_in[to][k][row][0], row, threadIdx.x % 8, n);
        }
        const uint16_t* bb = static_cast<const uint16_t*>(a.b.data) + next.b * a.b.stride + (first + tile) * a.b.ld;
        const uint16_t* cc = static_cast<const uint16_t*>(a.c.data) + next.b * a.c.stride + (first + tile) * a.c.ld;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = i * kScanThreads + threadIdx.x, k = at / N, m = at % N;
            const bool is = k < count && m < a.states;
            rb[i] = is ? PGT_LOAD(bb[k * a.b.ld + m]) : 0;
            if constexpr (!LOCAL) rc[i] = is ? PGT_LOAD(cc[k * a.c.ld + m]) : 0;
        }
    };
    auto advance = [&] {                               // to the tile after the one on its way; false if that was the last
        tile += kScanTile;
        if (tile < next.stop) return true;
        if (++ahead >= end) return false;
        next = item_at(ahead);
        tile = next.t0;
        return true;
    };
    ask(0);
    bool more = true;
    int64_t of = -1;                                   // worker and channels whose rates are here
    F2 rate[P / 2];
    float bias = 0.0f, skip = 0.0f;
    const bool wide = a.states % 4 == 0;
    for (uint32_t at = begin; at < end; ++at) {
        const Item item = next;                        // (its first tile is what is on its way)
        const int d = item.d0 + c, mine = d < a.channels ? there : 0;
        const bool is = d < a.channels, idle = item.d0 + threadIdx.x / 32 * (32 / LANES) >= a.channels;      // idle: the whole warp
        if (of != item.b * tiles + item.d0 / CH) {
            of = item.b * tiles + item.d0 / CH;
            const float* rates = static_cast<const float*>(a.a.data) + item.b * a.a.stride + d * a.a.ld + n0;
            load_states<P>(rates, mine, reinterpret_cast<uintptr_t>(rates) % 16 == 0, rate);
#pragma unroll
            for (int p = 0; p < P / 2; ++p) rate[p] = exponent_of(rate[p]);
            bias = is && a.delta_bias ? PGT_LOAD(a.delta_bias[item.b * a.delta_bias_stride + d]) : 0.0f;
            skip = is && a.skip ? PGT_LOAD(a.skip[item.b * a.skip_stride + d]) : 0.0f;
        }
        const int64_t held = (item.sequence * a.channels + d) * a.states + n0, chunk_at = (item.sequence * chunks + item.chunk) * a.channels + d;
        F2 h[P / 2];
#pragma unroll
        for (int p = 0; p < P / 2; ++p) h[p] = both(0.0f);
        if constexpr (!LOCAL) {
            if (chunks > 1) load_states<P>(states + chunk_at * a.states + n0, mine, wide, h);
            else if (a.state) load_states<P>(a.state + held, mine, wide && reinterpret_cast<uintptr_t>(a.state) % 16 == 0, h);
        }
        float sum = 0.0f;
        const int64_t first = static_cast<int64_t>(item.s) * a.length;
        uint16_t* y = LOCAL ? nullptr : static_cast<uint16_t*>(a.y.data) + item.b * a.y.stride + first * a.y.ld + d;
        int t = item.t0;
        do {                                           // (an item without tokens has a tile all the same, an empty one)
            copies_wait();
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int k = i * kScanThreads + threadIdx.x;
                (&s_b[buffer][0][0])[k] = Elem<H>::up(rb[i]);
                if constexpr (!LOCAL) (&s_c[LOCAL ? 0 : buffer][0][0])[k] = Elem<H>::up(rc[i]);
            }
            __syncthreads();                           // this tile is there, and nobody reads the one before it
            more = more && advance();
            if (more) ask(buffer ^ 1);
            const Rows<CH> ru(a.u, item.b, first + t, item.d0), rd(a.delta, item.b, first + t, item.d0);
            const Rows<CH> rz = LOCAL || !a.z.data ? Rows<CH>() : Rows<CH>(a.z, item.b, first + t, item.d0);
            const int count = idle ? 0 : min(kScanTile, item.stop - t);
            constexpr int U = 2;                       // tokens whose steps and gates are computed side by side; those behind the last change nothing
            uint16_t* to = LOCAL ? nullptr : y + t * a.y.ld;
            for (int k0 = 0; k0 < count; k0 += U) {
                F2 in[U / 2], step[U / 2], v[U / 2];
#pragma unroll
                for (int u = 0; u < U; u += 2) {
                    auto two = [&](const Rows<CH>& r, int which) {
                        return pair(Elem<H>::up(r.get(s_in[buffer][which][k0 + u], k0 + u, c)), Elem<H>::up(r.get(s_in[buffer][which][k0 + u + 1], k0 + u + 1, c)));
                    };
                    in[u / 2] = two(ru, 0);
                    step[u / 2] = softplus(add(two(rd, 1), both(bias)));
                    if constexpr (!LOCAL) v[u / 2] = a.z.data ? activate<PG_ACT_SILU>(two(rz, A - 1)) : both(1.0f);
                    if (k0 + U > count) {
                        float i0, i1, d0, d1;
                        split(in[u / 2], i0, i1);
                        split(step[u / 2], d0, d1);
                        const bool first_is = k0 + u < count, second_is = k0 + u + 1 < count;
                        in[u / 2] = pair(first_is ? i0 : 0.0f, second_is ? i1 : 0.0f);
                        step[u / 2] = pair(first_is ? d0 : 0.0f, second_is ? d1 : 0.0f);
                    }
                }
                float outs[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float lo, hi, lo2, hi2;
                    split(step[u / 2], lo, hi);
                    split(mul(step[u / 2], in[u / 2]), lo2, hi2);
                    const F2 steps = both(u & 1 ? hi : lo), drive = both(u & 1 ? hi2 : lo2);
                    F2 out[2] = {both(0.0f), both(0.0f)};
                    const ulonglong2* bk = reinterpret_cast<const ulonglong2*>(&s_b[buffer][k0 + u][n0]);
                    const ulonglong2* ck = reinterpret_cast<const ulonglong2*>(&s_c[LOCAL ? 0 : buffer][LOCAL ? 0 : k0 + u][LOCAL ? 0 : n0]);
#pragma unroll
                    for (int p = 0; p < P / 4; ++p) {
                        const ulonglong2 bv = bk[p];
                        h[2 * p] = fma(ex2(mul(steps, rate[2 * p])), h[2 * p], mul(drive, F2{bv.x}));
                        h[2 * p + 1] = fma(ex2(mul(steps, rate[2 * p + 1])), h[2 * p + 1], mul(drive, F2{bv.y}));
                        if constexpr (!LOCAL) {
                            const ulonglong2 cv = ck[p];
                            out[0] = fma(h[2 * p], F2{cv.x}, out[0]);
                            out[1] = fma(h[2 * p + 1], F2{cv.y}, out[1]);
                        }
                    }
                    if constexpr (LOCAL) sum += u & 1 ? hi : lo;
                    else outs[u] = sum2(add(out[0], out[1]));
                }
                if constexpr (!LOCAL) {
#pragma unroll
                    for (int u = 0; u < U; u += 2) {
#pragma unroll
                        for (int o = 1; o < LANES; o <<= 1) {
                            outs[u] += __shfl_xor_sync(0xffffffffu, outs[u], o);
                            outs[u + 1] += __shfl_xor_sync(0xffffffffu, outs[u + 1], o);
                        }
                        const uint32_t w = Elem<H>::down2(mul(fma(both(skip), in[u / 2], pair(outs[u], outs[u + 1])), v[u / 2]));
                        if (is && n0 == 0) {
                            if (k0 + u < count) PGT_STORE(to[0], static_cast<uint16_t>(w & 0xffffu));
                            if (k0 + u + 1 < count) PGT_STORE(to[a.y.ld], static_cast<uint16_t>(w >> 16));
                        }
                        to += 2 * a.y.ld;
                    }
                }
            }
            t += kScanTile;
            buffer ^= 1;
        } while (t < item.stop);
        if constexpr (LOCAL) {
            store_states<P>(states + chunk_at * a.states + n0, mine, wide, h);
            if (is && n0 == 0) PGT_STORE(sums[chunk_at], sum);
        } else {
            if (is && n0 == 0)
                for (int k = item.stop; k < item.t1; ++k) PGT_STORE(y[k * a.y.ld], static_cast<uint16_t>(0));
            if (a.state_out && item.chunk == chunks - 1) store_states<P>(a.state_out + held, mine, wide && reinterpret_cast<uintptr_t>(a.state_out) % 16 == 0, h);
        }
    }
}

// From the chunks' own parts to the states before them, in place; carries: backwards, from the adjoints' own parts to what reaches
// a chunk from those behind it.  A chunk's decay is the square of 2 to half its exponent, at most 2^254: where a state grows beyond fp32's range over a
// chunk, what is zero before it stays zero.
__global__ void __launch_bounds__(128)
join_chunks_kernel(const pg_matrix rates, const float* __restrict__ state, float* __restrict__ states, float* __restrict__ carries, const float* __restrict__ sums,
                   int sequences, int channels, int n_states, int chunks) {
    const int64_t width = static_cast<int64_t>(channels) * n_states;
    const uint32_t blocks = static_cast<uint32_t>((width + 127) / 128);                  // of a sequence
    const int64_t sequence = blockIdx.x / blocks, b = sequence / sequences, at = static_cast<int64_t>(blockIdx.x % blocks) * 128 + threadIdx.x;
    if (at >= width) return;
    const int64_t d = at / n_states, n = at % n_states;
    const float rate = exponent_of(PGT_LOAD(static_cast<const float*>(rates.data)[b * rates.stride + d * rates.ld + n]));
    const int64_t first = sequence * chunks;
    constexpr int U = 8;                               // chunks whose numbers are on their way at once
    auto join = [&](float* v, float carry, int64_t from, int64_t step) {       // from chunk `from` on, forwards or backwards
        float* mine = v + (first + from) * width + at;
        const float* steps = sums + (first + from) * channels + d;
        const int64_t by = step * width, steps_by = step * channels;
        for (int left = chunks; left > 0; left -= U, mine += U * by, steps += U * steps_by) {
            float own[U], keep[U];
            auto load = [&](auto place) {
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    own[i] = PGT_LOAD(mine[place(i) * by]);
                    keep[i] = PGT_LOAD(steps[place(i) * steps_by]);
                }
            };
            if (left >= U) load([](int i) { return i; });
            else load([&](int i) { return min(i, left - 1); });
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const float sum = keep[i], half = 0.5f * (sum * rate);         // (0: no tokens, which keep everything whatever the rate is)
                keep[i] = ex2(sum == 0.0f ? 0.0f : half > 127.0f ? 127.0f : half);
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (i < left) PGT_STORE(mine[i * by], carry);
                carry = fmaf(keep[i] * carry, keep[i], own[i]);
            }
        }
    };
    join(states, state ? PGT_LOAD(state[sequence * width + at]) : 0.0f, 0, 1);
    if (carries) join(carries, 0.0f, chunks - 1, -1);
}

// ---------------------------------------------------------------- scan gradient
// Backwards along a chunk with g_t = exp(D_t+1 A) g_t+1 + C_t dv_t the gradient of h_t (dv: of y before the gate):
//     dC_t = sum over channels of dv_t h_t,  dB_t = sum over channels of g_t D_t u_t
//     du_t = D_t (g_t . B_t) + skip dv_t
//     dD_t = u_t (g_t . B_t) + sum over states of A e_t,   e_t = g_t h_t-1 exp(D_t A)
//     dA = sum over tokens of D_t e_t,  dskip = sum of dv_t u_t,  ddelta_t = dD_t sigmoid(delta_t + delta_bias)
// The states before groups of kGroup tokens are kept in shared memory on a way forward through the chunk; backwards the
// states of a group are computed once more.  32 x 700 tokens x 1300 channels x 16 states: 1042 us, 640 us with lengths drawn from 0 to 35;
// issue slots are 51 % busy with the twelve warps that registers and shared memory leave room for.  With 4, 8, 32 and 64 states: 816, 829, 1959
// and 5910 us.
constexpr int kGradStates = 8;                         // states of a thread
constexpr int kGroup = 4;
// Tokens of a chunk at most, and of a sequence that is a chunk of its own: at 16 states shared memory holds three blocks of 36 tokens, two of
// 52.  Chunks cost a pass over the tokens before.  Of 32 x 1300 channels 17 sequences of 40, 14 of 48, 12 of 54 and 9 of 72, alone: 1301,
// 1234, 2145 and 2059 us, in chunks: 1702, 1593, 1559 and 1436; a sequence of 8192 in chunks of 36, 40 and 20: 559, 812 and 636 us.
// All of these were measured with 16 states.  Others fit differently: to 8 states an SM holds two blocks of 36 tokens and one of 52, from 17 to 32
// three and two, above two of either.
constexpr int kGradChunk = 36, kGradAlone = 52;
constexpr int kGradBlocks = 3;                         // resident per SM

// Every token and channel of a chunk once, into shared memory ([token][channel]): the step, what reaches y before the gate, u as it is, and (s_dz)
// what dz is a multiple of.  A thread has channel d.  The chunk's tokens are the last `count` of `rows`; in place of those before them, and of channels
// that are not there: zeros.
template <typename H, int LANES>
__device__ __forceinline__ void prepare_chunk(const pg_scan_grad_args& a, int64_t b, int64_t at, int count, int rows, int d, float bias, float* s_step, float* s_dv,
                                              float* s_dz, uint16_t* s_u) {
    constexpr int CH = kScanThreads / LANES, U = 4;    // tokens on their way at once
    const bool gated = a.z.data != nullptr, is = d < a.channels;
    const int pad = rows - count;
    auto rows_of = [&](const pg_matrix& m) { return static_cast<const uint16_t*>(m.data) + b * m.stride + (at - pad) * m.ld + d; };
    const uint16_t *u = rows_of(a.u), *delta = rows_of(a.delta), *dy = rows_of(a.dy), *z = gated ? rows_of(a.z) : nullptr;
    for (int k0 = threadIdx.x / CH; k0 < rows; k0 += U * LANES) {
        uint16_t ru[U], rd[U], rg[U], rz[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int k = k0 + i * LANES;
            const bool there = is && k >= pad && k < rows;
            ru[i] = there ? PGT_LOAD(u[k * a.u.ld]) : 0;
            rd[i] = there ? PGT_LOAD(delta[k * a.delta.ld]) : 0;
            rg[i] = there ? PGT_LOAD(dy[k * a.dy.ld]) : 0;
            rz[i] = there && gated ? PGT_LOAD(z[k * a.z.ld]) : 0;
        }
#pragma unroll
        for (int i = 0; i < U; i += 2) {
            float step[2], dv[2], dz[2] = {0.0f, 0.0f};
            split(softplus(pair(Elem<H>::up(rd[i]) + bias, Elem<H>::up(rd[i + 1]) + bias)), step[0], step[1]);
            const F2 gy = pair(Elem<H>::up(rg[i]), Elem<H>::up(rg[i + 1]));
            split(gy, dv[0], dv[1]);
            if (gated) {
                const F2 v = pair(Elem<H>::up(rz[i]), Elem<H>::up(rz[i + 1])), sig = sigmoid_of(mul(v, both(-kLog2e)));
                split(mul(gy, mul(v, sig)), dv[0], dv[1]);
                split(mul(gy, mul(sig, fma(v, fma(sig, both(-1.0f), both(1.0f)), both(1.0f)))), dz[0], dz[1]);
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int k = k0 + (i + w) * LANES, to = k * CH + threadIdx.x % CH;
                if (k < rows) {
                    s_step[to] = is && k >= pad ? step[w] : 0.0f;
                    s_dv[to] = dv[w];
                    if (s_dz) s_dz[to] = dz[w];
                    s_u[to] = ru[i + w];
                }
            }
        }
    }
}

// fp32's largest number in place of +inf.
__device__ __forceinline__ F2 finite(F2 v) {
    float a, b;
    split(v, a, b);
    return pair(a > 3.4028235e38f ? 3.4028235e38f : a, b > 3.4028235e38f ? 3.4028235e38f : b);
}

// Own parts of a chunk for the way in both directions: the last state from a zero one, and the gradient that reaches the state before it.
template <typename H, int LANES>
__global__ void __launch_bounds__(kScanThreads, 4)
scan_grad_local_kernel(const pg_scan_grad_args a, float* __restrict__ states, float* __restrict__ carries, float* __restrict__ sums, int chunk, int chunks) {
    constexpr int P = kGradStates, N = P * LANES, CH = kScanThreads / LANES;
    constexpr int kTile = 20;                          // tokens in shared memory at once
    __shared__ float s_step[kTile * CH], s_dv[kTile * CH];
    __shared__ uint16_t s_u[kTile * CH];
    __shared__ __align__(16) float s_b[kTile * N], s_c[kTile * N];
    const int64_t sequence = blockIdx.x / chunks;
    const int at_chunk = static_cast<int>(blockIdx.x % chunks);
    const int64_t b = sequence / a.sequences;
    const int s = static_cast<int>(sequence % a.sequences);
    const int d = blockIdx.y * CH + threadIdx.x / LANES, c = threadIdx.x / LANES, n0 = threadIdx.x % LANES * P, step_d = blockIdx.y * CH + threadIdx.x % CH;
    const bool is = d < a.channels;
    const int there = is ? min(max(a.states - n0, 0), P) : 0;
    const int have = tokens_of(a.lengths, b, a.sequences, s, a.length);
    const int t0 = at_chunk * chunk, count = max(0, min(min(a.length, t0 + chunk), have) - t0);
    const float bias = step_d < a.channels && a.delta_bias ? PGT_LOAD(a.delta_bias[b * a.delta_bias_stride + step_d]) : 0.0f;
    const float* rates = static_cast<const float*>(a.a.data) + b * a.a.stride + static_cast<int64_t>(d) * a.a.ld + n0;
    F2 rate[P / 2], h[P / 2], g[P / 2], product[P / 2];
    load_states<P>(rates, there, reinterpret_cast<uintptr_t>(rates) % 16 == 0, rate);
#pragma unroll
    for (int p = 0; p < P / 2; ++p) {
        rate[p] = exponent_of(rate[p]);
        h[p] = g[p] = both(0.0f);
        product[p] = both(1.0f);
    }
    bool growing = false;                              // a rate of the warp's is positive: the product may leave fp32's range
#pragma unroll
    for (int p = 0; p < P / 2; ++p) {
        float lo, hi;
        split(rate[p], lo, hi);
        growing = growing || lo > 0.0f || hi > 0.0f;
    }
    growing = __any_sync(0xffffffffu, growing);
    float sum = 0.0f;
    for (int from = 0; from < count; from += kTile) {
        const int64_t at = static_cast<int64_t>(s) * a.length + t0 + from;
        const int rows = min(kTile, count - from);
        const uint16_t* bb = static_cast<const uint16_t*>(a.b.data) + b * a.b.stride + at * a.b.ld;
        const uint16_t* cc = static_cast<const uint16_t*>(a.c.data) + b * a.c.stride + at * a.c.ld;
        __syncthreads();                               // (shared memory is free again)
#pragma unroll 4
        for (int i = threadIdx.x; i < rows * N; i += kScanThreads) {
            const int k = i / N, n = i % N;
            s_b[i] = n < a.states ? Elem<H>::up(PGT_LOAD(bb[k * a.b.ld + n])) : 0.0f;
            s_c[i] = n < a.states ? Elem<H>::up(PGT_LOAD(cc[k * a.c.ld + n])) : 0.0f;
        }
        prepare_chunk<H, LANES>(a, b, at, rows, rows, step_d, bias, s_step, s_dv, nullptr, s_u);
        __syncthreads();
        auto walk = [&](auto grows) {
#pragma unroll 2
            for (int k = 0; k < rows; ++k) {
                const float step = s_step[k * CH + c];
                const F2 steps = both(step), drive = both(step * Elem<H>::up(s_u[k * CH + c])), dv = both(s_dv[k * CH + c]);
                const ulonglong2* bk = reinterpret_cast<const ulonglong2*>(s_b + k * N + n0);
                const ulonglong2* ck = reinterpret_cast<const ulonglong2*>(s_c + k * N + n0);
                sum += step;
#pragma unroll
                for (int q = 0; q < P / 4; ++q) {
                    const ulonglong2 bv = bk[q], cv = ck[q];
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int p = 2 * q + w;
                        const F2 keep = ex2(mul(steps, rate[p]));
                        h[p] = fma(keep, h[p], mul(drive, F2{w ? bv.y : bv.x}));
                        product[p] = mul(product[p], keep);
                        if constexpr (decltype(grows)::value) product[p] = finite(product[p]);          // (0 times it is 0)
                        g[p] = fma(product[p], mul(dv, F2{w ? cv.y : cv.x}), g[p]);
                    }
                }
            }
        };
        if (growing) walk(std::true_type{});
        else walk(std::false_type{});
    }
    const int64_t to = static_cast<int64_t>(blockIdx.x) * a.channels + d;
    store_states<P>(states + to * a.states + n0, there, a.states % 4 == 0, h);
    store_states<P>(carries + to * a.states + n0, there, a.states % 4 == 0, g);
    if (is && n0 == 0) PGT_STORE(sums[to], sum);
}

// Sums v[0 .. 2P) over the warp's lanes with the same lane % LANES; a lane keeps 2P / (32 / LANES) of them, at least one: those from
// the returned index on.
template <int LANES, int V>
__device__ __forceinline__ int scatter_sums(float (&v)[V]) {
    const int lane = threadIdx.x & 31;
    int at = 0, count = V;
#pragma unroll
    for (int o = 16; o >= LANES; o >>= 1) {
        if (count > 1) {
            count >>= 1;
            const bool high = lane & o;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                if (i >= count) break;
                const float give = high ? v[i] : v[count + i], keep = high ? v[count + i] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
            at += high ? count : 0;
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        }
    }
    return at;
}

// Shared memory of a block for chunks of `rows` tokens, a multiple of kGroup; in bytes from the start.
template <int LANES>
struct GradLayout {
    static constexpr int kN = kGradStates * LANES, kCh = kScanThreads / LANES;
    static constexpr int kRed = kScanThreads / 32 * kGroup * 2 * kN * 4, kSlot = kGradStates * kScanThreads * 4;
    static constexpr int kSlots = (kRed + kSlot - 1) / kSlot;          // groups whose states leave room for a group's sums
    int u, dv, dz, b, c, h, red, all;                  // steps first; u in 16 bits; what dz is a multiple of; b and c; states before groups
    __host__ __device__ explicit GradLayout(int rows) {
        dv = rows * kCh * 4;
        dz = dv + rows * kCh * 4;
        u = dz + rows * kCh * 4;
        b = (u + rows * kCh * 2 + 15) / 16 * 16;
        c = b + rows * kN * 4;
        h = c + rows * kN * 4;
        red = h + rows / kGroup * kSlot;
        all = red + kSlots * kRed;
    }
};

// 1 - exp(-v), v >= 0: the softplus' slope where its value is v.  (Below 1/2 by its series, to v^8 / 8!; the difference would lose v's digits.)
__device__ __forceinline__ float slope_of_step(float v) {
    float p = -1.0f / 40320.0f;
    p = fmaf(p, v, 1.0f / 5040.0f);
    p = fmaf(p, v, -1.0f / 720.0f);
    p = fmaf(p, v, 1.0f / 120.0f);
    p = fmaf(p, v, -1.0f / 24.0f);
    p = fmaf(p, v, 1.0f / 6.0f);
    p = fmaf(p, v, -0.5f);
    p = fmaf(p, v, 1.0f);
    return v < 0.5f ? p * v : 1.0f - ex2(-kLog2e * v);
}

// A block has one share of a worker's chunks and CH channels, whose dA, dskip and ddelta_bias stay in registers.
// parts[block's channels][worker][token][2 N]: what these channels add to dB and dC.
// partial[worker][share][channels][states + 2]: dA, then dskip and ddelta_bias.
template <typename H, int LANES>
__global__ void __launch_bounds__(kScanThreads, kGradBlocks)
scan_grad_kernel(const pg_scan_grad_args a, const float* __restrict__ states, const float* __restrict__ carries, float* __restrict__ parts,
                 float* __restrict__ partial, int chunk, int chunks, int shares) {
    constexpr int P = kGradStates, N = P * LANES, G = 32 / LANES, V = 2 * P, kKept = V / G > 1 ? V / G : 1, CH = kScanThreads / LANES, kWarps = kScanThreads / 32;
    extern __shared__ __align__(16) char s_all[];
    const int rows = (chunk + kGroup - 1) / kGroup * kGroup;
    const GradLayout<LANES> layout(rows);
    float* s_step = reinterpret_cast<float*>(s_all);   // [token][channel], as are the next three
    float* s_dv = reinterpret_cast<float*>(s_all + layout.dv);
    float* s_dz = reinterpret_cast<float*>(s_all + layout.dz);
    uint16_t* s_u = reinterpret_cast<uint16_t*>(s_all + layout.u);
    float* s_b = reinterpret_cast<float*>(s_all + layout.b);
    float* s_c = reinterpret_cast<float*>(s_all + layout.c);
    float4* s_h = reinterpret_cast<float4*>(s_all + layout.h);
    float* s_red = reinterpret_cast<float*>(s_all + layout.red);
    const int64_t b = blockIdx.x / shares;
    const int share = static_cast<int>(blockIdx.x % shares);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = threadIdx.x / LANES, n0 = threadIdx.x % LANES * P;
    const int d0 = blockIdx.y * CH, d = d0 + c;
    const bool is = d < a.channels;
    const int there = is ? min(max(a.states - n0, 0), P) : 0, step_d = d0 + threadIdx.x % CH;
    const float step_bias = step_d < a.channels && a.delta_bias ? PGT_LOAD(a.delta_bias[b * a.delta_bias_stride + step_d]) : 0.0f;
    const float skip = is && a.skip ? PGT_LOAD(a.skip[b * a.skip_stride + d]) : 0.0f;
    const bool wide = a.states % 4 == 0;
    F2 rate[P / 2], da[P / 2];
    {
        const float* rates = static_cast<const float*>(a.a.data) + b * a.a.stride + static_cast<int64_t>(d) * a.a.ld + n0;
        load_states<P>(rates, there, reinterpret_cast<uintptr_t>(rates) % 16 == 0, rate);
#pragma unroll
        for (int p = 0; p < P / 2; ++p) {
            rate[p] = exponent_of(rate[p]);
            da[p] = both(0.0f);
        }
    }
    float dskip = 0.0f, dbias = 0.0f;
    const int64_t tokens = static_cast<int64_t>(a.sequences) * a.length;
    float* my_parts = parts + (static_cast<int64_t>(blockIdx.y) * a.batch + b) * tokens * 2 * N;
    const bool gated = a.z.data != nullptr;
    for (int64_t item = share; item < static_cast<int64_t>(a.sequences) * chunks; item += shares) {
        const int s = static_cast<int>(item / chunks), at_chunk = static_cast<int>(item % chunks);
        const int64_t sequence = b * a.sequences + s, first = static_cast<int64_t>(s) * a.length;
        const int have = tokens_of(a.lengths, b, a.sequences, s, a.length);
        const int t0 = at_chunk * chunk, t1 = min(a.length, t0 + chunk), count = max(0, min(t1, have) - t0);
        // Token k is at place k + pad, so that the last group is full.  The places before the first token change nothing: their step is zero, their
        // decay 1, and what they would add to dA is 0 times what the first token adds; behind the last one it would be 0 times a
        // state that dA does not depend on, and that may not be finite.
        const int groups = (count + kGroup - 1) / kGroup, pad = groups * kGroup - count;
        const int64_t at = first + t0;
        __syncthreads();                               // (shared memory is free again)
        const uint16_t* bb = static_cast<const uint16_t*>(a.b.data) + b * a.b.stride + at * a.b.ld;
        const uint16_t* cc = static_cast<const uint16_t*>(a.c.data) + b * a.c.stride + at * a.c.ld;
#pragma unroll 4
        for (int i = threadIdx.x; i < groups * kGroup * N; i += kScanThreads) {
            const int k = i / N, n = i % N;
            const bool is_there = k >= pad && n < a.states;
            s_b[i] = is_there ? Elem<H>::up(PGT_LOAD(bb[(k - pad) * a.b.ld + n])) : 0.0f;
            s_c[i] = is_there ? Elem<H>::up(PGT_LOAD(cc[(k - pad) * a.c.ld + n])) : 0.0f;
        }
        F2 h[P / 2], g[P / 2];
        const int64_t state_at = (sequence * a.channels + d) * a.states + n0, chunk_at = ((sequence * chunks + at_chunk) * a.channels + d) * a.states + n0;
#pragma unroll
        for (int p = 0; p < P / 2; ++p) h[p] = g[p] = both(0.0f);
        if (chunks > 1) {
            load_states<P>(states + chunk_at, there, wide, h);
            load_states<P>(carries + chunk_at, there, wide, g);
        } else if (a.state) {
            load_states<P>(a.state + state_at, there, wide && reinterpret_cast<uintptr_t>(a.state) % 16 == 0, h);
        }
        prepare_chunk<H, LANES>(a, b, at, count, groups * kGroup, step_d, step_bias, s_step, s_dv, s_dz, s_u);
        __syncthreads();
        for (int group = 0; group < groups; ++group) { // forward
#pragma unroll
            for (int q = 0; q < P / 4; ++q) {
                float4 f;
                split(h[2 * q], f.x, f.y);
                split(h[2 * q + 1], f.z, f.w);
                s_h[(group * (P / 4) + q) * kScanThreads + threadIdx.x] = f;
            }
            if (group + 1 == groups) break;
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
                const int k = group * kGroup + i;
                const float step = s_step[k * CH + c], in = Elem<H>::up(s_u[k * CH + c]);
                const F2 steps = both(step), drive = both(step * in);
                const ulonglong2* bk = reinterpret_cast<const ulonglong2*>(s_b + k * N + n0);
#pragma unroll
                for (int q = 0; q < P / 4; ++q) {
                    const ulonglong2 bv = bk[q];
                    h[2 * q] = fma(ex2(mul(steps, rate[2 * q])), h[2 * q], mul(drive, F2{bv.x}));
                    h[2 * q + 1] = fma(ex2(mul(steps, rate[2 * q + 1])), h[2 * q + 1], mul(drive, F2{bv.y}));
                }
            }
        }
        for (int group = groups - 1; group >= 0; --group) {
            F2 before[kGroup][P / 2], keep[kGroup][P / 2];
            float step[kGroup], in[kGroup], dv[kGroup], to_z[kGroup];
#pragma unroll
            for (int q = 0; q < P / 4; ++q) {
                const float4 f = s_h[(group * (P / 4) + q) * kScanThreads + threadIdx.x];
                h[2 * q] = pair(f.x, f.y);
                h[2 * q + 1] = pair(f.z, f.w);
            }
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
                const int k = group * kGroup + i;
                step[i] = s_step[k * CH + c];
                in[i] = Elem<H>::up(s_u[k * CH + c]);
                dv[i] = s_dv[k * CH + c];
                const F2 steps = both(step[i]), drive = both(step[i] * in[i]);
                const ulonglong2* bk = reinterpret_cast<const ulonglong2*>(s_b + k * N + n0);
                const ulonglong2* ck = reinterpret_cast<const ulonglong2*>(s_c + k * N + n0);
                F2 out = both(0.0f);
#pragma unroll
                for (int q = 0; q < P / 4; ++q) {
                    const ulonglong2 bv = bk[q], cv = ck[q];
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int p = 2 * q + w;
                        before[i][p] = h[p];
                        keep[i][p] = ex2(mul(steps, rate[p]));
                        h[p] = fma(keep[i][p], h[p], mul(drive, F2{w ? bv.y : bv.x}));
                        out = fma(h[p], F2{w ? cv.y : cv.x}, out);
                    }
                }
                if (gated) {
                    float v = sum2(out);
#pragma unroll
                    for (int o = 1; o < LANES; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                    to_z[i] = s_dz[k * CH + c] * fmaf(skip, in[i], v);
                }
            }
            // The sums go where the states of the groups behind this one were, or behind all states.
            constexpr int kSlots = GradLayout<LANES>::kSlots;
            float* reds = group + kSlots < groups ? reinterpret_cast<float*>(s_h + (group + 1) * (P / 4) * kScanThreads) : s_red + (groups - 1 - group) * (GradLayout<LANES>::kRed / 4);
            float* red = reds + warp * kGroup * 2 * N;
#pragma unroll
            for (int i = kGroup - 1; i >= 0; --i) {
                const int k = group * kGroup + i;
                const F2 steps = both(step[i]), drive = both(step[i] * in[i]), dvs = both(dv[i]);
                const ulonglong2* bk = reinterpret_cast<const ulonglong2*>(s_b + k * N + n0);
                const ulonglong2* ck = reinterpret_cast<const ulonglong2*>(s_c + k * N + n0);
                F2 drives = both(0.0f), slopes = both(0.0f);
                float v[V];
#pragma unroll
                for (int q = 0; q < P / 4; ++q) {
                    const ulonglong2 bv = bk[q], cv = ck[q];
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int p = 2 * q + w;
                        g[p] = fma(dvs, F2{w ? cv.y : cv.x}, g[p]);
                        split(mul(g[p], drive), v[2 * p], v[2 * p + 1]);
                        split(mul(dvs, i + 1 < kGroup ? before[i + 1 < kGroup ? i + 1 : i][p] : h[p]), v[P + 2 * p], v[P + 2 * p + 1]);
                        drives = fma(g[p], F2{w ? bv.y : bv.x}, drives);
                        g[p] = mul(g[p], keep[i][p]);
                        const F2 e = mul(g[p], before[i][p]);
                        slopes = fma(e, rate[p], slopes);
                        da[p] = fma(e, steps, da[p]);
                    }
                }
                float to_drive = sum2(drives), to_step = sum2(slopes);
#pragma unroll
                for (int o = 1; o < LANES; o <<= 1) {
                    to_drive += __shfl_xor_sync(0xffffffffu, to_drive, o);
                    to_step += __shfl_xor_sync(0xffffffffu, to_step, o);
                }
                if (n0 == 0) {                         // what the outputs are made of, in the places of what is used up
                    s_dv[k * CH + c] = fmaf(to_drive, step[i], skip * dv[i]);
                    s_step[k * CH + c] = fmaf(to_drive, in[i], to_step * kLn2) * slope_of_step(step[i]);
                    if (gated) s_dz[k * CH + c] = to_z[i];
                    dskip = fmaf(dv[i], in[i], dskip);
                }
                const int from = scatter_sums<LANES>(v);
#pragma unroll
                for (int w = 0; w < kKept; ++w)
                    if (V >= G || (lane & (G / V * LANES - 1)) < LANES)   // (of lanes that hold the same sum the first)
                        red[i * 2 * N + (from + w < P ? n0 + from + w : N + n0 + from + w - P)] = v[w];
            }
            __syncthreads();                           // (what the group before this one left is read by now)
            for (int i = threadIdx.x; i < kGroup * 2 * N; i += kScanThreads) {
                const int k = group * kGroup + i / (2 * N) - pad;
                const float* from = reds + i;
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) v += from[w * kGroup * 2 * N];
                if (k >= 0) PGT_STORE(my_parts[(at + k) * 2 * N + i % (2 * N)], v);
            }
            if constexpr (kSlots > 1) __syncthreads(); // (the next group's sums go over these)
        }
        __syncthreads();
        if (step_d < a.channels) {                     // outputs, rows behind the last token as zeros
            auto rows_of = [&](const pg_matrix& m) { return static_cast<uint16_t*>(m.data) + b * m.stride + (at + threadIdx.x / CH) * m.ld + step_d; };
            uint16_t *du = rows_of(a.du), *ddelta = rows_of(a.ddelta), *dz = gated ? rows_of(a.dz) : nullptr;
#pragma unroll 2
            for (int k = threadIdx.x / CH; k < t1 - t0; k += LANES) {
                const int s_at = (k + pad) * CH + threadIdx.x % CH;
                const bool is_there = k < count;
                const float dd = is_there ? s_step[s_at] : 0.0f;
                dbias += dd;
                PGT_STORE(du[0], Elem<H>::down(is_there ? s_dv[s_at] : 0.0f));
                PGT_STORE(ddelta[0], Elem<H>::down(dd));
                if (gated) PGT_STORE(dz[0], Elem<H>::down(is_there ? s_dz[s_at] : 0.0f));
                du += LANES * a.du.ld;
                ddelta += LANES * a.ddelta.ld;
                if (gated) dz += LANES * a.dz.ld;
            }
        }
        for (int i = count * 2 * N + threadIdx.x; i < (t1 - t0) * 2 * N; i += kScanThreads) PGT_STORE(my_parts[at * 2 * N + i], 0.0f);
    }
    __syncthreads();
    s_step[threadIdx.x] = dbias;                       // of channel threadIdx.x % CH
    __syncthreads();
    dbias = 0.0f;
#pragma unroll
    for (int i = 0; i < LANES; ++i) dbias += s_step[i * CH + c];
    float* mine = partial + (static_cast<int64_t>(blockIdx.x) * a.channels + d) * (a.states + 2);
    store_states<P>(mine + n0, there, false, da);
    if (is && n0 == 0) {
        PGT_STORE(mine[a.states], dskip);
        PGT_STORE(mine[a.states + 1], dbias);
    }
}

// dB and dC: the channel blocks' parts added up in order.
template <typename H>
__global__ void __launch_bounds__(256)
sum_bc_kernel(const pg_scan_grad_args a, const float* __restrict__ parts, int blocks, int n_padded) {
    const int64_t tokens = static_cast<int64_t>(a.sequences) * a.length, all = a.batch * tokens * 2 * n_padded;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= all) return;
    const int n = static_cast<int>(i % (2 * n_padded));
    const int64_t row = i / (2 * n_padded), b = row / tokens, t = row % tokens;
    float v = 0.0f;
#pragma unroll 4
    for (int k = 0; k < blocks; ++k) v += PGT_LOAD(parts[k * all + i]);
    const pg_matrix& m = n < n_padded ? a.db : a.dc;
    const int to = n < n_padded ? n : n - n_padded;
    if (to < a.states) PGT_STORE((static_cast<uint16_t*>(m.data) + b * m.stride + t * m.ld)[to], Elem<H>::down(v));
}

// ---------------------------------------------------------------- host
int current_device() {
    int d = 0;
    return cudaGetDevice(&d) == cudaSuccess ? d : -1;
}
constexpr int64_t kMaxBlocks = (int64_t{1} << 31) - 1;
constexpr int kMaxChannels = 1 << 19;
constexpr int kMaxStates = 64;

// Sizes of a batch of sequences; the product of sequences and length is the number of a worker's tokens.
bool sequence_sizes_ok(int64_t dtype, int64_t batch, int64_t sequences, int64_t length, int64_t channels) {
    return sizes_ok(dtype, batch, length, channels, 1) && sequences >= 0 && sequences <= kMaxDim && sequences * length <= kMaxDim;
}
bool array_ok(const void* p, uintptr_t align, int64_t count, int dev) { return count == 0 || device_pointer(p, align, dev); }
Operands& span(Operands& o, const void* p, int64_t bytes, bool output) {
    const pg_matrix m = {const_cast<void*>(p), bytes, 0};
    return output ? o.output(m, 1, 1, bytes, 1) : o.input(m, 1, 1, bytes, 1);
}

template <typename F>
void with_taps(int taps, F&& f) {
    using std::integral_constant;
    if (taps == 2) f(integral_constant<int, 2>{});
    else if (taps == 3) f(integral_constant<int, 3>{});
    else f(integral_constant<int, 4>{});
}
// Calls f with 2 if all rows of the matrix start on 4-byte boundaries, else with 1.
template <typename F>
void with_two(const pg_matrix& m, int64_t batch, F&& f) {
    using std::integral_constant;
    const uint64_t bits = reinterpret_cast<uintptr_t>(m.data) | static_cast<uint64_t>(m.ld) * 2 | (batch > 1 ? static_cast<uint64_t>(m.stride) * 2 : 0);
    if (bits % 4 == 0) f(integral_constant<int, 2>{});
    else f(integral_constant<int, 1>{});
}
template <typename F>
void with_kind(int dtype, F&& f) {
    if (dtype == PG_BF16) f(__nv_bfloat16{});
    else f(__half{});
}

int conv_strips(int channels) { return (channels + kStrip - 1) / kStrip; }
// Tokens of a run: kRun, fewer where there would not be 32 runs for every SM.  (Shorter runs read more of what is before and behind them.)
int conv_run(int64_t sequences, int64_t length, int64_t strips) {
    int run = static_cast<int>(std::min<int64_t>(kRun, std::max<int64_t>(length, 1)));
    while (run > 8 && sequences * ((length + run - 1) / run) * strips < int64_t{kSMs} * 32) run = (run + 1) / 2;
    return run;
}
// Blocks that share a worker's runs in the gradient: one for every four runs, to 1024 (a block's sums are small beside what its runs read).
int conv_parts(const pg_conv_grad_args& a, int runs) {
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(1024, (int64_t{a.sequences} * runs + 3) / 4)));
}

struct ScanPlan { int chunk, chunks, tiles; int64_t items; };
// Chunks of a sequence for the forward scan.  With chunks every token is gone through twice, so there are some only where they make the
// work of a block a third or less of a sequence.
ScanPlan scan_plan(const pg_scan_args& a, int lanes) {
    const int tiles = (a.channels + kScanThreads / lanes - 1) / (kScanThreads / lanes);
    const int64_t whole = std::max<int64_t>(1, int64_t{a.batch} * a.sequences * tiles), length = std::max(a.length, 1);
    int64_t chunks = std::min<int64_t>(int64_t{kSMs} * kScanBlocks / whole, length / 32);
    if (chunks < 3) chunks = 1;
    const int64_t chunk = (length + chunks - 1) / chunks;
    chunks = (length + chunk - 1) / chunk;
    return {static_cast<int>(chunk), static_cast<int>(chunks), tiles, int64_t{a.batch} * a.sequences * tiles * chunks};
}
template <typename Args>
int64_t join_blocks(const Args& a) { return int64_t{a.batch} * a.sequences * ((int64_t{a.channels} * a.states + 127) / 128); }
int lanes_of(int states, int per_thread) {
    int lanes = 1;
    while (lanes * per_thread < states) lanes *= 2;
    return lanes;
}
struct GradPlan { int chunk, chunks, lanes, shares; int64_t blocks; size_t states, sums, parts, partial; };
GradPlan grad_plan(const pg_scan_grad_args& a) {
    GradPlan p = {};
    p.lanes = lanes_of(a.states, kGradStates);
    const int64_t length = std::max(a.length, 1);
    p.chunks = length <= kGradAlone ? 1 : static_cast<int>((length + kGradChunk - 1) / kGradChunk);
    p.chunk = static_cast<int>((length + p.chunks - 1) / p.chunks);
    p.blocks = (int64_t{a.channels} * p.lanes + kScanThreads - 1) / kScanThreads;
    const int64_t items = int64_t{a.sequences} * p.chunks;
    // Shares of a worker's chunks: those whose waves of blocks take the fewest steps of a chunk, a block's start and end counted as a third of one.
    // At most 64, so that one sequence of 8192 and few channels leaves SMs idle: 154 us with 64 channels, 157 with 128 (559 with 1300).
    double least = 0.0;
    p.shares = 1;
    for (int64_t s = 1; s <= std::min<int64_t>(items, 64); ++s) {
        const double waves = static_cast<double>((p.blocks * a.batch * s + kSMs * kGradBlocks - 1) / (kSMs * kGradBlocks));
        const double cost = waves * (static_cast<double>((items + s - 1) / s) + 0.33);
        if (s == 1 || cost < least) {
            least = cost;
            p.shares = static_cast<int>(s);
        }
    }
    const size_t all = static_cast<size_t>(a.batch) * items;
    auto round = [](size_t n) { return (n + 255) / 256 * 256; };
    p.states = p.chunks > 1 ? round(sizeof(float) * all * a.channels * a.states) : 0;         // and as much for the carries
    p.sums = p.chunks > 1 ? round(sizeof(float) * all * a.channels) : 0;
    p.parts = round(sizeof(float) * p.blocks * a.batch * static_cast<size_t>(a.sequences) * a.length * 2 * kGradStates * p.lanes);
    p.partial = round(sizeof(float) * static_cast<size_t>(a.batch) * p.shares * a.channels * (a.states + 2));
    return p;
}

int conv_check(int dtype, int activation, int batch, int sequences, int length, int channels, int width) {
    if (!sequence_sizes_ok(dtype, batch, sequences, length, channels) || width < 2 || width > 4) return PG_ERR_INVALID;
    if (activation != PG_ACT_NONE && activation != PG_ACT_SILU) return PG_ERR_INVALID;
    return channels > kMaxChannels ? PG_ERR_TOO_LARGE : PG_OK;
}

template <typename Args>
int scan_check(const Args& a) {
    if (!sequence_sizes_ok(a.dtype, a.batch, a.sequences, a.length, a.channels) || a.states < 1) return PG_ERR_INVALID;
    return a.states > kMaxStates || a.channels > kMaxChannels ? PG_ERR_TOO_LARGE : PG_OK;
}
template <typename Args>
bool scan_inputs_ok(const Args& a, int dev) {
    const int64_t tokens = int64_t{a.sequences} * a.length, held = int64_t{a.batch} * a.sequences;
    if (!matrix_ok(a.u, a.batch, tokens, a.channels, 2, false, dev) || !matrix_ok(a.delta, a.batch, tokens, a.channels, 2, false, dev)) return false;
    if (!matrix_ok(a.b, a.batch, tokens, a.states, 2, false, dev) || !matrix_ok(a.c, a.batch, tokens, a.states, 2, false, dev)) return false;
    if (!matrix_ok(a.a, a.batch, a.channels, a.states, 4, false, dev)) return false;
    if (a.z.data && !matrix_ok(a.z, a.batch, tokens, a.channels, 2, false, dev)) return false;
    if (a.delta_bias && !vector_ok(a.delta_bias, a.delta_bias_stride, a.batch, a.channels, false, dev)) return false;
    if (a.skip && !vector_ok(a.skip, a.skip_stride, a.batch, a.channels, false, dev)) return false;
    if (a.lengths && !array_ok(a.lengths, 4, held, dev)) return false;
    return !a.state || array_ok(a.state, 4, held, dev);
}
template <typename Args>
void scan_inputs(Operands& o, const Args& a) {
    const int64_t tokens = int64_t{a.sequences} * a.length, held = int64_t{a.batch} * a.sequences;
    o.input(a.u, a.batch, tokens, a.channels, 2).input(a.delta, a.batch, tokens, a.channels, 2).input(a.z, a.batch, tokens, a.channels, 2);
    o.input(a.b, a.batch, tokens, a.states, 2).input(a.c, a.batch, tokens, a.states, 2).input(a.a, a.batch, a.channels, a.states, 4);
    o.input(a.delta_bias, a.delta_bias_stride, a.batch, a.channels).input(a.skip, a.skip_stride, a.batch, a.channels);
    span(o, a.lengths, held * 4, false);
    span(o, a.state, held * a.channels * a.states * 4, false);
}

}  // namespace

int take_sequence_errors(unsigned& value, cudaStream_t st) {
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

int pg_causal_conv(const pg_conv_args* args, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_conv_args& a = *args;
    const int dev = current_device(), rc = conv_check(a.dtype, a.activation, a.batch, a.sequences, a.length, a.channels, a.width);
    if (rc == PG_ERR_INVALID) return rc;
    const int64_t tokens = int64_t{a.sequences} * a.length, sequences = int64_t{a.batch} * a.sequences, held = sequences * (a.width - 1) * a.channels;
    if (!matrix_ok(a.x, a.batch, tokens, a.channels, 2, false, dev) || !matrix_ok(a.y, a.batch, tokens, a.channels, 2, true, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.weight, a.batch, a.channels, a.width, 4, false, dev)) return PG_ERR_INVALID;
    if (a.bias && !vector_ok(a.bias, a.bias_stride, a.batch, a.channels, false, dev)) return PG_ERR_INVALID;
    if ((a.lengths && !array_ok(a.lengths, 4, sequences, dev)) || (a.state && !array_ok(a.state, 2, held, dev)) ||
        (a.state_out && !array_ok(a.state_out, 2, held, dev)))
        return PG_ERR_INVALID;
    const int strips = conv_strips(a.channels), run = conv_run(sequences, a.length, strips);
    const int runs = std::max(1, (a.length + run - 1) / run);
    const int64_t blocks = (sequences * runs + 3) / 4;
    if (rc != PG_OK || blocks > kMaxBlocks) return PG_ERR_TOO_LARGE;
    if (sequences == 0 || (a.length == 0 && !a.state_out)) return PG_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Operands operands;
    operands.output(a.y, a.batch, tokens, a.channels, 2);
    span(operands, a.state_out, held * 2, true);
    operands.input(a.x, a.batch, tokens, a.channels, 2).input(a.weight, a.batch, a.channels, a.width, 4).input(a.bias, a.bias_stride, a.batch, a.channels);
    span(operands, a.lengths, sequences * 4, false);
    span(operands, a.state, held * 2, false);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    with_kind(a.dtype, [&](auto h) {
        with_two(a.y, a.batch, [&](auto two) {
            with_taps(a.width, [&](auto taps) {
                using H = decltype(h);
                constexpr int W = decltype(two)::value, TAPS = decltype(taps)::value;
                const dim3 grid(static_cast<unsigned>(blocks), strips);
                if (a.activation == PG_ACT_SILU) conv_kernel<H, W, TAPS, PG_ACT_SILU><<<grid, kConvThreads, 0, st>>>(a, run, runs);
                else conv_kernel<H, W, TAPS, PG_ACT_NONE><<<grid, kConvThreads, 0, st>>>(a, run, runs);
            });
        });
    });
    return launch_status();
}

int pg_causal_conv_grad_workspace_bytes(const pg_conv_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out) return PG_ERR_INVALID;
    const pg_conv_grad_args& a = *args;
    const int rc = conv_check(a.dtype, a.activation, a.batch, a.sequences, a.length, a.channels, a.width);
    if (rc != PG_OK) return rc;
    const int run = conv_run(int64_t{a.batch} * a.sequences, a.length, conv_strips(a.channels));
    *bytes_out = sizeof(float) * static_cast<size_t>(a.batch) * conv_parts(a, std::max(1, (a.length + run - 1) / run)) * (a.width + 1) * a.channels;
    return PG_OK;
}

int pg_causal_conv_grad(const pg_conv_grad_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_conv_grad_args& a = *args;
    size_t need = 0;
    const int dev = current_device(), rc = pg_causal_conv_grad_workspace_bytes(args, &need);
    if (rc != PG_OK) return rc;
    const int64_t tokens = int64_t{a.sequences} * a.length, sequences = int64_t{a.batch} * a.sequences, held = sequences * (a.width - 1) * a.channels;
    for (const pg_matrix* m : {&a.x, &a.dy})
        if (!matrix_ok(*m, a.batch, tokens, a.channels, 2, false, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.dx, a.batch, tokens, a.channels, 2, true, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.weight, a.batch, a.channels, a.width, 4, false, dev)) return PG_ERR_INVALID;
    if (a.dweight.data && !matrix_ok(a.dweight, a.batch, a.channels, a.width, 4, true, dev)) return PG_ERR_INVALID;
    if (a.bias && !vector_ok(a.bias, a.bias_stride, a.batch, a.channels, false, dev)) return PG_ERR_INVALID;
    if (a.dbias && !vector_ok(a.dbias, a.dbias_stride, a.batch, a.channels, true, dev)) return PG_ERR_INVALID;
    if ((a.lengths && !array_ok(a.lengths, 4, sequences, dev)) || (a.state && !array_ok(a.state, 2, held, dev))) return PG_ERR_INVALID;
    if (need > 0 && (workspace_bytes < need || !device_pointer(workspace, 16, dev))) return PG_ERR_WORKSPACE;
    if (a.batch == 0) return PG_OK;
    const int strips = conv_strips(a.channels), run = conv_run(sequences, a.length, strips);
    const int runs = std::max(1, (a.length + run - 1) / run), parts = conv_parts(a, runs);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    float* partial = static_cast<float*>(workspace);
    Operands operands;
    operands.output(a.dx, a.batch, tokens, a.channels, 2).output(a.dweight, a.batch, a.channels, a.width, 4).output(a.dbias, a.dbias_stride, a.batch, a.channels);
    span(operands, workspace, need, true);
    operands.input(a.x, a.batch, tokens, a.channels, 2).input(a.dy, a.batch, tokens, a.channels, 2).input(a.weight, a.batch, a.channels, a.width, 4);
    operands.input(a.bias, a.bias_stride, a.batch, a.channels);
    span(operands, a.lengths, sequences * 4, false);
    span(operands, a.state, held * 2, false);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    with_kind(a.dtype, [&](auto h) {
        with_two(a.dx, a.batch, [&](auto two) {
            with_taps(a.width, [&](auto taps) {
                using H = decltype(h);
                constexpr int W = decltype(two)::value, TAPS = decltype(taps)::value;
                const dim3 grid(a.batch * parts, strips);
                if (a.activation == PG_ACT_SILU) conv_grad_kernel<H, W, TAPS, PG_ACT_SILU><<<grid, kConvThreads, 0, st>>>(a, partial, run, runs, parts);
                else conv_grad_kernel<H, W, TAPS, PG_ACT_NONE><<<grid, kConvThreads, 0, st>>>(a, partial, run, runs, parts);
            });
        });
    });
    const int64_t size = int64_t{a.width + 1} * a.channels;
    if (a.dweight.data)
        sum_parts_kernel<<<dim3(static_cast<unsigned>((int64_t{a.channels} * a.width + 31) / 32), a.batch), 256, 0, st>>>(
            partial, parts, size, a.channels, a.width, 1, a.channels, true, static_cast<float*>(a.dweight.data), a.dweight.ld, a.dweight.stride, a.accumulate);
    if (a.dbias)
        sum_parts_kernel<<<dim3((a.channels + 31) / 32, a.batch), 256, 0, st>>>(partial + int64_t{a.width} * a.channels, parts, size, 1, a.channels, 0, 1, false,
                                                                                a.dbias, a.channels, a.dbias_stride, a.accumulate);
    return launch_status();
}

int pg_selective_scan_workspace_bytes(const pg_scan_args* args, size_t* bytes_out) {
    if (!args || !bytes_out) return PG_ERR_INVALID;
    const pg_scan_args& a = *args;
    const int rc = scan_check(a);
    if (rc != PG_OK) return rc;
    const ScanPlan p = scan_plan(a, lanes_of(a.states, 16));
    *bytes_out = p.chunks > 1 ? sizeof(float) * static_cast<size_t>(a.batch) * a.sequences * p.chunks * a.channels * (a.states + 1) : 0;
    return PG_OK;
}

int pg_selective_scan(const pg_scan_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_scan_args& a = *args;
    size_t need = 0;
    const int dev = current_device(), rc = pg_selective_scan_workspace_bytes(args, &need);
    if (rc != PG_OK) return rc;
    const int64_t tokens = int64_t{a.sequences} * a.length, sequences = int64_t{a.batch} * a.sequences, held = sequences * a.channels * a.states;
    if (!scan_inputs_ok(a, dev) || !matrix_ok(a.y, a.batch, tokens, a.channels, 2, true, dev)) return PG_ERR_INVALID;
    if (a.state_out && !array_ok(a.state_out, 4, held, dev)) return PG_ERR_INVALID;
    if (need > 0 && (workspace_bytes < need || !device_pointer(workspace, 16, dev))) return PG_ERR_WORKSPACE;
    const int lanes = lanes_of(a.states, 16);
    const ScanPlan p = scan_plan(a, lanes);
    if (p.items > kMaxBlocks || (p.chunks > 1 && join_blocks(a) > kMaxBlocks)) return PG_ERR_TOO_LARGE;
    if (sequences == 0 || (a.length == 0 && !a.state_out)) return PG_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Operands operands;
    operands.output(a.y, a.batch, tokens, a.channels, 2);
    span(operands, a.state_out, held * 4, true);
    span(operands, need > 0 ? workspace : nullptr, need, true);
    scan_inputs(operands, a);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    float* states = static_cast<float*>(workspace);
    float* sums = states + sequences * p.chunks * a.channels * a.states;
    with_kind(a.dtype, [&](auto h) {
        using H = decltype(h);
        auto launch = [&](auto per, auto lane) {
            constexpr int P = decltype(per)::value, LANES = decltype(lane)::value;
            const unsigned grid = static_cast<unsigned>(std::min<int64_t>(p.items, int64_t{kSMs} * kScanBlocks));
            if (p.chunks > 1) {
                scan_kernel<H, P, LANES, true><<<grid, kScanThreads, 0, st>>>(a, states, sums, p.chunk, p.chunks, p.tiles, static_cast<uint32_t>(p.items));
                join_chunks_kernel<<<static_cast<unsigned>(join_blocks(a)), 128, 0, st>>>(
                    a.a, a.state, states, nullptr, sums, a.sequences, a.channels, a.states, p.chunks);
            }
            scan_kernel<H, P, LANES, false><<<grid, kScanThreads, 0, st>>>(a, states, sums, p.chunk, p.chunks, p.tiles, static_cast<uint32_t>(p.items));
        };
        using std::integral_constant;
        if (a.states <= 8) launch(integral_constant<int, 8>{}, integral_constant<int, 1>{});
        else if (lanes == 1) launch(integral_constant<int, 16>{}, integral_constant<int, 1>{});
        else if (lanes == 2) launch(integral_constant<int, 16>{}, integral_constant<int, 2>{});
        else launch(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    });
    return launch_status();
}

int pg_selective_scan_grad_workspace_bytes(const pg_scan_grad_args* args, size_t* bytes_out) {
    if (!args || !bytes_out) return PG_ERR_INVALID;
    const int rc = scan_check(*args);
    if (rc != PG_OK) return rc;
    const GradPlan p = grad_plan(*args);
    *bytes_out = 2 * p.states + p.sums + p.parts + p.partial;
    return PG_OK;
}

int pg_selective_scan_grad(const pg_scan_grad_args* args, void* workspace, size_t workspace_bytes, void* stream) {
    if (!args) return PG_ERR_INVALID;
    const pg_scan_grad_args& a = *args;
    size_t need = 0;
    const int dev = current_device(), rc = pg_selective_scan_grad_workspace_bytes(args, &need);
    if (rc != PG_OK) return rc;
    const int64_t tokens = int64_t{a.sequences} * a.length, sequences = int64_t{a.batch} * a.sequences;
    if (!scan_inputs_ok(a, dev) || !matrix_ok(a.dy, a.batch, tokens, a.channels, 2, false, dev)) return PG_ERR_INVALID;
    for (const pg_matrix* m : {&a.du, &a.ddelta})
        if (!matrix_ok(*m, a.batch, tokens, a.channels, 2, true, dev)) return PG_ERR_INVALID;
    if (a.z.data && !matrix_ok(a.dz, a.batch, tokens, a.channels, 2, true, dev)) return PG_ERR_INVALID;
    for (const pg_matrix* m : {&a.db, &a.dc})
        if (!matrix_ok(*m, a.batch, tokens, a.states, 2, true, dev)) return PG_ERR_INVALID;
    if (!matrix_ok(a.da, a.batch, a.channels, a.states, 4, true, dev)) return PG_ERR_INVALID;
    if (a.dskip && !vector_ok(a.dskip, a.dskip_stride, a.batch, a.channels, true, dev)) return PG_ERR_INVALID;
    if (a.ddelta_bias && !vector_ok(a.ddelta_bias, a.ddelta_bias_stride, a.batch, a.channels, true, dev)) return PG_ERR_INVALID;
    if (need > 0 && (workspace_bytes < need || !device_pointer(workspace, 16, dev))) return PG_ERR_WORKSPACE;
    const GradPlan p = grad_plan(a);
    if (sequences * p.chunks > kMaxBlocks || int64_t{a.batch} * p.shares > kMaxBlocks || p.parts / 256 > static_cast<size_t>(kMaxBlocks) ||
        (p.chunks > 1 && join_blocks(a) > kMaxBlocks))
        return PG_ERR_TOO_LARGE;
    if (a.batch == 0) return PG_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Operands operands;
    operands.output(a.du, a.batch, tokens, a.channels, 2).output(a.ddelta, a.batch, tokens, a.channels, 2).output(a.db, a.batch, tokens, a.states, 2);
    operands.output(a.dc, a.batch, tokens, a.states, 2).output(a.da, a.batch, a.channels, a.states, 4);
    if (a.z.data) operands.output(a.dz, a.batch, tokens, a.channels, 2);
    operands.output(a.dskip, a.dskip_stride, a.batch, a.channels).output(a.ddelta_bias, a.ddelta_bias_stride, a.batch, a.channels);
    span(operands, workspace, need, true);
    operands.input(a.dy, a.batch, tokens, a.channels, 2);
    scan_inputs(operands, a);
    if (operands.publish(st) != PG_OK) return PG_ERR_CUDA;
    char* at = static_cast<char*>(workspace);
    float* states = reinterpret_cast<float*>(at);
    float* carries = reinterpret_cast<float*>(at + p.states);
    float* sums = reinterpret_cast<float*>(at + 2 * p.states);
    float* parts = reinterpret_cast<float*>(at + 2 * p.states + p.sums);
    float* partial = reinterpret_cast<float*>(at + 2 * p.states + p.sums + p.parts);
    int status = PG_OK;
    with_kind(a.dtype, [&](auto h) {
        using H = decltype(h);
        auto launch = [&](auto lane) {
            constexpr int LANES = decltype(lane)::value;
            if (p.chunks > 1 && sequences > 0) {
                scan_grad_local_kernel<H, LANES><<<dim3(static_cast<unsigned>(sequences * p.chunks), static_cast<unsigned>(p.blocks)), kScanThreads, 0, st>>>(
                    a, states, carries, sums, p.chunk, p.chunks);
                join_chunks_kernel<<<static_cast<unsigned>(join_blocks(a)), 128, 0, st>>>(
                    a.a, a.state, states, carries, sums, a.sequences, a.channels, a.states, p.chunks);
            }
            const size_t smem = GradLayout<LANES>((p.chunk + kGroup - 1) / kGroup * kGroup).all;
            const auto kernel = scan_grad_kernel<H, LANES>;
            static_assert(kGradAlone % kGroup == 0 && kGradChunk <= kGradAlone, "the most tokens of a chunk");
            static std::atomic<bool> allowed[64];
            if (smem > 48 * 1024 && !allow_shared_memory(reinterpret_cast<const void*>(kernel), GradLayout<LANES>(kGradAlone).all, allowed)) {
                status = PG_ERR_CUDA;
                return;
            }
            kernel<<<dim3(static_cast<unsigned>(a.batch * p.shares), static_cast<unsigned>(p.blocks)), kScanThreads, smem, st>>>(a, states, carries, parts, partial,
                                                                                                                               p.chunk, p.chunks, p.shares);
        };
        using std::integral_constant;
        if (p.lanes == 1) launch(integral_constant<int, 1>{});
        else if (p.lanes == 2) launch(integral_constant<int, 2>{});
        else if (p.lanes == 4) launch(integral_constant<int, 4>{});
        else launch(integral_constant<int, 8>{});
        const int n = kGradStates * p.lanes;
        const int64_t all = a.batch * tokens * 2 * n;
        if (all > 0) sum_bc_kernel<H><<<static_cast<unsigned>((all + 255) / 256), 256, 0, st>>>(a, parts, static_cast<int>(p.blocks), n);
    });
    if (status != PG_OK) return status;
    const int64_t row = a.states + 2, size = row * a.channels;
    sum_parts_kernel<<<dim3(static_cast<unsigned>((int64_t{a.channels} * a.states + 31) / 32), a.batch), 256, 0, st>>>(
        partial, p.shares, size, a.channels, a.states, row, 1, false, static_cast<float*>(a.da.data), a.da.ld, a.da.stride, a.accumulate);
    for (int i = 0; i < 2; ++i) {
        float* out = i ? a.ddelta_bias : a.dskip;
        if (out)
            sum_parts_kernel<<<dim3((a.channels + 31) / 32, a.batch), 256, 0, st>>>(partial + a.states + i, p.shares, size, 1, a.channels, 0, row, false, out, a.channels,
                                                                                    i ? a.ddelta_bias_stride : a.dskip_stride, a.accumulate);
    }
    return launch_status();
}

}  // extern "C"
