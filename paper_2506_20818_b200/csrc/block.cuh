// Dropout from a counter-based generator, and the norms around a residual block fused with its dropout, gate and sum.
//
//   dropout         out = in * f where u >= t, else 0;  t = round(65536 p), f = 65536 / (65536 - t)
//   residual norm   y = x + s gate * dropout(post(h)),  n = pre(y)
//
// The mask is never stored: u, sixteen bits per element, is a pure function of (seed, step, row, column), so the backward pass
// draws it again.  Eight neighbouring columns share one Philox4x32-10 block with counter (row, row >> 32, step,
// 5 | column / 8 << 8): with 32 bits per element the generator alone (about 85 instructions per block) would take as long as
// HBM takes for BF16 rows.  f is computed from t, so the expectation is exact although p is rounded to sixteen bits.
//
// Norms of a row v of D columns, weight w, bias b (parameters FP32):
//   RMS   : r = 1 / sqrt(mean(v^2) + eps),            out = w v r
//   layer : c = v - mean(v), r = 1 / sqrt(mean(c^2) + eps), out = w c r + b
// Backward, for a gradient q of out, u = w q, z = v r (c r):
//   dv = r (u - z mean(u z) [- mean(u)]),  dw = sum over rows of q z,  db = sum of q
// No statistics are kept from the forward pass: a row's sums come out of the same registers that its gradient needs anyway.
//
// A team of T threads (a power of two, eight columns each) holds a row in registers, so every array is read once and written
// once: bound by HBM.  Teams of up to 32 threads are parts of warps, larger ones whole blocks.
#pragma once
#include "common.cuh"
#include "sampler.cuh"

enum : uint32_t { DRAW_DROPOUT = 5 };

struct DropArgs {
    uint32_t key[20];    // of the ten rounds: constants beside the instructions that use them
    uint32_t step_lo;
    uint32_t threshold;  // 0 = nothing is dropped, 65536 = everything
    uint32_t below2;     // threshold - 1 in both halves: the largest u that is dropped
    float factor;
    int64_t row_base;
};

// the bits of the eight elements of this row and group of columns, two per word
LP_DEVINL uint4 drop_words(const DropArgs &d, int64_t row, uint32_t group)
{
    const uint64_t r = (uint64_t)(d.row_base + row);
    uint4 c = make_uint4((uint32_t)r, (uint32_t)(r >> 32), d.step_lo, DRAW_DROPOUT | group << 8);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ d.key[2 * i], (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ d.key[2 * i + 1], (uint32_t)a);
    }
    return c;
}
// zero in the place of the elements of v that are dropped (not for threshold 0)
LP_DEVINL void drop8(const DropArgs &d, const uint4 &x, float *v)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bool hi, lo;  // one instruction compares both halves of a word
        (void)__vibmin_u16x2(w[i], d.below2, &hi, &lo);
        v[2 * i] = lo ? 0.f : v[2 * i];
        v[2 * i + 1] = hi ? 0.f : v[2 * i + 1];
    }
}
// bit i: element i stays (not for threshold 0)
LP_DEVINL uint32_t drop_keep8(const DropArgs &d, const uint4 &x)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t keep = 0xffu;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bool hi, lo;
        (void)__vibmin_u16x2(w[i], d.below2, &hi, &lo);
        keep ^= lo ? 1u << (2 * i) : 0u;
        keep ^= hi ? 2u << (2 * i) : 0u;
    }
    return keep;
}

// The eight columns of a thread.  VEC (rows start on 16 bytes): neighbouring ones.  Otherwise `step` = min(T, 32) columns apart, so
// that a warp reads and writes runs of neighbouring elements.
template <bool VEC> struct Cols {
    int base, step, width;
    // t: thread of the team
    LP_DEVINL Cols(int t, int T, int width_) : width(width_)
    {
        if (VEC) { base = 8 * t; step = 1; }
        else { step = min(T, 32); base = (t / 32) * 256 + (t & (step - 1)); }
    }
    LP_DEVINL int at(int j) const { return base + j * step; }
    LP_DEVINL bool has(int j) const { return at(j) < width; }
    LP_DEVINL bool full() const { return VEC && base + 8 <= width; }
    // keep bits in the order of the thread's columns
    LP_DEVINL uint32_t keep(const DropArgs &d, int64_t row, int lane) const
    {
        if (VEC) return drop_keep8(d, drop_words(d, row, (uint32_t)(base >> 3)));
        // the thread draws the bits of the eight neighbouring columns that it would own under VEC and hands them round its team
        const int lane_t = lane & (step - 1), first = base - lane_t;
        const uint32_t mine = drop_keep8(d, drop_words(d, row, (uint32_t)(first / 8 + lane_t)));
        uint32_t keep = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = lane_t + j * step;
            keep |= ((__shfl_sync(0xffffffffu, mine, c >> 3, step) >> (c & 7)) & 1u) << j;
        }
        return keep;
    }
};

template <typename T, bool VEC> LP_DEVINL void load8(const T *row, const Cols<VEC> &c, float *v)
{
    if (c.full()) {
        constexpr int VN = Vec16<T>::N;
#pragma unroll
        for (int k = 0; k < 8 / VN; ++k) {
            Vec16<T> x;
            x.load_once(row + c.base + k * VN);
            x.to_float(v + k * VN);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c.has(j) ? to_f<T>(row[c.at(j)]) : 0.f;
    }
}
template <typename T, bool VEC> LP_DEVINL void store8(T *row, const Cols<VEC> &c, const float *v)
{
    if (c.full()) {
        constexpr int VN = Vec16<T>::N;
#pragma unroll
        for (int k = 0; k < 8 / VN; ++k) {
            Vec16<T> x;
            x.from_float(v + k * VN);
            x.store(row + c.base + k * VN);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.has(j)) row[c.at(j)] = from_f<T>(v[j]);
    }
}
// per-column parameter, `other` where there is none
template <bool VEC> LP_DEVINL void load_param8(const float *p, const Cols<VEC> &c, float other, float *v)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p && c.has(j) ? __ldg(p + c.at(j)) : other;
}

// ---------------------------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------------------------
constexpr int DROP_THREADS = 256;

struct DropoutParams {
    const void *in;
    void *out;
    int rows, width;
    int64_t ld_in, ld_out;
    int team;            // threads per row (a power of two, at most 256); wider rows are taken in pieces of 8 team columns
    DropArgs drop;
};

// A block takes DROP_ROWS rows per team, one after the other; the loads of all of them are under way while the bits are drawn.
constexpr int DROP_ROWS = 4;
template <typename T, bool VEC> __global__ void __launch_bounds__(DROP_THREADS) dropout_kernel(const DropoutParams p)
{
    LP_DEP_ENTER();
    const int t = threadIdx.x & (p.team - 1), lane = threadIdx.x & 31, teams = DROP_THREADS / p.team;
    const int64_t row0 = (int64_t)blockIdx.x * teams * DROP_ROWS + threadIdx.x / p.team;
    const bool drops = p.drop.threshold != 0;
    if (VEC) {
        constexpr int VN = Vec16<T>::N, NV = 8 / VN;
        for (int c0 = 8 * t; c0 < p.width; c0 += 8 * p.team) {
            const T *in = (const T *)p.in + row0 * p.ld_in + c0;
            T *out = (T *)p.out + row0 * p.ld_out + c0;
            if (c0 + 8 <= p.width) {
                Vec16<T> x[DROP_ROWS][NV];
#pragma unroll
                for (int i = 0; i < DROP_ROWS; ++i)
                    if (row0 + i * teams < p.rows)
#pragma unroll
                        for (int k = 0; k < NV; ++k) x[i][k].load_once(in + (int64_t)i * teams * p.ld_in + k * VN);
#pragma unroll
                for (int i = 0; i < DROP_ROWS; ++i) {
                    const int64_t row = row0 + i * teams;
                    if (row >= p.rows) break;
                    float v[8];
#pragma unroll
                    for (int k = 0; k < NV; ++k) x[i][k].to_float(v + k * VN);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] *= p.drop.factor;
                    if (drops) drop8(p.drop, drop_words(p.drop, row, (uint32_t)c0 >> 3), v);
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        x[i][k].from_float(v + k * VN);
                        x[i][k].store(out + (int64_t)i * teams * p.ld_out + k * VN);
                    }
                }
            } else {  // the end of a row whose width is no multiple of eight
                for (int i = 0; i < DROP_ROWS && row0 + i * teams < p.rows; ++i) {
                    const uint32_t keep = drops ? drop_keep8(p.drop, drop_words(p.drop, row0 + i * teams, (uint32_t)c0 >> 3)) : 0xffu;
                    for (int j = 0; c0 + j < p.width; ++j) {
                        const float x = to_f<T>(in[(int64_t)i * teams * p.ld_in + j]);
                        out[(int64_t)i * teams * p.ld_out + j] = from_f<T>((keep >> j) & 1u ? x * p.drop.factor : 0.f);
                    }
                }
            }
        }
        return;
    }
    for (int i = 0; i < DROP_ROWS; ++i) {
        const int64_t row = row0 + i * teams;
        for (int c0 = 0; c0 < p.width; c0 += 8 * p.team) {
            Cols<VEC> c(t, p.team, p.width);
            c.base += c0;
            float v[8];
            if (row < p.rows) load8<T, VEC>((const T *)p.in + row * p.ld_in, c, v);
            // the whole warp takes part in handing the bits round, rows that are not there too
            const uint32_t keep = drops ? c.keep(p.drop, row, lane) : 0xffu;
            if (row < p.rows) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (keep >> j) & 1u ? v[j] * p.drop.factor : 0.f;
                store8<T, VEC>((T *)p.out + row * p.ld_out, c, v);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// residual norm
// ---------------------------------------------------------------------------------------------
constexpr int RN_MAX_WIDTH = 8192;  // eight columns for each of 1024 threads
constexpr int64_t RN_MAX_PITCH = (int64_t)1 << 29;  // elements: a pitch in bytes fits 32 bits, and a row's offset is one multiplication
constexpr int RN_SUMS = 5;          // column sums of the backward pass: dpre, dpost, dgate, dpre_bias, dpost_bias

struct ResidualParams {
    int rows;
    int width, team;
    int pre_norm, post_norm;   // lp_norm
    float eps, inv_width, scale;
    DropArgs drop;
    const float *pre, *pre_bias, *post, *post_bias, *gate_vec;
    const void *gate;          // [rows, width], or null
    // pitches in bytes
    uint32_t ld_gate;
    // forward: x, h in, y, n out (null: not wanted); backward: dy, dn, y, h in, dx, dh, dgate out
    const void *x, *h, *dy, *dn;
    void *y, *n, *dx, *dh, *dgate;
    uint32_t ld_x, ld_h, ld_y, ld_n, ld_dy, ld_dn, ld_dx, ld_dh, ld_dgate;
    float *partial;            // [gridDim.x][RN_SUMS][width] column sums of each block
    int pieces, stages;        // of the rows under way: 16-byte pieces per thread and row, rows
    uint32_t at_x, at_h, at_gate, at_y, at_dn, at_dy;  // bytes to each array's pieces
};

// Rows on their way into shared memory: each thread copies its own eight columns of the arrays a row needs (16 bytes at a time;
// FP32 rows of any alignment 4 bytes at a time) several rows ahead and reads back only what it copied itself, so no barrier is
// needed, and what is under way takes no registers.  What lies beyond the row or the last row arrives as zeros.
// BF16 rows that do not start on 16 bytes cannot be copied this way and are loaded when they are needed.
template <typename T> constexpr int PIPE_PIECES = sizeof(T) == 4 ? 2 : 1;  // of 16 bytes
LP_DEVINL void copy_async_16(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
LP_DEVINL void copy_async_4(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <bool VEC> struct RowPipe {
    uint32_t base;       // of this thread's pieces
    uint32_t piece, stage_bytes;
    int stages, head;    // the stage that is read next
    LP_DEVINL RowPipe(uint8_t *smem, int pieces, int stages_)
        : base(smem_u32(smem) + threadIdx.x * 16), piece(blockDim.x * 16), stage_bytes(pieces * blockDim.x * 16), stages(stages_), head(0) {}
    LP_DEVINL uint32_t stage(int ahead) const
    {
        int s = head + ahead;
        if (s >= stages) s -= stages;
        return base + s * stage_bytes;
    }
    // `at`: bytes from the start of a stage to the array's pieces; `ld`: bytes between rows.  row: of an array's row that is there, live: false for zeros
    template <typename T> LP_DEVINL void copy(uint32_t st, uint32_t at, const void *array, uint32_t ld, uint32_t row, bool live, const Cols<VEC> &c) const
    {
        if (!VEC && sizeof(T) == 2) return;
        const char *src = (const char *)array + (uint64_t)row * ld;
        if (VEC) {
#pragma unroll
            for (int k = 0; k < PIPE_PIECES<T>; ++k) {
                const int col = c.base + k * (16 / (int)sizeof(T)), have = min(max(c.width - col, 0) * (int)sizeof(T), 16);
                copy_async_16(st + at + k * piece, src + (have ? col * (int)sizeof(T) : 0), live ? have : 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool has = c.has(j);
                copy_async_4(st + at + (j >> 2) * piece + (j & 3) * 4, src + (has ? c.at(j) * (int)sizeof(T) : 0), live && has ? 4 : 0);
            }
        }
    }
    template <typename T> LP_DEVINL void read(uint32_t st, uint32_t at, const void *array, uint32_t ld, uint32_t row, bool live, const Cols<VEC> &c, float *v) const
    {
        if (!VEC && sizeof(T) == 2) {
            const T *src = (const T *)((const char *)array + (uint64_t)row * ld);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = live && c.has(j) ? to_f<T>(src[c.at(j)]) : 0.f;
            return;
        }
#pragma unroll
        for (int k = 0; k < PIPE_PIECES<T>; ++k) {
            Vec16<T> x;
            uint32_t w[4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(st + at + k * piece) : "memory");
            memcpy(&x.v, w, 16);
            x.to_float(v + k * Vec16<T>::N);
        }
    }
    LP_DEVINL void commit() const { asm volatile("cp.async.commit_group;" ::: "memory"); }
    // the oldest row has arrived
    LP_DEVINL void wait() const
    {
        if (stages == 1) asm volatile("cp.async.wait_group 0;" ::: "memory");
        else if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else asm volatile("cp.async.wait_group 3;" ::: "memory");
    }
    LP_DEVINL void next() { head = head + 1 == stages ? 0 : head + 1; }
};

template <typename T> LP_DEVINL T *row_at(void *array, uint32_t row, uint32_t ld) { return (T *)((char *)array + (uint64_t)row * ld); }

// 1 / sqrt(x) of a positive x: the hardware's estimate and one Newton step, off by about 1.5 2^-24 (the correctly rounded square root and
// division took 35 instructions)
LP_DEVINL float inv_sqrt(float x)
{
    const float r = rsqrtf(x);
    return fmaf(r * fmaf(-x * r, r, 1.f), 0.5f, r);
}

// Sums of K values over a team, in every one of its threads.  A fixed tree, so the same bits in every run.
template <int K, bool BLOCK> LP_DEVINL void team_sum(float (&v)[K], int T, float *scratch, int &turn)
{
    if (!BLOCK) {
        if (T == 32) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
            return;
        }
        for (int o = T >> 1; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        return;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = T >> 5;
    float *s = scratch + (turn & 1) * 32 * 4;  // two areas in turn: one barrier per sum
    ++turn;
    if (lane == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) s[k * 32 + warp] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lane < warps ? s[k * 32 + lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
}

// v becomes z (the normalised row); returns r
template <bool VEC, bool BLOCK> LP_DEVINL float normalise(float *v, int kind, float eps, float inv_width, const Cols<VEC> &c, int T, float *scratch, int &turn)
{
    if (kind == LP_NORM_LAYER) {
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += v[j];
        team_sum<1, BLOCK>(s, T, scratch, turn);
        const float mean = s[0] * inv_width;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c.has(j) ? v[j] - mean : 0.f;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int j = 0; j < 8; ++j) q[0] = fmaf(v[j], v[j], q[0]);
    team_sum<1, BLOCK>(q, T, scratch, turn);
    const float r = inv_sqrt(fmaf(q[0], inv_width, eps));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= r;
    return r;
}

// MAXT: the largest team of the variant, 32 (parts of warps), 256 or 1024 (whole blocks).  BIAS: norms with a bias
template <typename TS, typename TD, bool VEC, int MAXT, bool BIAS> __global__ void __launch_bounds__(MAXT < 256 ? 256 : MAXT) residual_norm_kernel(const __grid_constant__ ResidualParams p)
{
    LP_DEP_ENTER();
    constexpr bool BLOCK = MAXT > 32;
    __shared__ float scratch[2 * 32 * 4];
    extern __shared__ __align__(16) uint8_t pipe_smem[];
    int turn = 0;
    const int T = p.team, t = threadIdx.x & (T - 1), lane = threadIdx.x & 31, teams = BLOCK ? 1 : blockDim.x / T;
    const Cols<VEC> c(t, T, p.width);
    float pre[8], pre_bias[8], post[8], post_bias[8], gate_vec[8];
    load_param8(p.pre, c, 1.f, pre);
    load_param8(p.post, c, 1.f, post);
    load_param8(p.gate_vec, c, 1.f, gate_vec);
    const float factor = p.h && p.drop.threshold ? p.scale * p.drop.factor : p.scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) gate_vec[j] *= factor;
    if (BIAS) {
        load_param8(p.pre_bias, c, 0.f, pre_bias);
        load_param8(p.post_bias, c, 0.f, post_bias);
    }
    const int stride = (int)gridDim.x * teams, rounds = (int)((p.rows + (int64_t)stride - 1) / stride);
    int64_t row = (int64_t)blockIdx.x * teams + (BLOCK ? 0 : threadIdx.x / T);
    RowPipe<VEC> pipe(pipe_smem, p.pieces, p.stages);
    auto fetch = [&](int64_t at, int ahead) {
        const uint32_t st = pipe.stage(ahead);
        const bool live = at < p.rows;
        const uint32_t r = live ? (uint32_t)at : 0u;
        pipe.template copy<TS>(st, p.at_x, p.x, p.ld_x, r, live, c);
        if (p.h) pipe.template copy<TD>(st, p.at_h, p.h, p.ld_h, r, live, c);
        if (p.gate) pipe.template copy<TD>(st, p.at_gate, p.gate, p.ld_gate, r, live, c);
        pipe.commit();
    };
    for (int i = 0; i < p.stages - 1; ++i) fetch(row + (int64_t)i * stride, i);
    for (int i = 0; i < rounds; ++i, row += stride, pipe.next()) {
        const bool live = row < p.rows;  // of a warp's teams some may be past the last row; they take part in the sums of the others
        fetch(row + (int64_t)(p.stages - 1) * stride, p.stages - 1);
        const uint32_t r = live ? (uint32_t)row : 0u;
        uint4 bits;
        if (VEC && p.drop.threshold) bits = drop_words(p.drop, row, (uint32_t)c.base >> 3);
        pipe.wait();
        const uint32_t st = pipe.stage(0);
        float y[8], b[8];
        pipe.template read<TS>(st, p.at_x, p.x, p.ld_x, r, live, c, y);
        if (p.h) {
            pipe.template read<TD>(st, p.at_h, p.h, p.ld_h, r, live, c, b);
            if (p.post_norm) {
                normalise<VEC, BLOCK>(b, p.post_norm, p.eps, p.inv_width, c, T, scratch, turn);
#pragma unroll
                for (int j = 0; j < 8; ++j) b[j] = BIAS ? fmaf(b[j], post[j], post_bias[j]) : b[j] * post[j];
            }
            if (p.drop.threshold) {
                if (VEC) {
                    drop8(p.drop, bits, b);
                } else {
                    const uint32_t keep = c.keep(p.drop, row, lane);
#pragma unroll
                    for (int j = 0; j < 8; ++j) b[j] = (keep >> j) & 1u ? b[j] : 0.f;
                }
            }
            if (p.gate) {
                float g[8];
                pipe.template read<TD>(st, p.at_gate, p.gate, p.ld_gate, r, live, c, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) b[j] *= g[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = fmaf(gate_vec[j], b[j], y[j]);  // with scale and dropout factor in it
            if (live && p.y) store8<TS, VEC>(row_at<TS>(p.y, r, p.ld_y), c, y);
        }
        if (p.pre_norm) {
            normalise<VEC, BLOCK>(y, p.pre_norm, p.eps, p.inv_width, c, T, scratch, turn);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = BIAS ? fmaf(y[j], pre[j], pre_bias[j]) : y[j] * pre[j];
            if (live) store8<TD, VEC>(row_at<TD>(p.n, r, p.ld_n), c, y);
        }
    }
}

// v: the row, becomes z.  q: gradient of the norm's output, becomes that of its input.  dw, db: column sums.
template <bool VEC, bool BLOCK, bool BIAS>
LP_DEVINL void norm_backward(float *v, float *q, const float *w, int kind, float eps, float inv_width, const Cols<VEC> &c, int T, float *scratch, int &turn, float *dw, float *db)
{
    const bool layer = kind == LP_NORM_LAYER;
    if (layer) {
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += v[j];
        team_sum<1, BLOCK>(s, T, scratch, turn);
        const float mean = s[0] * inv_width;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c.has(j) ? v[j] - mean : 0.f;
    }
    float s[2] = {0.f, 0.f}, mean_u = 0.f;
    if (layer) {
        float x[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float u = w[j] * q[j];
            x[0] = fmaf(v[j], v[j], x[0]);
            x[1] = fmaf(u, v[j], x[1]);
            x[2] += u;
        }
        team_sum<3, BLOCK>(x, T, scratch, turn);
        s[0] = x[0];
        s[1] = x[1];
        mean_u = x[2] * inv_width;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[0] = fmaf(v[j], v[j], s[0]);
            s[1] = fmaf(w[j] * q[j], v[j], s[1]);
        }
        team_sum<2, BLOCK>(s, T, scratch, turn);
    }
    const float r = inv_sqrt(fmaf(s[0], inv_width, eps));
    const float along = s[1] * inv_width * r;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] *= r;
        dw[j] = fmaf(q[j], v[j], dw[j]);
        if (BIAS) db[j] += q[j];
        q[j] = r * (fmaf(-v[j], along, w[j] * q[j]) - mean_u);
    }
}

// BIAS: column sums of the biases too (sixteen more registers).  MAXT as above, and 256: blocks of 1024 threads leave 64 registers
// for each, which the column sums do not fit into.
template <typename TS, typename TD, bool VEC, int MAXT, bool BIAS>
__global__ void __launch_bounds__(MAXT < 256 ? 256 : MAXT) residual_norm_grad_kernel(const __grid_constant__ ResidualParams p)
{
    LP_DEP_ENTER();
    constexpr bool BLOCK = MAXT > 32;
    __shared__ float scratch[2 * 32 * 4];
    __shared__ float sums[BLOCK ? 1 : 8 * 256];
    extern __shared__ __align__(16) uint8_t pipe_smem[];
    int turn = 0;
    const int T = p.team, t = threadIdx.x & (T - 1), lane = threadIdx.x & 31, teams = BLOCK ? 1 : blockDim.x / T;
    const Cols<VEC> c(t, T, p.width);
    float pre[8], post[8], post_bias[8], gate_vec[8];
    load_param8(p.pre, c, 1.f, pre);
    load_param8(p.post, c, 1.f, post);
    load_param8(p.gate_vec, c, 1.f, gate_vec);
    if (BIAS) load_param8(p.post_bias, c, 0.f, post_bias);
    const float factor = p.scale * p.drop.factor;  // the factor is 1 where nothing is dropped
    float acc[RN_SUMS][8];
#pragma unroll
    for (int k = 0; k < RN_SUMS; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[k][j] = 0.f;
    const int stride = (int)gridDim.x * teams, rounds = (int)((p.rows + (int64_t)stride - 1) / stride);
    int64_t row = (int64_t)blockIdx.x * teams + (BLOCK ? 0 : threadIdx.x / T);
    RowPipe<VEC> pipe(pipe_smem, p.pieces, p.stages);
    auto fetch = [&](int64_t at, int ahead) {
        const uint32_t st = pipe.stage(ahead);
        const bool live = at < p.rows;
        const uint32_t r = live ? (uint32_t)at : 0u;
        if (p.pre_norm) {
            pipe.template copy<TD>(st, p.at_dn, p.dn, p.ld_dn, r, live, c);
            pipe.template copy<TS>(st, p.at_y, p.y, p.ld_y, r, live, c);
        }
        if (p.dy) pipe.template copy<TS>(st, p.at_dy, p.dy, p.ld_dy, r, live, c);
        if (p.h) pipe.template copy<TD>(st, p.at_h, p.h, p.ld_h, r, live, c);
        if (p.gate) pipe.template copy<TD>(st, p.at_gate, p.gate, p.ld_gate, r, live, c);
        pipe.commit();
    };
    for (int i = 0; i < p.stages - 1; ++i) fetch(row + (int64_t)i * stride, i);
    for (int i = 0; i < rounds; ++i, row += stride, pipe.next()) {
        const bool live = row < p.rows;
        fetch(row + (int64_t)(p.stages - 1) * stride, p.stages - 1);
        const uint32_t r = live ? (uint32_t)row : 0u;
        const uint32_t keep = p.drop.threshold ? c.keep(p.drop, row, lane) : 0xffu;
        pipe.wait();
        const uint32_t st = pipe.stage(0);
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 0.f;
        if (p.pre_norm) {
            float y[8];
            pipe.template read<TD>(st, p.at_dn, p.dn, p.ld_dn, r, live, c, g);
            pipe.template read<TS>(st, p.at_y, p.y, p.ld_y, r, live, c, y);
            norm_backward<VEC, BLOCK, BIAS>(y, g, pre, p.pre_norm, p.eps, p.inv_width, c, T, scratch, turn, acc[0], acc[3]);
        }
        if (p.dy) {
            float d[8];
            pipe.template read<TS>(st, p.at_dy, p.dy, p.ld_dy, r, live, c, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] += d[j];
        }
        if (p.dx && live) store8<TS, VEC>(row_at<TS>(p.dx, r, p.ld_dx), c, g);
        if (!p.h) continue;
        // the branch: g -> gradient of h
        float m[8], z[8], q[8];
        pipe.template read<TD>(st, p.at_h, p.h, p.ld_h, r, live, c, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            g[j] = (keep >> j) & 1u ? factor * g[j] : 0.f;   // times gate: gradient of post(h)
            q[j] = g[j] * gate_vec[j];
        }
        if (p.gate) {
            pipe.template read<TD>(st, p.at_gate, p.gate, p.ld_gate, r, live, c, m);
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] *= m[j];
        }
        if (p.post_norm) norm_backward<VEC, BLOCK, BIAS>(z, q, post, p.post_norm, p.eps, p.inv_width, c, T, scratch, turn, acc[1], acc[4]);
        if (p.dh && live) store8<TD, VEC>(row_at<TD>(p.dh, r, p.ld_dh), c, q);
        if (p.dgate || p.gate_vec) {
#pragma unroll
            for (int j = 0; j < 8; ++j) m[j] = (keep >> j) & 1u ? g[j] * (BIAS ? fmaf(z[j], post[j], post_bias[j]) : z[j] * post[j]) : 0.f;
            if (p.gate_vec) {
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[2][j] += m[j];
            } else if (live) {
                store8<TD, VEC>(row_at<TD>(p.dgate, r, p.ld_dgate), c, m);
            }
        }
    }
    // column sums of the block: its teams' added in order
#pragma unroll
    for (int k = 0; k < (BIAS ? 5 : 3); ++k) {
        float *dst = p.partial + ((size_t)blockIdx.x * RN_SUMS + k) * p.width;
        if (BLOCK) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c.has(j)) dst[c.at(j)] = acc[k][j];
        } else {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[(threadIdx.x / T) * 8 * T + c.at(j)] = acc[k][j];
            __syncthreads();
            for (int col = threadIdx.x; col < p.width; col += blockDim.x) {
                float s = 0.f;
                for (int q = 0; q < teams; ++q) s += sums[q * 8 * T + col];
                dst[col] = s;
            }
        }
    }
}

// out[k][col] (+)= sum over the blocks, in a fixed order: 32 columns per block, 32 threads share the blocks of a column
struct ResidualSums {
    float *out[RN_SUMS];
};
__global__ void __launch_bounds__(1024) residual_sums_kernel(const float *partial, int blocks, int width, const ResidualSums o, int accumulate)
{
    LP_DEP_ENTER();
    __shared__ float s[32][33];
    float *out = o.out[blockIdx.y];
    if (!out) return;
    const int col = blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (col < width)
        for (int b = threadIdx.y; b < blocks; b += 32) v += partial[((size_t)b * RN_SUMS + blockIdx.y) * width + col];
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    v = s[threadIdx.x][threadIdx.y];  // a warp holds the 32 shares of one column
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) v += __shfl_xor_sync(0xffffffffu, v, i);
    const int c = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && c < width) out[c] = accumulate ? out[c] + v : v;
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
static int pow2_at_least(int64_t n)
{
    int t = 1;
    while (t < n) t <<= 1;
    return t;
}
template <typename T> static bool on_16_bytes(const void *p, int64_t ld) { return !p || (((uintptr_t)p & 15) == 0 && ld * (int64_t)sizeof(T) % 16 == 0); }

template <typename T> static void dropout_launch(Exec &ex, DropoutParams &p)
{
    p.team = std::min(DROP_THREADS, pow2_at_least(ceil_div64(p.width, 8)));
    const int64_t blocks = ceil_div64(p.rows, DROP_THREADS / p.team * DROP_ROWS);
    const bool vec = on_16_bytes<T>(p.in, p.ld_in) && on_16_bytes<T>(p.out, p.ld_out);
    if (vec) launch_dep(dropout_kernel<T, true>, dim3((unsigned)blocks), dim3(DROP_THREADS), 0, ex.st, p);
    else launch_dep(dropout_kernel<T, false>, dim3((unsigned)blocks), dim3(DROP_THREADS), 0, ex.st, p);
    ex.launches += 1;
}

struct ResidualGrid {
    int team, threads, blocks;
    bool block;
};
static ResidualGrid residual_grid(int64_t rows, int width, int threads_per_sm)
{
    ResidualGrid g;
    g.team = pow2_at_least(ceil_div64(width, 8));
    g.block = g.team > 32;
    g.threads = g.block ? g.team : 256;
    const int64_t per_sm = std::max(1, threads_per_sm / g.threads);
    g.blocks = (int)std::min<int64_t>(ceil_div64(rows, g.threads / g.team), (int64_t)tc_sm_count() * per_sm);
    return g;
}

static bool residual_vec(const ResidualParams &p)
{
    auto ok = [](const void *array, uint32_t ld) { return !array || (((uintptr_t)array | ld) & 15) == 0; };
    return ok(p.x, p.ld_x) && ok(p.h, p.ld_h) && ok(p.y, p.ld_y) && ok(p.n, p.ld_n) && ok(p.dy, p.ld_dy) && ok(p.dn, p.ld_dn) && ok(p.dx, p.ld_dx) && ok(p.dh, p.ld_dh) &&
           ok(p.gate, p.ld_gate) && ok(p.dgate, p.ld_dgate);
}

// pieces of the rows under way and how many rows: `room` bytes of shared memory per thread keep as many blocks resident as registers do
template <typename TS, typename TD> static size_t residual_pipe(ResidualParams &p, const ResidualGrid &g, int room)
{
    const int s = PIPE_PIECES<TS>, d = PIPE_PIECES<TD>;
    int at = 0;
    auto place = [&](const void *array, int pieces) { const uint32_t here = (uint32_t)at * 16 * g.threads; if (array) at += pieces; return here; };
    p.at_x = place(p.x, s);
    p.at_dn = place(p.dn, d);
    p.at_y = place(p.dn ? p.y : nullptr, s);
    p.at_dy = place(p.dy, s);
    p.at_h = place(p.h, d);
    p.at_gate = place(p.gate, d);
    p.pieces = at;
    p.stages = std::max(2, std::min(4, room / (16 * at)));
    while (p.stages * at * 16 * g.threads > 216 * 1024) --p.stages;  // blocks of 1024 threads: down to one, nothing under way
    return (size_t)p.stages * at * 16 * g.threads;
}
template <typename... A, typename... P> static void launch_large(void (*kernel)(A...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, P &&...args)
{
    if (smem > 40 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    launch_dep(kernel, grid, block, smem, st, args...);
}

template <typename TS, typename TD, bool VEC, bool BIAS> static void residual_dispatch(Exec &ex, const ResidualParams &p, const ResidualGrid &g, size_t smem)
{
    const dim3 grid(g.blocks), block(g.threads);
    if (g.threads > 256) launch_large(residual_norm_kernel<TS, TD, VEC, 1024, BIAS>, grid, block, smem, ex.st, p);
    else if (g.block) launch_large(residual_norm_kernel<TS, TD, VEC, 256, BIAS>, grid, block, smem, ex.st, p);
    else launch_large(residual_norm_kernel<TS, TD, VEC, 32, BIAS>, grid, block, smem, ex.st, p);
}
template <typename TS, typename TD> static void residual_launch(Exec &ex, ResidualParams &p)
{
    const ResidualGrid g = residual_grid(p.rows, p.width, 768);
    p.team = g.team;
    const size_t smem = residual_pipe<TS, TD>(p, g, 256);
    const bool bias = p.pre_bias || p.post_bias;
    if (residual_vec(p)) {
        if (bias) residual_dispatch<TS, TD, true, true>(ex, p, g, smem);
        else residual_dispatch<TS, TD, true, false>(ex, p, g, smem);
    } else {
        if (bias) residual_dispatch<TS, TD, false, true>(ex, p, g, smem);
        else residual_dispatch<TS, TD, false, false>(ex, p, g, smem);
    }
    ex.launches += 1;
}

template <typename TS, typename TD, bool VEC, bool BIAS> static void residual_grad_dispatch(Exec &ex, const ResidualParams &p, const ResidualGrid &g, size_t smem)
{
    const dim3 grid(g.blocks), block(g.threads);
    if (g.threads > 256) launch_large(residual_norm_grad_kernel<TS, TD, VEC, 1024, BIAS>, grid, block, smem, ex.st, p);
    else if (g.block) launch_large(residual_norm_grad_kernel<TS, TD, VEC, 256, BIAS>, grid, block, smem, ex.st, p);
    else launch_large(residual_norm_grad_kernel<TS, TD, VEC, 32, BIAS>, grid, block, smem, ex.st, p);
}
template <typename TS, typename TD> static void residual_grad_launch(Exec &ex, ResidualParams &p, const ResidualGrid &g, const ResidualSums &o, int accumulate)
{
    p.team = g.team;
    const size_t smem = residual_pipe<TS, TD>(p, g, 380);
    const bool bias = o.out[3] || o.out[4] || p.post_bias;
    if (residual_vec(p)) {
        if (bias) residual_grad_dispatch<TS, TD, true, true>(ex, p, g, smem);
        else residual_grad_dispatch<TS, TD, true, false>(ex, p, g, smem);
    } else {
        if (bias) residual_grad_dispatch<TS, TD, false, true>(ex, p, g, smem);
        else residual_grad_dispatch<TS, TD, false, false>(ex, p, g, smem);
    }
    ex.launches += 1;
    int last = -1;
    for (int k = 0; k < RN_SUMS; ++k)
        if (o.out[k]) last = k;
    if (last < 0) return;
    launch_dep(residual_sums_kernel, dim3((unsigned)ceil_div64(p.width, 32), (unsigned)(last + 1)), dim3(32, 32), 0, ex.st, p.partial, g.blocks, p.width, o, accumulate);
    ex.launches += 1;
}
