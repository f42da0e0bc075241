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
//
// Measured on the device, launches one after the other (the copy rate is 6.55 TB/s):
//   dropout, 1,000,000 x 256 BF16                                    185 us, 5.5 TB/s: 64 of 112 instructions per eight elements are the
//                                                                    generator's, whose multiplications keep their pipe busy
//   residual norm, 196,608 x 256, FP32 sums, BF16 blocks, both norms, dropout, gate per column    106 us, 5.7 TB/s
//     FP32 blocks 156 us, 5.2 TB/s; BF16 sums 101 us, 4.0 TB/s: the same instructions for two thirds of the bytes
//   its gradient                                                     173 us, 5.2 TB/s, and 4 us for the column sums of the blocks: 580
//                                                                    instructions per row of a warp at 16 warps per SM (128 registers)
//     FP32 blocks 203 us, 5.9 TB/s; BF16 sums 173 us, 3.5 TB/s
//   gradient, 50,001 x 417 FP32, layer norms, gate per element       183 us, 3.6 TB/s, and 6 us: 53 of a team's 64 threads have columns,
//                                                                    single elements loaded from shared memory and stored, four barriers a row
//     FP32 sums and BF16 blocks 179 us, BF16 sums 190 us: as many instructions for fewer bytes
#pragma once
#include "gemm_tc.cuh"

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

template <typename T, bool VEC> LP_DEVINL void store8(T *row, const Cols<VEC> &c, const float *v)
{
    if (c.full()) {
        if (sizeof(T) == 4 && ((uintptr_t)row & 31) == 0) {  // a whole sector in one instruction
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + c.base), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]),
                         "f"(v[6]), "f"(v[7])
                         : "memory");
            return;
        }
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
// Eight columns at once, two per instruction (sm_100 has FP32 multiplications and additions on pairs; one instruction per element made
// these kernels wait for the scheduler rather than for HBM).
LP_DEVINL float2 pair(const float *v, int k) { return make_float2(v[2 * k], v[2 * k + 1]); }
LP_DEVINL void set_pair(float *v, int k, float2 x) { v[2 * k] = x.x; v[2 * k + 1] = x.y; }
LP_DEVINL void mul8(float *v, const float *w)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) set_pair(v, k, __fmul2_rn(pair(v, k), pair(w, k)));
}
LP_DEVINL void scale8(float *v, float f)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) set_pair(v, k, __fmul2_rn(pair(v, k), make_float2(f, f)));
}
LP_DEVINL void add8(float *v, const float *w)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) set_pair(v, k, __fadd2_rn(pair(v, k), pair(w, k)));
}
LP_DEVINL void shift8(float *v, float f)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) set_pair(v, k, __fadd2_rn(pair(v, k), make_float2(f, f)));
}
LP_DEVINL void fma8(const float *a, const float *b, float *acc)  // acc += a b
{
#pragma unroll
    for (int k = 0; k < 4; ++k) set_pair(acc, k, __ffma2_rn(pair(a, k), pair(b, k), pair(acc, k)));
}
LP_DEVINL float sum8(const float *v)
{
    const float2 a = __fadd2_rn(__fadd2_rn(pair(v, 0), pair(v, 1)), __fadd2_rn(pair(v, 2), pair(v, 3)));
    return a.x + a.y;
}
LP_DEVINL float dot8(const float *a, const float *b)
{
    float2 x = __fmul2_rn(pair(a, 0), pair(b, 0));
#pragma unroll
    for (int k = 1; k < 4; ++k) x = __ffma2_rn(pair(a, k), pair(b, k), x);
    return x.x + x.y;
}
// per-column parameter, `other` where there is none; zeros beyond the row, so that nothing there enters a sum
template <bool VEC> LP_DEVINL void load_param8(const float *p, const Cols<VEC> &c, float other, float *v)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = !c.has(j) ? 0.f : p ? __ldg(p + c.at(j)) : other;
}

// ---------------------------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------------------------
constexpr int DROP_THREADS = 256;

struct DropoutParams {
    const void *in;
    void *out;
    int rows, width;
    uint32_t ld_in, ld_out;  // bytes
    int shift;               // 2^shift threads per row, at most 256; wider rows are taken in pieces of eight times as many columns
    DropArgs drop;
};

// A block takes DROP_ROWS rows per team, one after the other; the loads of all of them are under way while the bits are drawn.
constexpr int DROP_ROWS = 4;
template <typename T, bool VEC> __global__ void __launch_bounds__(DROP_THREADS, 4) dropout_kernel(const __grid_constant__ DropoutParams p)
{
    LP_DEP_ENTER();
    const int team = 1 << p.shift, teams = DROP_THREADS >> p.shift, t = threadIdx.x & (team - 1), lane = threadIdx.x & 31;
    const uint32_t row0 = blockIdx.x * (uint32_t)(teams * DROP_ROWS) + (threadIdx.x >> p.shift);  // rows < 2^31: no overflow
    const bool drops = p.drop.threshold != 0;
    if constexpr (VEC) {
        constexpr int VN = Vec16<T>::N, NV = 8 / VN;
        for (int c0 = 8 * t; c0 < p.width; c0 += 8 * team) {
            const char *in = (const char *)p.in + c0 * sizeof(T);
            char *out = (char *)p.out + c0 * sizeof(T);
            if (c0 + 8 <= p.width) {
                Vec16<T> x[DROP_ROWS][NV];
#pragma unroll
                for (int i = 0; i < DROP_ROWS; ++i)
                    if (row0 + i * teams < (uint32_t)p.rows)
#pragma unroll
                        for (int k = 0; k < NV; ++k) x[i][k].load_once((const T *)(in + (uint64_t)(row0 + i * teams) * p.ld_in) + k * VN);
#pragma unroll
                for (int i = 0; i < DROP_ROWS; ++i) {
                    const uint32_t row = row0 + i * teams;
                    if (row >= (uint32_t)p.rows) break;
                    float v[8];
#pragma unroll
                    for (int k = 0; k < NV; ++k) x[i][k].to_float(v + k * VN);
                    scale8(v, p.drop.factor);
                    if (drops) drop8(p.drop, drop_words(p.drop, row, (uint32_t)c0 >> 3), v);
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        x[i][k].from_float(v + k * VN);
                        x[i][k].store((T *)(out + (uint64_t)row * p.ld_out) + k * VN);
                    }
                }
            } else {  // the end of a row whose width is no multiple of eight
                for (int i = 0; i < DROP_ROWS && row0 + i * teams < (uint32_t)p.rows; ++i) {
                    const uint32_t row = row0 + i * teams, keep = drops ? drop_keep8(p.drop, drop_words(p.drop, row, (uint32_t)c0 >> 3)) : 0xffu;
                    for (int j = 0; c0 + j < p.width; ++j) {
                        const float x = to_f<T>(((const T *)(in + (uint64_t)row * p.ld_in))[j]);
                        ((T *)(out + (uint64_t)row * p.ld_out))[j] = from_f<T>((keep >> j) & 1u ? x * p.drop.factor : 0.f);
                    }
                }
            }
        }
    } else {
        for (int i = 0; i < DROP_ROWS; ++i) {
            const uint32_t row = row0 + i * teams;
            for (int c0 = 0; c0 < p.width; c0 += 8 * team) {
                Cols<VEC> c(t, team, p.width);
                c.base += c0;
                float v[8];
                const T *in = (const T *)((const char *)p.in + (uint64_t)row * p.ld_in);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = row < (uint32_t)p.rows && c.has(j) ? to_f<T>(in[c.at(j)]) : 0.f;
                // the whole warp takes part in handing the bits round, rows that are not there too
                const uint32_t keep = drops ? c.keep(p.drop, row, lane) : 0xffu;
                if (row < (uint32_t)p.rows) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = (keep >> j) & 1u ? v[j] * p.drop.factor : 0.f;
                    store8<T, VEC>((T *)((char *)p.out + (uint64_t)row * p.ld_out), c, v);
                }
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

struct PipeArray {        // of a kernel's arrays
    const char *at;
    uint32_t ld;          // bytes between rows
    uint32_t row_bytes;   // of a row
    uint32_t slot_bytes;  // of its place in a stage
    uint32_t offset;      // of the first team's place
};

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
    // rows under way: how many, bytes of a unit's rows of all arrays
    int stages;
    uint32_t stage_bytes;
    uint32_t copy_bytes;       // VEC: of one row of all arrays
    int unit_teams;            // teams of a unit
    PipeArray pipe[5];         // forward: x, h, gate; backward: dn, y, dy, h, gate
    int *err;
    unsigned long long wait_ns;
    uint32_t extra_tx;         // diagnostics: the first row's wait expires
};


// Rows on their way into shared memory, several ahead of the one that is worked on, so that what is under way takes no registers: one
// bulk copy per row and array, counted on a barrier of the unit (the warp, or the block of a large team) and row.  (Copies by every
// thread took about 150 instructions per row and, of FP32, asked for every sector twice.)  Bulk copies are made of aligned pieces of
// 16 bytes.  Rows that are not come with the bytes beside them in their first and last piece, which nobody looks at; a piece with a
// byte of the row lies in the row's page.
LP_DEVINL void copy_row(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
LP_DEVINL void mbar_expect_more(uint32_t bar, uint32_t bytes) { asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
template <bool VEC, bool BLOCK> struct RowPipe {
    const ResidualParams &p;
    uint32_t first, in, out, end;   // of the unit: where the next row goes, where the oldest lies
    uint32_t bar_in, bar_out, bars; // the same of the barriers
    uint32_t parity;
    bool ok;
    LP_DEVINL RowPipe(const ResidualParams &p_, uint8_t *smem) : p(p_), parity(0), ok(true)
    {
        const uint32_t unit = BLOCK ? 0 : threadIdx.x >> 5, units = BLOCK ? 1 : blockDim.x >> 5;
        first = in = out = smem_u32(smem) + unit * p.stages * p.stage_bytes;
        end = first + p.stages * p.stage_bytes;
        bars = bar_in = bar_out = smem_u32(smem) + units * p.stages * p.stage_bytes + unit * p.stages * 8;
        if (BLOCK ? threadIdx.x == 0 : (threadIdx.x & 31) == 0) {
            for (int i = 0; i < p.stages; ++i) mbar_init(bars + 8 * i, 1);
            fence_barrier_init();
            fence_async_proxy();
        }
        sync();
    }
    // the threads that share the rows of a stage
    LP_DEVINL void sync() const
    {
        if (BLOCK) __syncthreads();
        else __syncwarp();
    }
    // the next row of every team of the unit; `row` is this thread's.  extra: bytes that are announced and never come (diagnostics)
    template <int N> LP_DEVINL void fetch(const PipeArray (&arrays)[N], int64_t row, int t, int team, uint32_t extra = 0)
    {
        const bool sends = t == 0 && row < p.rows;
        if (VEC) {
            // the unit's first thread says how much is on its way
            if (t == 0 && team == 0) mbar_expect_tx(bar_in, p.copy_bytes * (uint32_t)min(max((int64_t)p.rows - row, (int64_t)0), (int64_t)p.unit_teams) + extra);
        } else {
            if (sends) {
                uint32_t bytes = extra;
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (arrays[k].at) {
                        const uint32_t at = (uint32_t)(uintptr_t)arrays[k].at + (uint32_t)row * arrays[k].ld;  // the low bits of the address
                        bytes += ((at & 15) + arrays[k].row_bytes + 15) & ~15u;
                    }
                mbar_expect_more(bar_in, bytes);
            }
            if (!BLOCK) __syncwarp();
            if (t == 0 && team == 0) mbar_arrive(bar_in);
        }
        if (sends)
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (arrays[k].at) {
                    const uint64_t at = (uint64_t)arrays[k].at + (uint64_t)(uint32_t)row * arrays[k].ld;
                    copy_row(in + arrays[k].offset + team * arrays[k].slot_bytes, (const void *)(VEC ? at : at & ~(uint64_t)15),
                             VEC ? arrays[k].row_bytes : (((uint32_t)at & 15) + arrays[k].row_bytes + 15) & ~15u, bar_in);
                }
        in += p.stage_bytes;
        bar_in += 8;
        if (in == end) { in = first; bar_in = bars; }
    }
    template <typename T> LP_DEVINL void read(const PipeArray &a, int64_t row, int team, const Cols<VEC> &c, float *v) const
    {
        const bool live = row < p.rows;
        uint32_t src = out + a.offset + team * a.slot_bytes;
        if (VEC) {
            constexpr int VN = Vec16<T>::N;
            src += c.base * (uint32_t)sizeof(T);
#pragma unroll
            for (int k = 0; k < 8 / VN; ++k) {
                Vec16<T> x;
                x.zero();
                if (live && c.base + k * VN < c.width) {
                    uint32_t w[4];
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(src + 16 * k) : "memory");
                    memcpy(&x.v, w, 16);
                }
                x.to_float(v + k * VN);
            }
        } else {
            src += (((uint32_t)(uintptr_t)a.at + (uint32_t)row * a.ld) & 15) + c.base * (uint32_t)sizeof(T);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = 0.f;
                if (live && c.has(j)) {
                    if (sizeof(T) == 4) {
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[j]) : "r"(src + j * c.step * 4) : "memory");
                    } else {
                        uint16_t h;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(src + j * c.step * 2) : "memory");
                        v[j] = __uint_as_float((uint32_t)h << 16);
                    }
                }
            }
        }
    }
    // the oldest row has arrived; false when the wait ran out (in all threads of the unit)
    LP_DEVINL bool wait()
    {
        ok = false;
        for (int i = 0; i < 256 && !ok; ++i) ok = mbar_try_wait(bar_out, parity);  // reading the time takes longer than most waits do
        if (!ok) ok = mbar_wait(bar_out, parity, p.wait_ns);
        ok = BLOCK ? __syncthreads_and(ok) != 0 : __all_sync(0xffffffffu, ok) != 0;
        return ok;
    }
    // the oldest row's place is free again
    LP_DEVINL void next()
    {
        sync();
        out += p.stage_bytes;
        bar_out += 8;
        if (out == end) { out = first; bar_out = bars; parity ^= 1; }
    }
    // what is under way lands before the block goes (after a wait that ran out; else nothing is)
    LP_DEVINL void drain()
    {
        for (int i = 0; i < p.stages; ++i) {
            mbar_wait(bar_out, parity, p.wait_ns);
            next();
        }
    }
};

template <typename T> LP_DEVINL T *row_at(void *array, uint32_t row, uint32_t ld) { return (T *)((char *)array + (uint64_t)row * ld); }

// 1 / sqrt(x) of a positive x: the hardware's estimate and one step of Newton-Raphson (on 1 / r^2 - x), off by about 1.5 2^-24 (the correctly rounded square root and
// division took 35 instructions); 0 for a sum that is infinite
LP_DEVINL float inv_sqrt(float x)
{
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r == 0.f ? 0.f : fmaf(r * fmaf(-x * r, r, 1.f), 0.5f, r);
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

// v less its mean over the row
template <bool VEC, bool BLOCK> LP_DEVINL void centre(float *v, float inv_width, const Cols<VEC> &c, int T, float *scratch, int &turn)
{
    float s[1] = {sum8(v)};
    team_sum<1, BLOCK>(s, T, scratch, turn);
    shift8(v, -s[0] * inv_width);
    if (!c.full())
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c.has(j) ? v[j] : 0.f;
}

// v becomes w times the normalised row (w: the weight)
template <bool VEC, bool BLOCK>
LP_DEVINL void normalise(float *v, const float *w, int kind, float eps, float inv_width, const Cols<VEC> &c, int T, float *scratch, int &turn)
{
    if (kind == LP_NORM_LAYER) centre<VEC, BLOCK>(v, inv_width, c, T, scratch, turn);
    float q[1] = {dot8(v, v)};
    team_sum<1, BLOCK>(q, T, scratch, turn);
    scale8(v, inv_sqrt(fmaf(q[0], inv_width, eps)));
    mul8(v, w);
}

// MAXT: the largest team of the variant, 32 (parts of warps), 256 or 1024 (whole blocks).  BIAS: norms with a bias
template <typename TS, typename TD, bool VEC, int MAXT, bool BIAS> __global__ void __launch_bounds__(MAXT < 256 ? 256 : MAXT, MAXT > 256 ? 1 : 3) residual_norm_kernel(const __grid_constant__ ResidualParams p)
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
    RowPipe<VEC, BLOCK> pipe(p, pipe_smem);
    const PipeArray arrays[3] = {p.pipe[0], p.pipe[1], p.pipe[2]};
    const int team = BLOCK ? 0 : lane / T;
    for (int i = 0; i < p.stages; ++i) pipe.fetch(arrays, row + (int64_t)i * stride, t, team, i == 0 && blockIdx.x == 0 ? p.extra_tx : 0u);
    for (int i = 0; i < rounds; ++i, row += stride) {
        const bool live = row < p.rows;  // of a warp's teams some may be past the last row; they take part in the sums of the others
        const uint32_t r = live ? (uint32_t)row : 0u;
        uint4 bits;
        if (VEC && p.drop.threshold) bits = drop_words(p.drop, row, (uint32_t)c.base >> 3);
        if (!pipe.wait()) break;
        float y[8], b[8];
        pipe.template read<TS>(arrays[0], row, team, c, y);
        if (p.h) {
            pipe.template read<TD>(arrays[1], row, team, c, b);
            if (p.post_norm) {
                normalise<VEC, BLOCK>(b, post, p.post_norm, p.eps, p.inv_width, c, T, scratch, turn);
                if (BIAS) add8(b, post_bias);
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
                pipe.template read<TD>(arrays[2], row, team, c, g);
                mul8(b, g);
            }
            fma8(gate_vec, b, y);  // scale and dropout factor are in it
            if (live && p.y) store8<TS, VEC>(row_at<TS>(p.y, r, p.ld_y), c, y);
        }
        if (p.pre_norm) {
            normalise<VEC, BLOCK>(y, pre, p.pre_norm, p.eps, p.inv_width, c, T, scratch, turn);
            if (BIAS) add8(y, pre_bias);
            if (live) store8<TD, VEC>(row_at<TD>(p.n, r, p.ld_n), c, y);
        }
        pipe.next();
        pipe.fetch(arrays, row + (int64_t)p.stages * stride, t, team);
    }
    if (!pipe.ok && threadIdx.x % 32 == 0) atomicExch(p.err, 8);
    pipe.drain();
}

// v: the row, becomes z.  q: gradient of the norm's output, becomes that of its input.  dw, db: column sums.
template <bool VEC, bool BLOCK, bool BIAS>
LP_DEVINL void norm_backward(float *v, float *q, const float *w, int kind, float eps, float inv_width, const Cols<VEC> &c, int T, float *scratch, int &turn, float *dw, float *db)
{
    float u[8], r, along, mean_u = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = w[j];
    mul8(u, q);
    if (kind == LP_NORM_LAYER) {
        centre<VEC, BLOCK>(v, inv_width, c, T, scratch, turn);
        float s[3] = {dot8(v, v), dot8(u, v), sum8(u)};
        team_sum<3, BLOCK>(s, T, scratch, turn);
        r = inv_sqrt(fmaf(s[0], inv_width, eps));
        along = s[1] * inv_width * r;
        mean_u = s[2] * inv_width;
    } else {
        float s[2] = {dot8(v, v), dot8(u, v)};
        team_sum<2, BLOCK>(s, T, scratch, turn);
        r = inv_sqrt(fmaf(s[0], inv_width, eps));
        along = s[1] * inv_width * r;
    }
    scale8(v, r);
    fma8(q, v, dw);
    if (BIAS) add8(db, q);
    // r (u - z along - mean(u))
    const float2 minus = make_float2(-along * r, -along * r), rr = make_float2(r, r);
    const float off = -mean_u * r;
#pragma unroll
    for (int k = 0; k < 4; ++k) set_pair(q, k, __ffma2_rn(pair(v, k), minus, __ffma2_rn(pair(u, k), rr, make_float2(off, off))));
}

// BIAS: column sums of the biases too (sixteen more registers: 384 threads per SM instead of 512).  MAXT as above, and 128 and 256:
// blocks of 1024 threads leave 64 registers for each, which the column sums do not fit into.
template <int MAXT, bool BIAS> constexpr int RN_GRAD_THREADS = MAXT > 32 ? MAXT : BIAS ? 128 : 256;
template <bool BIAS> constexpr int RN_GRAD_RESIDENT = BIAS ? 384 : 512;
template <typename TS, typename TD, bool VEC, int MAXT, bool BIAS>
__global__ void __launch_bounds__(RN_GRAD_THREADS<MAXT, BIAS>, MAXT > 256 ? 1 : RN_GRAD_RESIDENT<BIAS> / RN_GRAD_THREADS<MAXT, BIAS>) residual_norm_grad_kernel(const __grid_constant__ ResidualParams p)
{
    LP_DEP_ENTER();
    constexpr bool BLOCK = MAXT > 32;
    __shared__ float scratch[2 * 32 * 4];
    __shared__ float sums[BLOCK ? 1 : 8 * RN_GRAD_THREADS<MAXT, BIAS>];
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
    RowPipe<VEC, BLOCK> pipe(p, pipe_smem);
    const PipeArray arrays[5] = {p.pipe[0], p.pipe[1], p.pipe[2], p.pipe[3], p.pipe[4]};
    const int team = BLOCK ? 0 : lane / T;
    for (int i = 0; i < p.stages; ++i) pipe.fetch(arrays, row + (int64_t)i * stride, t, team, i == 0 && blockIdx.x == 0 ? p.extra_tx : 0u);
    for (int i = 0; i < rounds; ++i, row += stride) {
        const bool live = row < p.rows;
        const uint32_t r = live ? (uint32_t)row : 0u;
        const uint32_t keep = p.drop.threshold ? c.keep(p.drop, row, lane) : 0xffu;
        if (!pipe.wait()) break;
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 0.f;
        if (p.pre_norm) {
            float y[8];
            pipe.template read<TD>(arrays[0], row, team, c, g);
            pipe.template read<TS>(arrays[1], row, team, c, y);
            norm_backward<VEC, BLOCK, BIAS>(y, g, pre, p.pre_norm, p.eps, p.inv_width, c, T, scratch, turn, acc[0], acc[3]);
        }
        if (p.dy) {
            float d[8];
            pipe.template read<TS>(arrays[2], row, team, c, d);
            add8(g, d);
        }
        if (p.dx && live) store8<TS, VEC>(row_at<TS>(p.dx, r, p.ld_dx), c, g);
        if (p.h) {  // the branch: g -> gradient of h
            float m[8], z[8], q[8];
            pipe.template read<TD>(arrays[3], row, team, c, z);
            scale8(g, factor);
            if (p.drop.threshold)
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = (keep >> j) & 1u ? g[j] : 0.f;   // times gate: gradient of post(h)
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = g[j];
            mul8(q, gate_vec);
            if (p.gate) {
                pipe.template read<TD>(arrays[4], row, team, c, m);
                mul8(q, m);
            }
            if (p.post_norm) norm_backward<VEC, BLOCK, BIAS>(z, q, post, p.post_norm, p.eps, p.inv_width, c, T, scratch, turn, acc[1], acc[4]);
            if (p.dh && live) store8<TD, VEC>(row_at<TD>(p.dh, r, p.ld_dh), c, q);
            if (p.dgate || p.gate_vec) {
                // gradient of the gate: g post(h), where nothing was dropped
                if (BIAS) {
                    mul8(z, post);
                    add8(z, post_bias);
                }
                if (p.drop.threshold)
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = (keep >> j) & 1u ? z[j] : 0.f;
                if (p.gate_vec) {
                    fma8(g, z, acc[2]);  // without a bias the weight is the same for all rows and comes in at the end
                } else {
                    if (!BIAS) mul8(z, post);
                    mul8(z, g);
                    if (live) store8<TD, VEC>(row_at<TD>(p.dgate, r, p.ld_dgate), c, z);
                }
            }
        }
        pipe.next();
        pipe.fetch(arrays, row + (int64_t)p.stages * stride, t, team);
    }
    if (!pipe.ok && lane == 0) atomicExch(p.err, 8);
    pipe.drain();
    if (!BIAS) mul8(acc[2], post);
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
    p.shift = 0;
    while ((8 << p.shift) < p.width && p.shift < 8) ++p.shift;
    const int64_t blocks = ceil_div64(p.rows, (DROP_THREADS >> p.shift) * DROP_ROWS);
    const bool vec = (((uintptr_t)p.in | (uintptr_t)p.out | p.ld_in | p.ld_out) & 15) == 0;
    if (vec) launch_dep(dropout_kernel<T, true>, dim3((unsigned)blocks), dim3(DROP_THREADS), 0, ex.st, p);
    else launch_dep(dropout_kernel<T, false>, dim3((unsigned)blocks), dim3(DROP_THREADS), 0, ex.st, p);
    ex.launches += 1;
}

struct ResidualGrid {
    int team, threads, blocks;
    bool block;
};
// `threads` per block where the teams are parts of warps, `resident` per SM
static ResidualGrid residual_grid(int64_t rows, int width, int threads, int resident)
{
    ResidualGrid g;
    g.team = pow2_at_least(ceil_div64(width, 8));
    g.block = g.team > 32;
    g.threads = g.block ? g.team : threads;
    g.blocks = (int)std::min<int64_t>(ceil_div64(rows, g.threads / g.team), (int64_t)tc_sm_count() * std::max(1, resident / g.threads));
    return g;
}
static ResidualGrid residual_grad_grid(int64_t rows, int width, bool bias)
{
    return bias ? residual_grid(rows, width, RN_GRAD_THREADS<32, true>, RN_GRAD_RESIDENT<true>) : residual_grid(rows, width, RN_GRAD_THREADS<32, false>, RN_GRAD_RESIDENT<false>);
}

// every row of every array starts on 16 bytes and is made of pieces of 16
static bool residual_vec(const ResidualParams &p, int size_d)
{
    if (p.width * size_d % 16 != 0) return false;  // else rows of the sum's type, as wide or twice as wide, are too
    auto ok = [](const void *array, uint32_t ld) { return !array || (((uintptr_t)array | ld) & 15) == 0; };
    return ok(p.x, p.ld_x) && ok(p.h, p.ld_h) && ok(p.y, p.ld_y) && ok(p.n, p.ld_n) && ok(p.dy, p.ld_dy) && ok(p.dn, p.ld_dn) && ok(p.dx, p.ld_dx) && ok(p.dh, p.ld_dh) &&
           ok(p.gate, p.ld_gate) && ok(p.dgate, p.ld_dgate);
}

// Rows under way (one row of all arrays is at most 160 KiB and 80 bytes) and their barriers, up to eight of eight units
constexpr int RN_MAX_ROWS_SMEM = 208 * 1024, RN_MAX_SMEM = RN_MAX_ROWS_SMEM + 8 * 8 * 8;

// Places of the arrays in the ring of rows and how many rows it holds: `room` bytes of shared memory per thread keep as many blocks
// resident as registers do.  Returns the bytes of shared memory of a block.
static size_t residual_pipe(ResidualParams &p, const ResidualGrid &g, bool vec, bool forward, int size_s, int size_d, int room)
{
    const int units = g.block ? 1 : g.threads / 32, teams = g.block ? 1 : 32 / g.team;
    uint32_t at = 0;
    auto place = [&](PipeArray &a, const void *array, uint32_t ld, int size) {
        const uint32_t row = (uint32_t)p.width * size;
        a = PipeArray{(const char *)array, ld, row, vec ? row : (row + 30) & ~15u, at};
        if (array) at += teams * a.slot_bytes;
    };
    int k = 0;
    if (forward) {
        place(p.pipe[k++], p.x, p.ld_x, size_s);
    } else {
        place(p.pipe[k++], p.pre_norm ? p.dn : nullptr, p.ld_dn, size_d);
        place(p.pipe[k++], p.pre_norm ? p.y : nullptr, p.ld_y, size_s);
        place(p.pipe[k++], p.dy, p.ld_dy, size_s);
    }
    place(p.pipe[k++], p.h, p.ld_h, size_d);
    place(p.pipe[k++], p.gate, p.ld_gate, size_d);
    p.copy_bytes = vec ? at / teams : 0;
    p.unit_teams = teams;
    p.stage_bytes = std::max(at, 16u);
    const int64_t all = (int64_t)p.stage_bytes * units;
    p.stages = (int)std::max<int64_t>(2, std::min<int64_t>(8, (int64_t)room * g.threads / all));
    while (p.stages > 1 && p.stages * all > RN_MAX_ROWS_SMEM) --p.stages;  // blocks of 1024 threads: down to one, nothing under way
    return (size_t)(p.stages * (all + 8 * units));
}

// Which variant: the biases' registers are spared where rows are on 16 bytes and of at most 2,048 columns; the others (half as many
// variants to build) are bound by other things.
static bool residual_bias(bool wanted, bool vec, int width) { return wanted || !vec || width > 8 * 256; }

typedef void (*ResidualKernel)(ResidualParams);
template <typename TS, typename TD, bool VEC, bool BIAS> static ResidualKernel residual_kernel(int threads, bool block)
{
    if (threads > 256) return residual_norm_kernel<TS, TD, VEC, 1024, true>;
    return block ? residual_norm_kernel<TS, TD, VEC, 256, BIAS> : residual_norm_kernel<TS, TD, VEC, 32, BIAS>;
}
template <typename TS, typename TD> static ResidualKernel residual_kernel(bool vec, bool bias, int threads, bool block)
{
    if (!vec) return residual_kernel<TS, TD, false, true>(threads, block);
    return bias ? residual_kernel<TS, TD, true, true>(threads, block) : residual_kernel<TS, TD, true, false>(threads, block);
}
template <typename TS, typename TD> static void residual_launch(Exec &ex, ResidualParams &p)
{
    const ResidualGrid g = residual_grid(p.rows, p.width, 256, 768);
    p.team = g.team;
    const bool vec = residual_vec(p, sizeof(TD)), bias = residual_bias(p.pre_bias || p.post_bias, vec, p.width);
    const size_t smem = residual_pipe(p, g, vec, true, sizeof(TS), sizeof(TD), 256);
    launch_dep(residual_kernel<TS, TD>(vec, bias, g.threads, g.block), dim3(g.blocks), dim3(g.threads), smem, ex.st, p);
    ex.launches += 1;
}

template <typename TS, typename TD, bool VEC, bool BIAS> static ResidualKernel residual_grad_kernel(int threads, bool block)
{
    if (threads > 256) return residual_norm_grad_kernel<TS, TD, VEC, 1024, true>;
    if (!block) return residual_norm_grad_kernel<TS, TD, VEC, 32, BIAS>;
    return threads > 128 ? residual_norm_grad_kernel<TS, TD, VEC, 256, BIAS> : residual_norm_grad_kernel<TS, TD, VEC, 128, BIAS>;
}
template <typename TS, typename TD> static ResidualKernel residual_grad_kernel(bool vec, bool bias, int threads, bool block)
{
    if (!vec) return residual_grad_kernel<TS, TD, false, true>(threads, block);
    return bias ? residual_grad_kernel<TS, TD, true, true>(threads, block) : residual_grad_kernel<TS, TD, true, false>(threads, block);
}
// vec, bias: residual_vec, residual_bias of this call
template <typename TS, typename TD> static void residual_grad_launch(Exec &ex, ResidualParams &p, const ResidualGrid &g, const ResidualSums &o, bool vec, bool bias, int accumulate)
{
    p.team = g.team;
    const size_t smem = residual_pipe(p, g, vec, false, sizeof(TS), sizeof(TD), 190 * 1024 / (bias ? RN_GRAD_RESIDENT<true> : RN_GRAD_RESIDENT<false>));
    launch_dep(residual_grad_kernel<TS, TD>(vec, bias, g.threads, g.block), dim3(g.blocks), dim3(g.threads), smem, ex.st, p);
    ex.launches += 1;
    int last = -1;
    for (int k = 0; k < RN_SUMS; ++k)
        if (o.out[k]) last = k;
    if (last < 0) return;
    launch_dep(residual_sums_kernel, dim3((unsigned)ceil_div64(p.width, 32), (unsigned)(last + 1)), dim3(32, 32), 0, ex.st, p.partial, g.blocks, p.width, o, accumulate);
    ex.launches += 1;
}

// The shared memory limit of every variant, once for a device: a limit set for one call could be lowered by a call of another thread
// before its launch.
template <typename TS, typename TD> static bool residual_init_types()
{
    const int threads[] = {256, 128, 256, 1024};  // parts of warps, and blocks of each kind
    for (int i = 0; i < 4; ++i)
        for (int k = 0; k < 4; ++k)
            for (ResidualKernel f : {residual_kernel<TS, TD>(i & 1, i & 2, threads[k], k > 0), residual_grad_kernel<TS, TD>(i & 1, i & 2, threads[k], k > 0)})
                if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, RN_MAX_SMEM) != cudaSuccess) return false;
    return true;
}
static bool residual_init(std::string &err)
{
    if (residual_init_types<float, float>() && residual_init_types<float, bf16>() && residual_init_types<bf16, bf16>()) return true;
    err = "cannot raise the dynamic shared memory limit of the residual norms";
    return false;
}
