// Products with one weight matrix per group of rows, and their weight gradients, on the tensor cores.
//
//   grouped linear       rows offsets[g] .. offsets[g + 1] - 1:  C = act(A B[g] + bias[g])    (B[g] [K, N], or [N, K]: transposed)
//   grouped weight grad  dW[g] = A_g^T dZ_g,  dbias[g] = column sums of dZ_g
//
// The accumulator of the matrix instructions rounds towards zero, so what it adds up drifts by up to 2^-23 per addition of 16 terms.  BF16
// operands go to the matrix instructions as they are, 512 terms at a time, and these sums are added in FP32 registers (in one
// accumulator 2^20 terms of one sign came out 0.6 % too small; 65,536 x 1,024 x 1,024 takes 109 us where one accumulator took 106).
// FP32 operands are split into three BF16 numbers of eight bits each, x = x0 + x1 + x2 exactly (the upper half of the word, of the
// rest, and of the rest's rest), and of the nine products the six larger ones are taken, so that a product is off by about 2^-23; the
// accumulator adds up 64 terms, small products first.
//
// Persistent blocks of 20 warps, one per SM.  Sizes of the groups are on the device: one warp walks the offsets, 32 groups at a time,
// and finds the block's tiles (linear) or its share of the 64-row blocks of all tiles (weight gradient) without any plan or host read.
// It runs a few tiles ahead of the others, who read where they lie from shared memory (every role walking for itself took 2,500 cycles
// a tile, four times what a block of 64 terms takes).
//   warp 0    operands by TMA         warp 1   matrix instructions        warp 2   where the tiles lie
//   others    sums and results; FP32: the last eight bring in the operands that have to be split, through registers
// Large BF16 products take pairs of SMs (cta_group::2) and tiles of 256 x 256: a 64-term block then costs 32 KiB of operands per SM for
// 512 cycles of products, where a block of its own with 128 x 256 would need 48 KiB.
// Of FP32 operands one is split into its parts before (the matrices B; A of the weight gradient) and comes by TMA, the other is split on
// its way through registers.  BF16 operands whose rows do not start on 16 bytes are copied to rows that do (TMA takes no others), FP32
// ones, too, so that they can be read 16 bytes at a time.
// The weight gradient deals out equal shares of 64-row blocks: a tile that lies in several shares is written as partial tiles,
// added in a fixed order by a second kernel.  Bits do not depend on anything but the sizes.
//
// Measured on the device at 1,965 MHz (copy rate 6.55 TB/s, BF16 products 1,648 TFLOP/s); thousands of the large calls in a row meet the
// power cap, which takes the clock to 1,500 to 1,800 MHz:
//   linear, BF16, 196,608 rows, 256 -> 256, 8 groups       37 us: 5.5 TB/s, either layout of B
//   linear, BF16, 30,011 rows, 1,999 -> 1,000, transposed, 40 groups   111 us: 1.1 PFLOP/s (610 cycles per block of 64 terms, 512 of them
//                                                          products), after 94 us that copy both operands to aligned rows; 230 us in all under the cap
//   weight gradient, BF16, 196,608 rows, 256 x 256, 8 groups   59 us and 11 us for shared tiles: 1,200 cycles per block of 64 rows where HBM
//                                                          allows 1,400 at best, then 3 us to start, 7 us to write 19 MB of partial tiles
//   linear, FP32, 100,003 rows, 256 -> 512, 16 groups      199 us (216 under the cap): 790 TFLOP/s of BF16 products.  A block of 64 terms
//                                                          takes 2,500 cycles, 1,536 of them products.  Without the loads of A 157 us, without its
//                                                          stores either 141, with one of the six products 200 (of 212): the ways through shared
//                                                          memory (320 KB a block by count) and two stages share the time.  Transposed, 512 -> 256: 209
//   weight gradient, FP32, 30,011 rows, 417 x 1,000, 40 groups    362 us, and 29 us before and after it; 100,003 rows, 256 x 512, 16 groups
//                                                          264 us, 36 us for the parts of A before it and 9 us after it
//   196,608 rows, 64 -> 64 BF16 (weight gradient), rows spread evenly over 1,000 groups 38 us (59), 10,000 groups 207 us (345), 100,000
//                                                          groups 2.6 ms (3.9): tiles of a few rows; the walk takes about half a microsecond per 32
//                                                          groups, 16 ms (37, it walks twice) for 2^20
// Tried for FP32 and not faster (product, weight gradient; 64 terms with two stages and all loaders on one block: 210 to 218, 425 to 433 us):
// blocks of 32 terms with four stages 249, 558, and with four groups of loaders that take blocks in turn 235, 495; two such groups with
// blocks of 64 terms 222, 413 (and 17 instead of 15 us for 768 rows); the next tile's rows asked into L2 one tile earlier 237, 469.
#pragma once
#include "gemm_tc.cuh"
#include "orthogonal.cuh"

enum { GP_NN = 0, GP_NT = 1, GP_WGRAD = 2 };
constexpr int GP_THREADS = 640;
// Registers of the warpgroups: 5 x 96 at the launch, moved to those that hold sums and pieces of operands
constexpr int GP_REGS_CONTROL = 48, GP_REGS_SUMS = 104, GP_REGS_LOADS = 112;
static_assert(GP_REGS_CONTROL + 2 * GP_REGS_SUMS + 2 * GP_REGS_LOADS <= 5 * 96 && GP_REGS_CONTROL + 4 * GP_REGS_SUMS <= 5 * 96, "the block was launched with fewer");
template <int N> LP_DEVINL void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> LP_DEVINL void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <bool WIDE> constexpr int GP_EXTRA_SMEM = WIDE ? 65536 : 32768;  // results on their way out (WIDE: 128 bytes of a row at a time), sums of columns
constexpr int GP_JOBS = 4;  // tiles that are known ahead
constexpr int GP_MAX_STAGES = 8;
constexpr int GP_MAX_GROUPS = 1 << 20;
template <typename T> constexpr int GP_FLUSH = sizeof(T) == 4 ? 1 : 8;  // blocks of 64 terms that an accumulator adds up

struct GroupedSplit {  // a tile of the weight gradient that several blocks share, noted by the first of them; first_slot < 0: none
    int group, kt, nt, first_slot, last_block;
    int64_t blocks;    // 64-row blocks of the whole launch, from which the shares follow
};

struct GroupedParams {
    const int *offsets;      // [groups + 1]
    int groups;
    int rows;                // of A; offsets are clamped to [0, rows]
    int N, K;                // linear: columns of C, of A; weight gradient: columns of dZ, of A
    int tiles_n, tiles_k;    // tiles_k: weight gradient only
    const float *reg;        // FP32: the operand that comes through registers (A; dZ of the weight gradient), rows on 16 bytes
    int64_t ld_reg;
    int stages, flush;       // flush: GP_FLUSH
    // linear
    const float *bias;
    int relu;
    void *C;
    int64_t ldc;
    int vec_c, vec_bias;     // rows on 16 bytes
    int tma_c;               // whole tiles of rows leave by TMA
    // weight gradient
    float *dW, *dbias;
    int accumulate;
    float *slots;            // partial tiles, two per block
    GroupedSplit *splits;    // one per block
    int *offsets_err;
    int *err;
    unsigned long long wait_ns;
    int extra_tx;
};

// ---------------------------------------------------------------------------------------------
// who works on what
// ---------------------------------------------------------------------------------------------
// A warp's window of 32 groups.  Offsets that decrease or leave [0, rows] count as the nearest ones that do not, so that no tile can
// leave the arrays and no two groups share a row.
template <bool WGRAD, int ROWS> struct GroupWalk {  // ROWS: of a tile (linear)
    const int *off;
    int groups, rows;
    int g0, before, last;        // first group of the window, tiles before it, end of the group before it
    int begin, end, incl, total; // of this lane's group; tiles up to and with it; tiles of the window
    LP_DEVINL int count(int size) const { return WGRAD ? max(1, (size + 63) >> 6) : (size + ROWS - 1) / ROWS; }
    LP_DEVINL void window()
    {
        const int lane = threadIdx.x & 31, g = g0 + lane;
        end = g < groups ? min(max(off[g + 1], last), rows) : last;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, end, o);
            if (lane >= o) end = max(end, x);
        }
        begin = __shfl_up_sync(0xffffffffu, end, 1);
        if (lane == 0) begin = last;
        incl = g < groups ? count(end - begin) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        total = __shfl_sync(0xffffffffu, incl, 31);
    }
    LP_DEVINL GroupWalk(const GroupedParams &p) : off(p.offsets), groups(p.groups), rows(p.rows), g0(0), before(0)
    {
        last = min(max(off[0], 0), rows);
        window();
    }
    LP_DEVINL bool step()
    {
        if (g0 + 32 >= groups) return false;
        last = __shfl_sync(0xffffffffu, end, 31);
        before += total;
        g0 += 32;
        window();
        return true;
    }
    // group that holds tile t (not below an earlier one), its rows, and the tiles before it
    LP_DEVINL bool seek(int t, int &g, int &b, int &e, int &pre)
    {
        while (t >= before + total)
            if (!step()) return false;
        const int l = __ffs(__ballot_sync(0xffffffffu, before + incl > t)) - 1;
        g = g0 + l;
        b = __shfl_sync(0xffffffffu, begin, l);
        e = __shfl_sync(0xffffffffu, end, l);
        pre = before + __shfl_sync(0xffffffffu, incl, l) - count(e - b);
        return true;
    }
    LP_DEVINL int all()
    {
        while (step()) {}
        return before + total;
    }
};

struct GroupedJob {
    int g, row0, row_end;  // linear: rows of the tile; weight gradient: rows of the share.  g < 0: no more
    int kt, nt, kbs;       // tile, blocks of 64 terms
    int slot;              // weight gradient: partial tile of the worker, or -1: the whole tile is in this share
    int unused;
};

// `worker` of `workers`: block or pair of blocks
template <int MODE, int ROWS> struct GroupedJobs {
    GroupWalk<MODE == GP_WGRAD, ROWS> walk;
    const GroupedParams &p;
    int worker, workers;
    int mt, nt;              // linear: next tile
    int64_t u, lo, hi, all;  // weight gradient: 64-row blocks of this share and of all
    GroupedSplit split;      // ... the tile that this worker begins and others go on with
    LP_DEVINL GroupedJobs(const GroupedParams &p_, int worker_, int workers_) : walk(p_), p(p_), worker(worker_), workers(workers_), split{0, 0, 0, -1, 0, 0}
    {
        if (MODE == GP_WGRAD) {
            GroupWalk<MODE == GP_WGRAD, ROWS> w(walk);
            all = (int64_t)w.all() * p.tiles_k * p.tiles_n;
            u = lo = all * worker / workers;
            hi = all * (worker + 1) / workers;
        } else {
            mt = worker / p.tiles_n;
            nt = worker - mt * p.tiles_n;
        }
    }
    LP_DEVINL bool next(GroupedJob &j)
    {
        int b, e, pre;
        if (MODE != GP_WGRAD) {
            if (!walk.seek(mt, j.g, b, e, pre)) return false;
            j.nt = nt;
            j.row0 = b + (mt - pre) * ROWS;
            j.row_end = min(e, j.row0 + ROWS);
            j.kt = 0;
            j.kbs = (p.K + 63) >> 6;
            j.slot = -1;
            const int step = workers / p.tiles_n;
            mt += step;
            nt += workers - step * p.tiles_n;
            if (nt >= p.tiles_n) { nt -= p.tiles_n; ++mt; }
            return true;
        }
        if (u >= hi) return false;
        const int tiles = p.tiles_k * p.tiles_n;
        if (!walk.seek((int)(u / tiles), j.g, b, e, pre)) return false;
        const int blocks = walk.count(e - b);
        const int64_t q = u - (int64_t)pre * tiles;
        const int tile = (int)(q / blocks), kb0 = (int)(q - (int64_t)tile * blocks);
        j.kbs = (int)min((int64_t)(blocks - kb0), hi - u);
        j.kt = tile / p.tiles_n;
        j.nt = tile - j.kt * p.tiles_n;
        j.row0 = b + kb0 * 64;
        j.row_end = min(e, j.row0 + j.kbs * 64);
        j.slot = kb0 == 0 && j.kbs == blocks ? -1 : 2 * worker + (u == lo ? 0 : 1);
        // only the last share of a worker can begin a tile that others go on with: up to the one that has its last block
        if (kb0 == 0 && j.slot >= 0) split = GroupedSplit{j.g, j.kt, j.nt, j.slot, (int)(((u + blocks) * workers - 1) / all), all};
        u += j.kbs;
        return true;
    }
};

// Bounded wait that looks at the time only after some thousand cycles: reading it takes longer than most waits do.
LP_DEVINL bool wait_bar(uint32_t bar, uint32_t parity, unsigned long long limit_ns)
{
    for (int i = 0; i < 512; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait(bar, parity, limit_ns);
}

// ---------------------------------------------------------------------------------------------
// operands through registers
// ---------------------------------------------------------------------------------------------
// eight neighbouring elements of an FP32 row on 16 bytes, zeros beyond its end
struct Piece8 {
    float v[8];
    LP_DEVINL void load(const float *row, int col, int limit)
    {
        const int n = limit - col;  // > 0
        const float4 a = __ldg(reinterpret_cast<const float4 *>(row + col));
        const float4 b = n > 4 ? __ldg(reinterpret_cast<const float4 *>(row + col) + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        if (n < 8)  // of the last 16 bytes, which lie on one page, some may not be the row's
#pragma unroll
            for (int i = 1; i < 8; ++i) v[i] = i < n ? v[i] : 0.f;
    }
    LP_DEVINL void zero()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    // part q of the values goes to put(q, 16 bytes)
    template <typename F> LP_DEVINL void parts(F put) const
    {
        float r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = v[i];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            uint32_t x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __byte_perm(__float_as_uint(r[2 * i]), __float_as_uint(r[2 * i + 1]), 0x7632);  // the upper halves
            put(q, make_uint4(x[0], x[1], x[2], x[3]));
            if (q < 2)
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] -= __uint_as_float(__float_as_uint(r[i]) & 0xffff0000u);  // exact
        }
    }
};

// A matrix copied to rows that start on 16 bytes: `width` elements in rows of `ld_out`, 16 bytes per thread out of the one or two aligned
// pieces of 16 bytes that hold them (word by word the loads took a third longer than HBM does).  A piece with a byte of the row lies in
// the row's page.
template <typename T> __global__ void __launch_bounds__(256) grouped_align_kernel(const T *in, int64_t rows, int width, int64_t ld_in, T *out, int64_t ld_out)
{
    LP_DEP_ENTER();
    constexpr int E = 16 / sizeof(T);
    const int64_t per = ld_out / E, i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per;
    if (row >= rows) return;
    const int col = (int)(i - row * per) * E, n = min(E, width - col);
    const uintptr_t src = (uintptr_t)(in + row * ld_in + col);
    const int m = (int)(src & 15);
    const uint4 *piece = reinterpret_cast<const uint4 *>(src & ~(uintptr_t)15);
    const uint4 a = __ldg(piece), b = m + n * (int)sizeof(T) > 16 ? __ldg(piece + 1) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int k = 0; k < 6; ++k) w[k] = m & 8 ? w[k + 2] : w[k];
#pragma unroll
    for (int k = 0; k < 5; ++k) w[k] = m & 4 ? w[k + 1] : w[k];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], 8 * (m & 3));
    *reinterpret_cast<uint4 *>(out + row * ld_out + col) = make_uint4(w[0], w[1], w[2], w[3]);
}

// An FP32 matrix as its three parts, each in rows of `ld_out` BF16 numbers, `part` elements apart
__global__ void __launch_bounds__(256) grouped_split_kernel(const float *in, int64_t rows, int width, int64_t ld_in, int vec, bf16 *out, int64_t ld_out, int64_t part)
{
    LP_DEP_ENTER();
    const int64_t per = ld_out / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per;
    if (row >= rows) return;
    const int col = (int)(i - row * per) * 8;
    Piece8 x;
    if (vec) {
        x.load(in + row * ld_in, col, width);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x.v[k] = col + k < width ? __ldg(in + row * ld_in + col + k) : 0.f;
    }
    x.parts([&](int q, const uint4 &w) { *reinterpret_cast<uint4 *>(out + q * part + row * ld_out + col) = w; });
}

// ---------------------------------------------------------------------------------------------
// results
// ---------------------------------------------------------------------------------------------
// A warp's results leave through shared memory, 32 rows of RB (64 or 128) bytes at a time: a lane puts its row there, and then the
// whole runs of a few rows are written: by one TMA store, or 512 bytes per store instruction where only some of the rows are the
// tile's (the end of a group) or the old values are added, or element by element where the rows of the result do not start on 16 bytes.
// The code is kept short: the roles of a block run different parts of it, and when these did not fit into the instruction cache together
// the results of an FP32 tile took 18,000 cycles.
template <typename T, int RB> constexpr int PUT_COLS = RB / sizeof(T);
template <int RB> LP_DEVINL int stage_place(int r, int q) { return r * RB + ((q ^ (RB == 128 ? r & 7 : (r >> 1) & 3)) << 4); }  // no two of eight lanes in the same banks
// N columns of the lane's row, from column c on
template <typename T, int RB, int N> LP_DEVINL void stage_columns(int c, const float *v, uint8_t *stage)
{
    constexpr int VN = Vec16<T>::N;
#pragma unroll
    for (int q = 0; q < N / VN; ++q) {
        Vec16<T> o;
        o.from_float(v + q * VN);
        *reinterpret_cast<decltype(o.v) *>(stage + stage_place<RB>(threadIdx.x & 31, c / VN + q)) = o.v;
    }
}
// the staged rows below `rows` and columns below `cols`
template <typename T, int RB> LP_DEVINL void put_staged(T *dst, int64_t ld, int rows, int cols, int vec, const uint8_t *stage, bool accumulate)
{
    constexpr int VN = Vec16<T>::N, PIECES = RB / 16, AT_ONCE = 32 / PIECES;  // rows of a store instruction
    const int lane = threadIdx.x & 31;
    __syncwarp();
    if (vec) {
        const int q = lane & (PIECES - 1);
        T *d = dst + (int64_t)(lane / PIECES) * ld + q * VN;
#pragma unroll 4
        for (int r = lane / PIECES; r < (q * VN < cols ? rows : 0) && r < 32; r += AT_ONCE, d += AT_ONCE * ld) {
            Vec16<T> o;
            o.v = *reinterpret_cast<const decltype(o.v) *>(stage + stage_place<RB>(r, q));
            if (accumulate) {
                Vec16<T> old;
                old.v = *reinterpret_cast<const decltype(o.v) *>(d);
                float x[VN], y[VN];
                old.to_float(x);
                o.to_float(y);
#pragma unroll
                for (int k = 0; k < VN; ++k) y[k] += x[k];
                o.from_float(y);
            }
            o.store(d);
        }
    } else {
        // a lane stays in its column
        constexpr int W = PUT_COLS<T, RB> < 32 ? PUT_COLS<T, RB> : 32, STEP = 32 / W;
#pragma unroll
        for (int first = 0; first < PUT_COLS<T, RB>; first += W) {
            const int c = first + lane % W, n = c < cols ? min(rows, 32) : 0;
            const uint8_t *src = stage + c % VN * (int)sizeof(T);
            T *d = dst + (int64_t)(lane / W) * ld + c;
#pragma unroll 8
            for (int r = lane / W; r < n; r += STEP, d += STEP * ld) {
                const T x = *reinterpret_cast<const T *>(src + stage_place<RB>(r, c / VN));
                *d = accumulate ? from_f<T>(to_f<T>(*d) + to_f<T>(x)) : x;
            }
        }
    }
    __syncwarp();
}
// all TMA stores of the warp but the last N have read their rows
template <int N> LP_DEVINL void stage_free()
{
    if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
    __syncwarp();
}
// ... by TMA where `map` says so and all 32 rows are the tile's
template <typename T, int RB>
LP_DEVINL void put_rows(const CUtensorMap *map, int col, int row, T *dst, int64_t ld, int rows, int cols, int vec, const uint8_t *stage)
{
    if (map && rows >= 32) {
        fence_async_proxy();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) {
            tma_store_2d(map, smem_u32(stage), col, row);
            tma_store_commit();
        }
    } else {
        put_staged<T, RB>(dst, ld, rows, cols, vec, stage, false);
    }
}
// bias and ReLU of N columns
template <int N> LP_DEVINL void finish_columns(float *v, const float *bias, int vec, int cols, int relu)
{
    if (bias) {
        if (vec && cols >= N) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float4 x = __ldg(reinterpret_cast<const float4 *>(bias + i));
                v[i] += x.x; v[i + 1] += x.y; v[i + 2] += x.z; v[i + 3] += x.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += i < cols ? __ldg(bias + i) : 0.f;
        }
    }
    if (relu)
#pragma unroll
        for (int i = 0; i < N; ++i) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(v[i]));  // NaN stays
}

// ---------------------------------------------------------------------------------------------
// kernel
// ---------------------------------------------------------------------------------------------
// copies into this block's shared memory, counted on a barrier of this block or (PAIR) of the pair's first
template <bool PAIR> LP_DEVINL void tile_2d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    if (PAIR) tma_load_2d_pair(dst, map, bar, x, y);
    else tma_load_2d(dst, map, bar, x, y);
}
template <bool PAIR> LP_DEVINL void tile_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    if (PAIR)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map),
                     "r"(bar), "r"(x), "r"(y), "r"(z)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map),
                     "r"(bar), "r"(x), "r"(y), "r"(z)
                     : "memory");
}

// A worker (a block, or a pair of blocks) multiplies tiles of ROWS x BN.  BH: columns of B that a block brings in.
template <typename T> constexpr int GP_PARTS = sizeof(T) == 4 ? 3 : 1;
template <bool PAIR> constexpr int GP_BN = PAIR ? 256 : 128;
template <typename T> constexpr int GP_STAGE_BYTES = GP_PARTS<T> * (128 + 128) * 128;

template <int MODE, bool PAIR> constexpr bool GP_WIDE = MODE != GP_WGRAD && PAIR;

template <int MODE, typename T, bool PAIR>
__global__ void __launch_bounds__(GP_THREADS, 1) grouped_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
                                                                 const __grid_constant__ CUtensorMap mapC, const __grid_constant__ GroupedParams p)
{
    LP_DEP_ENTER();
    constexpr int PARTS = GP_PARTS<T>, BN = GP_BN<PAIR>, BH = 128, ROWS = PAIR ? 256 : 128, ACCS = 512 / BN;  // accumulators used in turn: all of tensor memory
    constexpr bool WGRAD = MODE == GP_WGRAD, SPLIT = PARTS == 3, TMA_A = !SPLIT || WGRAD, TMA_B = !SPLIT || !WGRAD;
    constexpr bool A_MN = WGRAD, B_MN = MODE != GP_NT;
    constexpr int EPI = SPLIT ? 8 : 16, COLS = BN * 4 / EPI;  // warps of sums and results, columns of each
    constexpr int LOADERS = SPLIT ? 8 : 0;
    constexpr uint32_t a_bytes = 128 * 128, b_bytes = BH * 128, stage_bytes = GP_STAGE_BYTES<T>, tma_bytes = (TMA_A ? PARTS * a_bytes : 0) + (TMA_B ? PARTS * b_bytes : 0);
    static_assert(!PAIR || PARTS == 1, "pairs take BF16 operands");
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_full[GP_MAX_STAGES], bar_empty[GP_MAX_STAGES], bar_read[GP_MAX_STAGES], bar_acc_full[ACCS], bar_acc_empty[ACCS], bar_sum_full, bar_sum_empty,
        bar_done, bar_tail[GP_MAX_STAGES];
    __shared__ __align__(8) uint64_t bar_job_full[GP_JOBS], bar_job_empty[GP_JOBS];
    __shared__ __align__(16) GroupedJob jobs_s[GP_JOBS];
    __shared__ uint32_t tmem_base_s;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)cluster_cta_rank() : 0, worker = PAIR ? blockIdx.x >> 1 : blockIdx.x, workers = PAIR ? gridDim.x >> 1 : gridDim.x;
    const bool leader = rank == 0;  // of a pair: issues its matrix instructions
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int S = p.stages;
    uint8_t *extra = smem + (size_t)S * stage_bytes;
    const bool sums = WGRAD && p.dbias != nullptr;

    if (warp == 2) {
        // ---- where the tiles lie (the first is found while the others set the block up)
        GroupedJobs<MODE, ROWS> jobs(p, worker, workers);
        GroupedJob w{};
        bool more = jobs.next(w), ok = true;
        if (blockIdx.x == 0) {
            bool bad = false;
            for (int g = lane; g <= p.groups; g += 32) bad |= p.offsets[g] < (g ? p.offsets[g - 1] : 0) || p.offsets[g] > p.rows;
            if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.offsets_err, 4);
        }
        tc_fence_before();
        __syncthreads();
        if (PAIR) cluster_barrier();
        fewer_registers<GP_REGS_CONTROL>();
        for (int at = 0, round = 0; ok;) {
            if (round > 0) {
                ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_job_empty[at]), (round & 1) ^ 1, p.wait_ns));
                if (!ok) { if (lane == 0) atomicExch(p.err, 9); break; }
            }
            if (!more) w.g = -1;
            if (lane == 0) {
                jobs_s[at] = w;
                mbar_arrive(smem_u32(&bar_job_full[at]));
            }
            __syncwarp();
            if (!more) break;
            more = jobs.next(w);
            if (++at == GP_JOBS) { at = 0; ++round; }
        }
        if (WGRAD && lane == 0) p.splits[blockIdx.x] = jobs.split;
        __syncwarp();
        __syncthreads();
        if (PAIR) cluster_barrier();
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(smem_u32(&bar_full[s]), (PAIR ? 2 : 1) + LOADERS);
            mbar_init(smem_u32(&bar_empty[s]), 1);
            mbar_init(smem_u32(&bar_read[s]), EPI);
            mbar_init(smem_u32(&bar_tail[s]), 1);
        }
        for (int b = 0; b < ACCS; ++b) {
            mbar_init(smem_u32(&bar_acc_full[b]), 1);
            mbar_init(smem_u32(&bar_acc_empty[b]), PAIR ? 2 * EPI : EPI);
        }
        mbar_init(smem_u32(&bar_sum_full), SPLIT ? LOADERS : EPI);
        mbar_init(smem_u32(&bar_sum_empty), BH / 32);
        for (int i = 0; i < GP_JOBS; ++i) {
            mbar_init(smem_u32(&bar_job_full[i]), 1);
            mbar_init(smem_u32(&bar_job_empty[i]), 1 + (leader ? 1 : 0) + (WGRAD ? 1 : 0) + EPI + LOADERS);
        }
        mbar_init(smem_u32(&bar_done), 1);
        fence_barrier_init();
        fence_async_proxy();
        if (TMA_A) tma_prefetch_desc(&mapA);
        if (TMA_B) tma_prefetch_desc(&mapB);
        if (!WGRAD && p.tma_c) tma_prefetch_desc(&mapC);
    }
    if (warp == 0) {
        __syncwarp();
        if (PAIR) tmem_alloc_pair(smem_u32(&tmem_base_s), ACCS * BN);
        else tmem_alloc(smem_u32(&tmem_base_s), ACCS * BN);
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_barrier();  // both blocks' barriers are there before either uses the other's
    tc_fence_after();
    const uint32_t tmem = tmem_base_s;
    GroupedJob j;
    int job_at = 0, job_round = 0;
    // this warp's next tile; false: there is none, or the wait ran out
    auto next_job = [&]() {
        bool there = wait_bar(smem_u32(&bar_job_full[job_at]), job_round & 1, p.wait_ns);
        there = __all_sync(0xffffffffu, there);
        if (!there) {
            if (lane == 0) atomicExch(p.err, 9);
            return false;
        }
        j = jobs_s[job_at];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar_job_empty[job_at]));
        if (++job_at == GP_JOBS) { job_at = 0; ++job_round; }
        return j.g >= 0;
    };

    if (warp == 0) {
        fewer_registers<GP_REGS_CONTROL>();
        {
            // ---- operands by TMA: this block's 128 rows (weight gradient: columns) of A and its BH columns of B
            int s = 0, round = 0;
            bool ok = true, first = blockIdx.x == (WGRAD ? gridDim.x - 1 : 0);  // a block that has work in any case
            while (ok && next_job()) {
                for (int kb = 0; kb < j.kbs && ok; ++kb) {
                    if (round > 0) {
                        ok = wait_bar(smem_u32(&bar_empty[s]), (round & 1) ^ 1, p.wait_ns) && (SPLIT || !sums || wait_bar(smem_u32(&bar_read[s]), (round & 1) ^ 1, p.wait_ns));
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) { if (lane == 0) atomicExch(p.err, 1); break; }
                    }
                    const uint32_t sa = smem_u32(smem) + s * stage_bytes, sb = sa + PARTS * a_bytes;
                    uint32_t bar = smem_u32(&bar_full[s]);
                    const int have = j.row_end - (j.row0 + kb * 64);
                    const bool tail = WGRAD && have < 64;  // the last rows of a group: warp 3 gets them first
                    if (elect_one()) {
                        const uint32_t more = first ? (uint32_t)p.extra_tx : 0u;
                        if (tail) {
                            mbar_expect_tx(smem_u32(&bar_tail[s]), tma_bytes + more);
                            bar = smem_u32(&bar_tail[s]);
                            if (PAIR) bar = map_to_cta(bar, rank);
                        } else if (PAIR) {
                            bar = map_to_cta(bar, 0);
                            mbar_expect_tx_remote(bar, tma_bytes + more);
                        } else {
                            mbar_expect_tx(bar, tma_bytes + more);
                        }
                        if (WGRAD) {
                            const int row = j.row0 + kb * 64;
#pragma unroll
                            for (int q = 0; q < PARTS; ++q)
#pragma unroll
                                for (int c = 0; c < 2; ++c) tile_3d<PAIR>(sa + q * a_bytes + c * 8192, &mapA, bar, j.kt * ROWS + rank * 128 + c * 64, row, q);
                            if (TMA_B)
#pragma unroll
                                for (int c = 0; c < 2; ++c) tile_2d<PAIR>(sb + c * 8192, &mapB, bar, j.nt * BN + rank * BH + c * 64, row);
                        } else {
                            if (TMA_A) tile_2d<PAIR>(sa, &mapA, bar, kb * 64, j.row0 + rank * 128);
#pragma unroll
                            for (int q = 0; q < PARTS; ++q) {
                                if (B_MN) {
#pragma unroll
                                    for (int c = 0; c < 2; ++c) tile_3d<PAIR>(sb + q * b_bytes + c * 8192, &mapB, bar, j.nt * BN + rank * BH + c * 64, kb * 64, q * p.groups + j.g);
                                } else {
                                    tile_3d<PAIR>(sb + q * b_bytes, &mapB, bar, kb * 64, j.nt * BN + rank * BH, q * p.groups + j.g);
                                }
                            }
                        }
                    }
                    __syncwarp();
                    first = false;
                    if (++s == S) { s = 0; ++round; }
                }
            }
            // copies under way land before the block gives up its shared memory (after a wait that ran out; else they long have; those of
            // a group's last block warp 3 waits for)
            if (lane == 0 && leader)
                for (int i = 0; i < S; ++i) {
                    const int at = s - 1 - i < 0 ? s - 1 - i + S : s - 1 - i, r = s - 1 - i < 0 ? round - 1 : round;
                    if (r >= 0) wait_bar(smem_u32(&bar_full[at]), r & 1, p.wait_ns);
                }
            __syncwarp();
        }
    } else if (warp == 1) {
        fewer_registers<GP_REGS_CONTROL>();
        // ---- products
        int s = 0, round = 0, use = 0;
        bool ok = true;
        const uint32_t idesc = (PAIR ? make_idesc_bf16_pair(BN) : make_idesc_bf16(BN, false, false)) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u);
        const uint64_t desc_a = make_smem_desc(smem_u32(smem), A_MN ? 8192 : 16, 1024), desc_b = make_smem_desc(smem_u32(smem) + PARTS * a_bytes, B_MN ? 8192 : 16, 1024);
        constexpr uint64_t step_a = (A_MN ? 2048 : 32) >> 4, step_b = (B_MN ? 2048 : 32) >> 4;
        auto product = [&](uint32_t acc, uint64_t da, uint64_t db, bool more) {
            if (PAIR) umma_bf16_pair(acc, da, db, idesc, more ? 1u : 0u);
            else umma_bf16(acc, da, db, idesc, more ? 1u : 0u);
        };
        auto commit = [&](uint64_t &bar) {
            if (PAIR) umma_commit_pair(smem_u32(&bar));
            else umma_commit(smem_u32(&bar));
        };
        while (leader && ok && next_job()) {
            int in_flush = 0;
            for (int kb = 0; kb < j.kbs && ok; ++kb) {
                const int b = use % ACCS;
                if (in_flush == 0 && use >= ACCS && !wait_bar(smem_u32(&bar_acc_empty[b]), ((use / ACCS) & 1) ^ 1, p.wait_ns)) {
                    if (lane == 0) atomicExch(p.err, 5);
                    ok = false;
                }
                if (ok && !wait_bar(smem_u32(&bar_full[s]), round & 1, p.wait_ns)) {
                    if (lane == 0) atomicExch(p.err, 2);
                    ok = false;
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const bool done = in_flush == p.flush - 1 || kb == j.kbs - 1;
                if (elect_one()) {
                    const uint64_t da = desc_a + ((s * stage_bytes) >> 4), db = desc_b + ((s * stage_bytes) >> 4);
                    const uint32_t acc = tmem + b * BN;
                    if (PARTS == 1) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) product(acc, da + i * step_a, db + i * step_b, in_flush != 0 || i != 0);
                    } else {
                        // parts 0 2, 2 0, 1 1, 0 1, 1 0, 0 0: the small products first, while the sums are small
#pragma unroll 1
                        for (int q = 0; q < 6; ++q) {
                            const uint64_t qa = da + ((0x021010u >> 4 * (5 - q)) & 3u) * (a_bytes >> 4), qb = db + ((0x201100u >> 4 * (5 - q)) & 3u) * (b_bytes >> 4);
#pragma unroll
                            for (int i = 0; i < 4; ++i) product(acc, qa + i * step_a, qb + i * step_b, in_flush != 0 || q != 0 || i != 0);
                        }
                    }
                    commit(bar_empty[s]);
                    if (done) commit(bar_acc_full[b]);
                }
                __syncwarp();
                in_flush = done ? 0 : in_flush + 1;
                if (done) ++use;
                if (++s == S) { s = 0; ++round; }
            }
        }
        // products under way are done with the memory of both blocks before they go, also after a wait that ran out
        if (leader) {
            if (elect_one()) commit(bar_done);
            __syncwarp();
            wait_bar(smem_u32(&bar_done), 0, p.wait_ns);
        }
        __syncwarp();
    } else if (warp == 3) {
        fewer_registers<GP_REGS_CONTROL>();
        if (WGRAD) {
            // ---- the last block of a group, before it is multiplied: rows behind the group belong to the next one (or to nobody): zeros in what TMA
            // brought, whatever they hold
            int at = 0;
            uint32_t phase = 0;  // of each stage's barrier
            bool ok = true;
            while (ok && next_job()) {
                const int kb = j.kbs - 1, have = j.row_end - (j.row0 + kb * 64);
                at += j.kbs;
                if (have >= 64) continue;
                const int s = (at - 1) % S;
                ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_tail[s]), phase >> s & 1, p.wait_ns));
                if (!ok) { if (lane == 0) atomicExch(p.err, 2); break; }
                phase ^= 1u << s;
                uint8_t *st = smem + (size_t)s * stage_bytes + max(have, 0) * 128;
                for (int i = lane; i < (64 - max(have, 0)) * 8; i += 32)
#pragma unroll
                    for (int c = 0; c < (SPLIT ? 6 : 4); ++c) *reinterpret_cast<uint4 *>(st + c * 8192 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                fence_async_proxy();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) mbar_arrive_remote(map_to_cta(smem_u32(&bar_full[s]), 0));
                    else mbar_arrive(smem_u32(&bar_full[s]));
                }
            }
        }
    } else if (warp < 4 + EPI) {
        more_registers<GP_REGS_SUMS>();
        // ---- sums and results: 32 rows x COLS columns per warp
        const int quarter = warp & 3, part = (warp - 4) >> 2;
        const int epi_thread = threadIdx.x - 128;
        constexpr int OUT = GP_WIDE<MODE, PAIR> || (SPLIT && !WGRAD) ? 4096 : 2048;  // bytes of a warp's results on their way
        uint8_t *stage = extra + (warp - 4) * OUT;
        const uint32_t acc_free = PAIR ? map_to_cta(smem_u32(&bar_acc_empty[0]), 0) : smem_u32(&bar_acc_empty[0]);
        int use = 0, s = 0, round = 0, summed = 0;
        bool ok = true;
        // the accumulator that holds the next sums; false when the wait ran out
        auto take = [&](uint32_t &at) {
            const int b = use % ACCS;
            ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_acc_full[b]), (use / ACCS) & 1, p.wait_ns));
            if (!ok) { if (lane == 0) atomicExch(p.err, 3); return false; }
            tc_fence_after();
            at = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(b * BN + part * COLS);
            return true;
        };
        auto give_back = [&]() {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR) mbar_arrive_remote(acc_free + (use % ACCS) * 8);
                else mbar_arrive(acc_free + (use % ACCS) * 8);
            }
            ++use;
        };
        while (ok && next_job()) {
            const int c0 = j.nt * BN + part * COLS;  // first column of this warp
            if (!WGRAD && PARTS == 1 && j.kbs <= p.flush) {
                // one accumulator holds all terms: from tensor memory straight to the result
                const int row = j.row0 + rank * 128 + quarter * 32;
                T *dst = (T *)p.C + (int64_t)row * p.ldc + c0;
                const float *bias = p.bias ? p.bias + (int64_t)j.g * p.N + c0 : nullptr;
                uint32_t at;
                if (!take(at)) break;
                if (p.tma_c) stage_free<0>();
#pragma unroll 1
                for (int c = 0; c < COLS; c += 32) {
                    float v[32];
                    tmem_ld_32x16(at + c, v);
                    tmem_ld_32x16(at + c + 16, v + 16);
                    tmem_ld_wait();
                    if (c + 32 >= COLS) give_back();
                    finish_columns<32>(v, bias ? bias + c : nullptr, p.vec_bias, p.N - (c0 + c), p.relu);
                    stage_columns<T, COLS * 2, 32>(c, v, stage);
                }
                if (c0 < p.N) put_rows<T, COLS * 2>(p.tma_c ? &mapC : nullptr, c0, row, dst, p.ldc, j.row_end - row, p.N - c0, p.vec_c, stage);
                continue;
            }
            float v[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) v[c] = 0.f;
            float col[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            const bool adds = sums && !SPLIT && j.kt == 0;
            int in_flush = 0;
            for (int kb = 0; kb < j.kbs && ok; ++kb) {
                if (!SPLIT && sums) {
                    // column sums of dZ out of the staged tiles, once their products are done: eight columns (a piece of 16 bytes) of two rows per thread
                    constexpr int PIECES = BH / 8, RPT = 64 * PIECES / (EPI * 32);
                    ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_empty[s]), round & 1, p.wait_ns));
                    if (!ok) { if (lane == 0) atomicExch(p.err, 4); break; }
                    if (adds) {
                        const int piece = epi_thread % PIECES, r0 = epi_thread / PIECES * RPT, have = j.row_end - (j.row0 + kb * 64);
                        const uint8_t *sb = smem + (size_t)s * stage_bytes + a_bytes + (piece >> 3) * 8192;
#pragma unroll
                        for (int i = 0; i < RPT; ++i) {
                            const int r = r0 + i;
                            if (r < have) {
                                Vec16<bf16> x;
                                x.v = *reinterpret_cast<const uint4 *>(sb + r * 128 + (((piece & 7) ^ (r & 7)) << 4));
                                float f[8];
                                x.to_float(f);
                                add8(col, f);
                            }
                        }
                        __syncwarp();
                    }
                    if (lane == 0) mbar_arrive(smem_u32(&bar_read[s]));
                    if (++s == S) { s = 0; ++round; }
                }
                const bool done = in_flush == p.flush - 1 || kb == j.kbs - 1;
                in_flush = done ? 0 : in_flush + 1;
                if (!done) continue;
                uint32_t at;
                if (!take(at)) break;
#pragma unroll
                for (int c = 0; c < COLS; c += 16) {
                    float x[16];
                    tmem_ld_32x16(at + c, x);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[c + i] += x[i];
                }
                give_back();
            }
            if (!ok) break;
            if (summed > 0) {  // the column sums of the job before have been read
                ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_sum_empty), (summed - 1) & 1, p.wait_ns));
                if (!ok) { if (lane == 0) atomicExch(p.err, 7); break; }
            }
            if (!WGRAD && PARTS == 1) {
                const int row = j.row0 + rank * 128 + quarter * 32;
                if (p.tma_c) stage_free<0>();
                finish_columns<COLS>(v, p.bias ? p.bias + (int64_t)j.g * p.N + c0 : nullptr, p.vec_bias, p.N - c0, p.relu);
                stage_columns<T, COLS * 2, COLS>(0, v, stage);
                if (c0 < p.N) put_rows<T, COLS * 2>(p.tma_c ? &mapC : nullptr, c0, row, (T *)p.C + (int64_t)row * p.ldc + c0, p.ldc, j.row_end - row, p.N - c0, p.vec_c, stage);
            } else if (!WGRAD) {
                const int row = j.row0 + quarter * 32;
                T *dst = (T *)p.C + (int64_t)row * p.ldc + c0;
                constexpr int PC = PUT_COLS<T, 64>;
                finish_columns<COLS>(v, p.bias ? p.bias + (int64_t)j.g * p.N + c0 : nullptr, p.vec_bias, p.N - c0, p.relu);
#pragma unroll
                for (int c = 0; c < COLS; c += PC) {
                    if (c0 + c < p.N) {
                        // Two halves in turn.  Before a half is written, the TMA stores that read it are done: at the first piece none of the tile before
                        // is left (whose last store may have read either half, or come before rows that left without TMA), and within a tile either every
                        // piece is a store, so that the one that may still be reading has the other half, or (fewer than 32 rows) none is.
                        uint8_t *half = stage + (c / PC & 1) * 2048;
                        if (p.tma_c) {
                            if (c == 0) stage_free<0>();
                            else stage_free<1>();
                        }
                        stage_columns<T, 64, PC>(0, v + c, half);
                        put_rows<T, 64>(p.tma_c ? &mapC : nullptr, c0 + c, row, dst + c, p.ldc, j.row_end - row, p.N - (c0 + c), p.vec_c, half);
                    }
                }
            } else {
                // the whole tile is this share's, or a partial tile of it
                const bool whole = j.slot < 0;
                const int row = j.kt * ROWS + rank * 128 + quarter * 32;
                float *dst = whole ? p.dW + ((int64_t)j.g * p.K + row) * p.N + c0
                                   : p.slots + (((size_t)j.slot * (ROWS / 128) + rank) * 129 + quarter * 32) * BN + part * COLS;
                const int ld = whole ? p.N : BN, rows = whole ? p.K - row : 32, cols = whole ? p.N - c0 : COLS, vec = whole ? p.vec_c : 1;
#pragma unroll
                for (int c = 0; c < COLS; c += 16)
                    if (c < cols) {
                        stage_columns<float, 64, 16>(0, v + c, stage);
                        put_staged<float, 64>(dst + c, ld, rows, cols - c, vec, stage, whole && p.accumulate != 0);
                    }
            }
            if (adds) {
                // every warp leaves its sums of a few rows in its own part of the area; the first BH threads add them up in order
                constexpr int PIECES = BH / 8, SHARES = EPI * 32 / PIECES;
                const float *area = reinterpret_cast<const float *>(extra);
                float *own = reinterpret_cast<float *>(stage);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) own[lane * 8 + i] = col[i];
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_sum_full));
                if (epi_thread < BH) {
                    ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_sum_full), summed & 1, p.wait_ns));
                    if (!ok) { if (lane == 0) atomicExch(p.err, 7); break; }
                    float x = 0.f;
#pragma unroll
                    for (int i = 0; i < SHARES; ++i) {
                        const int writer = i * PIECES + epi_thread / 8;  // thread that has these columns of share i
                        x += area[(writer >> 5) * (OUT / 4) + (writer & 31) * 8 + (epi_thread & 7)];
                    }
                    const int in_tile = rank * BH + epi_thread, c = j.nt * BN + in_tile;
                    if (j.slot >= 0) p.slots[(((size_t)j.slot * (ROWS / 128) + rank) * 129 + 128) * BN + in_tile] = x;
                    else if (c < p.N) {
                        float *d = p.dbias + (int64_t)j.g * p.N + c;
                        *d = p.accumulate ? *d + x : x;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bar_sum_empty));
                }
                ++summed;
            }
        }
        if (!WGRAD && lane == 0) tma_store_wait_all();
    } else if (SPLIT) {
        more_registers<GP_REGS_LOADS>();
        // ---- the FP32 operand that is split on its way: four pieces per thread and block of 64 terms.  While those of one block are put
        // down, those of the next are under way, and what comes after them is asked into L2.
        constexpr bool MN = WGRAD;
        constexpr uint32_t part = WGRAD ? b_bytes : a_bytes;
        const int lt = threadIdx.x - (4 + EPI) * 32;
        uint8_t *const first = smem + (WGRAD ? PARTS * a_bytes : 0);
        int s = 0, round = 0, summed = 0;
        bool ok = true;
        Piece8 x[4], y[4];
        float col[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        auto load = [&](Piece8 (&d)[4], int kb) {
            const int row = MN ? j.row0 + kb * 64 + (lt >> 4) : j.row0 + (lt >> 3), c = MN ? j.nt * 128 + 8 * (lt & 15) : kb * 64 + 8 * (lt & 7), limit = MN ? p.N : p.K;
            const float *at = p.reg + (int64_t)row * p.ld_reg;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = (MN ? 16 : 32) * i;
                if (row + r < j.row_end && c < limit) d[i].load(at + (int64_t)r * p.ld_reg, c, limit);
                else d[i].zero();
            }
        };
        auto ahead = [&](int kb) {  // into L2: 32 columns (a line) of one row per thread
            const int row = MN ? j.row0 + kb * 64 + (lt >> 2) : j.row0 + (lt >> 1), c = MN ? j.nt * 128 + 32 * (lt & 3) : kb * 64 + 32 * (lt & 1);
            if (row < j.row_end && c < (MN ? p.N : p.K)) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.reg + (int64_t)row * p.ld_reg + c));
        };
        auto put = [&](const Piece8 (&d)[4]) {
            uint8_t *dst = first + (size_t)s * stage_bytes;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int q = lt + 256 * i, r = MN ? q >> 4 : q >> 3, c = MN ? q & 15 : q & 7;
                uint8_t *at = dst + (c >> 3) * 8192 + r * 128 + (((c & 7) ^ (r & 7)) << 4);
                d[i].parts([&](int k, const uint4 &w) { *reinterpret_cast<uint4 *>(at + k * part) = w; });
            }
        };
        int kb = 0, done_kt = 0, done_nt = 0, done_g = 0, done_slot = 0;
        bool more = next_job(), last = false;
        constexpr int AHEAD = 6;  // blocks that are asked into L2
        auto open_job = [&]() {
            for (int i = 0; i < AHEAD && i < j.kbs; ++i) ahead(i);
        };
        if (more) {
            open_job();
            load(x, 0);
        }
        // one block: the pieces in `cur` go into the stage, the next block's into `nxt`
        auto step = [&](Piece8 (&cur)[4], Piece8 (&nxt)[4]) {
            done_kt = j.kt; done_nt = j.nt; done_g = j.g; done_slot = j.slot;
            last = ++kb == j.kbs;
            if (last) {
                kb = 0;
                more = next_job();
                if (more) open_job();
            } else if (kb + AHEAD - 1 < j.kbs) {
                ahead(kb + AHEAD - 1);
            }
            if (more) load(nxt, kb);
            if (round > 0) {
                ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_empty[s]), (round & 1) ^ 1, p.wait_ns));
                if (!ok) { if (lane == 0) atomicExch(p.err, 1); return; }
            }
            put(cur);
            fence_async_proxy();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_full[s]));
            if (++s == S) { s = 0; ++round; }
            if (!sums || done_kt != 0) return;
#pragma unroll
            for (int i = 0; i < 4; ++i) add8(col, cur[i].v);
            if (!last) return;
            // a thread has the rows 16 i + lt / 16 of its eight columns: sixteen sums per column, added up in order
            float *area = reinterpret_cast<float *>(extra + EPI * 2048);
            if (summed > 0) ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_sum_empty), (summed - 1) & 1, p.wait_ns));
            if (ok) {
#pragma unroll
                for (int i = 0; i < 8; ++i) { area[(lt >> 4) * 128 + (lt & 15) * 8 + i] = col[i]; col[i] = 0.f; }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_sum_full));
                if (lt < 128) {
                    ok = __all_sync(0xffffffffu, wait_bar(smem_u32(&bar_sum_full), summed & 1, p.wait_ns));
                    if (ok) {
                        float v = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) v += area[i * 128 + lt];
                        const int c = done_nt * 128 + lt;
                        if (done_slot >= 0) p.slots[((size_t)done_slot * 129 + 128) * BN + lt] = v;
                        else if (c < p.N) {
                            float *d = p.dbias + (int64_t)done_g * p.N + c;
                            *d = p.accumulate ? *d + v : v;
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&bar_sum_empty));
                    }
                }
            }
            if (!ok && lane == 0) atomicExch(p.err, 7);
            ++summed;
        };
        while (more && ok) {
            step(x, y);
            if (!more || !ok) break;
            step(y, x);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_barrier();  // neither block frees tensor memory, or leaves with barriers the other may still signal, before both are done
    if (warp == 0) {
        __syncwarp();
        if (PAIR) tmem_dealloc_pair(tmem, ACCS * BN);
        else tmem_dealloc(tmem, ACCS * BN);
    }
}

// tiles that several workers share: their partial tiles added in the order of the workers.  gridDim.x = blocks of the product
template <bool PAIR> __global__ void __launch_bounds__(256) grouped_splits_kernel(const __grid_constant__ GroupedParams p)
{
    LP_DEP_ENTER();
    const GroupedSplit sp = p.splits[blockIdx.x];
    if (sp.first_slot < 0) return;
    constexpr int BN = GP_BN<PAIR>, BLOCKS = PAIR ? 2 : 1, AT_ONCE = 8, size = 129 * BN / 4;  // BLOCKS: of a worker; sizes in float4
    const int worker = blockIdx.x / BLOCKS, rank = blockIdx.x % BLOCKS, workers = gridDim.x / BLOCKS;
    const int at = blockIdx.y * 256 + threadIdx.x;
    if (at >= size) return;
    const float4 *slots = reinterpret_cast<const float4 *>(p.slots);
    const bool gaps = sp.blocks < workers;  // some workers have no share
    float4 v = slots[((size_t)sp.first_slot * BLOCKS + rank) * size + at];
    for (int c = worker + 1; c <= sp.last_block; c += AT_ONCE) {
        float4 x[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const bool there = c + k <= sp.last_block && !(gaps && sp.blocks * (c + k) / workers == sp.blocks * (c + k + 1) / workers);
            x[k] = there ? slots[((size_t)(2 * (c + k)) * BLOCKS + rank) * size + at] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) { v.x += x[k].x; v.y += x[k].y; v.z += x[k].z; v.w += x[k].w; }
    }
    const int row = at * 4 / BN, in_tile = at * 4 % BN, col = sp.nt * BN + in_tile, k = (sp.kt * BLOCKS + rank) * 128 + row;
    float *d;
    if (row < 128) {
        if (k >= p.K) return;
        d = p.dW + ((int64_t)sp.group * p.K + k) * p.N + col;
    } else {
        if (!p.dbias || sp.kt != 0 || in_tile / 128 != rank) return;  // a block adds up the 128 columns it brings in
        d = p.dbias + (int64_t)sp.group * p.N + col;
    }
    const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < p.N) d[i] = p.accumulate ? d[i] + w[i] : w[i];
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
template <int MODE, typename T, bool PAIR> static bool grouped_init_one(std::string &err)
{
    if (cudaFuncSetAttribute(grouped_kernel<MODE, T, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 1536) == cudaSuccess) return true;
    err = "cannot raise the dynamic shared memory limit of the grouped products";
    return false;
}
template <int MODE> static bool grouped_init_mode(std::string &err)
{
    return grouped_init_one<MODE, bf16, false>(err) && grouped_init_one<MODE, bf16, true>(err) && grouped_init_one<MODE, float, false>(err);
}
static bool grouped_init(std::string &err) { return grouped_init_mode<GP_NN>(err) && grouped_init_mode<GP_NT>(err) && grouped_init_mode<GP_WGRAD>(err); }

// tensor map over [matrices][rows][cols] BF16 matrices behind one another in rows of ld
static bool grouped_map_3d(const TcState &tc, CUtensorMap *map, const bf16 *base, int64_t matrices, int64_t rows, int64_t cols, int64_t ld, int box_rows, std::string &err)
{
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)matrices};
    cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * (cuuint64_t)rows * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
    if (tc.encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, (void *)base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS)
        return true;
    err = "cuTensorMapEncodeTiled failed";
    return false;
}

template <int MODE, typename T, bool PAIR> static void grouped_launch_one(Exec &ex, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &c, GroupedParams &p, int blocks)
{
    constexpr int stage = GP_STAGE_BYTES<T>;
    constexpr int extra = GP_EXTRA_SMEM<GP_WIDE<MODE, PAIR>>;
    p.stages = std::min(GP_MAX_STAGES, (227 * 1024 - 1536 - 1024 - extra) / stage);
    const size_t smem = (size_t)p.stages * stage + extra + 1024;
    if (PAIR) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)blocks);
        cfg.blockDim = dim3(GP_THREADS);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = ex.st;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        cudaLaunchKernelEx(&cfg, grouped_kernel<MODE, T, PAIR>, a, b, c, p);
    } else {
        launch_dep(grouped_kernel<MODE, T, PAIR>, dim3((unsigned)blocks), dim3(GP_THREADS), smem, ex.st, a, b, c, p);
    }
    ex.launches += 1;
    if (MODE == GP_WGRAD) {
        launch_dep(grouped_splits_kernel<PAIR>, dim3((unsigned)blocks, (unsigned)ceil_div64(129 * GP_BN<PAIR>, 1024)), dim3(256), 0, ex.st, p);
        ex.launches += 1;
    }
}

// an operand and, where its rows have to be copied or split first, its place in the workspace
struct GroupedOperand {
    const void *at;
    int64_t matrices, rows;    // rows: of a matrix
    int cols;
    int64_t ld;
    bool split;                // FP32 into three BF16 parts
    bool copied = false;
    size_t bytes = 0, offset = 0;
};
template <typename T> static GroupedOperand grouped_operand(const void *at, int64_t matrices, int64_t rows, int cols, int64_t ld, bool split, size_t &ws)
{
    GroupedOperand o{at, matrices, rows, cols, ld, split};
    o.copied = split || !on_16_bytes<T>(at, ld);
    if (o.copied) {
        const int64_t step = split ? 8 : 16 / (int64_t)sizeof(T);
        o.ld = ceil_div64(cols, step) * step;
        o.bytes = (size_t)(o.ld * rows * matrices) * (split ? 6 : sizeof(T));
        o.offset = ws;
        ws += (o.bytes + 255) & ~(size_t)255;
    }
    return o;
}
// makes the copy; the operand is then where `at` says
template <typename T> static void grouped_prepare(Exec &ex, GroupedOperand &o, int64_t ld_in, uint8_t *ws)
{
    if (!o.copied) return;
    const int64_t rows = o.matrices * o.rows;
    void *out = ws + o.offset;
    if (o.split) {
        launch_dep(grouped_split_kernel, dim3((unsigned)ceil_div64(rows * (o.ld / 8), 256)), dim3(256), 0, ex.st, (const float *)o.at, rows, o.cols, ld_in,
                   (int)(on_16_bytes<float>(o.at, ld_in)), (bf16 *)out, o.ld, o.ld * rows);
    } else {
        constexpr int E = 16 / sizeof(T);
        launch_dep(grouped_align_kernel<T>, dim3((unsigned)ceil_div64(rows * (o.ld / E), 256)), dim3(256), 0, ex.st, (const T *)o.at, rows, o.cols, ld_in, (T *)out, o.ld);
    }
    ex.launches += 1;
    o.at = out;
}

struct GroupedPlan {
    bool pair;
    int blocks;
    GroupedOperand a, b;
    size_t slots, splits, bytes;  // places in the workspace and its size
};
// Pairs of SMs and tiles of 256 x 256 where those keep most SMs busy (weight gradient: where the matrix fills such a tile), blocks of their
// own and tiles of 128 x 128 elsewhere and for FP32
template <int MODE, typename T> static GroupedPlan grouped_plan(int64_t rows, int64_t groups, int N, int K, const void *A, int64_t lda, const void *B, int64_t ldb)
{
    constexpr bool WGRAD = MODE == GP_WGRAD;
    GroupedPlan g{};
    g.a = grouped_operand<T>(A, 1, rows, K, lda, sizeof(T) == 4 && WGRAD, g.bytes);
    g.b = WGRAD ? grouped_operand<T>(B, 1, rows, N, ldb, false, g.bytes)
                : grouped_operand<T>(B, groups, MODE == GP_NN ? K : N, MODE == GP_NN ? N : K, ldb, sizeof(T) == 4, g.bytes);
    const int64_t sms = tc_sm_count(), busy = std::min(rows, groups);
    auto tiles = [&](int side) { return (WGRAD ? (ceil_div64(rows, 64) + groups) * ceil_div64(K, side) : ceil_div64(rows, side) + busy) * ceil_div64(N, side); };
    g.pair = sizeof(T) == 2 && N > 128 && (WGRAD ? K > 128 && rows >= 2048 : ceil_div64(rows, 256) * ceil_div64(N, 256) * 4 >= sms);
    g.blocks = g.pair ? 2 * (int)std::min<int64_t>(sms / 2, std::max<int64_t>(1, tiles(256))) : (int)std::min<int64_t>(sms, std::max<int64_t>(1, tiles(128)));
    if (WGRAD) {
        g.slots = g.bytes;
        g.splits = g.slots + sizeof(float) * (size_t)2 * g.blocks * 129 * (g.pair ? 256 : 128);
        g.bytes = g.splits + sizeof(GroupedSplit) * (size_t)g.blocks;
    }
    return g;
}
template <int MODE, typename T> static bool grouped_launch(TcState &tc, Exec &ex, GroupedParams &p, GroupedPlan &g, int64_t lda, int64_t ldb, uint8_t *ws, std::string &err)
{
    CUtensorMap a{}, b{}, c{};
    constexpr bool WGRAD = MODE == GP_WGRAD, SPLIT = sizeof(T) == 4;
    const int side = g.pair ? 256 : 128;
    p.tiles_n = (int)ceil_div64(p.N, side);
    p.tiles_k = (int)ceil_div64(p.K, side);
    p.err = tc.err_word;
    p.wait_ns = tc.wait_limit_ns;
    p.extra_tx = tc.overdeclare_tx;
    grouped_prepare<T>(ex, g.a, lda, ws);
    grouped_prepare<T>(ex, g.b, ldb, ws);
    p.slots = (float *)(ws + g.slots);
    p.splits = (GroupedSplit *)(ws + g.splits);
    const GroupedOperand &reg = WGRAD ? g.b : g.a;
    if (SPLIT) { p.reg = (const float *)reg.at; p.ld_reg = reg.ld; }
    // operands that come by TMA
    if (WGRAD) {
        if (!grouped_map_3d(tc, &a, (const bf16 *)g.a.at, GP_PARTS<T>, p.rows, p.K, g.a.ld, 64, err)) return false;
        if (!SPLIT && !tc_make_map(tc, &b, (const bf16 *)g.b.at, p.rows, p.N, g.b.ld, 64, 64, err)) return false;
    } else {
        if (!SPLIT && !tc_make_map(tc, &a, (const bf16 *)g.a.at, p.rows, p.K, g.a.ld, 64, 128, err)) return false;
        if (!grouped_map_3d(tc, &b, (const bf16 *)g.b.at, p.groups * (int64_t)GP_PARTS<T>, g.b.rows, g.b.cols, g.b.ld, MODE == GP_NN ? 64 : 128, err)) return false;
    }
    p.tma_c = !WGRAD && p.vec_c;
    if (p.tma_c) {  // boxes of a warp: 32 rows, 64 or 128 bytes wide, laid out as they are staged
        const bool wide = g.pair;
        cuuint64_t dims[2] = {(cuuint64_t)p.N, (cuuint64_t)p.rows}, strides[1] = {(cuuint64_t)p.ldc * sizeof(T)};
        cuuint32_t box[2] = {(cuuint32_t)((wide ? 128 : 64) / sizeof(T)), 32}, estr[2] = {1, 1};
        if (tc.encode(&c, SPLIT ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.C, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      wide ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            p.tma_c = 0;  // a pitch that no tensor map takes: rows leave one by one
    }
    if (p.extra_tx) tc.overdeclare_tx = 0;
    if constexpr (sizeof(T) == 2) {
        if (g.pair) {
            grouped_launch_one<MODE, T, true>(ex, a, b, c, p, g.blocks);
            return true;
        }
    }
    grouped_launch_one<MODE, T, false>(ex, a, b, c, p, g.blocks);
    return true;
}
