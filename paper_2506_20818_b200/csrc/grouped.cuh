// Products with one weight matrix per group of rows, and their weight gradients, on the tensor cores.
//
//   grouped linear       rows offsets[g] .. offsets[g + 1] - 1:  C = act(A B[g] + bias[g])    (B[g] [K, N], or [N, K]: transposed)
//   grouped weight grad  dW[g] = A_g^T dZ_g,  dbias[g] = column sums of dZ_g
//
// BF16 operands go to the matrix instructions as they are.  FP32 operands are split into three BF16 numbers of eight bits each,
// x = x0 + x1 + x2 exactly (the upper half of the word, of the rest, and of the rest's rest), and of the nine products the six
// larger ones are taken, so that a product is off by about 2^-23; the accumulator of the matrix instructions rounds towards
// zero, so it adds up 64 terms, small products first, and those sums are added in FP32 registers.
//
// One persistent block per SM, 18 warps.  Sizes of the groups are on the device: every role walks the offsets itself, 32 groups at a
// time, and finds its tiles (linear) or its share of the 64-row blocks of all tiles (weight gradient) without any plan or host read.
//   warp 0    operands by TMA (BF16, rows on 16 bytes)         warp 1   matrix instructions
//   others    sums and results; without TMA the last eight bring in the operands through registers
// The weight gradient deals out equal shares of 64-row blocks: a tile that lies in several shares is written as partial tiles,
// added in a fixed order by a second kernel.  Bits do not depend on anything but the sizes.
#pragma once
#include "gemm_tc.cuh"
#include "orthogonal.cuh"

enum { GP_NN = 0, GP_NT = 1, GP_WGRAD = 2 };
constexpr int GP_THREADS = 576;
constexpr int GP_EXTRA_SMEM = 32768;  // results that are written element by element, sums of columns
constexpr int GP_MAX_STAGES = 8;
constexpr int GP_MAX_GROUPS = 1 << 20;

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
    const void *A, *B;       // register loads only (B: dZ of the weight gradient)
    int64_t lda, ldb, stride_b;
    int vec_a, vec_b;        // rows on 16 bytes
    int stages, flush;       // blocks of 64 terms that an accumulator adds up
    // linear
    const float *bias;
    int relu;
    void *C;
    int64_t ldc;
    int vec_c;
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
template <bool WGRAD> struct GroupWalk {
    const int *off;
    int groups, rows;
    int g0, before, last;        // first group of the window, tiles before it, end of the group before it
    int begin, end, incl, total; // of this lane's group; tiles up to and with it; tiles of the window
    LP_DEVINL int count(int size) const { return WGRAD ? max(1, (size + 63) >> 6) : (size + 127) >> 7; }
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
    int g, row0, row_end;  // linear: rows of the tile; weight gradient: rows of the share
    int kt, nt, kbs;       // tile, blocks of 64 terms
    int slot;              // weight gradient: partial tile, or -1: the whole tile is in this share
    bool begins;           // ... the share begins the tile, which ends before block tile_end of all
    int64_t tile_end;
};

template <int MODE> struct GroupedJobs {
    GroupWalk<MODE == GP_WGRAD> walk;
    const GroupedParams &p;
    int64_t t;           // linear: next tile of this block
    int64_t u, lo, hi;   // weight gradient: 64-row blocks of this share
    LP_DEVINL GroupedJobs(const GroupedParams &p_, int64_t lo_, int64_t hi_) : walk(p_), p(p_), t(blockIdx.x), u(lo_), lo(lo_), hi(hi_) {}
    LP_DEVINL bool next(GroupedJob &j)
    {
        int b, e, pre;
        if (MODE != GP_WGRAD) {
            const int mt = (int)(t / p.tiles_n);
            j.nt = (int)(t - (int64_t)mt * p.tiles_n);
            if (!walk.seek(mt, j.g, b, e, pre)) return false;
            j.row0 = b + (mt - pre) * 128;
            j.row_end = min(e, j.row0 + 128);
            j.kt = 0;
            j.kbs = (p.K + 63) >> 6;
            j.slot = -1;
            t += gridDim.x;
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
        j.slot = kb0 == 0 && j.kbs == blocks ? -1 : 2 * (int)blockIdx.x + (u == lo ? 0 : 1);
        j.begins = kb0 == 0;
        j.tile_end = u - kb0 + blocks;
        u += j.kbs;
        return true;
    }
};

// ---------------------------------------------------------------------------------------------
// operands through registers
// ---------------------------------------------------------------------------------------------
// eight neighbouring elements of a row, zeros beyond its end
template <typename T> struct Piece8;
template <> struct Piece8<bf16> {
    uint4 w;
    LP_DEVINL void load(const bf16 *row, int col, int limit, int vec)
    {
        const int n = limit - col;
        if (vec && n >= 8) {
            w = __ldg(reinterpret_cast<const uint4 *>(row + col));
        } else {
            uint32_t x[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) x[i >> 1] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short *>(row + col) + i) << (16 * (i & 1));
            w = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }
    LP_DEVINL void zero() { w = make_uint4(0u, 0u, 0u, 0u); }
    LP_DEVINL void store(uint8_t *s, uint32_t) const { *reinterpret_cast<uint4 *>(s) = w; }
    LP_DEVINL void add_to(float *acc) const
    {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc[2 * i] += __uint_as_float(x[i] << 16);
            acc[2 * i + 1] += __uint_as_float(x[i] & 0xffff0000u);
        }
    }
};
template <> struct Piece8<float> {
    float v[8];
    LP_DEVINL void load(const float *row, int col, int limit, int vec)
    {
        const int n = limit - col;
        if (vec && n >= 8) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(row + col)), b = __ldg(reinterpret_cast<const float4 *>(row + col) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? __ldg(row + col + i) : 0.f;
        }
    }
    LP_DEVINL void zero()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    // the three parts lie `part` bytes apart
    LP_DEVINL void store(uint8_t *s, uint32_t part) const
    {
        float r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = v[i];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            uint32_t x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __byte_perm(__float_as_uint(r[2 * i]), __float_as_uint(r[2 * i + 1]), 0x7632);  // the upper halves
            *reinterpret_cast<uint4 *>(s + q * part) = make_uint4(x[0], x[1], x[2], x[3]);
            if (q < 2)
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] -= __uint_as_float(__float_as_uint(r[i]) & 0xffff0000u);  // exact
        }
    }
    LP_DEVINL void add_to(float *acc) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += v[i];
    }
};

// ---------------------------------------------------------------------------------------------
// results
// ---------------------------------------------------------------------------------------------
// sixteen neighbouring columns of a warp's 32 rows, a row per lane: rows below `rows`, columns below `cols`
template <typename T> LP_DEVINL void put16(T *dst, int64_t ld, int rows, int cols, const float *v, int vec, float *stage, bool accumulate)
{
    const int lane = threadIdx.x & 31;
    if (vec) {
        if (lane < rows) {
            T *d = dst + (int64_t)lane * ld;
            constexpr int VN = Vec16<T>::N;
#pragma unroll
            for (int c = 0; c < 16; c += VN)
                if (c < cols) {
                    Vec16<T> o;
                    float w[VN];
#pragma unroll
                    for (int i = 0; i < VN; ++i) w[i] = v[c + i];
                    if (accumulate) {
                        o.v = *reinterpret_cast<decltype(o.v) *>(d + c);
                        float x[VN];
                        o.to_float(x);
#pragma unroll
                        for (int i = 0; i < VN; ++i) w[i] += x[i];
                    }
                    o.from_float(w);
                    o.store(d + c);
                }
        }
        return;
    }
    // through shared memory, so that a store instruction writes runs of sixteen elements of two rows
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 16; ++c) stage[lane * 16 + (c ^ (lane & 15))] = v[c];
    __syncwarp();
    const int c = lane & 15;
    if (c < cols)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 2 * i + (lane >> 4);
            if (r < rows) {
                T *d = dst + (int64_t)r * ld + c;
                const float x = stage[r * 16 + (c ^ (r & 15))];
                *d = from_f<T>(accumulate ? to_f<T>(*d) + x : x);
            }
        }
}

// ---------------------------------------------------------------------------------------------
// kernel
// ---------------------------------------------------------------------------------------------
LP_DEVINL void tma_load_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map),
                 "r"(bar), "r"(x), "r"(y), "r"(z)
                 : "memory");
}

template <typename T> constexpr int GP_PARTS = sizeof(T) == 4 ? 3 : 1;
template <typename T, int BN> constexpr int GP_STAGE_BYTES = GP_PARTS<T> * (128 + BN) * 128;

template <int MODE, typename T, int BN, bool TMA>
__global__ void __launch_bounds__(GP_THREADS, 1) grouped_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
                                                                 const __grid_constant__ GroupedParams p)
{
    LP_DEP_ENTER();
    constexpr int PARTS = GP_PARTS<T>;
    constexpr bool WGRAD = MODE == GP_WGRAD;
    constexpr bool A_MN = WGRAD, B_MN = MODE != GP_NT;
    constexpr int EPI = TMA ? 16 : 8, COLS = BN * 4 / EPI;  // warps of sums and results, columns of each
    constexpr int LOADERS = TMA ? 0 : 8;
    constexpr uint32_t a_bytes = 128 * 128, b_bytes = BN * 128, stage_bytes = GP_STAGE_BYTES<T, BN>;
    static_assert(TMA ? PARTS == 1 : BN == 128, "TMA brings in BF16 operands, registers tiles of 128 columns");
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_full[GP_MAX_STAGES], bar_empty[GP_MAX_STAGES], bar_acc_full[2], bar_acc_empty[2], bar_sum_full, bar_sum_empty, bar_done;
    __shared__ uint32_t tmem_base_s;
    __shared__ int blocks_s;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int S = p.stages;
    uint8_t *extra = smem + (size_t)S * stage_bytes;
    const bool sums = WGRAD && p.dbias != nullptr;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(smem_u32(&bar_full[s]), TMA ? 1 : LOADERS);
            mbar_init(smem_u32(&bar_empty[s]), TMA && sums ? 1 + EPI : 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bar_acc_full[b]), 1);
            mbar_init(smem_u32(&bar_acc_empty[b]), EPI);
        }
        mbar_init(smem_u32(&bar_sum_full), TMA ? EPI : LOADERS);
        mbar_init(smem_u32(&bar_sum_empty), BN / 32);
        mbar_init(smem_u32(&bar_done), 1);
        fence_barrier_init();
        fence_async_proxy();
        if (TMA) {
            tma_prefetch_desc(&mapA);
            tma_prefetch_desc(&mapB);
        }
    }
    if (warp == 0) {
        __syncwarp();
        tmem_alloc(smem_u32(&tmem_base_s), 2 * BN);
    } else if (warp == 1) {
        if (WGRAD) {
            GroupWalk<true> w(p);
            const int n = w.all();
            if (lane == 0) blocks_s = n;
        }
    } else if (warp == 2 && blockIdx.x == 0) {
        bool bad = false;
        for (int g = lane; g <= p.groups; g += 32) bad |= p.offsets[g] < (g ? p.offsets[g - 1] : 0) || p.offsets[g] > p.rows;
        if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.offsets_err, 4);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_s;
    int64_t lo = 0, hi = 0, all = 0;
    if (WGRAD) {
        all = (int64_t)blocks_s * p.tiles_k * p.tiles_n;
        lo = all * blockIdx.x / gridDim.x;
        hi = all * (blockIdx.x + 1) / gridDim.x;
    }
    GroupedJobs<MODE> jobs(p, lo, hi);
    GroupedJob j;

    if (warp == 0) {
        if (TMA) {
            // ---- operands
            int s = 0, round = 0;
            bool ok = true, first = blockIdx.x == (WGRAD ? gridDim.x - 1 : 0);  // a block that has work in any case
            const bool chosen = elect_one();
            const int chosen_lane = __ffs(__ballot_sync(0xffffffffu, chosen)) - 1;
            while (ok && jobs.next(j)) {
                if (chosen) {
                    for (int kb = 0; kb < j.kbs; ++kb) {
                        if (round > 0 && !mbar_wait(smem_u32(&bar_empty[s]), (round & 1) ^ 1, p.wait_ns)) { atomicExch(p.err, 1); ok = false; break; }
                        const uint32_t sa = smem_u32(smem) + s * stage_bytes, sb = sa + a_bytes, bar = smem_u32(&bar_full[s]);
                        mbar_expect_tx(bar, stage_bytes + (first ? (uint32_t)p.extra_tx : 0u));
                        first = false;
                        if (WGRAD) {
                            const int row = j.row0 + kb * 64;
#pragma unroll
                            for (int c = 0; c < 2; ++c) tma_load_2d(sa + c * 8192, &mapA, bar, j.kt * 128 + c * 64, row);
#pragma unroll
                            for (int c = 0; c < BN / 64; ++c) tma_load_2d(sb + c * 8192, &mapB, bar, j.nt * BN + c * 64, row);
                        } else {
                            tma_load_2d(sa, &mapA, bar, kb * 64, j.row0);
                            if (B_MN) {
#pragma unroll
                                for (int c = 0; c < BN / 64; ++c) tma_load_3d(sb + c * 8192, &mapB, bar, j.nt * BN + c * 64, kb * 64, j.g);
                            } else {
                                tma_load_3d(sb, &mapB, bar, kb * 64, j.nt * BN, j.g);
                            }
                        }
                        if (++s == S) { s = 0; ++round; }
                    }
                }
                __syncwarp();
                ok = __all_sync(0xffffffffu, ok);
            }
            s = __shfl_sync(0xffffffffu, s, chosen_lane);
            round = __shfl_sync(0xffffffffu, round, chosen_lane);
            // copies under way land before the block gives up its shared memory (after a wait that ran out; else they long have)
            if (lane == 0)
                for (int i = 0; i < S; ++i) {
                    const int at = s - 1 - i < 0 ? s - 1 - i + S : s - 1 - i, r = s - 1 - i < 0 ? round - 1 : round;
                    if (r >= 0) mbar_wait(smem_u32(&bar_full[at]), r & 1, p.wait_ns);
                }
            __syncwarp();
        }
    } else if (warp == 1) {
        // ---- products
        int s = 0, round = 0, use = 0;
        bool ok = true;
        constexpr uint32_t idesc_mn = (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u);
        const uint32_t idesc = make_idesc_bf16(BN, false, false) | idesc_mn;
        const uint64_t desc_a = make_smem_desc(smem_u32(smem), A_MN ? 8192 : 16, 1024), desc_b = make_smem_desc(smem_u32(smem) + PARTS * a_bytes, B_MN ? 8192 : 16, 1024);
        constexpr uint64_t step_a = (A_MN ? 2048 : 32) >> 4, step_b = (B_MN ? 2048 : 32) >> 4;
        while (ok && jobs.next(j)) {
            for (int kb = 0; kb < j.kbs && ok; ++kb) {
                const int b = use & 1, in_flush = kb % p.flush;
                if (in_flush == 0 && use >= 2 && !mbar_wait(smem_u32(&bar_acc_empty[b]), ((use >> 1) & 1) ^ 1, p.wait_ns)) {
                    if (lane == 0) atomicExch(p.err, 5);
                    ok = false;
                }
                if (ok && !mbar_wait(smem_u32(&bar_full[s]), round & 1, p.wait_ns)) {
                    if (lane == 0) atomicExch(p.err, 2);
                    ok = false;
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if (WGRAD && TMA) {
                    // rows behind the group belong to the next one (or to nobody): zeros in both operands, whatever they hold
                    const int have = j.row_end - (j.row0 + kb * 64);
                    if (have < 64) {
                        uint8_t *st = smem + (size_t)s * stage_bytes;
                        for (int i = lane; i < (64 - max(have, 0)) * 8; i += 32)
#pragma unroll
                            for (int c = 0; c < 2 + BN / 64; ++c) *reinterpret_cast<uint4 *>(st + c * 8192 + max(have, 0) * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                        fence_async_proxy();
                        __syncwarp();
                    }
                }
                const bool done = in_flush == p.flush - 1 || kb == j.kbs - 1;
                if (elect_one()) {
                    const uint64_t da = desc_a + ((s * stage_bytes) >> 4), db = desc_b + ((s * stage_bytes) >> 4);
                    const uint32_t acc = tmem + b * BN;
                    if (PARTS == 1) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) umma_bf16(acc, da + i * step_a, db + i * step_b, idesc, in_flush != 0 || i != 0 ? 1u : 0u);
                    } else {
                        constexpr int first[6] = {0, 2, 1, 0, 1, 0}, second[6] = {2, 0, 1, 1, 0, 0};  // the small products first, while the sums are small
#pragma unroll
                        for (int q = 0; q < 6; ++q)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                umma_bf16(acc, da + first[q] * (a_bytes >> 4) + i * step_a, db + second[q] * (b_bytes >> 4) + i * step_b, idesc,
                                          in_flush != 0 || q != 0 || i != 0 ? 1u : 0u);
                    }
                    umma_commit(smem_u32(&bar_empty[s]));
                    if (done) umma_commit(smem_u32(&bar_acc_full[b]));
                }
                __syncwarp();
                if (done) ++use;
                if (++s == S) { s = 0; ++round; }
            }
        }
        // products under way are done with the block's memory before it goes, also after a wait that ran out
        if (elect_one()) umma_commit(smem_u32(&bar_done));
        __syncwarp();
        mbar_wait(smem_u32(&bar_done), 0, p.wait_ns);
        __syncwarp();
    } else if (warp < 2 + EPI) {
        // ---- sums and results: 32 rows x COLS columns per warp
        const int quarter = warp & 3, part = (warp - 2) >> 2;
        const int epi_thread = threadIdx.x - 64;
        float *stage = reinterpret_cast<float *>(extra) + (warp - 2) * 512;
        int use = 0, s = 0, round = 0, summed = 0;
        bool ok = true;
        GroupedSplit split{0, 0, 0, -1, 0, 0};
        while (ok && jobs.next(j)) {
            float v[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) v[c] = 0.f;
            float col[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            const bool adds = sums && TMA && j.kt == 0;
            for (int kb = 0; kb < j.kbs && ok; ++kb) {
                if (TMA && sums) {
                    // column sums of dZ out of the staged tiles: eight columns (piece of 16 bytes) of a few rows per thread
                    constexpr int PIECES = BN / 8, ROWS = 64 * PIECES / (EPI * 32);
                    ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_full[s]), round & 1, p.wait_ns));
                    if (!ok) { if (lane == 0) atomicExch(p.err, 4); break; }
                    if (adds) {
                        const int piece = epi_thread % PIECES, r0 = epi_thread / PIECES * ROWS, have = j.row_end - (j.row0 + kb * 64);
                        const uint8_t *sb = smem + (size_t)s * stage_bytes + a_bytes + (piece >> 3) * 8192;
#pragma unroll
                        for (int i = 0; i < ROWS; ++i) {
                            const int r = r0 + i;
                            if (r < have) {
                                Piece8<bf16> x;
                                x.w = *reinterpret_cast<const uint4 *>(sb + r * 128 + (((piece & 7) ^ (r & 7)) << 4));
                                x.add_to(col);
                            }
                        }
                        __syncwarp();
                    }
                    if (lane == 0) mbar_arrive(smem_u32(&bar_empty[s]));
                    if (++s == S) { s = 0; ++round; }
                }
                if (kb % p.flush != p.flush - 1 && kb != j.kbs - 1) continue;
                const int b = use & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_acc_full[b]), (use >> 1) & 1, p.wait_ns));
                if (!ok) { if (lane == 0) atomicExch(p.err, 3); break; }
                tc_fence_after();
                const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(b * BN + part * COLS);
#pragma unroll
                for (int c = 0; c < COLS; c += 16) {
                    float x[16];
                    tmem_ld_32x16(at + c, x);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[c + i] += x[i];
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_acc_empty[b]));
                ++use;
            }
            if (!ok) break;
            if (summed > 0) {  // the column sums of the job before have been read
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_sum_empty), (summed - 1) & 1, p.wait_ns));
                if (!ok) { if (lane == 0) atomicExch(p.err, 7); break; }
            }
            const int c0 = j.nt * BN + part * COLS;  // first column of this warp
            if (!WGRAD) {
                const int row = j.row0 + quarter * 32;
                T *dst = (T *)p.C + (int64_t)row * p.ldc + c0;
                const float *bias = p.bias ? p.bias + (int64_t)j.g * p.N + c0 : nullptr;
#pragma unroll
                for (int c = 0; c < COLS; c += 16) {
                    if (c0 + c >= p.N) break;
                    if (bias)
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[c + i] += c0 + c + i < p.N ? __ldg(bias + c + i) : 0.f;
                    if (p.relu)
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[c + i] = v[c + i] > 0.f || v[c + i] != v[c + i] ? v[c + i] : 0.f;  // NaN stays
                    put16<T>(dst + c, p.ldc, j.row_end - row, p.N - (c0 + c), v + c, p.vec_c, stage, false);
                }
            } else if (j.slot < 0) {
                const int row = j.kt * 128 + quarter * 32;
                float *dst = p.dW + ((int64_t)j.g * p.K + row) * p.N + c0;
#pragma unroll
                for (int c = 0; c < COLS; c += 16)
                    if (c0 + c < p.N) put16<float>(dst + c, p.N, p.K - row, p.N - (c0 + c), v + c, p.vec_c, stage, p.accumulate != 0);
            } else {
                float *dst = p.slots + ((size_t)j.slot * 129 + quarter * 32 + lane) * BN + part * COLS;
#pragma unroll
                for (int c = 0; c < COLS; c += 4) *reinterpret_cast<float4 *>(dst + c) = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
            }
            if (adds) {
                // every warp leaves its sums of a few rows in its own part of the area; the first BN threads add them up in order
                constexpr int PIECES = BN / 8, SHARES = EPI * 32 / PIECES;
                float *area = reinterpret_cast<float *>(extra);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) stage[lane * 8 + i] = col[i];
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_sum_full));
                if (epi_thread < BN) {
                    ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_sum_full), summed & 1, p.wait_ns));
                    if (!ok) { if (lane == 0) atomicExch(p.err, 7); break; }
                    float x = 0.f;
#pragma unroll
                    for (int i = 0; i < SHARES; ++i) {
                        const int writer = i * PIECES + epi_thread / 8;  // thread that has these columns of share i
                        x += area[(writer >> 5) * 512 + (writer & 31) * 8 + (epi_thread & 7)];
                    }
                    const int c = j.nt * BN + epi_thread;
                    if (j.slot >= 0) p.slots[((size_t)j.slot * 129 + 128) * BN + epi_thread] = x;
                    else if (c < p.N) {
                        float *d = p.dbias + (int64_t)j.g * p.N + c;
                        *d = p.accumulate ? *d + x : x;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bar_sum_empty));
                }
                ++summed;
            }
            // of the shares of a block only the last can begin a tile that others go on with
            if (WGRAD && j.slot >= 0 && j.begins)
                split = GroupedSplit{j.g, j.kt, j.nt, j.slot, (int)((j.tile_end * gridDim.x - 1) / all), all};
        }
        if (WGRAD && warp == 2 && lane == 0) p.splits[blockIdx.x] = split;
    } else if (!TMA) {
        // ---- operands through registers: four pieces of each operand per thread and block of 64 terms.  The pieces of the second
        // operand are under way while those of the first are put down, and the first's next ones while those of the second are.
        const int lt = threadIdx.x - (2 + EPI) * 32;
        int s = 0, round = 0, summed = 0;
        bool ok = true;
        Piece8<T> a[4], bq[4];
        float col[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        auto load = [&](Piece8<T> (&x)[4], const T *base, int64_t ld, int row, int row_end, int col0, int limit, int vec, bool mn) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int q = lt + 256 * i, r = row + (mn ? q >> 4 : q >> 3), c = col0 + 8 * (mn ? q & 15 : q & 7);
                if (r < row_end && c < limit) x[i].load(base + (int64_t)r * ld, c, limit, vec);
                else x[i].zero();
            }
        };
        auto load_a = [&](const GroupedJob &w, int kb) {
            if (WGRAD) load(a, (const T *)p.A, p.lda, w.row0 + kb * 64, w.row_end, w.kt * 128, p.K, p.vec_a, true);
            else load(a, (const T *)p.A, p.lda, w.row0, w.row_end, kb * 64, p.K, p.vec_a, false);
        };
        auto load_b = [&](const GroupedJob &w, int kb) {
            const T *b = (const T *)p.B + (WGRAD ? 0 : (int64_t)w.g * p.stride_b);
            if (WGRAD) load(bq, b, p.ldb, w.row0 + kb * 64, w.row_end, w.nt * 128, p.N, p.vec_b, true);
            else if (MODE == GP_NN) load(bq, b, p.ldb, kb * 64, p.K, w.nt * 128, p.N, p.vec_b, true);
            else load(bq, b, p.ldb, w.nt * 128, p.N, kb * 64, p.K, p.vec_b, false);
        };
        auto put = [&](const Piece8<T> (&x)[4], uint8_t *dst, uint32_t part, bool mn) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int q = lt + 256 * i, r = mn ? q >> 4 : q >> 3, c = mn ? q & 15 : q & 7;
                x[i].store(dst + (c >> 3) * 8192 + r * 128 + (((c & 7) ^ (r & 7)) << 4), part);
            }
        };
        int kb = 0;
        bool more = jobs.next(j);
        if (more) load_a(j, 0);
        while (more && ok) {
            load_b(j, kb);
            if (round > 0) {
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_empty[s]), (round & 1) ^ 1, p.wait_ns));
                if (!ok) { if (lane == 0) atomicExch(p.err, 1); break; }
            }
            uint8_t *st = smem + (size_t)s * stage_bytes;
            put(a, st, a_bytes, A_MN);
            const GroupedJob cur = j;
            const bool last = ++kb == j.kbs;
            if (last) {
                kb = 0;
                more = jobs.next(j);
            }
            if (more) load_a(j, kb);
            put(bq, st + PARTS * a_bytes, b_bytes, B_MN);
            fence_async_proxy();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_full[s]));
            if (++s == S) { s = 0; ++round; }
            if (sums && cur.kt == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) bq[i].add_to(col);
                if (last) {
                    // a thread has the rows 16 i + lt / 16 of its eight columns: sixteen sums per column, added up in order
                    float *area = reinterpret_cast<float *>(extra) + EPI * 512;
                    if (summed > 0) {
                        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_sum_empty), (summed - 1) & 1, p.wait_ns));
                        if (!ok) { if (lane == 0) atomicExch(p.err, 7); break; }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) { area[(lt >> 4) * 128 + (lt & 15) * 8 + i] = col[i]; col[i] = 0.f; }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bar_sum_full));
                    if (lt < 128) {
                        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_sum_full), summed & 1, p.wait_ns));
                        if (!ok) { if (lane == 0) atomicExch(p.err, 7); break; }
                        float x = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) x += area[i * 128 + lt];
                        const int c = cur.nt * 128 + lt;
                        if (cur.slot >= 0) p.slots[((size_t)cur.slot * 129 + 128) * BN + lt] = x;
                        else if (c < p.N) {
                            float *d = p.dbias + (int64_t)cur.g * p.N + c;
                            *d = p.accumulate ? *d + x : x;
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&bar_sum_empty));
                    }
                    ++summed;
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        __syncwarp();
        tmem_dealloc(tmem, 2 * BN);
    }
}

// tiles that several blocks share: their partial tiles added in the order of the blocks.  gridDim.x = blocks of the product
template <int BN> __global__ void __launch_bounds__(256) grouped_splits_kernel(const __grid_constant__ GroupedParams p)
{
    LP_DEP_ENTER();
    const GroupedSplit sp = p.splits[blockIdx.x];
    if (sp.first_slot < 0) return;
    constexpr int EACH = 4;
    float v[EACH];
    const int at = blockIdx.y * 256 * EACH + threadIdx.x, size = 129 * BN;
#pragma unroll
    for (int i = 0; i < EACH; ++i) v[i] = at + 256 * i < size ? p.slots[(size_t)sp.first_slot * size + at + 256 * i] : 0.f;
    for (int c = (int)blockIdx.x + 1; c <= sp.last_block; ++c) {
        if (sp.blocks * c / gridDim.x == sp.blocks * (c + 1) / gridDim.x) continue;  // a block without a share
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (at + 256 * i < size) v[i] += p.slots[(size_t)(2 * c) * size + at + 256 * i];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int row = (at + 256 * i) / BN, col = sp.nt * BN + (at + 256 * i) % BN, k = sp.kt * 128 + row;
        if (row > 128 || col >= p.N) continue;
        float *d;
        if (row < 128) {
            if (k >= p.K) continue;
            d = p.dW + ((int64_t)sp.group * p.K + k) * p.N + col;
        } else {
            if (!p.dbias || sp.kt != 0) continue;
            d = p.dbias + (int64_t)sp.group * p.N + col;
        }
        *d = p.accumulate ? *d + v[i] : v[i];
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
template <int MODE, typename T, int BN, bool TMA> static bool grouped_init_one(std::string &err)
{
    if (cudaFuncSetAttribute(grouped_kernel<MODE, T, BN, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 1024) == cudaSuccess) return true;
    err = "cannot raise the dynamic shared memory limit of the grouped products";
    return false;
}
template <int MODE> static bool grouped_init_mode(std::string &err)
{
    return grouped_init_one<MODE, bf16, 128, true>(err) && grouped_init_one<MODE, bf16, 256, true>(err) && grouped_init_one<MODE, bf16, 128, false>(err) &&
           grouped_init_one<MODE, float, 128, false>(err);
}
static bool grouped_init(std::string &err) { return grouped_init_mode<GP_NN>(err) && grouped_init_mode<GP_NT>(err) && grouped_init_mode<GP_WGRAD>(err); }

// tensor map over [groups][rows][cols] BF16 matrices behind one another
static bool grouped_map_3d(const TcState &tc, CUtensorMap *map, const bf16 *base, int64_t groups, int64_t rows, int64_t cols, int box_rows, std::string &err)
{
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)groups};
    cuuint64_t strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)cols * (cuuint64_t)rows * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
    if (tc.encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, (void *)base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS)
        return true;
    err = "cuTensorMapEncodeTiled failed";
    return false;
}

template <int MODE, typename T, int BN, bool TMA> static void grouped_launch_one(Exec &ex, const CUtensorMap &a, const CUtensorMap &b, GroupedParams &p, int blocks)
{
    constexpr int stage = GP_STAGE_BYTES<T, BN>;
    p.stages = std::min(GP_MAX_STAGES, (227 * 1024 - 1024 - 1024 - GP_EXTRA_SMEM) / stage);
    const size_t smem = (size_t)p.stages * stage + GP_EXTRA_SMEM + 1024;
    launch_dep(grouped_kernel<MODE, T, BN, TMA>, dim3((unsigned)blocks), dim3(GP_THREADS), smem, ex.st, a, b, p);
    ex.launches += 1;
    if (MODE == GP_WGRAD) {
        launch_dep(grouped_splits_kernel<BN>, dim3((unsigned)blocks, (unsigned)ceil_div64(129 * BN, 1024)), dim3(256), 0, ex.st, p);
        ex.launches += 1;
    }
}

struct GroupedPlan {
    bool tma;
    int bn, blocks;
    size_t slots_bytes;  // weight gradient; the notes on shared tiles follow
};
template <typename T> static bool grouped_tma(const void *A, int64_t lda, const void *B, int64_t ldb)
{
    return sizeof(T) == 2 && on_16_bytes<T>(A, lda) && on_16_bytes<T>(B, ldb);
}
// tiles of 256 columns where they keep every SM busy, of 128 elsewhere and for operands through registers
static GroupedPlan grouped_plan(bool tma, bool wgrad, int64_t rows, int64_t groups, int N, int K)
{
    GroupedPlan g{};
    const int64_t sms = tc_sm_count(), busy = std::min(rows, groups);
    g.tma = tma;
    auto tiles = [&](int bn) { return (wgrad ? (ceil_div64(rows, 64) + groups) * ceil_div64(K, 128) : ceil_div64(rows, 128) + busy) * ceil_div64(N, bn); };
    g.bn = tma && N > 128 && (wgrad || tiles(256) >= sms) ? 256 : 128;
    g.blocks = (int)std::min<int64_t>(sms, std::max<int64_t>(1, tiles(g.bn)));
    g.slots_bytes = wgrad ? sizeof(float) * (size_t)2 * g.blocks * 129 * g.bn : 0;
    return g;
}
template <int MODE, typename T> static bool grouped_launch(TcState &tc, Exec &ex, GroupedParams &p, const GroupedPlan &g, std::string &err)
{
    CUtensorMap a{}, b{};
    p.tiles_n = (int)ceil_div64(p.N, g.bn);
    p.tiles_k = (int)ceil_div64(p.K, 128);
    p.vec_a = on_16_bytes<T>(p.A, p.lda);
    p.vec_b = on_16_bytes<T>(p.B, p.ldb) && on_16_bytes<T>(p.B, p.stride_b);
    p.err = tc.err_word;
    p.wait_ns = tc.wait_limit_ns;
    p.extra_tx = g.tma ? tc.overdeclare_tx : 0;
    if (g.tma) {
        tc.overdeclare_tx = 0;
        const bf16 *A = (const bf16 *)p.A, *B = (const bf16 *)p.B;
        if (!tc_make_map(tc, &a, A, p.rows, p.K, p.lda, 64, MODE == GP_WGRAD ? 64 : 128, err)) return false;
        if (MODE == GP_WGRAD ? !tc_make_map(tc, &b, B, p.rows, p.N, p.ldb, 64, 64, err)
                             : !grouped_map_3d(tc, &b, B, p.groups, MODE == GP_NN ? p.K : p.N, MODE == GP_NN ? p.N : p.K, MODE == GP_NN ? 64 : g.bn, err))
            return false;
    }
    if (sizeof(T) == 4) grouped_launch_one<MODE, float, 128, false>(ex, a, b, p, g.blocks);
    else if (!g.tma) grouped_launch_one<MODE, bf16, 128, false>(ex, a, b, p, g.blocks);
    else if (g.bn == 256) grouped_launch_one<MODE, bf16, 256, true>(ex, a, b, p, g.blocks);
    else grouped_launch_one<MODE, bf16, 128, true>(ex, a, b, p, g.blocks);
    return true;
}
