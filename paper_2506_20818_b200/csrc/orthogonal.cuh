// Orthogonalisation of matrices by Newton-Schulz products, and the weight update built on it.
//
//   X_0 = U / (|U|_F + eps);   A = X X^T,  B = b A + c A^2,  X <- a X + B X     (steps times)
//
// maps every singular value s of X_0 through the odd polynomial a s + b s^3 + c s^5 again and again and leaves the
// singular vectors.  The products run on the tensor cores with FP16 operands and FP32 accumulators.  FP16 carries eleven
// significant bits where BF16 carries eight, at the same rate, and the range it lacks is not needed here: the values
// are bounded by the polynomial (the host refuses coefficients for which they are not), so X is held as 2^12 X and A and B
// as 2^8 A, 2^8 B, which keeps the parts that matter inside the normal numbers of FP16.
// X is always kept as a pair of FP16 numbers hi + lo (22 bits), and the term a X of every step is taken from both.
//   BF16 results : the products take the leading parts only, A and B are one FP16 number per value
//   FP32 results : A and B are pairs too, products hi*hi + hi*lo + lo*hi into one accumulator
// Why X keeps its low part where the products do not read it: rounding X to eleven bits would add a matrix of full rank, and
// whatever lies in directions that X hardly has is multiplied by a in every step (3.4^5 = 480 for five).  The errors of the
// products are of the form dB X and B dX, which vanish in such directions, so they stay at their own size.
// A matrix with more rows than columns is iterated transposed: m = min(rows, cols), n = max(rows, cols).
// A and B are symmetric, so only tiles on and above the diagonal are computed and the others are written by mirroring.
//
// All matrices of a call lie in common arenas (X: rows of `pitch_x`, A and B: rows of `pitch_a`), each padded with zeros
// to multiples of 64; the padding stays zero through every product.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "embed.cuh"
#include "gemm_tc.cuh"

constexpr int NS_MAX_MATS = 24;       // descriptors in one launch group (they travel as kernel arguments, 4 KiB in all)
constexpr float NS_X_SCALE = 4096.f;  // X is held as 2^12 X
constexpr float NS_A_SCALE = 256.f;   // A and B as 2^8 A, 2^8 B

struct NsMat {
    int m, n;              // oriented sizes, m <= n
    int mp, np;            // padded to multiples of 64
    int repeat;            // matrices of this shape, `src_stride` elements apart
    int tall;              // rows > cols: the arena holds the transpose
    int row_x, row_a;      // first arena row of the first repetition (mp rows each)
    int tiles_sym, tiles_x;    // tiles of one repetition: A or B (on and above the diagonal), X
    int first_sym, first_x;    // tiles before this descriptor
    int first_norm, first_conv;  // blocks of the norm and conversion kernels before this descriptor
    int norm_blocks, conv_blocks;  // blocks of one repetition
    long long src, src_stride, ld_src;  // element offset, distance of repetitions, row pitch of U
    long long dst, dst_stride, ld_dst;  // ... of the result
    float update;          // weight update: lr * sqrt(max(1, cols / rows))
};
struct NsGroup {
    int count;
    NsMat mat[NS_MAX_MATS];
};

// which descriptor holds item t, given the running starts
template <typename F> LP_DEVINL int ns_find(const NsGroup &g, int t, F first)
{
    int d = 0;
    while (d + 1 < g.count && t >= first(g.mat[d + 1])) ++d;
    return d;
}

constexpr int NS_X_PARTS = 2;

LP_DEVINL void ns_store_parts(float v, int parts, __half *hi, size_t lo_off)
{
    const __half h = __float2half_rn(v);
    *hi = h;
    if (parts == 2) hi[lo_off] = __float2half_rn(v - __half2float(h));
}

// ---------------------------------------------------------------------------------------------
// what the iteration starts from
// ---------------------------------------------------------------------------------------------
constexpr int NS_THREADS = 256;
constexpr int NS_NORM_ELEMS = 8192;  // elements of one block of the norm kernel

struct NsSource {          // where U comes from
    const void *u;         // the matrix itself (plain orthogonalisation)
    int bf16_u;
    // weight update: U = g + mu M' (nesterov) or M', with g = grad_scale * grads and M' = mu M + g
    const float *grads, *momentum;
    float *new_momentum;
    const float *adam_v;   // copied to new_adam_v where the two differ (the matrices have no second moment of their own)
    float *new_adam_v;
    float grad_scale, mu;
    int nesterov;
};

LP_DEVINL float ns_source(const NsSource &s, long long i)
{
    if (s.grads) {
        const float m = s.new_momentum[i];
        return s.nesterov ? fmaf(s.mu, m, s.grad_scale * s.grads[i]) : m;
    }
    return s.bf16_u ? __bfloat162float(((const bf16 *)s.u)[i]) : ((const float *)s.u)[i];
}

// partial[b] = sum of squares over the block's elements, in double: no overflow for any FP32 input.  The weight update also
// writes M' here.
__global__ void __launch_bounds__(NS_THREADS) ns_norm_kernel(const NsSource s, const __grid_constant__ NsGroup g, double *__restrict__ partial)
{
    LP_DEP_ENTER();
    const int t = blockIdx.x;
    const int d = ns_find(g, t, [](const NsMat &m) { return m.first_norm; });
    const NsMat &mat = g.mat[d];
    const int rep = (t - mat.first_norm) / mat.norm_blocks, blk = (t - mat.first_norm) % mat.norm_blocks;
    const long long rows = mat.tall ? mat.n : mat.m, cols = mat.tall ? mat.m : mat.n;
    const long long e0 = (long long)blk * NS_NORM_ELEMS, e1 = min(e0 + NS_NORM_ELEMS, rows * cols);
    const long long base = mat.src + rep * mat.src_stride;
    double acc = 0.0;
    for (long long e = e0 + threadIdx.x; e < e1; e += NS_THREADS) {
        const long long r = e / cols, i = base + r * mat.ld_src + (e - r * cols);
        if (s.grads) {
            s.new_momentum[i] = fmaf(s.mu, s.momentum[i], s.grad_scale * s.grads[i]);
            if (s.new_adam_v) s.new_adam_v[i] = s.adam_v[i];
        }
        const double x = (double)ns_source(s, i);
        acc = fma(x, x, acc);
    }
    __shared__ double sw[NS_THREADS / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if ((threadIdx.x & 31) == 0) sw[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (int w = 0; w < NS_THREADS / 32; ++w) sum += sw[w];
        partial[t] = sum;
    }
}

// X_0 as FP16 parts, oriented and padded with zeros.  A block writes 64 rows x 64 columns of the arena.
__global__ void __launch_bounds__(NS_THREADS) ns_convert_kernel(const NsSource s, const __grid_constant__ NsGroup g, const double *__restrict__ partial, float eps,
                                                                __half *__restrict__ X, int pitch_x, size_t lo_off)
{
    LP_DEP_ENTER();
    const int t = blockIdx.x;
    const int d = ns_find(g, t, [](const NsMat &m) { return m.first_conv; });
    const NsMat &mat = g.mat[d];
    const int rep = (t - mat.first_conv) / mat.conv_blocks, blk = (t - mat.first_conv) % mat.conv_blocks;
    __shared__ double sw[NS_THREADS / 32];
    __shared__ float tile[64][65];
    double acc = 0.0;
    for (int b = threadIdx.x; b < mat.norm_blocks; b += NS_THREADS) acc += partial[mat.first_norm + rep * mat.norm_blocks + b];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if ((threadIdx.x & 31) == 0) sw[threadIdx.x >> 5] = acc;
    __syncthreads();
    acc = 0.0;
    for (int w = 0; w < NS_THREADS / 32; ++w) acc += sw[w];
    const double scale = (double)NS_X_SCALE / (sqrt(acc) + (double)eps);
    const int cb = mat.np / 64;
    const int i0 = (blk / cb) * 64, j0 = (blk % cb) * 64;
    const long long base = mat.src + rep * mat.src_stride;
    const int lx = threadIdx.x & 63, ly = threadIdx.x >> 6;
    if (mat.tall) {  // U is [n, m]: read rows of U (j), columns i consecutive, and turn the tile in shared memory
        for (int y = ly; y < 64; y += 4) {
            const int j = j0 + y, i = i0 + lx;
            tile[lx][y] = (j < mat.n && i < mat.m) ? ns_source(s, base + (long long)j * mat.ld_src + i) : 0.f;
        }
    } else {
        for (int y = ly; y < 64; y += 4) {
            const int i = i0 + y, j = j0 + lx;
            tile[y][lx] = (i < mat.m && j < mat.n) ? ns_source(s, base + (long long)i * mat.ld_src + j) : 0.f;
        }
    }
    __syncthreads();
    for (int y = ly; y < 64; y += 4)
        ns_store_parts((float)((double)tile[y][lx] * scale), NS_X_PARTS, X + (size_t)(mat.row_x + rep * mat.mp + i0 + y) * pitch_x + j0 + lx, lo_off);
}

// ---------------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------------
enum { NS_GRAM = 0, NS_POLY = 1, NS_APPLY = 2, NS_LAST = 3 };

struct NsPhase {
    int kind;
    int parts;                           // FP16 parts that the products read
    float a, b, c;
    int part_rows_a, part_rows_b;        // rows between the hi and lo parts of the first and second operand's arena
    int row_off_b;                       // first row of the X buffer that is read (X lives in two buffers used in turn)
    const __half *addend;                // POLY: A; APPLY, LAST: X
    __half *out;                         // GRAM: A, POLY: B, APPLY: the other X buffer
    int pitch;                           // of addend and out
    size_t lo_off;                       // elements between the parts of addend and out
    // LAST
    void *dst;
    int bf16_dst;
    const float *params;                 // weight update: dst = keep * params - update * result
    float keep;
    int stages;
    int *err;
    unsigned long long wait_ns;
    int extra_tx;
};

static __host__ __device__ inline uint32_t make_idesc_f16(int m, int n, bool b_mn)
{
    uint32_t d = 0;
    d |= 1u << 4;                      // accumulator format F32; A and B formats F16 (0)
    d |= (b_mn ? 1u : 0u) << 16;
    d |= (uint32_t)(n >> 3) << 17;
    d |= (uint32_t)(m >> 4) << 24;
    return d;
}

// tile t of the upper triangle (rows i <= columns j) of a T x T grid, row by row
LP_DEVINL void ns_triangle(int t, int T, int &i, int &j)
{
    i = 0;
    while (t >= T - i) { t -= T - i; ++i; }
    j = i + t;
}

LP_DEVINL void ns_load32(const __half *hi, int parts, size_t lo_off, float *v)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint4 w = *reinterpret_cast<const uint4 *>(hi + 8 * q);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&x[k]));
            v[8 * q + 2 * k] = f.x;
            v[8 * q + 2 * k + 1] = f.y;
        }
    }
    if (parts == 2) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4 w = *reinterpret_cast<const uint4 *>(hi + lo_off + 8 * q);
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&x[k]));
                v[8 * q + 2 * k] += f.x;
                v[8 * q + 2 * k + 1] += f.y;
            }
        }
    }
}
LP_DEVINL void ns_store32(const float *v, int parts, __half *hi, size_t lo_off)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float x = v[8 * q + 2 * k], y = v[8 * q + 2 * k + 1];
            const __half2 p = __floats2half2_rn(x, y);
            const float2 f = __half22float2(p);
            const __half2 r = __floats2half2_rn(x - f.x, y - f.y);
            h[k] = *reinterpret_cast<const uint32_t *>(&p);
            l[k] = *reinterpret_cast<const uint32_t *>(&r);
        }
        *reinterpret_cast<uint4 *>(hi + 8 * q) = make_uint4(h[0], h[1], h[2], h[3]);
        if (parts == 2) *reinterpret_cast<uint4 *>(hi + lo_off + 8 * q) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// One CTA per 128 x 128 tile.  Warp 0 brings the operand tiles in by TMA (both parts of each), warp 1 issues the matrix
// instructions, all four warps write the result.
__global__ void __launch_bounds__(TC_THREADS) ns_product_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const NsPhase p,
                                                                const __grid_constant__ NsGroup g)
{
    LP_DEP_ENTER();
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_full[8], bar_empty[8], bar_acc;
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const bool sym = p.kind == NS_GRAM || p.kind == NS_POLY;
    const int t = blockIdx.x;
    const int d = sym ? ns_find(g, t, [](const NsMat &m) { return m.first_sym; }) : ns_find(g, t, [](const NsMat &m) { return m.first_x; });
    const NsMat &mat = g.mat[d];
    const int per = sym ? mat.tiles_sym : mat.tiles_x, first = sym ? mat.first_sym : mat.first_x;
    const int rep = (t - first) / per, tt = (t - first) % per;
    const int T = (mat.mp + 127) / 128;
    int ti, tj;
    if (sym) ns_triangle(tt, T, ti, tj);
    else { ti = tt % T; tj = tt / T; }
    const int K = p.kind == NS_GRAM ? mat.np : mat.mp;
    const int num_kb = K / TC_BK;
    const int slot_x = mat.row_x + rep * mat.mp, slot_a = mat.row_a + rep * mat.mp;
    const int row_a0 = (p.kind == NS_GRAM ? p.row_off_b + slot_x : slot_a) + ti * 128;
    const bool b_mn = !sym;
    const int row_b0 = p.kind == NS_GRAM ? p.row_off_b + slot_x + tj * 128 : slot_a + tj * 128;  // K-major second operand
    const int parts = p.parts, S = p.stages;
    const uint32_t tile_bytes = 128 * TC_BK * 2;
    const uint32_t stage_bytes = 2 * parts * tile_bytes;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 1);
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        mbar_init(smem_u32(&bar_acc), 1);
        abort_s = 0;
        fence_barrier_init();
        fence_async_proxy();
    }
    if (warp == 0) {
        __syncwarp();
        tmem_alloc(smem_u32(&tmem_base_s), 128);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_d = tmem_base_s;

    if (warp == 0 && lane == 0) {
        for (int kb = 0; kb < num_kb; ++kb) {
            const int s = kb % S;
            if (kb >= S && !mbar_wait(smem_u32(&bar_empty[s]), ((kb / S) & 1) ^ 1, p.wait_ns)) {
                atomicExch(p.err, 1);
                abort_s = 1;
                break;
            }
            const uint32_t base = smem_u32(smem + (size_t)s * stage_bytes);
            const uint32_t bar = smem_u32(&bar_full[s]);
            mbar_expect_tx(bar, stage_bytes + (kb == 0 && t == 0 ? (uint32_t)p.extra_tx : 0u));
            const int kk = kb * TC_BK;
            for (int q = 0; q < parts; ++q) {
                tma_load_2d(base + q * tile_bytes, &mapA, bar, kk, row_a0 + q * p.part_rows_a);
                const uint32_t sb = base + (parts + q) * tile_bytes;
                if (!b_mn) {
                    tma_load_2d(sb, &mapB, bar, kk, row_b0 + q * p.part_rows_b);
                } else {  // X as the second operand: 64 rows of K, two boxes of 64 columns
                    const int row = p.row_off_b + slot_x + kk + q * p.part_rows_b;
                    tma_load_2d(sb, &mapB, bar, tj * 128, row);
                    tma_load_2d(sb + 8192, &mapB, bar, tj * 128 + 64, row);
                }
            }
        }
    } else if (warp == 1 && lane == 0) {
        const uint32_t idesc = make_idesc_f16(128, 128, b_mn);
        bool ok = true;
        for (int kb = 0; kb < num_kb; ++kb) {
            const int s = kb % S;
            if (!mbar_wait(smem_u32(&bar_full[s]), (kb / S) & 1, p.wait_ns)) {
                atomicExch(p.err, 2);
                abort_s = 1;
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t sa = smem_u32(smem + (size_t)s * stage_bytes), sb = sa + parts * tile_bytes;
#pragma unroll
            for (int k = 0; k < TC_BK / TC_UMMA_K; ++k) {
                const uint64_t da = make_smem_desc(sa + k * 32, 16, 1024);
                const uint64_t db = b_mn ? make_smem_desc(sb + k * 2048, 8192, 1024) : make_smem_desc(sb + k * 32, 16, 1024);
                umma_bf16(tmem_d, da, db, idesc, (kb | k) != 0 ? 1u : 0u);
                if (parts == 2) {
                    const uint64_t la = make_smem_desc(sa + tile_bytes + k * 32, 16, 1024);
                    const uint64_t lb = b_mn ? make_smem_desc(sb + tile_bytes + k * 2048, 8192, 1024) : make_smem_desc(sb + tile_bytes + k * 32, 16, 1024);
                    umma_bf16(tmem_d, da, lb, idesc, 1u);
                    umma_bf16(tmem_d, la, db, idesc, 1u);
                }
            }
            umma_commit(smem_u32(&bar_empty[s]));
        }
        if (ok) umma_commit(smem_u32(&bar_acc));
    }
    __syncwarp();
    const bool done = mbar_wait(smem_u32(&bar_acc), 0, p.wait_ns);
    if (!done) {
        if (lane == 0) atomicExch(p.err, 3);
        abort_s = 1;
    }
    __syncthreads();
    if (abort_s == 0) {
        tc_fence_after();
        const int row = ti * 128 + warp * 32 + lane;
        const int slot = sym ? slot_a : slot_x, stored = sym ? parts : NS_X_PARTS;
        for (int c0 = 0; c0 < 128; c0 += 32) {
            float v[32];
            __syncwarp();
            tmem_ld_32x32(tmem_d + ((uint32_t)(warp * 32) << 16) + c0, v);
            const int col = tj * 128 + c0;
            const int width = sym ? mat.mp : mat.np;
            if (row >= mat.mp || col >= width) continue;
            const size_t at = (size_t)(slot + row) * p.pitch + col;
            if (p.kind == NS_GRAM) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] *= NS_A_SCALE / (NS_X_SCALE * NS_X_SCALE);
            } else {
                float x[32];
                ns_load32(p.addend + at, stored, p.lo_off, x);
                const float f = p.kind == NS_POLY ? p.c / NS_A_SCALE : 1.f / NS_A_SCALE;
                const float h = p.kind == NS_POLY ? p.b : p.a;
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = fmaf(h, x[i], f * v[i]);
            }
            if (p.kind != NS_LAST) {
                ns_store32(v, stored, p.out + at, p.lo_off);
                if (sym && ti != tj) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) ns_store_parts(v[i], stored, p.out + (size_t)(slot + col + i) * p.pitch + row, p.lo_off);
                }
            } else if (row < mat.m) {
                const long long base = mat.dst + rep * mat.dst_stride;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    if (col + i < mat.n) {
                        const long long o = base + (mat.tall ? (long long)(col + i) * mat.ld_dst + row : (long long)row * mat.ld_dst + col + i);
                        const float r = v[i] * (1.f / NS_X_SCALE);
                        if (p.params) ((float *)p.dst)[o] = fmaf(-mat.update, r, p.keep * p.params[o]);
                        else if (p.bf16_dst) ((bf16 *)p.dst)[o] = __float2bfloat16_rn(r);
                        else ((float *)p.dst)[o] = r;
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        __syncwarp();
        tmem_dealloc(tmem_d, 128);
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
static bool ns_init(std::string &err)
{
    if (cudaFuncSetAttribute(ns_product_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024) != cudaSuccess) {
        err = "cannot raise the dynamic shared memory limit of the Newton-Schulz products";
        return false;
    }
    return true;
}

// 2-D FP16 tensor map over a row-major arena [rows, pitch]; box {64 columns, box_rows}, 128-byte swizzle
static bool ns_make_map(const TcState &tc, CUtensorMap *map, const __half *base, int64_t rows, int64_t pitch, int box_rows)
{
    cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)pitch * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return tc.encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, (void *)base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Bounds of the iteration: with |X| <= 1 at the start, every later |X| must stay below 2 and |B| below 200 for the FP16
// scales above.  The largest value of |a s + b s^3 + c s^5| on [0, top] is at an end or where its derivative vanishes.
static bool ns_coefficients_ok(double a, double b, double c, int steps)
{
    if (!(std::isfinite(a) && std::isfinite(b) && std::isfinite(c))) return false;
    double top = 1.0;
    for (int k = 0; k < steps; ++k) {
        if (std::fabs(b) * top * top + std::fabs(c) * top * top * top * top > 200.0) return false;
        auto f = [&](double s) { return std::fabs(s * (a + s * s * (b + s * s * c))); };
        double best = f(top);
        const double disc = 9.0 * b * b - 20.0 * a * c;
        double roots[2] = {-1.0, -1.0};
        if (c != 0.0 && disc >= 0.0) {
            roots[0] = (-3.0 * b - std::sqrt(disc)) / (10.0 * c);
            roots[1] = (-3.0 * b + std::sqrt(disc)) / (10.0 * c);
        } else if (c == 0.0 && b != 0.0) {
            roots[0] = -a / (3.0 * b);
        }
        for (double t : roots)
            if (t > 0.0 && t < top * top) best = std::max(best, f(std::sqrt(t)));
        if (best > 2.0) return false;
        top = std::max(best, 1e-30);
    }
    return true;
}

struct NsLayout {  // sizes of the arenas of a group
    int rows_x = 0, rows_a = 0, pitch_x = 0, pitch_a = 0, norm_blocks = 0;
    size_t x_elems() const { return (size_t)2 * NS_X_PARTS * rows_x * pitch_x; }
    size_t a_elems(int parts) const { return (size_t)parts * rows_a * pitch_a; }
    static size_t up(size_t b) { return (b + 1023) & ~(size_t)1023; }
    size_t bytes(int parts) const { return up(2 * x_elems()) + 2 * up(2 * a_elems(parts)) + up(sizeof(double) * (size_t)std::max(norm_blocks, 1)); }
};

// fills the derived fields of the descriptors (m, n, repeat, tall given)
static NsLayout ns_layout(NsGroup &g)
{
    NsLayout l;
    int sym = 0, xt = 0, conv = 0;
    for (int d = 0; d < g.count; ++d) {
        NsMat &m = g.mat[d];
        m.mp = (m.m + 63) / 64 * 64;
        m.np = (m.n + 63) / 64 * 64;
        m.row_x = l.rows_x;
        m.row_a = l.rows_a;
        l.rows_x += m.mp * m.repeat;
        l.rows_a += m.mp * m.repeat;
        l.pitch_x = std::max(l.pitch_x, m.np);
        l.pitch_a = std::max(l.pitch_a, m.mp);
        const int T = (m.mp + 127) / 128;
        m.tiles_sym = T * (T + 1) / 2;
        m.tiles_x = T * ((m.np + 127) / 128);
        m.first_sym = sym;
        m.first_x = xt;
        sym += m.tiles_sym * m.repeat;
        xt += m.tiles_x * m.repeat;
        m.norm_blocks = (int)ceil_div64((int64_t)m.m * m.n, NS_NORM_ELEMS);
        m.conv_blocks = (m.mp / 64) * (m.np / 64);
        m.first_norm = l.norm_blocks;
        m.first_conv = conv;
        l.norm_blocks += m.norm_blocks * m.repeat;
        conv += m.conv_blocks * m.repeat;
    }
    return l;
}

struct NsTarget {
    void *dst;
    int bf16_dst;
    const float *params;
    float keep;
};

static bool ns_run(TcState &tc, Exec &ex, const NsSource &src, NsGroup &g, const NsLayout &l, int parts, int steps, double a, double b, double c, double eps,
                   const NsTarget &out, uint8_t *ws, std::string &err)
{
    __half *X = (__half *)ws;
    __half *A = (__half *)(ws + NsLayout::up(2 * l.x_elems()));
    __half *B = (__half *)((uint8_t *)A + NsLayout::up(2 * l.a_elems(parts)));
    double *partial = (double *)((uint8_t *)B + NsLayout::up(2 * l.a_elems(parts)));
    const size_t lo_x = (size_t)l.rows_x * l.pitch_x, lo_a = (size_t)l.rows_a * l.pitch_a;
    CUtensorMap xk, xmn, ak, bk;
    if (!ns_make_map(tc, &xk, X, (int64_t)2 * NS_X_PARTS * l.rows_x, l.pitch_x, 128) || !ns_make_map(tc, &xmn, X, (int64_t)2 * NS_X_PARTS * l.rows_x, l.pitch_x, 64) ||
        !ns_make_map(tc, &ak, A, (int64_t)parts * l.rows_a, l.pitch_a, 128) || !ns_make_map(tc, &bk, B, (int64_t)parts * l.rows_a, l.pitch_a, 128)) {
        err = "cuTensorMapEncodeTiled failed";
        return false;
    }
    int sym = 0, xt = 0, conv = 0;
    for (int d = 0; d < g.count; ++d) {
        sym += g.mat[d].tiles_sym * g.mat[d].repeat;
        xt += g.mat[d].tiles_x * g.mat[d].repeat;
        conv += g.mat[d].conv_blocks * g.mat[d].repeat;
    }
    launch_dep(ns_norm_kernel, dim3(l.norm_blocks), dim3(NS_THREADS), 0, ex.st, src, g, partial);
    launch_dep(ns_convert_kernel, dim3(conv), dim3(NS_THREADS), 0, ex.st, src, g, partial, (float)eps, X, l.pitch_x, lo_x);
    ex.launches += 2;
    NsPhase p{};
    p.parts = parts;
    p.a = (float)a; p.b = (float)b; p.c = (float)c;
    p.stages = parts == 2 ? 3 : 6;
    p.err = tc.err_word;
    p.wait_ns = tc.wait_limit_ns;
    const size_t smem = (size_t)p.stages * 2 * parts * 128 * TC_BK * 2 + 1024;
    for (int k = 0; k < steps; ++k) {
        const int cur = k & 1;
        p.row_off_b = cur * NS_X_PARTS * l.rows_x;
        p.extra_tx = tc.overdeclare_tx;
        tc.overdeclare_tx = 0;
        p.kind = NS_GRAM;
        p.part_rows_a = p.part_rows_b = l.rows_x;
        p.addend = nullptr; p.out = A; p.pitch = l.pitch_a; p.lo_off = lo_a;
        launch_dep(ns_product_kernel, dim3(sym), dim3(TC_THREADS), smem, ex.st, xk, xk, p, g);
        p.extra_tx = 0;
        p.kind = NS_POLY;
        p.part_rows_a = p.part_rows_b = l.rows_a;
        p.addend = A; p.out = B;
        launch_dep(ns_product_kernel, dim3(sym), dim3(TC_THREADS), smem, ex.st, ak, ak, p, g);
        p.kind = k + 1 == steps ? NS_LAST : NS_APPLY;
        p.part_rows_b = l.rows_x;
        p.addend = X + (size_t)cur * NS_X_PARTS * lo_x; p.out = X + (size_t)(cur ^ 1) * NS_X_PARTS * lo_x; p.pitch = l.pitch_x; p.lo_off = lo_x;
        p.dst = out.dst; p.bf16_dst = out.bf16_dst; p.params = out.params; p.keep = out.keep;
        launch_dep(ns_product_kernel, dim3(xt), dim3(TC_THREADS), smem, ex.st, bk, xmn, p, g);
        ex.launches += 3;
    }
    return true;
}

// ---------------------------------------------------------------------------------------------
// weight update: every parameter that belongs to no matrix takes an Adam step
// ---------------------------------------------------------------------------------------------
struct NsSpans {  // the stretches of the flat vector between the matrices
    int count;
    long long begin[NS_MAX_MATS + 1], first[NS_MAX_MATS + 2];  // first element, and elements before the stretch; first[count] = all
};
__global__ void ns_adam_kernel(const float *__restrict__ p, const float *__restrict__ m, const float *__restrict__ v, const float *__restrict__ grad, const NsSpans spans,
                               float scale, float lr, float b1, float one_minus_b1, float b2, float one_minus_b2, float eps, float inv_c1, float inv_c2,
                               float *__restrict__ pn, float *__restrict__ mn, float *__restrict__ vn)
{
    LP_DEP_ENTER();
    const long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (e >= spans.first[spans.count]) return;
    int s = 0;
    while (e >= spans.first[s + 1]) ++s;
    const long long i = spans.begin[s] + (e - spans.first[s]);
    const float g = scale * grad[i];
    const float mi = b1 * m[i] + one_minus_b1 * g;
    const float vi = b2 * v[i] + one_minus_b2 * g * g;
    const float pi = p[i] - lr * (mi * inv_c1) / (sqrtf(vi * inv_c2) + eps);
    mn[i] = mi;
    vn[i] = vi;
    pn[i] = pi;
}
