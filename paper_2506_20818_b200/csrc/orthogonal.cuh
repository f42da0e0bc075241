// Orthogonalisation of matrices by Newton-Schulz products, and the weight update built on it.
//
//   X_0 = U / (|U|_F + eps);   A = X X^T,  B = b A + c A^2,  X <- a X + B X     (steps times)
//
// maps every singular value s of X_0 through the odd polynomial a s + b s^3 + c s^5 again and again and leaves the
// singular vectors.  The products run on the tensor cores with FP16 operands and FP32 accumulators.  FP16 carries eleven
// significant bits where BF16 carries eight, at the same rate, and the range it lacks is not needed here: the values
// are bounded by the polynomial (the host refuses coefficients for which they are not), so X is held as 2^14 X, A as 2^13 A and B as
// 2^8 B to 2^13 B, as far as its coefficients' bound allows (2^12 B for the default): the largest values lie just below the end of FP16.
// What a matrix holds far below its largest values ends at FP16's 2^-24: FP32 rows of 1e-5 of the others are 3e-7 to 9e-6 off, relative
// to themselves, rows of 1e-6 2e-6 to 9e-5 (64 x 64 to 2048 x 2048; with 2^12 X and 2^8 A, B thirty times that), where FP32 products
// are 3e-7 to 2.5e-6 off for rows of any size.  Of the whole matrix these errors are 1e-9.
// X is kept twice: in FP32, from which the term a X of every step is taken, and as FP16 operands.
//   BF16 results : X, A and B are one FP16 number per value in the products
//   FP32 results : pairs of FP16 numbers hi + lo (22 bits), products hi*lo + lo*hi + hi*hi; the accumulator of the matrix
//                  instructions rounds towards zero, so it only adds up 32 to 64 terms at a time and those sums are
//                  added in FP32 registers (1000 x 417: error 1.3e-5 with one accumulator for all of K, 1e-6 this way)
// Why X keeps more bits than its operands: rounding X to eleven bits would add a matrix of full rank, and whatever lies
// in directions that X hardly has is multiplied by a in every step (3.4^5 = 480 for five).  The errors of the products are
// of the form dB X and B dX, which vanish in such directions, so they stay at their own size.  For the same reason X_0 is
// U times a power of two 2^14 r / |U|, r in [1/2, 1), which is exact; b / r^2 and c / r^4 in the place of b and c keep r X
// going in the place of X, and the result is divided by r.
// A matrix with more rows than columns is iterated transposed: m = min(rows, cols), n = max(rows, cols).
//
// All matrices of a call lie in common arenas (X: rows of `pitch_x`, A and B: rows of `pitch_a`), each padded with zeros
// to multiples of 64; the padding stays zero through every product.
#pragma once
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.cuh"
#include "embed.cuh"
#include "gemm_tc.cuh"

constexpr int NS_MAX_MATS = 16;       // descriptors in one launch group (they travel as kernel arguments, 4 KiB in all)
constexpr float NS_X_SCALE = 16384.f;  // X is held as 2^14 X: |X| <= 2
constexpr float NS_A_SCALE = 8192.f;   // A as 2^13 A: |A| <= 4

struct NsMat {
    int m, n;              // oriented sizes, m <= n
    int mp, np;            // padded to multiples of 64
    int repeat;            // matrices of this shape, `src_stride` elements apart
    int tall;              // rows > cols: the arena holds the transpose
    int row_x, row_a;      // first arena row of the first repetition (mp rows each)
    int tiles_a, tiles_x;      // tiles of one repetition: A or B, X
    int first_a, first_x;      // tiles before this descriptor
    int first_norm, first_conv;  // blocks of the norm and conversion kernels before this descriptor
    int norm_blocks, conv_blocks;  // blocks of one repetition
    int norm_elems;        // elements of one block of the norm kernel
    int index;             // matrices before this descriptor
    long long src, src_stride, ld_src;  // element offset, distance of repetitions, row pitch of U
    long long dst, dst_stride, ld_dst;  // ... of the result
    float update;          // weight update: lr * sqrt(max(1, cols / rows))
};
struct NsGroup {
    int count;
    NsMat mat[NS_MAX_MATS];
};

struct NsPoly {          // X <- a X + B X, B = b A + c A^2, in the scales that X, A and B are held in
    float a, b, c;
    float unscale;       // of B
};

struct NsX {             // one of the two buffers of X
    float *full;
    __half *hi;
    size_t lo_off;       // the low parts lie this many elements behind the high ones
    int pitch;
};

// which descriptor holds item t, given the running starts
template <typename F> LP_DEVINL int ns_find(const NsGroup &g, int t, F first)
{
    int d = 0;
    while (d + 1 < g.count && t >= first(g.mat[d + 1])) ++d;
    return d;
}

// ---------------------------------------------------------------------------------------------
// what the iteration starts from
// ---------------------------------------------------------------------------------------------
constexpr int NS_THREADS = 256;
constexpr int NS_NORM_ELEMS = 2048;   // elements of one block of the norm kernel, more where a matrix would need over 1024 blocks
constexpr int NS_NORM_BLOCKS = 1024;

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
        const float m = __ldcg(s.new_momentum + i);  // written by other blocks, in the chain kernel of the same launch
        return s.nesterov ? fmaf(s.mu, m, s.grad_scale * s.grads[i]) : m;
    }
    return s.bf16_u ? __bfloat162float(((const bf16 *)s.u)[i]) : ((const float *)s.u)[i];
}

// The weight update's other parameters: Adam over the stretches of the flat vector between the matrices.
struct NsSpans {
    int count;
    long long begin[NS_MAX_MATS + 1], first[NS_MAX_MATS + 2];  // first element, and elements before the stretch; first[count] = all
};
struct NsAdam {
    const float *p, *m, *v, *grad;
    float *pn, *mn, *vn;
    float scale, lr, b1, one_minus_b1, b2, one_minus_b2, eps, inv_c1, inv_c2;
    NsSpans spans;
};
constexpr int NS_ADAM_ELEMS = 1024;  // elements of one block

template <int T> LP_DEVINL void ns_sync() { __syncwarp(); asm volatile("bar.sync 1, %0;" ::"n"(T) : "memory"); }  // the threads that share a block of work

// ... the same with the OR of a condition over them, so that all take the same branch after it
template <int T> LP_DEVINL bool ns_any(bool x)
{
    uint32_t r;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.aligned.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)x), "n"(T) : "memory");
    return r != 0;
}

template <int T> LP_DEVINL void ns_adam_block(const NsAdam &a, int blk, int tid)
{
    for (int u = 0; u < NS_ADAM_ELEMS / T; ++u) {
        const long long e = (long long)blk * NS_ADAM_ELEMS + u * T + tid;
        if (e >= a.spans.first[a.spans.count]) return;
        int s = 0;
        while (e >= a.spans.first[s + 1]) ++s;
        const long long i = a.spans.begin[s] + (e - a.spans.first[s]);
        const float g = a.scale * a.grad[i];
        const float mi = a.b1 * a.m[i] + a.one_minus_b1 * g;
        const float vi = a.b2 * a.v[i] + a.one_minus_b2 * g * g;
        const float pi = a.p[i] - a.lr * (mi * a.inv_c1) / (sqrtf(vi * a.inv_c2) + a.eps);
        a.mn[i] = mi;
        a.vn[i] = vi;
        a.pn[i] = pi;
    }
}

// partial[t] = sum of squares over the block's elements, in double: no overflow for any FP32 input.  The weight update also
// writes M' here.
template <int T> LP_DEVINL void ns_norm_block(const NsSource &s, const NsGroup &g, int t, int tid, double *__restrict__ partial, double *sw)
{
    const int d = ns_find(g, t, [](const NsMat &m) { return m.first_norm; });
    const NsMat &mat = g.mat[d];
    const int rep = (t - mat.first_norm) / mat.norm_blocks, blk = (t - mat.first_norm) % mat.norm_blocks;
    const long long rows = mat.tall ? mat.n : mat.m, cols = mat.tall ? mat.m : mat.n;
    const long long e0 = (long long)blk * mat.norm_elems, e1 = min(e0 + mat.norm_elems, rows * cols);
    const long long base = mat.src + rep * mat.src_stride;
    double acc = 0.0;
    constexpr int U = 4;  // elements (or runs of four) in flight per thread
    if (!s.grads && mat.ld_src == cols && ((base + e0) & 3) == 0 && ((uintptr_t)s.u & 15) == 0) {  // dense rows: four neighbours per load
        for (long long e = e0 + 4 * tid; e < e1; e += U * 4 * T) {
            float x[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long i = e + u * 4 * T;
                if (i + 4 <= e1) {
                    if (s.bf16_u) load_elems<bf16, 4>((const bf16 *)s.u + base + i, x[u]);
                    else load_elems<float, 4>((const float *)s.u + base + i, x[u]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[u][k] = i + k < e1 ? ns_source(s, base + i + k) : 0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc = fma((double)x[u][k], (double)x[u][k], acc);
        }
    } else
    for (long long e = e0 + tid; e < e1; e += U * T) {
        long long at[U];
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = e + u * T;
            if (mat.ld_src == cols) at[u] = base + i;
            else { const long long r = i / cols; at[u] = base + r * mat.ld_src + (i - r * cols); }
            if (i >= e1) at[u] = -1;
        }
        if (s.grads) {
            float gr[U], mo[U], av[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                gr[u] = at[u] >= 0 ? s.grad_scale * s.grads[at[u]] : 0.f;
                mo[u] = at[u] >= 0 ? s.momentum[at[u]] : 0.f;
                if (s.new_adam_v) av[u] = at[u] >= 0 ? s.adam_v[at[u]] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float m = fmaf(s.mu, mo[u], gr[u]);
                if (at[u] >= 0) {
                    s.new_momentum[at[u]] = m;
                    if (s.new_adam_v) s.new_adam_v[at[u]] = av[u];
                }
                x[u] = s.nesterov ? fmaf(s.mu, m, gr[u]) : m;
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = at[u] >= 0 ? ns_source(s, at[u]) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) acc = fma((double)x[u], (double)x[u], acc);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if ((tid & 31) == 0) sw[tid >> 5] = acc;
    ns_sync<T>();
    if (tid == 0) {
        double sum = 0.0;
        for (int w = 0; w < T / 32; ++w) sum += sw[w];
        partial[t] = sum;
    }
    ns_sync<T>();
}

// |U| + eps = 2^e r with r in [1/2, 1): X_0 is held as 2^14 2^-e U, which is 2^14 r times U / (|U| + eps)
LP_DEVINL void ns_start_scale(double norm, float &r, double &pow2)
{
    int e = 0;
    const double f = frexp(norm, &e);  // norm = f 2^e, f in [1/2, 1)
    if (norm == 0.0 || !isfinite(norm)) {  // zeros with eps = 0 stay zeros; a norm of infinity or NaN makes the products NaN
        r = 1.f;
        pow2 = norm == 0.0 ? 0.0 : (double)NS_X_SCALE / norm;
        return;
    }
    r = (float)f;
    pow2 = ldexp((double)NS_X_SCALE, -e);
}

// X_0, oriented and padded with zeros: 64 rows x 64 columns of the arena.  `tile` holds 64 x 65 floats, `sw` T / 32 doubles.
template <int PARTS, int T>
LP_DEVINL void ns_convert_block(const NsSource &s, const NsGroup &g, int t, int tid, const double *partial, double eps, const NsX &X, float *inv_r, float *tile, double *sw)
{
    const int d = ns_find(g, t, [](const NsMat &m) { return m.first_conv; });
    const NsMat &mat = g.mat[d];
    const int rep = (t - mat.first_conv) / mat.conv_blocks, blk = (t - mat.first_conv) % mat.conv_blocks;
    double acc = 0.0;
    for (int b = tid; b < mat.norm_blocks; b += T) acc += __ldcg(partial + mat.first_norm + rep * mat.norm_blocks + b);
    const int cb = mat.np / 64;
    const int i0 = (blk / cb) * 64, j0 = (blk % cb) * 64;
    const long long base = mat.src + rep * mat.src_stride;
    // a thread holds R runs of four neighbours in a row of U; tall: U is [n, m], and the tile is turned in shared memory
    constexpr int R = 1024 / T, STEP = T / 16;
    const int lx = (tid & 15) * 4, ly = tid >> 4;
    float u[R][4];
    const bool wide = !s.grads && (mat.ld_src & 3) == 0 && (base & 3) == 0 && ((uintptr_t)s.u & 15) == 0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int row = (mat.tall ? j0 : i0) + ly + STEP * k, col = (mat.tall ? i0 : j0) + lx;
        const int rows = mat.tall ? mat.n : mat.m, cols = mat.tall ? mat.m : mat.n;
        const long long at = base + (long long)row * mat.ld_src + col;
        if (wide && row < rows && col + 4 <= cols) {
            if (s.bf16_u) load_elems<bf16, 4>((const bf16 *)s.u + at, u[k]);
            else load_elems<float, 4>((const float *)s.u + at, u[k]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) u[k][j] = row < rows && col + j < cols ? ns_source(s, at + j) : 0.f;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if ((tid & 31) == 0) sw[tid >> 5] = acc;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int y = ly + STEP * k;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (mat.tall) tile[(lx + j) * 65 + y] = u[k][j]; else tile[y * 65 + lx + j] = u[k][j];
        }
    }
    ns_sync<T>();
    acc = 0.0;
    for (int w = 0; w < T / 32; ++w) acc += sw[w];
    float r;
    double pow2;
    ns_start_scale(sqrt(acc) + eps, r, pow2);
    if (blk == 0 && tid == 0) inv_r[mat.index + rep] = 1.f / r;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int y = ly + STEP * k;
        float a[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = (float)(tile[y * 65 + lx + j] * pow2);
        const size_t at = (size_t)(mat.row_x + rep * mat.mp + i0 + y) * X.pitch + j0 + lx;
        store_elems<float, 4>(X.full + at, a);
        const __half2 h0 = __floats2half2_rn(a[0], a[1]), h1 = __floats2half2_rn(a[2], a[3]);
        *reinterpret_cast<uint2 *>(X.hi + at) = make_uint2(*reinterpret_cast<const uint32_t *>(&h0), *reinterpret_cast<const uint32_t *>(&h1));
        if (PARTS == 2) {
            const float2 f0 = __half22float2(h0), f1 = __half22float2(h1);
            const __half2 l0 = __floats2half2_rn(a[0] - f0.x, a[1] - f0.y), l1 = __floats2half2_rn(a[2] - f1.x, a[3] - f1.y);
            *reinterpret_cast<uint2 *>(X.hi + X.lo_off + at) = make_uint2(*reinterpret_cast<const uint32_t *>(&l0), *reinterpret_cast<const uint32_t *>(&l1));
        }
    }
    ns_sync<T>();
}

// the two steps as kernels of their own, for matrices too large for the chain kernel; blocks from `norm_blocks` on take Adam steps
__global__ void __launch_bounds__(NS_THREADS) ns_norm_kernel(const NsSource s, const __grid_constant__ NsGroup g, const __grid_constant__ NsAdam adam, int norm_blocks,
                                                             double *__restrict__ partial)
{
    LP_DEP_ENTER();
    __shared__ double sw[NS_THREADS / 32];
    if ((int)blockIdx.x < norm_blocks) ns_norm_block<NS_THREADS>(s, g, blockIdx.x, threadIdx.x, partial, sw);
    else ns_adam_block<NS_THREADS>(adam, blockIdx.x - norm_blocks, threadIdx.x);
}
template <int PARTS>
__global__ void __launch_bounds__(NS_THREADS) ns_convert_kernel(const NsSource s, const __grid_constant__ NsGroup g, const double *partial, double eps, const NsX X,
                                                                float *inv_r)
{
    LP_DEP_ENTER();
    __shared__ double sw[NS_THREADS / 32];
    __shared__ float tile[64 * 65];
    ns_convert_block<PARTS, NS_THREADS>(s, g, blockIdx.x, threadIdx.x, partial, eps, X, inv_r, tile, sw);
}

// ---------------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------------
enum { NS_GRAM = 0, NS_POLY = 1, NS_APPLY = 2, NS_LAST = 3 };

struct NsPhase {
    int kind;
    NsPoly poly;
    int lo_rows_a, lo_rows_b;            // rows between the hi and lo parts of the first and second operand's arena
    int x_row0;                          // first row of the X buffer that is read
    const __half *A;                     // POLY: the addend b A
    const float *X;                      // APPLY, LAST: the addend a X
    __half *out;                         // GRAM: A, POLY: B
    int pitch_a;
    size_t lo_off_a;                     // elements between the parts of A and B
    NsX next;                            // APPLY: the other X buffer
    const float *inv_r;                  // 1 / r of every matrix
    // LAST
    void *dst;
    int bf16_dst;
    const float *params;                 // weight update: dst = keep * params - update * result
    float keep;
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

// eight FP16 values (one 16-byte piece) as floats, added to v
LP_DEVINL void ns_add8(const uint4 &w, float *v)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&x[k]));
        v[2 * k] += f.x;
        v[2 * k + 1] += f.y;
    }
}
// 8 values as FP16 parts
template <int PARTS> LP_DEVINL void ns_store8(const float *v, __half *hi, size_t lo_off)
{
    uint32_t h[4], l[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __half2 p = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
        h[k] = *reinterpret_cast<const uint32_t *>(&p);
        if (PARTS == 2) {
            const float2 f = __half22float2(p);
            const __half2 r = __floats2half2_rn(v[2 * k] - f.x, v[2 * k + 1] - f.y);
            l[k] = *reinterpret_cast<const uint32_t *>(&r);
        }
    }
    *reinterpret_cast<uint4 *>(hi) = make_uint4(h[0], h[1], h[2], h[3]);
    if (PARTS == 2) *reinterpret_cast<uint4 *>(hi + lo_off) = make_uint4(l[0], l[1], l[2], l[3]);
}

// ---------------------------------------------------------------------------------------------
// The whole iteration in one launch, for matrices whose products leave SMs idle.
//
// Every launch of a product costs two to three microseconds before its first operand arrives, which is more than such a
// product takes: 17 launches took 63 us for one 64 x 64 matrix and 134 us for the four matrices of a 128-256-256 encoder.
// Here the blocks stay resident (cooperative launch) and step from phase to phase -- norm, conversion, and per step A, B and
// the new X -- through a counter in global memory.  The blocks form clusters of C that split the K range of a 128 x 64 tile:
// each adds up its share in tensor memory, all of them put the sums into shared memory, and each finishes 64 / C columns
// from everybody's (distributed shared memory), so that operands, products and epilogue are all spread C ways.
//   warp 0 operands by TMA, warp 1 matrix instructions, warps 2-17 sums and results (and the first two phases)
// Every wait is bounded; a block that gives up reports it and leaves, and the others run into their own limits.
// ---------------------------------------------------------------------------------------------
constexpr int NSC_THREADS = 576;
constexpr int NSC_WORKERS = 512;  // threads of warps 2-17
constexpr int NSC_BN = 64;
constexpr int NSC_KEPT = 4;  // tiles of A and of X whose description a block keeps
constexpr int NSC_ACCS = 4;  // accumulators used in turn
template <int PARTS> constexpr int NSC_ACC_COLS = PARTS * NSC_BN;  // PARTS = 2: the two halves of a 64-term block are added up apart
constexpr int NSC_SUM_BYTES = 128 * NSC_BN * 4;  // the sums of a tile
constexpr int NSC_BARRIERS = 256;  // counters of one call: 1 + 3 * steps are used, the last one counts the blocks that are done with them

struct NsChainIo {       // of one kind of phase; the addend has the rows, columns and pitch of the output
    const __half *add_h;   // B: A (parts out_lo apart)
    const float *add_f;    // new X: X
    __half *out_h;         // operands of a later phase
    float *out_f;          // new X in FP32
    long long out_lo;      // elements between the parts of out_h
    int pitch;
};
struct NsChain {
    NsChainIo io[2][3];                  // [step parity][kind], read from constant memory where needed: pointers held in registers spill
    int parts_rows_x, parts_rows_a;      // rows between the hi and lo parts of X and of A, B
    int steps;
    NsPoly poly;
    double eps;
    NsX X0;
    double *partial;
    float *inv_r;
    int norm_blocks, adam_blocks, conv_blocks, tiles_a, tiles_x;
    void *dst;
    int bf16_dst;
    const float *params;
    float keep;
    unsigned *counters;  // NSC_BARRIERS of them, zero between launches
    int *err;
    unsigned long long wait_ns;
    int extra_tx;
};

LP_DEVINL unsigned ld_acquire_gpu(const unsigned *p)
{
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
LP_DEVINL void red_release_gpu(unsigned *p)
{
    asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p) : "memory");
}
// A block that will not wait for the counters again says so; the last one puts them back to zero, while the last products are still
// under way.  So a launch leaves them as it found them, also one that a captured graph replays.
LP_DEVINL void ns_leave(unsigned *counters, int used, int count)
{
    unsigned before;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(counters + count) : "memory");
    if (before != gridDim.x - 1) return;
#pragma unroll 1
    for (int i = 0; i < used; ++i) counters[i] = 0;
    counters[count] = 0;
}
LP_DEVINL void fence_async_proxy_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }
LP_DEVINL bool counter_wait(const unsigned *p, unsigned want, unsigned long long limit_ns)
{
    if (ld_acquire_gpu(p) >= want) return true;
    const unsigned long long t0 = global_timer_ns();
    for (;;) {
        for (int i = 0; i < 16; ++i)
            if (ld_acquire_gpu(p) >= want) return true;
        if (global_timer_ns() - t0 > limit_ns) return false;
    }
}
LP_DEVINL void mbar_arrive_cluster(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
LP_DEVINL bool mbar_wait_cluster(uint32_t bar, uint32_t parity, unsigned long long limit_ns)
{
    unsigned long long t0 = 0;
    for (;;) {
        for (int i = 0; i < 64; ++i) {
            uint32_t ok;
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                         : "=r"(ok)
                         : "r"(bar), "r"(parity)
                         : "memory");
            if (ok) return true;
        }
        if (t0 == 0) t0 = global_timer_ns();
        else if (global_timer_ns() - t0 > limit_ns) return false;
    }
}
// this block's shared memory into that of a block of the cluster, counted in bytes on that block's barrier
LP_DEVINL void copy_to_cta(uint32_t dst_cluster, uint32_t src, uint32_t bytes, uint32_t bar_cluster)
{
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst_cluster), "r"(src), "r"(bytes), "r"(bar_cluster)
                 : "memory");
}
// one lane of the (converged) warp, by the instruction whose branch the compiler knows to be taken by a single lane: the operands
// of the matrix and copy instructions behind it stay in uniform registers (a branch on the lane number: 146 cycles per matrix
// instruction instead of 50)
LP_DEVINL bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
LP_DEVINL void tmem_ld_32x16(uint32_t taddr, float *v)
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
LP_DEVINL void tmem_ld_32x8(uint32_t a, float *v)
{
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(a)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
LP_DEVINL void tmem_ld_32x8_pair(uint32_t a, uint32_t b, float *v, float *w)
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(a)
                 : "memory");
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(b)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = __uint_as_float(r[i]);
        w[i] = __uint_as_float(r[8 + i]);
    }
}
// sum + lost becomes sum + lost + x, the rounding of the new sum added to lost (exact whatever the magnitudes)
LP_DEVINL void ns_two_sum(float &sum, float &lost, float x)
{
    const float t = sum + x, b = t - sum;
    lost += (sum - (t - b)) + (x - b);
    sum = t;
}

// the phase's tiles: where a tile lies and what it is made of
struct NsTile {
    int d, rep, ti, tj, slot_x, slot_a, mp, np, m, n, tall, index;
    LP_DEVINL int num_kb(int kind) const { return (kind == NS_GRAM ? np : mp) / TC_BK; }
};
LP_DEVINL NsTile ns_tile(const NsGroup &g, int kind, int t)
{
    const bool square = kind == NS_GRAM || kind == NS_POLY;
    NsTile r;
    r.d = square ? ns_find(g, t, [](const NsMat &m) { return m.first_a; }) : ns_find(g, t, [](const NsMat &m) { return m.first_x; });
    const NsMat &mat = g.mat[r.d];
    const int per = square ? mat.tiles_a : mat.tiles_x, local = t - (square ? mat.first_a : mat.first_x);
    const int T = (mat.mp + 127) / 128;
    r.rep = local / per;
    const int tt = local - r.rep * per;
    r.ti = tt % T;
    r.tj = tt / T;
    r.slot_x = mat.row_x + r.rep * mat.mp;
    r.slot_a = mat.row_a + r.rep * mat.mp;
    r.mp = mat.mp; r.np = mat.np; r.m = mat.m; r.n = mat.n;
    r.tall = mat.tall;
    r.index = mat.index + r.rep;
    return r;
}

// eight columns of the result (kept out of line: the code that every phase runs has to stay in the instruction cache)
__device__ __noinline__ void ns_result8(const NsChain &p, const NsMat &mat, int rep, int row, int col, const float4 lo, const float4 hi, float scale)
{
    float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    // read once: behind a store the compiler would fetch them again
    const long long base = mat.dst + rep * mat.dst_stride, ld = mat.ld_dst;
    const float *const params = p.params;
    void *const dst = p.dst;
    const bool to_bf16 = p.bf16_dst != 0, tall = mat.tall != 0;
    const float update = mat.update, keep = p.keep;
    const int n = mat.n;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= scale;
    if (tall || col + 8 > n) {
        const long long o = base + (tall ? (long long)col * ld + row : (long long)row * ld + col), step = tall ? ld : 1;
        float old[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) old[i] = params && col + i < n ? params[o + i * step] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (col + i >= n) continue;
            if (params) ((float *)dst)[o + i * step] = fmaf(-update, v[i], keep * old[i]);
            else if (to_bf16) ((bf16 *)dst)[o + i * step] = __float2bfloat16_rn(v[i]);
            else ((float *)dst)[o + i * step] = v[i];
        }
        return;
    }
    const long long o = base + (long long)row * ld + col;
    if (to_bf16) {
        bf16 *q = (bf16 *)dst + o;
        if (((uintptr_t)q & 15) == 0) {
            store_elems<bf16, 8>(q, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = __float2bfloat16_rn(v[i]);
        }
        return;
    }
    float *q = (float *)dst + o;
    const bool wide = (((uintptr_t)q | (uintptr_t)(params ? params + o : nullptr)) & 15) == 0;
    if (params) {
        float old[8];
        if (wide) {
            load_elems<float, 4>(params + o, old);
            load_elems<float, 4>(params + o + 4, old + 4);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) old[i] = params[o + i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(-update, v[i], keep * old[i]);
    }
    if (wide) {
        store_elems<float, 4>(q, v);
        store_elems<float, 4>(q + 4, v + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = v[i];
    }
}

template <int PARTS> constexpr int NSC_STAGE_BYTES = PARTS * (128 + NSC_BN) * TC_BK * 2;
template <int PARTS> constexpr int NSC_STAGES = PARTS == 2 ? 3 : 6;  // 144 KiB beside 64 KiB of sums (this block's and those it receives)

// the first two phases
LP_DEVINL void ns_chain_norm(const NsSource &src, const NsGroup &g, const NsAdam &adam, const NsChain &p, int tid, double *sw)
{
    for (int t = blockIdx.x; t < p.norm_blocks + p.adam_blocks; t += gridDim.x) {
        if (t < p.norm_blocks) ns_norm_block<NSC_WORKERS>(src, g, t, tid, p.partial, sw);
        else ns_adam_block<NSC_WORKERS>(adam, t - p.norm_blocks, tid);
    }
}
template <int PARTS> LP_DEVINL void ns_chain_convert(const NsSource &src, const NsGroup &g, const NsChain &p, int tid, float *tile, double *sw)
{
    for (int t = blockIdx.x; t < p.conv_blocks; t += gridDim.x) ns_convert_block<PARTS, NSC_WORKERS>(src, g, t, tid, p.partial, p.eps, p.X0, p.inv_r, tile, sw);
}

// After a wait that ran out somewhere in the block, copies into its shared memory and products may still be under way; both are waited
// for (again not longer than the limit) before the block gives up its shared and tensor memory.  Without such a wait they have
// long been used and nothing is waited for here.
// copies: stages that the last S uses of the ring filled; `s`, `round`: where the ring would go on
template <int S> LP_DEVINL void ns_drain_copies(const uint64_t *bar_full, int s, int round, unsigned long long limit_ns)
{
#pragma unroll 1
    for (int i = 0; i < S; ++i) {
        const int use = i < s ? round : round - 1;
        if (use >= 0) mbar_wait(smem_u32(bar_full + i), use & 1, limit_ns);
    }
}
// products: the last commit covers all of them
template <int S> LP_DEVINL void ns_drain_products(const uint64_t *bar_empty, int s, int round, unsigned long long limit_ns)
{
    const int last = s > 0 ? s - 1 : S - 1, use = s > 0 ? round : round - 1;
    if (use >= 0) mbar_wait(smem_u32(bar_empty + last), use & 1, limit_ns);
}

template <int PARTS, int C>
__global__ void __launch_bounds__(NSC_THREADS, 1) ns_chain_kernel(const __grid_constant__ CUtensorMap mapX128, const __grid_constant__ CUtensorMap mapX64,
                                                                  const __grid_constant__ CUtensorMap mapA128, const __grid_constant__ CUtensorMap mapA64,
                                                                  const __grid_constant__ CUtensorMap mapB128, const __grid_constant__ NsSource src,
                                                                  const __grid_constant__ NsGroup g,
                                                                  const __grid_constant__ NsAdam adam, const __grid_constant__ NsChain p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_full[8], bar_empty[8], bar_acc_full[NSC_ACCS], bar_acc_empty[NSC_ACCS], bar_xfull, bar_xfree;
    __shared__ uint32_t tmem_base_s;
    __shared__ double sw[NSC_WORKERS / 32];
    __shared__ NsTile kept_s[2][NSC_KEPT], later_s;
    __shared__ int left_s, announced_s;  // the workers wait for no counter any more; the others' sums of this tile are announced and not yet here
    constexpr int S = NSC_STAGES<PARTS>;
    constexpr uint32_t a_bytes = 128 * TC_BK * 2, b_bytes = NSC_BN * TC_BK * 2, stage_bytes = NSC_STAGE_BYTES<PARTS>;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    float *mine = reinterpret_cast<float *>(smem + (size_t)S * stage_bytes), *theirs = mine + NSC_SUM_BYTES / 4;
    const int rank = C > 1 ? (int)cluster_cta_rank() : 0;
    const int cluster = blockIdx.x / C, n_clusters = gridDim.x / C;
    const unsigned everybody = gridDim.x;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 1);
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        for (int b = 0; b < NSC_ACCS; ++b) {
            mbar_init(smem_u32(&bar_acc_full[b]), 1);
            mbar_init(smem_u32(&bar_acc_empty[b]), NSC_WORKERS / 32);
        }
        mbar_init(smem_u32(&bar_xfull), 1);
        mbar_init(smem_u32(&bar_xfree), C);
        left_s = announced_s = 0;
        fence_barrier_init();
        fence_async_proxy();
        tma_prefetch_desc(&mapX128);
        tma_prefetch_desc(&mapX64);
        tma_prefetch_desc(&mapA128);
        tma_prefetch_desc(&mapA64);
        tma_prefetch_desc(&mapB128);
    }
    if (warp == 0) {
        __syncwarp();
        tmem_alloc(smem_u32(&tmem_base_s), NSC_ACCS * NSC_ACC_COLS<PARTS>);
    }
    // every step visits the same tiles: the first ones of A, B and of X are looked up once
    if (threadIdx.x >= 64 && threadIdx.x < 64 + 2 * NSC_KEPT) {
        const int i = (threadIdx.x - 64) % NSC_KEPT, of_x = (threadIdx.x - 64) / NSC_KEPT, t = cluster + i * n_clusters;
        if (t < (of_x ? p.tiles_x : p.tiles_a)) kept_s[of_x][i] = ns_tile(g, of_x ? NS_APPLY : NS_GRAM, t);
    }
    tc_fence_before();
    __syncthreads();
    if (C > 1) cluster_barrier();
    tc_fence_after();
    const uint32_t tmem = tmem_base_s;

    if (warp == 0) {
        if (elect_one()) {
            // ---- operands
            int s = 0, round = 0;  // stage, and how often the ring has gone round
            bool ok = true, first = true;
            for (int k = 0; k < p.steps && ok; ++k) {
                const int x0 = (k & 1) * PARTS * p.parts_rows_x;
                for (int kind = NS_GRAM; kind <= NS_APPLY && ok; ++kind) {
                    const int phase = 2 + 3 * k + kind;
                    if (!counter_wait(p.counters + phase - 1, everybody, p.wait_ns)) { atomicExch(p.err, 6); ok = false; break; }
                    fence_async_proxy_global();
                    const int tiles = kind == NS_APPLY ? p.tiles_x : p.tiles_a;
                    const CUtensorMap *map_a = kind == NS_GRAM ? &mapX128 : kind == NS_POLY ? &mapA128 : &mapB128;
                    const CUtensorMap *map_b = kind == NS_POLY ? &mapA64 : &mapX64;
                    const int lo_a = kind == NS_GRAM ? p.parts_rows_x : p.parts_rows_a, lo_b = kind == NS_POLY ? p.parts_rows_a : p.parts_rows_x;
                    int i = 0;
                    for (int t = cluster; t < tiles && ok; t += n_clusters, ++i) {
                        const NsTile tl = i < NSC_KEPT ? kept_s[kind == NS_APPLY][i] : ns_tile(g, kind, t);
                        const int kbs = tl.num_kb(kind), kb0 = kbs * rank / C, kb1 = kbs * (rank + 1) / C;
                        const int row_a = (kind == NS_GRAM ? x0 + tl.slot_x : tl.slot_a) + tl.ti * 128;
                        // X as the second operand of the new X is read across: 64 rows of K, 64 columns
                        const int row_b = kind == NS_GRAM ? x0 + tl.slot_x + tl.tj * NSC_BN : kind == NS_POLY ? tl.slot_a + tl.tj * NSC_BN : x0 + tl.slot_x;
                        for (int kb = kb0; kb < kb1; ++kb) {
                            if (round > 0 && !mbar_wait(smem_u32(&bar_empty[s]), (round & 1) ^ 1, p.wait_ns)) { atomicExch(p.err, 1); ok = false; break; }
                            const uint32_t sa = smem_u32(smem) + s * stage_bytes, sb = sa + PARTS * a_bytes, bar = smem_u32(&bar_full[s]);
                            mbar_expect_tx(bar, stage_bytes + (first && blockIdx.x == 0 ? (uint32_t)p.extra_tx : 0u));
                            first = false;
                            const int kk = kb * TC_BK;
                            const int xb = kind == NS_APPLY ? tl.tj * NSC_BN : kk, yb = kind == NS_APPLY ? row_b + kk : row_b;
#pragma unroll
                            for (int q = 0; q < PARTS; ++q) {
                                tma_load_2d(sa + q * a_bytes, map_a, bar, kk, row_a + q * lo_a);
                                tma_load_2d(sb + q * b_bytes, map_b, bar, xb, yb + q * lo_b);
                            }
                            if (++s == S) { s = 0; ++round; }
                        }
                    }
                }
            }
            // the last operands are requested; the other thread of this block that waits for the counters is done with them, too, once it
            // has seen the last one or given up, each of its waits being limited
            const unsigned long long t0 = global_timer_ns();
            bool others = *(volatile int *)&left_s != 0;
            while (!others && global_timer_ns() - t0 <= 16 * p.wait_ns) others = *(volatile int *)&left_s != 0;
            __threadfence_block();
            if (others) ns_leave(p.counters, 1 + 3 * p.steps, NSC_BARRIERS - 1);
            ns_drain_copies<S>(bar_full, s, round, p.wait_ns);
        }
    } else if (warp == 1) {
        if (elect_one()) {
            // ---- products
            int s = 0, round = 0, use = 0;  // stage, rounds of the ring, accumulators handed over
            bool ok = true;
            const uint64_t desc_a = make_smem_desc(smem_u32(smem), 16, 1024), desc_bk = make_smem_desc(smem_u32(smem) + PARTS * a_bytes, 16, 1024),
                           desc_bm = make_smem_desc(smem_u32(smem) + PARTS * a_bytes, 8192, 1024);
            for (int k = 0; k < p.steps && ok; ++k) {
                for (int kind = NS_GRAM; kind <= NS_APPLY && ok; ++kind) {
                    const uint32_t idesc = make_idesc_f16(128, NSC_BN, kind == NS_APPLY);
                    const uint64_t desc_b = kind == NS_APPLY ? desc_bm : desc_bk;
                    const uint64_t step_b = kind == NS_APPLY ? 2048 >> 4 : 32 >> 4;  // 16 terms further
                    const int tiles = kind == NS_APPLY ? p.tiles_x : p.tiles_a;
                    int i = 0;
                    for (int t = cluster; t < tiles && ok; t += n_clusters, ++i) {
                        const NsTile tl = i < NSC_KEPT ? kept_s[kind == NS_APPLY][i] : ns_tile(g, kind, t);
                        const int kbs = tl.num_kb(kind), kb0 = kbs * rank / C, kb1 = kbs * (rank + 1) / C;
                        for (int kb = kb0; kb < kb1; ++kb) {
                            const int b = use % NSC_ACCS;
                            if ((PARTS == 2 || kb == kb0) && use >= NSC_ACCS && !mbar_wait(smem_u32(&bar_acc_empty[b]), ((use / NSC_ACCS) & 1) ^ 1, p.wait_ns)) {
                                atomicExch(p.err, 5);
                                ok = false;
                                break;
                            }
                            if (!mbar_wait(smem_u32(&bar_full[s]), round & 1, p.wait_ns)) { atomicExch(p.err, 2); ok = false; break; }
                            tc_fence_after();
                            const uint64_t da = desc_a + ((s * stage_bytes) >> 4), db = desc_b + ((s * stage_bytes) >> 4);
                            const uint32_t acc = tmem + b * NSC_ACC_COLS<PARTS>;
                            if (PARTS == 2) {
#pragma unroll
                                for (int i = 0; i < TC_BK / TC_UMMA_K; ++i) {  // the small terms first, while the sums are small
                                    const uint32_t half = acc + (i >> 1) * NSC_BN;
                                    umma_bf16(half, da + i * 2, db + (b_bytes >> 4) + i * step_b, idesc, i & 1);
                                    umma_bf16(half, da + (a_bytes >> 4) + i * 2, db + i * step_b, idesc, 1u);
                                }
#pragma unroll
                                for (int i = 0; i < TC_BK / TC_UMMA_K; ++i) umma_bf16(acc + (i >> 1) * NSC_BN, da + i * 2, db + i * step_b, idesc, 1u);
                            } else {
#pragma unroll
                                for (int i = 0; i < TC_BK / TC_UMMA_K; ++i) umma_bf16(acc, da + i * 2, db + i * step_b, idesc, kb != kb0 || i != 0 ? 1u : 0u);
                            }
                            umma_commit(smem_u32(&bar_empty[s]));
                            if (PARTS == 2 || kb + 1 == kb1) {
                                umma_commit(smem_u32(&bar_acc_full[b]));
                                ++use;
                            }
                            if (++s == S) { s = 0; ++round; }
                        }
                    }
                }
            }
            ns_drain_products<S>(bar_empty, s, round, p.wait_ns);
        }
    } else {
        // ---- norm and conversion, then sums and results
        const int tid = threadIdx.x - 64;
        bool ok = true;
        // ends phase i: everything this block wrote is visible to whoever sees the counter; begins phase i + 1
        auto arrive = [&](int i) {
            ns_sync<NSC_WORKERS>();
            if (tid == 0) red_release_gpu(p.counters + i);
        };
        auto await = [&](int i) {
            bool failed = false;
            if (tid == 0 && !counter_wait(p.counters + i, everybody, p.wait_ns)) { atomicExch(p.err, 6); failed = true; }
            return !ns_any<NSC_WORKERS>(failed);
        };
        ns_chain_norm(src, g, adam, p, tid, sw);
        arrive(0);
        ok = await(0);
        if (ok) {
            ns_chain_convert<PARTS>(src, g, p, tid, mine, sw);
            arrive(1);
        }
        const int q = warp & 3, quarter = (warp - 2) >> 2;  // the 32 rows that the warp may read from tensor memory, and its 16 columns
        int use = 0, tiles_done = 0;
        for (int k = 0; k < p.steps && ok; ++k) {
            for (int kind_ = NS_GRAM; kind_ <= NS_APPLY && ok; ++kind_) {
                const int phase = 2 + 3 * k + kind_;
                const int kind = kind_ == NS_APPLY && k + 1 == p.steps ? NS_LAST : kind_;
                const bool square = kind == NS_GRAM || kind == NS_POLY;
                ok = await(phase - 1);
                if (kind == NS_LAST && tid == 0) *(volatile int *)&left_s = 1;
                const int tiles = kind_ == NS_APPLY ? p.tiles_x : p.tiles_a;
                const NsChainIo &io = p.io[k & 1][kind_];
                int nth = 0;
                for (int t = cluster; t < tiles && ok; t += n_clusters, ++nth) {
                    if (nth >= NSC_KEPT) {
                        if (tid == 0) later_s = ns_tile(g, kind_, t);
                        ns_sync<NSC_WORKERS>();
                    }
                    const NsTile &tl = nth < NSC_KEPT ? kept_s[kind_ == NS_APPLY][nth] : later_s;  // read where it is needed, not held
                    const int kbs = tl.num_kb(kind_), kb0 = kbs * rank / C, kb1 = kbs * (rank + 1) / C;
                    const int width = square ? tl.mp : tl.np, slot = square ? tl.slot_a : tl.slot_x;
                    const float inv_r = kind == NS_POLY || kind == NS_LAST ? __ldcg(p.inv_r + tl.index) : 1.f;
                    // this block finishes 64 / C columns of the tile; a thread takes GPT groups of eight, neighbours along the rows
                    constexpr int GPR = 8 / C, GPT = C == 1 ? 2 : 1;  // groups per row, per thread (C = 4: half of the threads have none)
                    float add[GPT][8];
                    auto fetch = [&]() {
#pragma unroll
                        for (int i = 0; i < GPT; ++i) {
                            const int e = i * NSC_WORKERS + tid, row = tl.ti * 128 + e / GPR, col = tl.tj * NSC_BN + rank * (NSC_BN / C) + 8 * (e % GPR);
#pragma unroll
                            for (int j = 0; j < 8; ++j) add[i][j] = 0.f;
                            if (e < 128 * GPR && row < tl.mp && col < width) {
                                const size_t at = (size_t)(slot + row) * io.pitch + col;
                                if (kind == NS_POLY) {
                                    ns_add8(__ldcg(reinterpret_cast<const uint4 *>(io.add_h + at)), add[i]);
                                    if (PARTS == 2) ns_add8(__ldcg(reinterpret_cast<const uint4 *>(io.add_h + io.out_lo + at)), add[i]);
                                } else if (!square) {
                                    const float4 x = __ldcg(reinterpret_cast<const float4 *>(io.add_f + at)), y = __ldcg(reinterpret_cast<const float4 *>(io.add_f + at) + 1);
                                    add[i][0] = x.x; add[i][1] = x.y; add[i][2] = x.z; add[i][3] = x.w;
                                    add[i][4] = y.x; add[i][5] = y.y; add[i][6] = y.z; add[i][7] = y.w;
                                }
                            }
                        }
                    };
                    // requested before the products are waited for, unless that makes registers spill: a spilled value costs more
                    // than the wait, because every phase empties L1
                    constexpr bool EARLY = PARTS == 1 || C == 4;
                    if (EARLY) fetch();
                    float v[16], lost[16];  // running sums and what their roundings lost
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = lost[i] = 0.f;
                    const int chunks = kb1 <= kb0 ? 0 : PARTS == 2 ? kb1 - kb0 : 1;
                    bool failed = false;
                    for (int c = 0; c < chunks; ++c, ++use) {
                        const int b = use % NSC_ACCS;
                        failed = !__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_acc_full[b]), (use / NSC_ACCS) & 1, p.wait_ns));
                        if (failed) {
                            if (lane == 0) atomicExch(p.err, 3);
                            break;
                        }
                        tc_fence_after();
                        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16) + b * NSC_ACC_COLS<PARTS> + quarter * 16;
                        if (tl.ti * 128 + q * 32 >= tl.mp) {  // rows behind the matrix
                        } else if (PARTS == 1) {  // one chunk
                            tmem_ld_32x16(taddr, v);
                        } else {
#pragma unroll
                            for (int o = 0; o < 16; o += 8) {  // eight columns at a time: spills are dear, every barrier empties L1 (C = 1, 2: one register)
                                float r[8], r2[8];
                                tmem_ld_32x8_pair(taddr + o, taddr + NSC_BN + o, r, r2);
                                if (c == 0) {
#pragma unroll
                                    for (int i = 0; i < 8; ++i) v[o + i] = r[i] + r2[i];
                                } else {
#pragma unroll
                                    for (int i = 0; i < 8; ++i) ns_two_sum(v[o + i], lost[o + i], r[i] + r2[i]);
                                }
                            }
                        }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&bar_acc_empty[b]));
                    }
                    if (PARTS == 2 && C > 1) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] += lost[i];
                    }
                    const float r2 = inv_r * inv_r;
                    const float f = kind == NS_GRAM ? NS_A_SCALE / (NS_X_SCALE * NS_X_SCALE) : kind == NS_POLY ? p.poly.c * r2 * r2 : p.poly.unscale;
                    const float h = kind == NS_POLY ? p.poly.b * r2 : p.poly.a;
                    // the sums go to shared memory, [block that finishes][row][64 / C] with the 16-byte pieces of a row permuted by the
                    // row; every other block of the cluster gets its share by one bulk copy
                    constexpr int SHARE = 128 * NSC_BN / C, PIECES = 16 / C;
                    if (C > 1 && tiles_done > 0 && !mbar_wait_cluster(smem_u32(&bar_xfree), (tiles_done - 1) & 1, p.wait_ns)) { atomicExch(p.err, 7); failed = true; }
                    const int row_t = q * 32 + lane;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int piece = quarter * 4 + i, to = piece / PIECES, within = piece % PIECES;
                        *reinterpret_cast<float4 *>(mine + to * SHARE + row_t * (NSC_BN / C) + ((within ^ (row_t & (PIECES - 1))) << 2)) =
                            make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                        if (PARTS == 2 && C == 1 && chunks > 1)  // what the sums lost goes along in the second area
                            *reinterpret_cast<float4 *>(theirs + row_t * NSC_BN + ((within ^ (row_t & (PIECES - 1))) << 2)) =
                                make_float4(lost[4 * i], lost[4 * i + 1], lost[4 * i + 2], lost[4 * i + 3]);
                    }
                    if (!EARLY) fetch();
                    if (C > 1) fence_async_proxy();
                    ok = !ns_any<NSC_WORKERS>(failed);  // all sixteen warps go on or all leave
                    if (!ok) break;
                    if (C > 1) {
                        if (tid == 0) {
                            mbar_expect_tx(smem_u32(&bar_xfull), (C - 1) * SHARE * 4);
                            announced_s = 1;
                            for (int o = 1; o < C; ++o) {
                                const int to = (rank + o) % C;
                                copy_to_cta(map_to_cta(smem_u32(theirs + rank * SHARE), to), smem_u32(mine + to * SHARE), SHARE * 4, map_to_cta(smem_u32(&bar_xfull), to));
                            }
                        }
                        if (!mbar_wait_cluster(smem_u32(&bar_xfull), tiles_done & 1, p.wait_ns)) { atomicExch(p.err, 7); failed = true; }
                    }
#pragma unroll
                    for (int i = 0; i < GPT; ++i) {
                        const int e = i * NSC_WORKERS + tid;
                        if (e >= 128 * GPR) break;
                        const int r_t = e / GPR, piece = 2 * (e % GPR), row = tl.ti * 128 + r_t, col = tl.tj * NSC_BN + rank * (NSC_BN / C) + 4 * piece;
                        float sum[8], off[8];
#pragma unroll
                        for (int other = 0; other < (C == 1 ? PARTS : C); ++other) {
                            if (C == 1 && other == 1 && chunks <= 1) break;
                            const float *row_p = (other == rank ? mine : theirs) + (C == 1 ? 0 : other * SHARE) + r_t * (NSC_BN / C);
                            const float4 x = *reinterpret_cast<const float4 *>(row_p + ((piece ^ (r_t & (PIECES - 1))) << 2));
                            const float4 y = *reinterpret_cast<const float4 *>(row_p + (((piece + 1) ^ (r_t & (PIECES - 1))) << 2));
                            const float z[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                if (other == 0) { sum[j] = z[j]; off[j] = 0.f; }
                                else if (C == 1) off[j] = z[j];
                                else ns_two_sum(sum[j], off[j], z[j]);
                            }
                        }
                        if (row >= tl.mp || col >= width) continue;
                        const size_t at = (size_t)(slot + row) * io.pitch + col;
#pragma unroll
                        for (int j = 0; j < 8; ++j) sum[j] = fmaf(f, off[j], fmaf(h, add[i][j], f * sum[j]));  // f is a power of two where precision counts
                        if (kind != NS_LAST) {
                            ns_store8<PARTS>(sum, io.out_h + at, io.out_lo);
                            if (!square) {
                                store_elems<float, 4>(io.out_f + at, sum);
                                store_elems<float, 4>(io.out_f + at + 4, sum + 4);
                            }
                        } else if (row < tl.m && col < tl.n) {
                            ns_result8(p, g.mat[tl.d], tl.rep, row, col, make_float4(sum[0], sum[1], sum[2], sum[3]), make_float4(sum[4], sum[5], sum[6], sum[7]),
                                       inv_r / NS_X_SCALE);
                        }
                    }
                    ok = !ns_any<NSC_WORKERS>(failed);  // and the sums may be overwritten
                    if (!ok) break;
                    if (C > 1 && tid < C) mbar_arrive_cluster(map_to_cta(smem_u32(&bar_xfree), tid));
                    if (C > 1 && tid == 0) announced_s = 0;
                    ++tiles_done;
                }
                if (ok && kind != NS_LAST) arrive(phase);
            }
        }
        if (tid == 0) *(volatile int *)&left_s = 1;  // gave up before the last phase
        // this block gave up: sums that others of its cluster may have sent it meanwhile land before its shared memory goes
        if (C > 1 && !ok && tid == 0) {
            if (!announced_s) mbar_expect_tx(smem_u32(&bar_xfull), (C - 1) * (128 * NSC_BN / C) * 4);
            mbar_wait_cluster(smem_u32(&bar_xfull), tiles_done & 1, p.wait_ns);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (C > 1) cluster_barrier();  // nobody leaves while its sums may still be read
    if (warp == 0) {
        __syncwarp();
        tmem_dealloc(tmem, NSC_ACCS * NSC_ACC_COLS<PARTS>);
    }
}

// ---------------------------------------------------------------------------------------------
// The whole iteration of a matrix of up to 128 x 128 in one block, for calls whose matrices are all of that size.
//
// Such a matrix needs 17 dependent steps of next to no work, so the time is the way from one product to the next.  Through
// global memory and a counter (the chain kernel) that is 3.8 us; here X and A (then B, in its place) stay in shared memory as
// operands of the matrix instructions, X also in FP32, and a product follows the one before it after one barrier of the block.  The same copy of X serves both products: its rows are the K-major
// operands of X X^T, and read across, the MN-major second operand of B X.
//   every warp sums and results: 32 rows x every fourth group of eight columns; warp 3 also the matrix instructions
// PARTS = 2: every 32 terms have an accumulator of their own (four of 128 columns fill tensor memory).  Their four sums are added
// in pairs; carrying the roundings along, as the chain kernel does for longer sums, took 54 us for 128 x 128 and changes the
// error of a matrix of full rank from 6.4e-7 to 6.2e-7, of rank one from 2.3e-5 to 1.7e-5 (FP32 matrix products: 9.7e-5).
// Blocks from `matrices` on take Adam steps.
// Microseconds for five steps, FP32 (BF16), against the chain kernel: 64 x 64 24 (17) against 64 (47); 128 x 128 45 (27) against
// 95 (60); 200 of 128 x 128 90 (52) against 243 (155); 1,000 of 64 x 64 157 (110) against 312 (228).  A 64 x 64 product takes 2,300
// cycles: 930 for its twelve matrix instructions (50 each, the time in which shared memory delivers their operands) and their
// completion, 1,250 to 1,600 for the sums, the next operands' rounding and their stores, the rest barriers.  Of 128 x 128 the sums
// take most, and they are bound by instructions.
// ---------------------------------------------------------------------------------------------
constexpr int NSB_SIZE = 128;                // largest side
constexpr int NSB_THREADS = 512;
constexpr int NSB_COLS = NSB_SIZE * 64;      // elements of 64 columns of an operand
constexpr int NSB_PART = 2 * NSB_COLS;       // elements of a part of an operand
template <int PARTS> constexpr int NSB_SMEM = 2 * PARTS * NSB_PART * 2 + NSB_SIZE * NSB_SIZE * 4 + 1024;

struct NsBlock {
    int steps, matrices;
    NsPoly poly;
    double eps;
    void *dst;
    int bf16_dst;
    const float *params;
    float keep;
    int *err;
    unsigned long long wait_ns;
    int extra_tx;
};

template <int PARTS>
__global__ void __launch_bounds__(NSB_THREADS, 1) ns_block_kernel(const __grid_constant__ NsSource src, const __grid_constant__ NsGroup g, const __grid_constant__ NsAdam adam,
                                                                  const __grid_constant__ NsBlock p)
{
    LP_DEP_ENTER();
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_acc;
    __shared__ uint32_t tmem_base_s;
    __shared__ double sw[NSB_THREADS / 32];
    if ((int)blockIdx.x >= p.matrices) {
        ns_adam_block<NSB_THREADS>(adam, blockIdx.x - p.matrices, threadIdx.x);
        return;
    }
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const NsMat &mat = g.mat[ns_find(g, blockIdx.x, [](const NsMat &m) { return m.index; })];
    const int rep = blockIdx.x - mat.index, mp = mat.mp, np = mat.np, m = mat.m, n = mat.n;
    const bool tall = mat.tall != 0;
    __half *Xs = reinterpret_cast<__half *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023), *As = Xs + PARTS * NSB_PART;
    float4 *Xf = reinterpret_cast<float4 *>(As + PARTS * NSB_PART);  // [four columns][row]
    constexpr int TERMS = PARTS == 2 ? 32 : NSB_SIZE;                // terms of an accumulator
    const uint32_t tmem_cols = (uint32_t)max((np + TERMS - 1) / TERMS * mp, (mp + TERMS - 1) / TERMS * np);  // a power of two, np >= mp
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&bar_acc), p.extra_tx != 0 && blockIdx.x == 0 ? 2 : 1);
        fence_barrier_init();
    }
    if (warp == 0) {
        __syncwarp();
        tmem_alloc(smem_u32(&tmem_base_s), tmem_cols);
    }
    const int q = warp & 3, quarter = warp >> 2, row = q * 32 + lane;  // the rows that the warp may read from tensor memory
    const bool rows_here = q * 32 < mp;
    auto place = [&](__half *base, int group) {  // eight columns of this thread's row in an operand (128-byte swizzle)
        return base + (group >> 3) * NSB_COLS + row * 64 + (((group & 7) ^ (row & 7)) << 3);
    };
    float r;
    {
        constexpr int GROUPS = NSB_SIZE / 32;
        float x[GROUPS][8];
        const long long base = mat.src + rep * mat.src_stride, ld = mat.ld_src;
        const bool wide = !src.grads && !tall && (ld & 3) == 0 && (base & 3) == 0 && ((uintptr_t)src.u & 15) == 0;
        double acc = 0.0;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) {
            const int col = 8 * (quarter + 4 * i);
            if (wide && row < m && col + 8 <= n) {
                const long long at = base + row * ld + col;
                if (src.bf16_u) {
                    load_elems<bf16, 4>((const bf16 *)src.u + at, x[i]);
                    load_elems<bf16, 4>((const bf16 *)src.u + at + 4, x[i] + 4);
                } else {
                    load_elems<float, 4>((const float *)src.u + at, x[i]);
                    load_elems<float, 4>((const float *)src.u + at + 4, x[i] + 4);
                }
            } else if (!src.grads) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const long long at = base + (tall ? (col + j) * ld + row : row * ld + col + j);
                    const bool in = row < m && col + j < n;
                    x[i][j] = !in ? 0.f : src.bf16_u ? __bfloat162float(((const bf16 *)src.u)[at]) : ((const float *)src.u)[at];
                }
            } else {
                float gr[8], av[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const long long at = base + (tall ? (col + j) * ld + row : row * ld + col + j);
                    const bool in = row < m && col + j < n;
                    gr[j] = in ? src.grad_scale * src.grads[at] : 0.f;
                    x[i][j] = in ? src.momentum[at] : 0.f;
                    if (src.new_adam_v) av[j] = in ? src.adam_v[at] : 0.f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const long long at = base + (tall ? (col + j) * ld + row : row * ld + col + j);
                    const float mo = fmaf(src.mu, x[i][j], gr[j]);
                    if (row < m && col + j < n) {
                        src.new_momentum[at] = mo;
                        if (src.new_adam_v) src.new_adam_v[at] = av[j];
                    }
                    x[i][j] = src.nesterov ? fmaf(src.mu, mo, gr[j]) : mo;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < GROUPS; ++i)
#pragma unroll
            for (int j = 0; j < 8 && 32 * i < np; ++j) acc = fma((double)x[i][j], (double)x[i][j], acc);  // in double: no overflow for any FP32 input
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
        if (lane == 0) sw[warp] = acc;
        __syncthreads();
        acc = 0.0;
        for (int w = 0; w < NSB_THREADS / 32; ++w) acc += sw[w];
        double pow2;
        ns_start_scale(sqrt(acc) + p.eps, r, pow2);
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) {
            const int group = quarter + 4 * i;
            if (!rows_here || 32 * i >= np) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = (float)(x[i][j] * pow2);
            ns_store8<PARTS>(x[i], place(Xs, group), NSB_PART);
            Xf[2 * group * NSB_SIZE + row] = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
            Xf[(2 * group + 1) * NSB_SIZE + row] = make_float4(x[i][4], x[i][5], x[i][6], x[i][7]);
        }
    }
    const float inv_r = 1.f / r, r2 = inv_r * inv_r;
    const float bf = p.poly.b * r2, cf = p.poly.c * r2 * r2, af = p.poly.a;
    fence_async_proxy();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_s, lanes = (uint32_t)(q * 32) << 16;

    // one product: of the columns of this warp, the sums and what becomes of them
    auto finish = [&](auto kind_) {
        constexpr int kind = decltype(kind_)::value;
        constexpr bool square = kind == NS_GRAM || kind == NS_POLY;
        const int width = square ? mp : np, chunks = ((kind == NS_GRAM ? np : mp) + TERMS - 1) / TERMS;
        // the last product: where it goes (held in registers: a store may not change it)
        void *const dst = p.dst;
        const float *const params = p.params;
        const bool to_bf16 = p.bf16_dst != 0;
        const long long base = mat.dst + rep * mat.dst_stride, step = tall ? mat.ld_dst : 1;
        const float update = mat.update, keep = p.keep, unscale = inv_r / NS_X_SCALE;
#pragma unroll 1
        for (int group = quarter; 8 * group < width; group += 4) {
            const uint32_t taddr = tmem + lanes + 8 * group;
            float v[8], add[8];
            if (PARTS == 2) {
                float t[8], u[8];
                tmem_ld_32x8_pair(taddr, taddr + width, v, t);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += t[j];
                if (chunks > 2) {
                    tmem_ld_32x8_pair(taddr + 2 * width, taddr + 3 * width, t, u);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += t[j] + u[j];
                }
            } else {
                tmem_ld_32x8(taddr, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) add[j] = 0.f;
            if (kind == NS_POLY) {
                ns_add8(*reinterpret_cast<const uint4 *>(place(As, group)), add);
                if (PARTS == 2) ns_add8(*reinterpret_cast<const uint4 *>(place(As, group) + NSB_PART), add);
            } else if (!square) {
                const float4 x0 = Xf[2 * group * NSB_SIZE + row], x1 = Xf[(2 * group + 1) * NSB_SIZE + row];
                add[0] = x0.x; add[1] = x0.y; add[2] = x0.z; add[3] = x0.w;
                add[4] = x1.x; add[5] = x1.y; add[6] = x1.z; add[7] = x1.w;
            }
            const float f = kind == NS_GRAM ? NS_A_SCALE / (NS_X_SCALE * NS_X_SCALE) : kind == NS_POLY ? cf : p.poly.unscale;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] *= f;  // a power of two where precision counts
                if (kind != NS_GRAM) v[j] = fmaf(kind == NS_POLY ? bf : af, add[j], v[j]);
            }
            if (kind == NS_LAST) {
                const long long o = base + (tall ? (long long)8 * group * step + row : (long long)row * mat.ld_dst + 8 * group);
                const int live = row < m ? n - 8 * group : 0;  // columns inside the matrix
                float old[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) old[j] = params && j < live ? params[o + j * step] : 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] *= unscale;
                    if (params) v[j] = fmaf(-update, v[j], keep * old[j]);
                }
                if (!tall && live >= 8 && !to_bf16 && ((uintptr_t)((float *)dst + o) & 15) == 0) {
                    store_elems<float, 4>((float *)dst + o, v);
                    store_elems<float, 4>((float *)dst + o + 4, v + 4);
                } else if (!tall && live >= 8 && to_bf16 && ((uintptr_t)((bf16 *)dst + o) & 15) == 0) {
                    store_elems<bf16, 8>((bf16 *)dst + o, v);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (j >= live) continue;
                        if (to_bf16) ((bf16 *)dst)[o + j * step] = __float2bfloat16_rn(v[j]);
                        else ((float *)dst)[o + j * step] = v[j];
                    }
                }
            } else {
                ns_store8<PARTS>(v, place(square ? As : Xs, group), NSB_PART);
                if (!square) {
                    Xf[2 * group * NSB_SIZE + row] = make_float4(v[0], v[1], v[2], v[3]);
                    Xf[(2 * group + 1) * NSB_SIZE + row] = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
        }
    };
    int product = 0;
    for (int k = 0; k < p.steps; ++k) {
        bool failed = false;
        for (int kind = NS_GRAM; kind <= NS_APPLY; ++kind, ++product) {
            if (warp == 3) {  // without rows of its own where the matrix has 64
                if (elect_one()) {
                    const int terms = kind == NS_GRAM ? np : mp, width = kind == NS_APPLY ? np : mp;
                    const uint32_t idesc = make_idesc_f16(NSB_SIZE, width, kind == NS_APPLY);
                    const uint64_t da = make_smem_desc(smem_u32(kind == NS_GRAM ? Xs : As), 16, 1024);
                    const uint64_t db = kind == NS_APPLY ? make_smem_desc(smem_u32(Xs), NSB_COLS * 2, 1024) : da;
                    constexpr uint64_t lo = (NSB_PART * 2) >> 4;
                    for (int s = 0; s < terms / TC_UMMA_K; s += 2) {  // 32 terms
                        const uint64_t a0 = da + (s >> 2) * ((NSB_COLS * 2) >> 4) + (s & 3) * 2, a1 = a0 + 2;
                        const uint64_t step = kind == NS_APPLY ? 2048 >> 4 : 2;
                        const uint64_t b0 = kind == NS_APPLY ? db + s * step : a0, b1 = b0 + step;
                        const uint32_t acc = tmem + (PARTS == 2 ? (s >> 1) * width : 0);
                        if (PARTS == 2) {  // the small terms first, while the sums are small
                            umma_bf16(acc, a0, b0 + lo, idesc, 0u);
                            umma_bf16(acc, a0 + lo, b0, idesc, 1u);
                            umma_bf16(acc, a1, b1 + lo, idesc, 1u);
                            umma_bf16(acc, a1 + lo, b1, idesc, 1u);
                        }
                        umma_bf16(acc, a0, b0, idesc, PARTS == 2 || s != 0 ? 1u : 0u);
                        umma_bf16(acc, a1, b1, idesc, 1u);
                    }
                    umma_commit(smem_u32(&bar_acc));
                }
                __syncwarp();
            }
            if (rows_here) {
                failed = !__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_acc), product & 1, p.wait_ns));
                tc_fence_after();
                if (failed) {
                    if (lane == 0) atomicExch(p.err, 3);
                } else if (kind == NS_GRAM) {
                    finish(std::integral_constant<int, NS_GRAM>());
                } else if (kind == NS_POLY) {
                    finish(std::integral_constant<int, NS_POLY>());
                } else if (k + 1 < p.steps) {
                    finish(std::integral_constant<int, NS_APPLY>());
                } else {
                    finish(std::integral_constant<int, NS_LAST>());
                }
            }
            fence_async_proxy();
            tc_fence_before();
            failed = __syncthreads_or(failed) != 0;  // all go on or all leave
            tc_fence_after();
            if (failed) break;
        }
        if (failed) break;
    }
    if (warp == 0) {
        __syncwarp();
        tmem_dealloc(tmem, tmem_cols);
    }
}

// ---------------------------------------------------------------------------------------------
// products of large matrices: one launch per product, persistent pairs of SMs (clusters of two CTAs, cta_group::2)
//
// A pair multiplies tiles of 256 x 256 (PARTS = 2: 256 x 128): each CTA brings in 128 rows of the first operand and half of the
// second, so a 64-term block costs 32 KiB per CTA for 512 cycles of products (48 KiB for 768).  PARTS = 1: two accumulators of
// 256 columns fill tensor memory, and a tile's is drained while the next tile's products run.  PARTS = 2: the accumulators
// (four of 128 columns) change hands after every 64-term block and sixteen warps add the blocks up in registers (32
// columns per thread, which spills 16 registers; 64, for tiles of 256 x 256, spilled far more).
// A and B are symmetric: only tiles on and above the diagonal are computed, the others are written turned.
//   warp 0 operands, warp 1 matrix instructions (of the pair's first CTA), warps 2-17 results: 32 rows x 64 (32) columns each, turned
//   through 2 KiB of shared memory per warp, 16 columns at a time, so that rows are written in pieces of 64 bytes
// ---------------------------------------------------------------------------------------------
constexpr int NSP_THREADS = 576;
template <int PARTS> constexpr int NSP_BN = PARTS == 2 ? 128 : 256;
template <int PARTS> constexpr int NSP_STAGES = PARTS == 2 ? 4 : 6;  // 192 KiB in flight (4096 x 4096 with 96, 128, 160 KiB: 1.48, 1.37, 1.32 ms)
template <int PARTS> constexpr int NSP_ACCS = PARTS == 2 ? 4 : 2;  // accumulators used in turn: all 512 columns of tensor memory
template <int PARTS> constexpr int NSP_STAGE_BYTES = PARTS * (128 + NSP_BN<PARTS> / 2) * TC_BK * 2;
constexpr int NSP_TURN_BYTES = 16 * 2048;
template <int PARTS> constexpr int NSP_SMEM = NSP_STAGES<PARTS> * NSP_STAGE_BYTES<PARTS> + NSP_TURN_BYTES + 1024;

// tile t of the upper triangle (rows i <= columns j) of a T x T grid, row by row
LP_DEVINL void ns_triangle(int t, int T, int &i, int &j)
{
    i = 0;
    while (t >= T - i) { t -= T - i; ++i; }
    j = i + t;
}

// one element of the result
LP_DEVINL void ns_result(const NsPhase &p, const NsMat &mat, long long o, float v)
{
    if (p.params) ((float *)p.dst)[o] = fmaf(-mat.update, v, p.keep * p.params[o]);
    else if (p.bf16_dst) ((bf16 *)p.dst)[o] = __float2bfloat16_rn(v);
    else ((float *)p.dst)[o] = v;
}

template <int PARTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NSP_THREADS, 1)
    ns_pair_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ NsPhase p, const __grid_constant__ NsGroup g, int tiles)
{
    LP_DEP_ENTER();
    extern __shared__ uint8_t smem_raw[];
    constexpr int S = NSP_STAGES<PARTS>, ACCS = NSP_ACCS<PARTS>;
    __shared__ __align__(8) uint64_t bar_full[S], bar_empty[S], bar_acc_full[ACCS], bar_acc_empty[ACCS];
    __shared__ uint32_t tmem_base_s;
    constexpr int BN = NSP_BN<PARTS>, COLS = BN / 4;  // COLS: columns of a warp
    constexpr uint32_t a_bytes = 128 * TC_BK * 2, b_bytes = BN / 2 * TC_BK * 2, stage_bytes = NSP_STAGE_BYTES<PARTS>;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = (int)cluster_cta_rank();
    const bool leader = rank == 0;
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const bool square = p.kind == NS_GRAM || p.kind == NS_POLY;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 2);   // one announcement per CTA of the pair (used in the leader only)
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        for (int b = 0; b < ACCS; ++b) {
            mbar_init(smem_u32(&bar_acc_full[b]), 1);
            mbar_init(smem_u32(&bar_acc_empty[b]), 32);  // sixteen warps in each CTA (used in the leader only)
        }
        fence_barrier_init();
        fence_async_proxy();
        tma_prefetch_desc(&mapA);
        tma_prefetch_desc(&mapB);
    }
    if (warp == 0) {
        __syncwarp();
        tmem_alloc_pair(smem_u32(&tmem_base_s), ACCS * BN);
    }
    tc_fence_before();
    __syncthreads();
    cluster_barrier();  // both CTAs' barriers are initialised before either announces anything on them
    tc_fence_after();
    const uint32_t tmem = tmem_base_s;

    // where tile t lies: descriptor, repetition, tile row and column, blocks of 64 terms
    auto locate = [&](int t, int &rep, int &ti, int &tj) {
        const int d = square ? ns_find(g, t, [](const NsMat &m) { return m.first_a; }) : ns_find(g, t, [](const NsMat &m) { return m.first_x; });
        const NsMat &mat = g.mat[d];
        const int per = square ? mat.tiles_a : mat.tiles_x, local = t - (square ? mat.first_a : mat.first_x);
        rep = local / per;
        const int tt = local - rep * per, T = (mat.mp + 255) / 256;
        if (square) {  // blocks of 256 x 256 on and above the diagonal, 256 / BN tiles each
            ns_triangle(tt / (256 / BN), T, ti, tj);
            tj = tj * (256 / BN) + tt % (256 / BN);
        }
        else { ti = tt % T; tj = tt / T; }
        return d;
    };

    if (warp == 0) {
        if (elect_one()) {
            // ---- operands: this CTA's 128 rows of the first and 128 rows (or columns) of the second
            int s = 0, round = 0;
            bool ok = true, first = true;
            for (int t = pair; t < tiles && ok; t += n_pairs) {
                int rep, ti, tj;
                const NsMat &mat = g.mat[locate(t, rep, ti, tj)];
                const int slot_x = mat.row_x + rep * mat.mp, slot_a = mat.row_a + rep * mat.mp;
                const int kbs = (p.kind == NS_GRAM ? mat.np : mat.mp) / TC_BK;
                const int row_a = (p.kind == NS_GRAM ? p.x_row0 + slot_x : slot_a) + ti * 256 + rank * 128;
                const int at_b = tj * BN + rank * (BN / 2);
                for (int kb = 0; kb < kbs; ++kb) {
                    if (round > 0 && !mbar_wait(smem_u32(&bar_empty[s]), (round & 1) ^ 1, p.wait_ns)) { atomicExch(p.err, 1); ok = false; break; }
                    const uint32_t sa = smem_u32(smem) + s * stage_bytes, sb = sa + PARTS * a_bytes, bar = map_to_cta(smem_u32(&bar_full[s]), 0);
                    mbar_expect_tx_remote(bar, stage_bytes + (first && blockIdx.x == 0 ? (uint32_t)p.extra_tx : 0u));
                    first = false;
                    const int kk = kb * TC_BK;
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) {
                        tma_load_2d_pair(sa + q * a_bytes, &mapA, bar, kk, row_a + q * p.lo_rows_a);
                        if (square) {
                            tma_load_2d_pair(sb + q * b_bytes, &mapB, bar, kk, (p.kind == NS_GRAM ? p.x_row0 + slot_x : slot_a) + at_b + q * p.lo_rows_b);
                        } else {  // X across: 64 rows of K, boxes of 64 columns
                            const int row = p.x_row0 + slot_x + kk + q * p.lo_rows_b;
#pragma unroll
                            for (int c = 0; c < BN / 128; ++c) tma_load_2d_pair(sb + q * b_bytes + c * 8192, &mapB, bar, at_b + c * 64, row);
                        }
                    }
                    if (++s == S) { s = 0; ++round; }
                }
            }
            if (leader) ns_drain_copies<S>(bar_full, s, round, p.wait_ns);  // both CTAs' copies count on the leader's barriers
        }
    } else if (warp == 1) {
        if (leader && elect_one()) {
            // ---- products of the pair
            int s = 0, round = 0, use = 0;
            bool ok = true;
            const uint32_t idesc = make_idesc_f16(256, BN, !square);
            const uint64_t desc_a = make_smem_desc(smem_u32(smem), 16, 1024), desc_b = make_smem_desc(smem_u32(smem) + PARTS * a_bytes, square ? 16 : 8192, 1024);
            const uint64_t step_b = square ? 32 >> 4 : 2048 >> 4;
            for (int t = pair; t < tiles && ok; t += n_pairs) {
                int rep, ti, tj;
                const NsMat &mat = g.mat[locate(t, rep, ti, tj)];
                const int kbs = (p.kind == NS_GRAM ? mat.np : mat.mp) / TC_BK;
                for (int kb = 0; kb < kbs; ++kb) {
                    const int b = use % ACCS;
                    if ((PARTS == 2 || kb == 0) && use >= ACCS && !mbar_wait(smem_u32(&bar_acc_empty[b]), ((use / ACCS) & 1) ^ 1, p.wait_ns)) {
                        atomicExch(p.err, 5);
                        ok = false;
                        break;
                    }
                    if (!mbar_wait(smem_u32(&bar_full[s]), round & 1, p.wait_ns)) { atomicExch(p.err, 2); ok = false; break; }
                    tc_fence_after();
                    const uint64_t da = desc_a + ((s * stage_bytes) >> 4), db = desc_b + ((s * stage_bytes) >> 4);
                    const uint32_t acc = tmem + b * BN;
                    if (PARTS == 2) {  // the small terms first, while the sums are small
#pragma unroll
                        for (int i = 0; i < TC_BK / TC_UMMA_K; ++i) {
                            umma_bf16_pair(acc, da + i * 2, db + (b_bytes >> 4) + i * step_b, idesc, i != 0 ? 1u : 0u);
                            umma_bf16_pair(acc, da + (a_bytes >> 4) + i * 2, db + i * step_b, idesc, 1u);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < TC_BK / TC_UMMA_K; ++i) umma_bf16_pair(acc, da + i * 2, db + i * step_b, idesc, PARTS == 2 || kb != 0 || i != 0 ? 1u : 0u);
                    umma_commit_pair(smem_u32(&bar_empty[s]));
                    if (PARTS == 2 || kb + 1 == kbs) {
                        umma_commit_pair(smem_u32(&bar_acc_full[b]));
                        ++use;
                    }
                    if (++s == S) { s = 0; ++round; }
                }
            }
            ns_drain_products<S>(bar_empty, s, round, p.wait_ns);
        }
    } else {
        // ---- results: warp (q, cg) holds rows 32 q .. of this CTA's 128 and columns 64 cg .. of the tile's 256
        const int q = warp & 3, cg = (warp - 2) >> 2;
        float *turn = reinterpret_cast<float *>(smem + (size_t)S * stage_bytes) + (warp - 2) * 512;
        const int r_sub = lane >> 2, piece = lane & 3;  // after turning: rows 8 i + r_sub, columns 4 piece ..
        int use = 0;
        bool ok = true;
        for (int t = pair; t < tiles && ok; t += n_pairs) {
            int rep, ti, tj;
            const int d = locate(t, rep, ti, tj);
            const NsMat &mat = g.mat[d];
            const int kbs = (p.kind == NS_GRAM ? mat.np : mat.mp) / TC_BK;
            const int slot = square ? mat.row_a + rep * mat.mp : mat.row_x + rep * mat.mp;
            const int width = square ? mat.mp : mat.np;
            const int row0 = ti * 256 + rank * 128 + q * 32, col0 = tj * BN + cg * COLS;
            const bool live = row0 < mat.mp && col0 < width;  // whole blocks (sizes are padded to multiples of 64)
            const float inv_r = p.inv_r[mat.index + rep], r2 = inv_r * inv_r;
            const float f = p.kind == NS_GRAM ? NS_A_SCALE / (NS_X_SCALE * NS_X_SCALE) : p.kind == NS_POLY ? p.poly.c * r2 * r2 : p.poly.unscale;
            const float h = p.kind == NS_POLY ? p.poly.b * r2 : p.poly.a;
            const int pitch = square ? p.pitch_a : p.next.pitch;
            float v[PARTS == 2 ? COLS : 16];
            // the addends of 16 columns, as they lie in memory (POLY: 4 + 4 FP16, else 4 FP32), one block of columns ahead of their use
            uint4 ahead[2][4];
            auto fetch = [&](int blk) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const size_t at = (size_t)(slot + row0 + 8 * i + r_sub) * pitch + col0 + blk * 16 + 4 * piece;
                    if (p.kind == NS_POLY) {
                        const uint2 hi = *reinterpret_cast<const uint2 *>(p.A + at);
                        const uint2 lo = PARTS == 2 ? *reinterpret_cast<const uint2 *>(p.A + p.lo_off_a + at) : make_uint2(0u, 0u);
                        ahead[blk & 1][i] = make_uint4(hi.x, hi.y, lo.x, lo.y);
                    } else if (!square) {
                        ahead[blk & 1][i] = *reinterpret_cast<const uint4 *>(p.X + at);
                    }
                }
            };
            if (live && PARTS == 1) fetch(0);
            const int chunks = PARTS == 2 ? kbs : 1;
            for (int c = 0; c < chunks; ++c, ++use) {
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_acc_full[use % ACCS]), (use / ACCS) & 1, p.wait_ns));
                if (!ok) {
                    if (lane == 0) atomicExch(p.err, 3);
                    break;
                }
                tc_fence_after();
                if (PARTS == 2) {
                    const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16) + (use % ACCS) * BN + cg * 32;
#pragma unroll
                    for (int o = 0; o < 32; o += 16) {
                        float r[16];
                        tmem_ld_32x16(taddr + o, r);
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[o + i] = c == 0 ? r[i] : v[o + i] + r[i];
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(map_to_cta(smem_u32(&bar_acc_empty[use % ACCS]), 0));
                }
            }
            if (!ok) break;
            const bool mirror = square && ti != tj / (256 / BN), last = p.kind == NS_LAST;
            if (live && PARTS == 2) fetch(0);
#pragma unroll
            for (int blk = 0; blk < COLS / 16; ++blk) {
                const int col = col0 + blk * 16;
                if (PARTS == 1) {
                    tmem_ld_32x16(tmem + ((uint32_t)(q * 32) << 16) + ((use - 1) % ACCS) * BN + cg * COLS + blk * 16, v);
                    if (blk == COLS / 16 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_remote(map_to_cta(smem_u32(&bar_acc_empty[(use - 1) % ACCS]), 0));
                    }
                }
                if (!live) continue;
                if (blk + 1 < COLS / 16) fetch(blk + 1);
                __syncwarp();
                const float *w = v + (PARTS == 2 ? blk * 16 : 0);
#pragma unroll
                for (int i = 0; i < 4; ++i)  // 16-byte piece i of row `lane` lies at i ^ (lane / 2 mod 4)
                    *reinterpret_cast<float4 *>(turn + lane * 16 + ((i ^ ((lane >> 1) & 3)) << 2)) = make_float4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 8 * i + r_sub, row = row0 + r, c = col + 4 * piece;
                    float4 *place = reinterpret_cast<float4 *>(turn + r * 16 + ((piece ^ ((r >> 1) & 3)) << 2));
                    const float4 x = *place;
                    float y[4] = {f * x.x, f * x.y, f * x.z, f * x.w};
                    const size_t at = (size_t)(slot + row) * pitch + c;
                    const uint4 ad = ahead[blk & 1][i];
                    if (p.kind == NS_POLY) {
                        float2 a0 = __half22float2(*reinterpret_cast<const __half2 *>(&ad.x)), a1 = __half22float2(*reinterpret_cast<const __half2 *>(&ad.y));
                        if (PARTS == 2) {
                            const float2 l0 = __half22float2(*reinterpret_cast<const __half2 *>(&ad.z)), l1 = __half22float2(*reinterpret_cast<const __half2 *>(&ad.w));
                            a0.x += l0.x; a0.y += l0.y; a1.x += l1.x; a1.y += l1.y;
                        }
                        y[0] = fmaf(h, a0.x, y[0]); y[1] = fmaf(h, a0.y, y[1]); y[2] = fmaf(h, a1.x, y[2]); y[3] = fmaf(h, a1.y, y[3]);
                    } else if (!square) {
                        y[0] = fmaf(h, __uint_as_float(ad.x), y[0]); y[1] = fmaf(h, __uint_as_float(ad.y), y[1]);
                        y[2] = fmaf(h, __uint_as_float(ad.z), y[2]); y[3] = fmaf(h, __uint_as_float(ad.w), y[3]);
                    }
                    if (!last) {
                        if (!square) store_elems<float, 4>(p.next.full + at, y);
                        __half *o = (square ? p.out : p.next.hi) + at;
                        const size_t lo = square ? p.lo_off_a : p.next.lo_off;
                        const __half2 h0 = __floats2half2_rn(y[0], y[1]), h1 = __floats2half2_rn(y[2], y[3]);
                        *reinterpret_cast<uint2 *>(o) = make_uint2(*reinterpret_cast<const uint32_t *>(&h0), *reinterpret_cast<const uint32_t *>(&h1));
                        if (PARTS == 2) {
                            const float2 f0 = __half22float2(h0), f1 = __half22float2(h1);
                            const __half2 l0 = __floats2half2_rn(y[0] - f0.x, y[1] - f0.y), l1 = __floats2half2_rn(y[2] - f1.x, y[3] - f1.y);
                            *reinterpret_cast<uint2 *>(o + lo) = make_uint2(*reinterpret_cast<const uint32_t *>(&l0), *reinterpret_cast<const uint32_t *>(&l1));
                        }
                    }
                    if (mirror || last) *place = make_float4(y[0], y[1], y[2], y[3]);
                }
                if (mirror) {  // lane = turned row and eight of its elements: stores of 16 bits cost as much as stores of 16 bytes
                    __syncwarp();
                    const int c = lane & 15;
#pragma unroll
                    for (int it = 0; it < 2; ++it) {
                        const int r0 = 8 * ((lane >> 4) + 2 * it);
                        float y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = turn[(r0 + j) * 16 + ((((c >> 2) ^ (j >> 1)) & 3) << 2) + (c & 3)];
                        ns_store8<PARTS>(y, p.out + (size_t)(slot + col + c) * pitch + row0 + r0, p.lo_off_a);
                    }
                } else if (last && mat.tall) {  // lane = row: 32 neighbouring elements of every turned row
                    __syncwarp();
                    const int row = row0 + lane;
                    const bool odd = (lane & 1) != 0;
                    // BF16 in pairs where they are aligned: of two columns, the lane of the even row takes the first for both rows, the
                    // lane of the odd row the second
                    const bool pairs = p.bf16_dst && ((mat.dst + rep * mat.dst_stride) & 1) == 0 && (mat.ld_dst & 1) == 0 && ((uintptr_t)p.dst & 3) == 0;
                    const float scale = inv_r / NS_X_SCALE;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 x = *reinterpret_cast<const float4 *>(turn + lane * 16 + ((i ^ ((lane >> 1) & 3)) << 2));
                        const float y[4] = {x.x * scale, x.y * scale, x.z * scale, x.w * scale};
                        if (pairs) {
#pragma unroll
                            for (int j = 0; j < 4; j += 2) {
                                const float got = __shfl_xor_sync(0xffffffffu, odd ? y[j] : y[j + 1], 1);
                                const float lo = odd ? got : y[j], hi = odd ? y[j + 1] : got;  // rows row & ~1 and row | 1
                                const int c = col + 4 * i + j + (odd ? 1 : 0), even = row & ~1;
                                if (c < mat.n && even < mat.m) {
                                    bf16 *o = (bf16 *)p.dst + mat.dst + rep * mat.dst_stride + (long long)c * mat.ld_dst + even;
                                    if (even + 1 < mat.m) *reinterpret_cast<uint32_t *>(o) = pack_bf16(lo, hi);
                                    else *o = __float2bfloat16_rn(lo);
                                }
                            }
                        } else if (row < mat.m) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int c = col + 4 * i + j;
                                if (c < mat.n) ns_result(p, mat, mat.dst + rep * mat.dst_stride + (long long)c * mat.ld_dst + row, y[j]);
                            }
                        }
                    }
                } else if (last) {
                    __syncwarp();
                    const long long base = mat.dst + rep * mat.dst_stride;
                    const float scale = inv_r / NS_X_SCALE;
                    if (p.bf16_dst && (base & 1) == 0 && (mat.ld_dst & 1) == 0 && ((uintptr_t)p.dst & 3) == 0) {  // two columns per lane, four rows at a time
                        const int e = lane & 7, c = col + 2 * e;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int r = 4 * i + (lane >> 3), row = row0 + r;
                            const float2 y = *reinterpret_cast<const float2 *>(turn + r * 16 + (((e >> 1) ^ ((r >> 1) & 3)) << 2) + 2 * (e & 1));
                            bf16 *o = (bf16 *)p.dst + base + (long long)row * mat.ld_dst + c;
                            if (row < mat.m && c + 1 < mat.n) *reinterpret_cast<uint32_t *>(o) = pack_bf16(y.x * scale, y.y * scale);
                            else if (row < mat.m && c < mat.n) *o = __float2bfloat16_rn(y.x * scale);
                        }
                    } else {  // lane = column, two rows at a time
                        const int c = col + (lane & 15);
#pragma unroll 8
                        for (int i = 0; i < 16; ++i) {
                            const int r = 2 * i + (lane >> 4), row = row0 + r;
                            const float y = turn[r * 16 + ((((lane & 15) >> 2) ^ ((r >> 1) & 3)) << 2) + (lane & 3)];
                            if (row < mat.m && c < mat.n) ns_result(p, mat, base + (long long)row * mat.ld_dst + c, y * scale);
                        }
                    }
                }
                __syncwarp();
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_barrier();  // neither CTA frees tensor memory, or leaves with barriers the other may still signal, before both are done
    if (warp == 0) {
        __syncwarp();
        tmem_dealloc_pair(tmem, ACCS * BN);
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
template <int PARTS> constexpr int NSC_SMEM = NSC_STAGES<PARTS> * NSC_STAGE_BYTES<PARTS> + 2 * NSC_SUM_BYTES + 1024;

template <int PARTS, int C> static bool ns_chain_init()
{
    return cudaFuncSetAttribute(ns_chain_kernel<PARTS, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, NSC_SMEM<PARTS>) == cudaSuccess;
}

template <int PARTS, int C> static cudaLaunchConfig_t ns_chain_config(int clusters, cudaStream_t st, cudaLaunchAttribute (&attr)[2])
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(clusters * C);
    cfg.blockDim = dim3(NSC_THREADS);
    cfg.dynamicSmemBytes = NSC_SMEM<PARTS>;
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeCooperative;
    attr[1].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cfg;
}

// clusters of C blocks that are resident at the same time on the current device
template <int PARTS, int C> static int ns_chain_room()
{
    int room = 0;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = ns_chain_config<PARTS, C>(1, nullptr, attr);
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&room, ns_chain_kernel<PARTS, C>, &cfg) != cudaSuccess) { cudaGetLastError(); room = 0; }
    return room;
}

struct NsState {                  // of a context
    unsigned *counters = nullptr; // barrier counters of the chain kernel, zero between its launches
    int room[2][3] = {};          // [parts - 1][log2 of the cluster size]: ns_chain_room of the context's device
};

static bool ns_init(NsState &ns, std::string &err)
{
    if (!ns_chain_init<1, 1>() || !ns_chain_init<1, 2>() || !ns_chain_init<1, 4>() || !ns_chain_init<2, 1>() || !ns_chain_init<2, 2>() || !ns_chain_init<2, 4>() ||
        cudaFuncSetAttribute(ns_block_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, NSB_SMEM<1>) != cudaSuccess ||
        cudaFuncSetAttribute(ns_block_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, NSB_SMEM<2>) != cudaSuccess ||
        cudaFuncSetAttribute(ns_pair_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, NSP_SMEM<1>) != cudaSuccess ||
        cudaFuncSetAttribute(ns_pair_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, NSP_SMEM<2>) != cudaSuccess) {
        err = "cannot raise the dynamic shared memory limit of the Newton-Schulz products";
        return false;
    }
    if (cudaMalloc((void **)&ns.counters, NSC_BARRIERS * sizeof(unsigned)) != cudaSuccess || cudaMemset(ns.counters, 0, NSC_BARRIERS * sizeof(unsigned)) != cudaSuccess) {
        err = "allocation of the counters of the Newton-Schulz products failed";
        return false;
    }
    ns.room[0][0] = ns_chain_room<1, 1>(); ns.room[0][1] = ns_chain_room<1, 2>(); ns.room[0][2] = ns_chain_room<1, 4>();
    ns.room[1][0] = ns_chain_room<2, 1>(); ns.room[1][1] = ns_chain_room<2, 2>(); ns.room[1][2] = ns_chain_room<2, 4>();
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

// Bounds of the iteration: with |X| <= 1 at the start, every later |X| must stay below 2 and |B| below 200 for FP16 to
// hold them.  The largest value of |a s + b s^3 + c s^5| on [0, top] is at an end or where its derivative vanishes.
static bool ns_coefficients_ok(double a, double b, double c, int steps, NsPoly &poly)
{
    if (!(std::isfinite(a) && std::isfinite(b) && std::isfinite(c))) return false;
    double top = 1.0, largest_b = 0.0;
    for (int k = 0; k < steps; ++k) {
        largest_b = std::max(largest_b, std::fabs(b) * top * top + std::fabs(c) * top * top * top * top);
        if (largest_b > 200.0) return false;
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
    float b_scale = 256.f;  // the largest power of two for which B stays inside FP16 (65,504), the roundings of A and B included
    while (b_scale < NS_A_SCALE && 2.0 * b_scale * largest_b <= 60000.0) b_scale *= 2.f;
    poly = {(float)a, (float)b * (b_scale / NS_A_SCALE), (float)c * (b_scale / (NS_A_SCALE * NS_A_SCALE)), 1.f / b_scale};
    return true;
}

struct NsLayout {  // sizes of the arenas of a group
    int rows_x = 0, rows_a = 0, pitch_x = 0, pitch_a = 0, norm_blocks = 0, conv_blocks = 0, matrices = 0;
    size_t x_elems() const { return (size_t)rows_x * pitch_x; }
    size_t a_elems() const { return (size_t)rows_a * pitch_a; }
    static size_t up(size_t b) { return (b + 1023) & ~(size_t)1023; }
    // two FP32 copies of X, two of its operands, A, B, the norm partials, 1 / r
    size_t bytes(int parts) const
    {
        return 2 * up(4 * x_elems()) + up((size_t)4 * parts * x_elems()) + 2 * up((size_t)2 * parts * a_elems()) + up(sizeof(double) * (size_t)norm_blocks) +
               up(sizeof(float) * (size_t)matrices);
    }
};

// fills the derived fields of the descriptors (m, n, repeat, tall given)
static NsLayout ns_layout(NsGroup &g)
{
    NsLayout l;
    for (int d = 0; d < g.count; ++d) {
        NsMat &m = g.mat[d];
        m.mp = (m.m + 63) / 64 * 64;
        m.np = (m.n + 63) / 64 * 64;
        m.row_x = l.rows_x;
        m.row_a = l.rows_a;
        m.index = l.matrices;
        l.rows_x += m.mp * m.repeat;
        l.rows_a += m.mp * m.repeat;
        l.pitch_x = std::max(l.pitch_x, m.np);
        l.pitch_a = std::max(l.pitch_a, m.mp);
        const int64_t elems = (int64_t)m.m * m.n;
        m.norm_elems = (int)std::max<int64_t>(NS_NORM_ELEMS, ceil_div64(ceil_div64(elems, NS_NORM_BLOCKS), NS_THREADS) * NS_THREADS);
        m.norm_blocks = (int)ceil_div64(elems, m.norm_elems);
        m.conv_blocks = (m.mp / 64) * (m.np / 64);
        m.first_norm = l.norm_blocks;
        m.first_conv = l.conv_blocks;
        l.norm_blocks += m.norm_blocks * m.repeat;
        l.conv_blocks += m.conv_blocks * m.repeat;
        l.matrices += m.repeat;
    }
    return l;
}

// tiles of the products for tiles of bm x bn; `half`: of A only those of the blocks of bm x bm on and above the diagonal.  Returns the
// numbers of tiles of A and of X
static void ns_tiles(NsGroup &g, int bm, int bn, bool half, int &tiles_a, int &tiles_x)
{
    tiles_a = tiles_x = 0;
    for (int d = 0; d < g.count; ++d) {
        NsMat &m = g.mat[d];
        const int T = (m.mp + bm - 1) / bm;
        m.tiles_a = half ? T * (T + 1) / 2 * (bm / bn) : T * ((m.mp + bn - 1) / bn);
        m.tiles_x = T * ((m.np + bn - 1) / bn);
        m.first_a = tiles_a;
        m.first_x = tiles_x;
        tiles_a += m.tiles_a * m.repeat;
        tiles_x += m.tiles_x * m.repeat;
    }
}

// all matrices go to the one-block kernel: faster wherever it applies (figures at the kernel), and it needs no workspace
static bool ns_small(const NsGroup &g)
{
    for (int d = 0; d < g.count; ++d)
        if (g.mat[d].n > NSB_SIZE) return false;
    return g.count > 0;
}
static size_t ns_workspace(const NsGroup &g, const NsLayout &l, int parts) { return ns_small(g) ? 0 : l.bytes(parts); }

struct NsTarget {
    void *dst;
    int bf16_dst;
    const float *params;
    float keep;
};

// Which kernel: estimated microseconds of one step, a fixed time per phase, a time per tile that a block (or pair) takes in turn and
// one per 64 terms, fitted to runs of 64 x 64 to 2048 x 2048 and of batches.  Measured, BF16 (FP32), microseconds for five steps:
//                     chain, C = 1     C = 2          C = 4          pair
//   64 x 64           52 (69)          72 (82)        81 (87)        112 (113)
//   64 x 1024         70 (121)         80 (107)       87 (101)       139 (150)
//   768 x 768         103 (201)        101 (152)      199 (268)      235 (250)
//   1024 x 1024       124 (248)        156 (286)      257 (381)      252 (278)
//   2048 x 2048       549 (1497)       517 (1471)     1029 (2117)    350 (551)
//   16 of 512 x 512   242 (552)        404 (645)      961 (1176)     241 (393)
struct NsCost {
    double phase, tile, kb;
    double step(const NsGroup &g, int room, int tiles_a, int tiles_x, int split) const
    {
        int kb_m = 0, kb_n = 0;
        for (int d = 0; d < g.count; ++d) { kb_m = std::max(kb_m, g.mat[d].mp / 64); kb_n = std::max(kb_n, g.mat[d].np / 64); }
        auto one = [&](int tiles, int blocks) { return phase + ((tiles + room - 1) / room) * (tile + kb * ((blocks + split - 1) / split)); };
        return one(tiles_a, kb_n) + one(tiles_a, kb_m) + one(tiles_x, kb_m);
    }
};
static NsCost ns_chain_cost(int parts, int c)
{
    const double tile = c == 1 ? 1.0 : c == 2 ? 2.0 : 2.5;
    return parts == 2 ? NsCost{2.9, tile, 0.75} : NsCost{2.4, tile, 0.26};
}
static NsCost ns_pair_cost(int parts) { return parts == 2 ? NsCost{8.0, 5.0, 0.42} : NsCost{13.0, 0.5, 0.29}; }

template <int PARTS>
static bool ns_run(TcState &tc, Exec &ex, const NsSource &src, NsGroup &g, const NsLayout &l, const NsAdam &adam, const NsState &ns, int steps,
                   const NsPoly &poly, double eps, const NsTarget &out, uint8_t *ws, std::string &err)
{
    const size_t nx = l.x_elems(), na = l.a_elems();
    NsX X[2];
    X[0].full = (float *)ws;
    X[1].full = (float *)(ws + NsLayout::up(4 * nx));
    __half *ops = (__half *)(ws + 2 * NsLayout::up(4 * nx));
    for (int i = 0; i < 2; ++i) {
        X[i].hi = ops + (size_t)i * PARTS * nx;
        X[i].lo_off = nx;
        X[i].pitch = l.pitch_x;
    }
    __half *A = (__half *)((uint8_t *)ops + NsLayout::up((size_t)4 * PARTS * nx));
    __half *B = (__half *)((uint8_t *)A + NsLayout::up((size_t)2 * PARTS * na));
    double *partial = (double *)((uint8_t *)B + NsLayout::up((size_t)2 * PARTS * na));
    float *inv_r = (float *)((uint8_t *)partial + NsLayout::up(sizeof(double) * (size_t)l.norm_blocks));
    const int adam_blocks = (int)ceil_div64(adam.spans.first[adam.spans.count], NS_ADAM_ELEMS);
    if (ns_small(g)) {
        NsBlock p{};
        p.steps = steps; p.matrices = l.matrices;
        p.poly = poly; p.eps = eps;
        p.dst = out.dst; p.bf16_dst = out.bf16_dst; p.params = out.params; p.keep = out.keep;
        p.err = tc.err_word; p.wait_ns = tc.wait_limit_ns; p.extra_tx = tc.overdeclare_tx;
        tc.overdeclare_tx = 0;
        launch_dep(ns_block_kernel<PARTS>, dim3(l.matrices + adam_blocks), dim3(NSB_THREADS), NSB_SMEM<PARTS>, ex.st, src, g, adam, p);
        ex.launches += 1;
        return true;
    }
    CUtensorMap x128, x64, a128, a64, b128;
    if (g.count > 0 && (!ns_make_map(tc, &x128, ops, (int64_t)2 * PARTS * l.rows_x, l.pitch_x, 128) || !ns_make_map(tc, &x64, ops, (int64_t)2 * PARTS * l.rows_x, l.pitch_x, 64) ||
                        !ns_make_map(tc, &a128, A, (int64_t)PARTS * l.rows_a, l.pitch_a, 128) || !ns_make_map(tc, &a64, A, (int64_t)PARTS * l.rows_a, l.pitch_a, 64) ||
                        !ns_make_map(tc, &b128, B, (int64_t)PARTS * l.rows_a, l.pitch_a, 128))) {
        err = "cuTensorMapEncodeTiled failed";
        return false;
    }
    const int pairs = std::max(1, tc_sm_count() / 2);
    int tiles_a = 0, tiles_x = 0, best = -1;  // best: log2 of the chain kernel's cluster size, -1 = pair kernel
    ns_tiles(g, 256, NSP_BN<PARTS>, true, tiles_a, tiles_x);
    double cost = ns_pair_cost(PARTS).step(g, pairs, tiles_a, tiles_x, 1);
    ns_tiles(g, 128, NSC_BN, false, tiles_a, tiles_x);
    const int(&rooms)[3] = ns.room[PARTS - 1];
    for (int i = 0; i < 3; ++i) {
        if (rooms[i] <= 0) continue;
        const double t = ns_chain_cost(PARTS, 1 << i).step(g, rooms[i], tiles_a, tiles_x, 1 << i);
        if (t < cost) { cost = t; best = i; }
    }
    if (best >= 0 && g.count > 0) {
        NsChain p{};
        for (int par = 0; par < 2; ++par) {
            p.io[par][NS_GRAM] = {nullptr, nullptr, A, nullptr, (long long)na, l.pitch_a};
            p.io[par][NS_POLY] = {A, nullptr, B, nullptr, (long long)na, l.pitch_a};
            p.io[par][NS_APPLY] = {nullptr, X[par].full, X[par ^ 1].hi, X[par ^ 1].full, (long long)nx, l.pitch_x};
        }
        p.parts_rows_x = l.rows_x; p.parts_rows_a = l.rows_a;
        p.steps = steps;
        p.poly = poly; p.eps = eps;
        p.X0 = X[0];
        p.partial = partial; p.inv_r = inv_r;
        p.norm_blocks = l.norm_blocks; p.adam_blocks = adam_blocks; p.conv_blocks = l.conv_blocks; p.tiles_a = tiles_a; p.tiles_x = tiles_x;
        p.dst = out.dst; p.bf16_dst = out.bf16_dst; p.params = out.params; p.keep = out.keep;
        p.counters = ns.counters;
        p.err = tc.err_word; p.wait_ns = tc.wait_limit_ns; p.extra_tx = tc.overdeclare_tx;
        tc.overdeclare_tx = 0;
        const int cl = 1 << best;
        const int clusters = std::min(rooms[best], std::max({tiles_a, tiles_x, (l.conv_blocks + cl - 1) / cl, (l.norm_blocks + adam_blocks + cl - 1) / cl}));
        cudaLaunchAttribute attr[2];
        cudaError_t e = cudaSuccess;
#define LP_CHAIN(C_)                                                                                                                                 \
    do {                                                                                                                                             \
        cudaLaunchConfig_t cfg = ns_chain_config<PARTS, C_>(clusters, ex.st, attr);                                                                  \
        e = cudaLaunchKernelEx(&cfg, ns_chain_kernel<PARTS, C_>, x128, x64, a128, a64, b128, src, g, adam, p);                                        \
    } while (0)
        if (best == 0) LP_CHAIN(1); else if (best == 1) LP_CHAIN(2); else LP_CHAIN(4);
#undef LP_CHAIN
        if (e != cudaSuccess) {
            cudaGetLastError();
            err = std::string("launch of the chain kernel: ") + cudaGetErrorString(e);
            return false;
        }
        ex.launches += 1;
        return true;
    }
    launch_dep(ns_norm_kernel, dim3(std::max(1, l.norm_blocks + adam_blocks)), dim3(NS_THREADS), 0, ex.st, src, g, adam, l.norm_blocks, partial);
    ex.launches += 1;
    if (g.count == 0) return true;
    ns_tiles(g, 256, NSP_BN<PARTS>, true, tiles_a, tiles_x);
    launch_dep(ns_convert_kernel<PARTS>, dim3(l.conv_blocks), dim3(NS_THREADS), 0, ex.st, src, g, partial, eps, X[0], inv_r);
    ex.launches += 1;
    NsPhase p{};
    p.poly = poly;
    p.err = tc.err_word;
    p.wait_ns = tc.wait_limit_ns;
    p.pitch_a = l.pitch_a;
    p.lo_off_a = na;
    p.inv_r = inv_r;
    p.dst = out.dst; p.bf16_dst = out.bf16_dst; p.params = out.params; p.keep = out.keep;
    auto product = [&](int kind, int tiles, const CUtensorMap &ma, const CUtensorMap &mb) {
        p.kind = kind;
        p.extra_tx = tc.overdeclare_tx;
        tc.overdeclare_tx = 0;
        launch_dep(ns_pair_kernel<PARTS>, dim3(2 * std::min(tiles, pairs)), dim3(NSP_THREADS), NSP_SMEM<PARTS>, ex.st, ma, mb, p, g, tiles);
        ex.launches += 1;
    };
    for (int k = 0; k < steps; ++k) {
        const int cur = k & 1;
        p.x_row0 = cur * PARTS * l.rows_x;
        p.lo_rows_a = p.lo_rows_b = l.rows_x;
        p.out = A;
        p.next = X[cur ^ 1];
        product(NS_GRAM, tiles_a, x128, PARTS == 2 ? x64 : x128);
        p.lo_rows_a = p.lo_rows_b = l.rows_a;
        p.A = A; p.out = B;
        product(NS_POLY, tiles_a, a128, PARTS == 2 ? a64 : a128);
        p.lo_rows_b = l.rows_x;
        p.X = X[cur].full;
        product(k + 1 == steps ? NS_LAST : NS_APPLY, tiles_x, b128, x64);
    }
    return true;
}
