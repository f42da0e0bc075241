// Learned node features: rows of an embedding table scaled and gathered, and the gradient of the table.
//
//   lookup    out[i]  = scale * table[ids[i]]                     (zero for the padding id)
//   gradient  grad[v] = scale * sum over { i : ids[i] = v } of dout[i]   (zero for rows that no id names)
//
// The gradient is taken over the ids sorted stably, so the rows of one table row are added in the order of i and the
// result is the same bits in every run.  All sums are FP32; a BF16 result is rounded once, at the store.
#pragma once
#include "common.cuh"
#include "scan_sort.cuh"

// VE consecutive elements as floats; the address is aligned to min(16, VE * sizeof(T)) bytes
template <typename T, int VE> LP_DEVINL void load_elems(const T *p, float *f);
template <> LP_DEVINL void load_elems<float, 4>(const float *p, float *f)
{
    const float4 v = *reinterpret_cast<const float4 *>(p);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
}
template <> LP_DEVINL void load_elems<float, 2>(const float *p, float *f)
{
    const float2 v = *reinterpret_cast<const float2 *>(p);
    f[0] = v.x; f[1] = v.y;
}
template <> LP_DEVINL void load_elems<float, 1>(const float *p, float *f) { f[0] = *p; }
LP_DEVINL void bf16_pair(uint32_t w, float *f) { f[0] = __uint_as_float(w << 16); f[1] = __uint_as_float(w & 0xFFFF0000u); }
template <> LP_DEVINL void load_elems<bf16, 8>(const bf16 *p, float *f)
{
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    bf16_pair(v.x, f); bf16_pair(v.y, f + 2); bf16_pair(v.z, f + 4); bf16_pair(v.w, f + 6);
}
template <> LP_DEVINL void load_elems<bf16, 4>(const bf16 *p, float *f)
{
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    bf16_pair(v.x, f); bf16_pair(v.y, f + 2);
}
template <> LP_DEVINL void load_elems<bf16, 2>(const bf16 *p, float *f) { bf16_pair(*reinterpret_cast<const uint32_t *>(p), f); }
template <> LP_DEVINL void load_elems<bf16, 1>(const bf16 *p, float *f) { f[0] = __bfloat162float(*p); }

template <typename T, int VE> LP_DEVINL void store_elems(T *p, const float *f);
template <> LP_DEVINL void store_elems<float, 4>(float *p, const float *f) { *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]); }
template <> LP_DEVINL void store_elems<float, 8>(float *p, const float *f) { store_elems<float, 4>(p, f); store_elems<float, 4>(p + 4, f + 4); }
template <> LP_DEVINL void store_elems<float, 2>(float *p, const float *f) { *reinterpret_cast<float2 *>(p) = make_float2(f[0], f[1]); }
template <> LP_DEVINL void store_elems<float, 1>(float *p, const float *f) { *p = f[0]; }
template <> LP_DEVINL void load_elems<float, 8>(const float *p, float *f) { load_elems<float, 4>(p, f); load_elems<float, 4>(p + 4, f + 4); }
LP_DEVINL uint32_t pack_bf16(float a, float b)
{
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&h);
}
template <> LP_DEVINL void store_elems<bf16, 8>(bf16 *p, const float *f)
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
template <> LP_DEVINL void store_elems<bf16, 4>(bf16 *p, const float *f) { *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])); }
template <> LP_DEVINL void store_elems<bf16, 2>(bf16 *p, const float *f) { *reinterpret_cast<uint32_t *>(p) = pack_bf16(f[0], f[1]); }
template <> LP_DEVINL void store_elems<bf16, 1>(bf16 *p, const float *f) { *p = __float2bfloat16_rn(f[0]); }

// Largest VE (a power of two, at most `most`) such that rows of D elements at `base` with pitch ld can be read in aligned
// pieces of VE elements.
static int elems_per_piece(const void *base, int64_t ld, int D, size_t elem, int most)
{
    int ve = most;
    while (ve > 1 && (D % ve != 0 || ld % ve != 0 || (uintptr_t)base % std::min<size_t>(16, ve * elem) != 0)) ve >>= 1;
    return ve;
}

// lanes that share a row: the smallest power of two in 8..32 that covers the row's pieces in one step
static int lanes_per_row(int pieces) { return pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32; }

// ---------------------------------------------------------------------------------------------
// lookup.  A group of G lanes takes four ids at a time, so four row loads are in flight per lane.
// ---------------------------------------------------------------------------------------------
constexpr int EMB_THREADS = 256;
constexpr int EMB_ROWS = 4;

template <typename TT, typename TO, int VE>
__global__ void __launch_bounds__(EMB_THREADS) embed_kernel(const TT *__restrict__ table, int64_t V, int D, int64_t ldt, const int *__restrict__ ids,
                                                            int64_t N, int padding, float scale, TO *__restrict__ out, int64_t ldo, int G,
                                                            int *__restrict__ err)
{
    LP_DEP_ENTER();
    const int gl = threadIdx.x & (G - 1);
    const int64_t group = ((int64_t)blockIdx.x * EMB_THREADS + threadIdx.x) / G;
    const int64_t i0 = group * EMB_ROWS;
    int id[EMB_ROWS];
    bool live[EMB_ROWS];
#pragma unroll
    for (int r = 0; r < EMB_ROWS; ++r) {
        id[r] = i0 + r < N ? ids[i0 + r] : -1;
        live[r] = id[r] >= 0 && id[r] < V && id[r] != padding;
        if (i0 + r < N && !live[r] && gl == 0 && (id[r] != padding || padding == LP_NO_PADDING)) atomicOr(err, 1);
    }
    for (int c = gl * VE; c < D; c += G * VE) {
        float v[EMB_ROWS][VE];
#pragma unroll
        for (int r = 0; r < EMB_ROWS; ++r) {
            if (live[r]) {
                load_elems<TT, VE>(table + (int64_t)id[r] * ldt + c, v[r]);
            } else {
#pragma unroll
                for (int t = 0; t < VE; ++t) v[r][t] = 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < EMB_ROWS; ++r) {
            if (i0 + r < N) {
                if (live[r]) {
#pragma unroll
                    for (int t = 0; t < VE; ++t) v[r][t] *= scale;
                }
                store_elems<TO, VE>(out + (i0 + r) * ldo + c, v[r]);
            }
        }
    }
}

template <typename TT, typename TO>
static void embed_launch(Exec &ex, const TT *table, int64_t V, int D, int64_t ldt, const int *ids, int64_t N, int padding, float scale, TO *out, int64_t ldo,
                         int *err)
{
    constexpr int most = sizeof(TT) == 4 || sizeof(TO) == 4 ? 4 : 8;
    const int ve = std::min(elems_per_piece(table, ldt, D, sizeof(TT), most), elems_per_piece(out, ldo, D, sizeof(TO), most));
    const int G = lanes_per_row((D + ve - 1) / ve);
    const dim3 grid((unsigned)ceil_div64(N, (int64_t)EMB_THREADS / G * EMB_ROWS)), block(EMB_THREADS);
#define LP_EMBED(VE_) launch_dep(embed_kernel<TT, TO, VE_>, grid, block, 0, ex.st, table, V, D, ldt, ids, N, padding, scale, out, ldo, G, err)
    if (ve == 8) { if constexpr (most == 8) LP_EMBED(8); }
    else if (ve == 4) LP_EMBED(4);
    else if (ve == 2) LP_EMBED(2);
    else LP_EMBED(1);
#undef LP_EMBED
    ex.launches += 1;
}

// ---------------------------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------------------------
constexpr int EG_THREADS = 256;
constexpr int EG_CHUNK = 32;  // consecutive sorted ids that one group of lanes adds up
constexpr int EG_BATCH = 8;   // rows of dout requested together

// keys[i] = ids[i], or V (sorted behind every row) for the padding id and for ids outside the table; bit v of `named`
// is set when row v receives a gradient
__global__ void embed_keys_kernel(const int *__restrict__ ids, int64_t N, int64_t V, int padding, uint32_t *__restrict__ keys,
                                  uint32_t *__restrict__ vals, uint32_t *__restrict__ named, int *__restrict__ err)
{
    LP_DEP_ENTER();
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= N) return;
    const int id = ids[i];
    const bool live = id >= 0 && id < V && id != padding;
    if (!live && (id != padding || padding == LP_NO_PADDING)) atomicOr(err, 1);
    keys[i] = live ? (uint32_t)id : (uint32_t)V;
    vals[i] = (uint32_t)i;
    if (live) {
        const uint32_t bit = 1u << (id & 31);
        if (!(*(volatile uint32_t *)(named + (id >> 5)) & bit)) atomicOr(named + (id >> 5), bit);
    }
}

template <typename TG, int VE> LP_DEVINL void embed_grad_store(TG *p, const float *acc, float scale, bool accumulate)
{
    float o[VE];
    if (accumulate) {
        load_elems<TG, VE>(p, o);
#pragma unroll
        for (int t = 0; t < VE; ++t) o[t] = fmaf(scale, acc[t], o[t]);
    } else {
#pragma unroll
        for (int t = 0; t < VE; ++t) o[t] = scale * acc[t];
    }
    store_elems<TG, VE>(p, o);
}

// One group of G lanes adds the rows of EG_CHUNK consecutive sorted ids.  A run of equal ids that lies inside the chunk
// is written to the gradient; the part of a run that began in an earlier chunk goes to head[chunk], the part of a run that
// begins here and goes on goes to tail[chunk] (FP32, unscaled), and embed_grad_join_kernel adds those up.
template <typename TD, typename TG, int VE>
__global__ void __launch_bounds__(EG_THREADS) embed_grad_sum_kernel(const uint32_t *__restrict__ keys, const uint32_t *__restrict__ vals, int64_t N, int64_t V,
                                                                    const TD *__restrict__ dout, int64_t ldd, int D, float scale, TG *__restrict__ grad,
                                                                    int64_t ldg, int accumulate, float *__restrict__ head, float *__restrict__ tail, int G)
{
    LP_DEP_ENTER();
    const int gl = threadIdx.x & (G - 1);
    const int64_t chunk = ((int64_t)blockIdx.x * EG_THREADS + threadIdx.x) / G;
    const int64_t p0 = chunk * EG_CHUNK;
    if (p0 >= N) return;
    const int count = (int)min((int64_t)EG_CHUNK, N - p0);
    const uint32_t before = p0 > 0 ? keys[p0 - 1] : 0xFFFFFFFFu, after = p0 + count < N ? keys[p0 + count] : 0xFFFFFFFFu;
    const uint32_t first = keys[p0];
    for (int c = gl * VE; c < D; c += G * VE) {
        uint32_t cur = first;
        bool from_before = before == first;
        float acc[VE];
#pragma unroll
        for (int t = 0; t < VE; ++t) acc[t] = 0.f;
        for (int b = 0; b < count; b += EG_BATCH) {
            uint32_t k[EG_BATCH];
            float x[EG_BATCH][VE];
#pragma unroll
            for (int j = 0; j < EG_BATCH; ++j) {
                k[j] = b + j < count ? keys[p0 + b + j] : (uint32_t)V;
                if (k[j] < (uint32_t)V) load_elems<TD, VE>(dout + (int64_t)vals[p0 + b + j] * ldd + c, x[j]);
            }
#pragma unroll
            for (int j = 0; j < EG_BATCH; ++j) {
                if (k[j] != cur) {
                    if (cur < (uint32_t)V) {
                        if (from_before) store_elems<float, VE>(head + chunk * D + c, acc);
                        else embed_grad_store<TG, VE>(grad + (int64_t)cur * ldg + c, acc, scale, accumulate != 0);
                    }
                    from_before = false;
                    cur = k[j];
#pragma unroll
                    for (int t = 0; t < VE; ++t) acc[t] = 0.f;
                }
                if (k[j] < (uint32_t)V) {
#pragma unroll
                    for (int t = 0; t < VE; ++t) acc[t] += x[j][t];
                }
            }
        }
        if (cur < (uint32_t)V) {
            if (from_before) store_elems<float, VE>(head + chunk * D + c, acc);
            else if (after == cur) store_elems<float, VE>(tail + chunk * D + c, acc);
            else embed_grad_store<TG, VE>(grad + (int64_t)cur * ldg + c, acc, scale, accumulate != 0);
        }
    }
}

// Runs that cross chunks: for every chunk in which such a run begins, grad[run] = tail[chunk] + head[chunk + 1] + ...
template <typename TG, int VE>
__global__ void __launch_bounds__(EG_THREADS) embed_grad_join_kernel(const uint32_t *__restrict__ keys, int64_t N, int64_t V, int D, float scale,
                                                                     TG *__restrict__ grad, int64_t ldg, int accumulate, const float *__restrict__ head,
                                                                     const float *__restrict__ tail, int G)
{
    LP_DEP_ENTER();
    const int gl = threadIdx.x & (G - 1);
    const int64_t chunk = ((int64_t)blockIdx.x * EG_THREADS + threadIdx.x) / G;
    const int64_t p1 = (chunk + 1) * EG_CHUNK;
    if (p1 >= N) return;
    const uint32_t key = keys[p1 - 1];
    if (key >= (uint32_t)V || keys[p1] != key) return;                                  // no run goes on into the next chunk
    if (keys[p1 - EG_CHUNK] == key && chunk > 0 && keys[p1 - EG_CHUNK - 1] == key) return;  // it began in an earlier one
    // last chunk of the run: the chunks p with keys[p * EG_CHUNK] == key follow one another
    int64_t lo = chunk + 1, hi = (N + EG_CHUNK - 1) / EG_CHUNK;  // keys[lo * EG_CHUNK] == key; search the first chunk that does not begin with key
    int64_t end = lo + 1;
    while (lo + 1 < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (keys[mid * EG_CHUNK] == key) lo = mid; else hi = mid;
    }
    end = lo + 1;
    for (int c = gl * VE; c < D; c += G * VE) {
        float acc[VE];
        load_elems<float, VE>(tail + chunk * D + c, acc);
        for (int64_t q = chunk + 1; q < end; ++q) {
            float x[VE];
            load_elems<float, VE>(head + q * D + c, x);
#pragma unroll
            for (int t = 0; t < VE; ++t) acc[t] += x[t];
        }
        embed_grad_store<TG, VE>(grad + (int64_t)key * ldg + c, acc, scale, accumulate != 0);
    }
}

// zero rows that no id names
template <typename TG, int VE>
__global__ void __launch_bounds__(EG_THREADS) embed_grad_zero_kernel(const uint32_t *__restrict__ named, int64_t V, int D, TG *__restrict__ grad, int64_t ldg,
                                                                     int G)
{
    LP_DEP_ENTER();
    const int gl = threadIdx.x & (G - 1);
    const int64_t groups = (int64_t)gridDim.x * EG_THREADS / G;
    float z[VE];
#pragma unroll
    for (int t = 0; t < VE; ++t) z[t] = 0.f;
    for (int64_t v = ((int64_t)blockIdx.x * EG_THREADS + threadIdx.x) / G; v < V; v += groups) {
        if ((named[v >> 5] >> (v & 31)) & 1u) continue;
        for (int c = gl * VE; c < D; c += G * VE) store_elems<TG, VE>(grad + v * ldg + c, z);
    }
}

struct EmbedGradScratch {
    uint32_t *keys = nullptr, *vals = nullptr, *named = nullptr;
    SortScratch sort;
    float *head = nullptr, *tail = nullptr;
};

template <typename TD, typename TG, int VE>
static void embed_grad_rows(Exec &ex, const TD *dout, int64_t ldd, const uint32_t *keys, const uint32_t *vals, int64_t N, float scale, int64_t V, int D,
                            TG *grad, int64_t ldg, int accumulate, const EmbedGradScratch &s)
{
    const int G = lanes_per_row((D + VE - 1) / VE);
    const int64_t groups = EG_THREADS / G;
    if (!accumulate) {
        const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div64(V, groups), 148 * 8);
        launch_dep(embed_grad_zero_kernel<TG, VE>, dim3(blocks), dim3(EG_THREADS), 0, ex.st, s.named, V, D, grad, ldg, G);
        ex.launches += 1;
    }
    if (N == 0) return;
    const int64_t chunks = ceil_div64(N, EG_CHUNK);
    const unsigned blocks = (unsigned)ceil_div64(chunks, groups);
    launch_dep(embed_grad_sum_kernel<TD, TG, VE>, dim3(blocks), dim3(EG_THREADS), 0, ex.st, keys, vals, N, V, dout, ldd, D, scale, grad, ldg, accumulate, s.head,
               s.tail, G);
    ex.launches += 1;
    if (chunks > 1) {
        launch_dep(embed_grad_join_kernel<TG, VE>, dim3(blocks), dim3(EG_THREADS), 0, ex.st, keys, N, V, D, scale, grad, ldg, accumulate, s.head, s.tail, G);
        ex.launches += 1;
    }
}

template <typename TD, typename TG>
static void embed_grad_launch(Exec &ex, const TD *dout, int64_t ldd, const int *ids, int64_t N, int padding, float scale, int64_t V, int D, TG *grad, int64_t ldg,
                              int accumulate, const EmbedGradScratch &s, int *err)
{
    const uint32_t *keys = s.keys, *vals = s.vals;
    if (N > 0 || !accumulate) cudaMemsetAsync(s.named, 0, sizeof(uint32_t) * (size_t)ceil_div64(V, 32), ex.st);
    if (N > 0) {
        launch_dep(embed_keys_kernel, dim3((unsigned)ceil_div64(N, 256)), dim3(256), 0, ex.st, ids, N, V, padding, s.keys, s.vals, s.named, err);
        ex.launches += 1;
        if (!radix_sort_pairs(ex, s.keys, s.vals, N, bits_for(V + 1), s.sort)) { keys = s.sort.keys_alt; vals = s.sort.vals_alt; }
    }
    constexpr int most = sizeof(TD) == 4 || sizeof(TG) == 4 ? 4 : 8;
    const int ve = std::min(elems_per_piece(dout, ldd, D, sizeof(TD), most), elems_per_piece(grad, ldg, D, sizeof(TG), most));
    if (ve == 8) { if constexpr (most == 8) embed_grad_rows<TD, TG, 8>(ex, dout, ldd, keys, vals, N, scale, V, D, grad, ldg, accumulate, s); }
    else if (ve == 4) embed_grad_rows<TD, TG, 4>(ex, dout, ldd, keys, vals, N, scale, V, D, grad, ldg, accumulate, s);
    else if (ve == 2) embed_grad_rows<TD, TG, 2>(ex, dout, ldd, keys, vals, N, scale, V, D, grad, ldg, accumulate, s);
    else embed_grad_rows<TD, TG, 1>(ex, dout, ldd, keys, vals, N, scale, V, D, grad, ldg, accumulate, s);
}
