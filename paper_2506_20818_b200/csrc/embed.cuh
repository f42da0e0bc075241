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

// VE elements as they lie in memory (BF16 rows wait for their turn in half the registers that floats would take)
template <typename T, int VE> struct RawElems {
    T v[VE];
    LP_DEVINL void load(const T *p)
    {
        constexpr int BYTES = VE * (int)sizeof(T);
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) reinterpret_cast<uint4 *>(v)[i] = reinterpret_cast<const uint4 *>(p)[i];
        } else if constexpr (BYTES == 8) *reinterpret_cast<uint2 *>(v) = *reinterpret_cast<const uint2 *>(p);
        else if constexpr (BYTES == 4) *reinterpret_cast<uint32_t *>(v) = *reinterpret_cast<const uint32_t *>(p);
        else v[0] = *p;
    }
    LP_DEVINL void add_to(float *acc) const
    {
#pragma unroll
        for (int t = 0; t < VE; ++t) acc[t] += to_f<T>(v[t]);
    }
};
template <typename T, int VE> struct alignas(16) RawAligned : RawElems<T, VE> {};

// Largest VE (a power of two, at most `most`) such that rows of D elements at `base` with pitch ld can be read in aligned
// pieces of VE elements.
static int elems_per_piece(const void *base, int64_t ld, int D, size_t elem, int most)
{
    int ve = most;
    while (ve > 1 && (D % ve != 0 || ld % ve != 0 || (uintptr_t)base % std::min<size_t>(16, ve * elem) != 0)) ve >>= 1;
    return ve;
}

// Pieces of VE elements that a lane handles at a time, G * VE columns apart: four elements at least, so that rows whose width or
// address only allows narrow pieces have as many loads in flight as the others (gradient from 200,000 rows of 257 floats: 220 us
// with one piece, 180 so; of 101: 120 and 91)
template <int VE> constexpr int PIECES_PER_LANE = VE >= 4 ? 1 : 4 / VE;

// lanes that share a row: the smallest power of two in 8..32 that covers the row's pieces in one step
static int lanes_per_row(int pieces) { return pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32; }

// ---------------------------------------------------------------------------------------------
// lookup.  A group of G lanes takes four ids at a time, so four row loads are in flight per lane.  Bound by the bytes of the rows
// read and written: 196,608 ids, rows of 256 floats out of 1,000,000, stored as BF16, take 42 us, 303 MB at 7.1 TB/s (rows named
// twice come from L2; a plain copy of as many bytes takes 46 us).  768 rows of 64 floats take 2.3 us on the device, of 8 us that
// the call takes from Python.
// ---------------------------------------------------------------------------------------------
constexpr int EMB_THREADS = 256;
constexpr int EMB_ROWS = 4;

template <typename TT, typename TO, int VE, int U>
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
    for (int c0 = gl * VE; c0 < D; c0 += U * G * VE) {
        float v[EMB_ROWS][U][VE];
#pragma unroll
        for (int r = 0; r < EMB_ROWS; ++r) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * G * VE;
                if (live[r] && c < D) {
                    load_elems<TT, VE>(table + (int64_t)id[r] * ldt + c, v[r][u]);
                } else {
#pragma unroll
                    for (int t = 0; t < VE; ++t) v[r][u][t] = 0.f;
                }
            }
        }
#pragma unroll
        for (int r = 0; r < EMB_ROWS; ++r) {
            if (i0 + r >= N) continue;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * G * VE;
                if (c >= D) continue;
                if (live[r]) {
#pragma unroll
                    for (int t = 0; t < VE; ++t) v[r][u][t] *= scale;
                }
                store_elems<TO, VE>(out + (i0 + r) * ldo + c, v[r][u]);
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
#define LP_EMBED(VE_, U_) launch_dep(embed_kernel<TT, TO, VE_, U_>, grid, block, 0, ex.st, table, V, D, ldt, ids, N, padding, scale, out, ldo, G, err)
    // several pieces per lane pay for rows of floats wider than three pieces (200,000 rows of 257: 94 us with one, 76 with four; of
    // 33: 21 and 27) and not for rows of BF16 (257: 68 and 107)
    const bool several = sizeof(TT) == 4 && D >= 96;
    if (ve == 8) { if constexpr (most == 8) LP_EMBED(8, 1); }
    else if (ve == 4) LP_EMBED(4, 1);
    else if (ve == 2) { if (several) LP_EMBED(2, 2); else LP_EMBED(2, 1); }
    else if (several && sizeof(TO) == 4) LP_EMBED(1, 4);
    else LP_EMBED(1, 1);
#undef LP_EMBED
    ex.launches += 1;
}

// ---------------------------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------------------------
constexpr int EG_THREADS = 256;
constexpr int EG_CHUNK = 32;  // consecutive sorted ids that one group of lanes adds up
constexpr int EG_BATCH = 8;   // rows of dout requested together
constexpr int EG_PIECES = 8;  // chunks (or pieces of a list) that are joined in shared memory: fixed, so that the order of the
                              // additions, and with it every bit, is the same for every row width, pitch and alignment
constexpr int EG_SPAN = EG_PIECES * EG_CHUNK;
constexpr int EG_JOIN = 32;   // spans that one block looks at for runs to join
constexpr int EG_SHORT = 16;  // spans up to which a run is added up by one group of lanes

// Sorting.  Least significant digit first, up to eight bits a pass, one launch a pass: a block takes a tile of 2,048 pairs
// (by ticket, so it only waits for tiles that are running, and not beyond the context's limit), ranks them by digit, finds what
// earlier tiles hold of each digit by looking back over their published counts (eight at a time; thread d looks for digit d), and
// writes its pairs in digit order.
// The pass is bound by latency (1,966,080 pairs: 29 to 38 us, 200,000: 10 to 12).  Tried and no faster: nine-bit digits (200,000 ids
// 78 us for 80 in all, 1,966,080 ids 495 for 473), tiles of 4,096 pairs (86 for 80, 481 for 473).  The rows that no id
// names were once set to zero by further blocks of these launches: with 1,966,080 ids that hides nothing (234 us together, 101 and
// 110 alone), with fewer ids a part (96,035 ids, 701,850 rows of 64: 70 us so, 76 now), but noting the named rows before the sort
// takes a store per id, and they queue up at the lines of the hubs (849,408 ids on 2,749 rows: 96 us with the counts, 6 without).
// So the kernel that adds up the sorted rows notes them, once per run of equal ids, and the last launch sets the others to
// zero (200,001 ids: 80 -> 76 us; 849,408 on 2,749 rows: 229 -> 139).
constexpr int ES_ITEMS = 8;
constexpr int ES_TILE = EG_THREADS * ES_ITEMS;
constexpr int ES_DIGITS = 256;
constexpr unsigned ES_SUM = 1u << 30, ES_PREFIX = 2u << 30, ES_COUNT = (1u << 30) - 1;  // of a tile alone, of all tiles up to it

struct EmbedSort {
    int passes = 0, bits = 0;      // bits per pass
    int tiles = 0;
    uint32_t *keys[2] = {nullptr, nullptr}, *vals[2] = {nullptr, nullptr};
    uint8_t *named = nullptr;      // [rows] row v receives a gradient      } cleared together before the call's first kernel
    unsigned *hist = nullptr;      // [passes][256] keys per digit        }
    unsigned *ticket = nullptr;    // [passes]                            }
    unsigned *status = nullptr;    // [passes][tiles][256], cleared by the first kernel
    unsigned long long wait_ns = 0;  // limit of a tile's wait for the tiles before it
    int withhold = 0;              // self-test of that limit: the first tile of the first pass publishes nothing
};

// the key of an id: the id, or V (sorted behind every row) for the padding id and for ids outside the table
LP_DEVINL uint32_t embed_key(int id, int64_t V, int padding) { return id >= 0 && id < V && id != padding ? (uint32_t)id : (uint32_t)V; }

__global__ void __launch_bounds__(EG_THREADS) embed_hist_kernel(const int *__restrict__ ids, int64_t N, int64_t V, int padding, const EmbedSort s, int *__restrict__ err)
{
    LP_DEP_ENTER();
    __shared__ unsigned h[4][ES_DIGITS];
    for (int p = 0; p < s.passes; ++p) h[p][threadIdx.x] = 0;
    const int64_t words = (int64_t)s.passes * s.tiles * ES_DIGITS;
    for (int64_t i = (int64_t)blockIdx.x * EG_THREADS + threadIdx.x; i < words; i += (int64_t)gridDim.x * EG_THREADS) s.status[i] = 0;
    __syncthreads();
    const uint32_t mask = (1u << s.bits) - 1;
    int id[ES_ITEMS];
#pragma unroll
    for (int r = 0; r < ES_ITEMS; ++r) {
        const int64_t i = (int64_t)blockIdx.x * ES_TILE + r * EG_THREADS + threadIdx.x;
        id[r] = i < N ? ids[i] : -1;
    }
#pragma unroll
    for (int r = 0; r < ES_ITEMS; ++r) {
        if ((int64_t)blockIdx.x * ES_TILE + r * EG_THREADS + threadIdx.x < N) {
            const uint32_t key = embed_key(id[r], V, padding);
            if (key == (uint32_t)V && (id[r] != padding || padding == LP_NO_PADDING)) atomicOr(err, 1);
            for (int p = 0; p < s.passes; ++p) atomicAdd(&h[p][(key >> (p * s.bits)) & mask], 1u);
        }
    }
    __syncthreads();
    for (int p = 0; p < s.passes; ++p)
        if (h[p][threadIdx.x]) atomicAdd(s.hist + p * ES_DIGITS + threadIdx.x, h[p][threadIdx.x]);
}

// sets the rows that no id names to zero; `blocks` blocks share the work.  A warp reads the flags of 32
// rows at once and then only stores (a load per row: 218 us for 2.9 M rows of 512 bytes, this way 110 us)
template <typename TG, int VE>
LP_DEVINL void embed_zero_rows(const uint8_t *named, int64_t V, int D, TG *grad, int64_t ldg, int G, int block, int blocks)
{
    const int lane = threadIdx.x & 31, gl = lane & (G - 1), sub = lane / G, step = 32 / G;
    const int64_t warps = (int64_t)blocks * (EG_THREADS / 32), w1 = (V + 31) / 32;
    constexpr int ZE = VE * (int)sizeof(TG) > 16 ? 16 / (int)sizeof(TG) : VE;  // neighbouring lanes store neighbouring 16 bytes
    float z[ZE];
#pragma unroll
    for (int t = 0; t < ZE; ++t) z[t] = 0.f;
    int64_t w = (int64_t)block * (EG_THREADS / 32) + (threadIdx.x >> 5);
    uint32_t flag = w < w1 && w * 32 + lane < V ? named[w * 32 + lane] : 0u;
    while (w < w1) {
        const uint32_t next = w + warps < w1 && (w + warps) * 32 + lane < V ? named[(w + warps) * 32 + lane] : 0u;
        const uint32_t word = __ballot_sync(0xffffffffu, flag != 0u);
        const int rows = (int)min((int64_t)32, V - w * 32);
        TG *p = grad + (w * 32 + sub) * ldg;
        for (int r = sub; r < rows; r += step, p += (int64_t)step * ldg) {
            if ((word >> r) & 1u) continue;
            for (int c = gl * ZE; c < D; c += G * ZE) store_elems<TG, ZE>(p + c, z);
        }
        w += warps;
        flag = next;
    }
}

__global__ void __launch_bounds__(EG_THREADS) embed_sort_kernel(const int *__restrict__ ids, int64_t N, int64_t V, int padding, const EmbedSort s, int pass, int *__restrict__ err)
{
    LP_DEP_ENTER();
    __shared__ int warp_count[EG_THREADS / 32][ES_DIGITS];
    __shared__ int start_s[ES_DIGITS];               // where a digit begins in the tile's own order
    __shared__ int out_s[ES_DIGITS];                 // ... and its first place in the output, less start_s
    __shared__ uint32_t key_s[ES_TILE], val_s[ES_TILE];
    __shared__ int sw[8];
    __shared__ int tile_s;
    if (threadIdx.x == 0) tile_s = (int)atomicAdd(s.ticket + pass, 1u);
#pragma unroll
    for (int w = 0; w < EG_THREADS / 32; ++w) warp_count[w][threadIdx.x] = 0;
    __syncthreads();
    const int tile = tile_s, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int shift = pass * s.bits;
    const uint32_t mask = (1u << s.bits) - 1;
    const uint32_t *keys = pass & 1 ? s.keys[0] : s.keys[1], *vals = pass & 1 ? s.vals[0] : s.vals[1];  // the first pass reads the ids and writes set 0
    uint32_t key[ES_ITEMS], val[ES_ITEMS];
    int rank[ES_ITEMS];
    const int64_t base = (int64_t)tile * ES_TILE + warp * (32 * ES_ITEMS) + lane;  // a warp's pairs are consecutive: ranks keep the order
#pragma unroll
    for (int r = 0; r < ES_ITEMS; ++r) {
        const int64_t i = base + r * 32;
        if (i < N) {
            key[r] = pass == 0 ? embed_key(ids[i], V, padding) : keys[i];
            val[r] = pass == 0 ? (uint32_t)i : vals[i];
        }
    }
#pragma unroll
    for (int r = 0; r < ES_ITEMS; ++r) {
        const bool live = base + r * 32 < N;
        const unsigned digit = live ? (key[r] >> shift) & mask : ES_DIGITS;  // places behind the end match one another only
        const unsigned peers = __match_any_sync(0xffffffffu, digit);
        const int before = __popc(peers & ((1u << lane) - 1u));
        int have = 0;
        if (live) have = warp_count[warp][digit];
        __syncwarp();
        if (live && before == 0) warp_count[warp][digit] = have + __popc(peers);
        __syncwarp();
        rank[r] = have + before;
    }
    __syncthreads();
    const int d = threadIdx.x;
    int total = 0;
#pragma unroll
    for (int w = 0; w < EG_THREADS / 32; ++w) {
        const int c = warp_count[w][d];
        warp_count[w][d] = total;
        total += c;
    }
    unsigned *mine = s.status + ((int64_t)pass * s.tiles + tile) * ES_DIGITS + d;
    if (!s.withhold || tile > 0 || pass > 0)
        asm volatile("st.relaxed.gpu.global.u32 [%0], %1;" ::"l"(mine), "r"((tile == 0 ? ES_PREFIX : ES_SUM) | (unsigned)total) : "memory");
    int sum;
    const int start = block_exclusive_scan_256(total, sw, &sum);
    const int digit_base = block_exclusive_scan_256((int)s.hist[pass * ES_DIGITS + d], sw, &sum);
    start_s[d] = start;
#pragma unroll
    for (int r = 0; r < ES_ITEMS; ++r) rank[r] += base + r * 32 < N ? warp_count[warp][(key[r] >> shift) & mask] : 0;
    // look back
    unsigned prefix = 0;
    if (tile > 0) {
        int t = tile - 1;
        unsigned long long t0 = 0;
        bool done = false;
        while (!done) {
            unsigned w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[j] = ES_PREFIX;
                if (t - j >= 0) asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(w[j]) : "l"(mine - (int64_t)(tile - (t - j)) * ES_DIGITS) : "memory");
            }
            int used = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (done || used < j || (w[j] >> 30) == 0) continue;  // in order, up to the first one that is not there yet
                prefix += w[j] & ES_COUNT;
                used = j + 1;
                done = (w[j] >> 30) == 2;
            }
            t -= used;
            if (used == 0) {
                unsigned long long now;
                asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
                if (t0 == 0) t0 = now;
                else if (now - t0 > s.wait_ns) {  // give up, report, carry on: places outside the arrays are not written, and places that
                                                  // nobody writes hold anything, which the sums check before they use it
                    atomicOr(err, 2);
                    done = true;
                }
            }
        }
        asm volatile("st.relaxed.gpu.global.u32 [%0], %1;" ::"l"(mine), "r"(ES_PREFIX | (prefix + (unsigned)total)) : "memory");
    }
    out_s[d] = digit_base + (int)prefix - start;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ES_ITEMS; ++r) {
        if (base + r * 32 < N) {
            const int at = start_s[(key[r] >> shift) & mask] + rank[r];
            key_s[at] = key[r];
            val_s[at] = val[r];
        }
    }
    __syncthreads();
    const int count = (int)min((int64_t)ES_TILE, N - (int64_t)tile * ES_TILE);
    uint32_t *keys_out = pass & 1 ? s.keys[1] : s.keys[0], *vals_out = pass & 1 ? s.vals[1] : s.vals[0];
    for (int i = threadIdx.x; i < count; i += EG_THREADS) {
        const uint32_t k = key_s[i];
        const int64_t o = out_s[(k >> shift) & mask] + i;
        if (o < N) {
            keys_out[o] = k;
            vals_out[o] = val_s[i];
        }
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

// A group of G lanes adds the rows of EG_CHUNK consecutive sorted ids.  A run of equal ids inside the chunk is written to the
// gradient; runs that cross chunks of a span are joined in shared memory, and what crosses spans goes out unscaled in FP32:
// the part of a run that began in an earlier span to head[span], the part of one that begins here and goes on to tail[span].
// Bound by HBM: 1,966,080 BF16 rows of 128 read in sorted order, which is no order in memory, and the FP32 rows of 1.0 M ids
// written, 1.0 GB, take 186 us = 5.5 TB/s at 80 registers (rows wait as they lie in memory, EG_BATCH of them; as floats: 128
// registers and 330 us).  Dividing by ids and not by rows of the table is what keeps a hub's thousands of ids from one warp.
template <typename TD, typename TG, int VE>
__global__ void __launch_bounds__(EG_THREADS, 3) embed_grad_sum_kernel(const uint32_t *__restrict__ keys, const uint32_t *__restrict__ vals, int64_t N, int64_t V,
                                                                    const TD *__restrict__ dout, int64_t ldd, int D, float scale, TG *__restrict__ grad,
                                                                    int64_t ldg, int accumulate, float *__restrict__ head, float *__restrict__ tail, uint8_t *__restrict__ named, int G)
{
    LP_DEP_ENTER();
    constexpr int U = PIECES_PER_LANE<VE>, E = U * VE;
    __shared__ __align__(16) float head_s[EG_THREADS * E], tail_s[EG_THREADS * E];
    __shared__ uint32_t key_s[EG_THREADS / 8 * EG_CHUNK], val_s[EG_THREADS / 8 * EG_CHUNK];  // the block's sorted ids
    const int gl = threadIdx.x & (G - 1), group = threadIdx.x / G, g = group % EG_PIECES;
    const int64_t span = (int64_t)blockIdx.x * (EG_THREADS / G / EG_PIECES) + group / EG_PIECES;
    const int64_t span1 = min(N, (span + 1) * EG_SPAN);
    const int64_t p0 = span * EG_SPAN + (int64_t)g * EG_CHUNK;
    const int count = (int)max((int64_t)0, min((int64_t)EG_CHUNK, N - p0));
    const uint32_t none = 0xFFFFFFFFu;
    const uint32_t before = count > 0 && p0 > 0 ? keys[p0 - 1] : none, after = count > 0 && p0 + count < N ? keys[p0 + count] : none;
    const int64_t b0 = (int64_t)blockIdx.x * (EG_THREADS / G) * EG_CHUNK;
    const int ids = (int)min((int64_t)(EG_THREADS / G) * EG_CHUNK, N - b0);
    for (int i = threadIdx.x; i < ids; i += EG_THREADS) {
        const uint32_t val = vals[b0 + i];
        key_s[i] = val < (uint32_t)N ? keys[b0 + i] : (uint32_t)V;  // no such position: the sort gave up a wait (reported), the pair was never written
        val_s[i] = val;
    }
    __syncthreads();
    if (named && blockIdx.y == 0)  // rows with a gradient, at the first id of each
        for (int i = threadIdx.x; i < ids; i += EG_THREADS) {
            const uint32_t key = key_s[i];
            if (key < (uint32_t)V && (i > 0 ? key_s[i - 1] != key : b0 == 0 || keys[b0 - 1] != key)) named[key] = 1;
        }
    const uint32_t *ck = key_s + group * EG_CHUNK, *cv = val_s + group * EG_CHUNK;
    const uint32_t first = count > 0 ? ck[0] : none;
    // E sums of this lane to shared memory, to a row of FP32 partial sums, to the gradient
    auto keep = [&](float *to, const float *acc) {
#pragma unroll
        for (int u = 0; u < U; ++u) store_elems<float, VE>(to + threadIdx.x * E + u * VE, acc + u * VE);
    };
    for (int c0 = blockIdx.y * U * G * VE; c0 < D; c0 += gridDim.y * U * G * VE) {
        const int c = c0 + gl * VE;
        auto put = [&](float *row, const float *acc) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c + u * G * VE < D) store_elems<float, VE>(row + c + u * G * VE, acc + u * VE);
        };
        auto finish = [&](uint32_t v, const float *acc) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c + u * G * VE < D) embed_grad_store<TG, VE>(grad + (int64_t)v * ldg + c + u * G * VE, acc + u * VE, scale, accumulate != 0);
        };
        uint32_t open = none;  // the run that begins in this chunk, or before the span, and goes on
        if (count > 0 && c < D) {
            uint32_t cur = first;
            bool from_before = before == first;
            float acc[E];
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] = 0.f;
            for (int b = 0; b < count; b += EG_BATCH) {
                RawAligned<TD, VE> x[EG_BATCH][U];
#pragma unroll
                for (int j = 0; j < EG_BATCH; ++j)
                    if (b + j < count && ck[b + j] < (uint32_t)V) {
                        const TD *row = dout + (int64_t)cv[b + j] * ldd + c;
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            if (c + u * G * VE < D) x[j][u].load(row + u * G * VE);
                    }
#pragma unroll
                for (int j = 0; j < EG_BATCH; ++j) {
                    const uint32_t key = b + j < count ? ck[b + j] : (uint32_t)V;
                    if (key != cur) {
                        if (cur < (uint32_t)V) {
                            if (from_before) keep(head_s, acc);
                            else finish(cur, acc);
                        }
                        from_before = false;
                        cur = key;
#pragma unroll
                        for (int t = 0; t < E; ++t) acc[t] = 0.f;
                    }
                    if (key < (uint32_t)V) {
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            if (c + u * G * VE < D) x[j][u].add_to(acc + u * VE);
                    }
                }
            }
            if (cur < (uint32_t)V) {
                if (from_before) keep(head_s, acc);
                else if (after == cur) { keep(tail_s, acc); open = cur; }
                else finish(cur, acc);
            }
        }
        __syncthreads();
        // a run is finished by the group in whose chunk it begins; one that came in from an earlier span by its first group
        const bool came_in = g == 0 && count > 0 && before == first && first < (uint32_t)V;
        if ((open != none || came_in) && c < D) {
            const uint32_t run = came_in ? first : open;
            float acc[E];
            auto gather = [&](const float *own, uint32_t r) {  // this chunk's part and those of the chunks behind it that begin with the run
#pragma unroll
                for (int t = 0; t < E; ++t) acc[t] = own[threadIdx.x * E + t];
                int64_t q = p0 + EG_CHUNK;
                for (int o = g + 1; q < span1 && keys[q] == r; ++o, q += EG_CHUNK) {
#pragma unroll
                    for (int t = 0; t < E; ++t) acc[t] += head_s[((group - g + o) * G + gl) * E + t];
                }
            };
            auto goes_on = [&](uint32_t r) { return span1 < N && keys[span1 - 1] == r && keys[span1] == r; };
            gather(came_in ? head_s : tail_s, run);
            if (came_in) put(head + span * D, acc);
            else if (goes_on(run)) put(tail + span * D, acc);
            else finish(run, acc);
            if (came_in && open != none) {  // the first group may hold both: the run that came in and ended, and one that begins in its chunk and goes on
                gather(tail_s, open);
                if (goes_on(open)) put(tail + span * D, acc);
                else finish(open, acc);
            }
        }
        __syncthreads();
    }
}

// Runs that cross spans: for every span in which such a run begins, grad[run] = tail[span] + head[span + 1] + ...  A block
// looks at EG_JOIN spans; runs over few spans are added up by a group of lanes each, the others by EG_PIECES groups that
// take equal stretches.  Blocks from `joins` on set the rows that no id names to zero meanwhile: the joins are a chain of loads.
template <typename TG, int VE>
__global__ void __launch_bounds__(EG_THREADS) embed_grad_join_kernel(const uint32_t *__restrict__ keys, int64_t N, int64_t V, int D, float scale, TG *__restrict__ grad,
                                                                     int64_t ldg, int accumulate, const float *__restrict__ head, const float *__restrict__ tail, const uint8_t *__restrict__ named,
                                                                     int joins, int G)
{
    LP_DEP_ENTER();
    if ((int)blockIdx.x >= joins) {
        embed_zero_rows<TG, VE>(named, V, D, grad, ldg, G, (blockIdx.x - joins) * gridDim.y + blockIdx.y, (gridDim.x - joins) * gridDim.y);
        return;
    }
    __shared__ __align__(16) float part_s[EG_THREADS * VE];
    __shared__ uint32_t run_s[EG_JOIN];
    __shared__ int64_t last_s[EG_JOIN];  // last span of the run that begins in span i and goes on; -1: none
    const int gl = threadIdx.x & (G - 1), g = threadIdx.x / G, groups = EG_THREADS / G;
    const int64_t first = (int64_t)blockIdx.x * EG_JOIN;
    if (threadIdx.x < EG_JOIN) {
        const int64_t span = first + threadIdx.x, p1 = (span + 1) * EG_SPAN;
        int64_t last = -1;
        uint32_t key = 0;
        if (p1 < N) {
            key = keys[p1 - 1];
            const uint32_t next = keys[p1], begin = keys[p1 - EG_SPAN], before = span > 0 ? keys[p1 - EG_SPAN - 1] : 0xFFFFFFFFu;
            if (key < (uint32_t)V && next == key && !(begin == key && before == key)) {
                int64_t lo = span + 1, hi = (N + EG_SPAN - 1) / EG_SPAN;  // the first span behind that does not begin with the key
                for (int64_t step = 1; lo + step < hi && keys[(lo + step) * EG_SPAN] == key; step <<= 1) lo += step;
                while (lo + 1 < hi) {
                    const int64_t mid = (lo + hi) >> 1;
                    if (keys[mid * EG_SPAN] == key) lo = mid; else hi = mid;
                }
                last = lo;
            }
        }
        run_s[threadIdx.x] = key;
        last_s[threadIdx.x] = last;
    }
    __syncthreads();
    for (int i = g; i < EG_JOIN; i += groups) {
        const int64_t span = first + i, last = last_s[i];
        if (last < 0 || last - span > EG_SHORT) continue;
        for (int c = (blockIdx.y * G + gl) * VE; c < D; c += gridDim.y * G * VE) {
            float acc[VE];
            load_elems<float, VE>(tail + span * D + c, acc);
            for (int64_t q = span + 1; q <= last; ++q) {
                float x[VE];
                load_elems<float, VE>(head + q * D + c, x);
#pragma unroll
                for (int t = 0; t < VE; ++t) acc[t] += x[t];
            }
            embed_grad_store<TG, VE>(grad + (int64_t)run_s[i] * ldg + c, acc, scale, accumulate != 0);
        }
    }
    for (int i = 0; i < EG_JOIN; ++i) {
        const int64_t span = first + i, last = last_s[i];
        if (last < 0 || last - span <= EG_SHORT) continue;
        const int64_t share = (last - span + EG_PIECES - 1) / EG_PIECES, q0 = span + 1 + g * share, q1 = g < EG_PIECES ? min(last + 1, q0 + share) : q0;
        for (int c0 = blockIdx.y * G * VE; c0 < D; c0 += gridDim.y * G * VE) {
            const int c = c0 + gl * VE;
            float acc[VE];
#pragma unroll
            for (int t = 0; t < VE; ++t) acc[t] = 0.f;
            if (c < D) {
                if (g == 0) load_elems<float, VE>(tail + span * D + c, acc);
                for (int64_t q = q0; q < q1; q += EG_BATCH) {
                    float x[EG_BATCH][VE];
#pragma unroll
                    for (int j = 0; j < EG_BATCH; ++j)
                        if (q + j < q1) load_elems<float, VE>(head + (q + j) * D + c, x[j]);
#pragma unroll
                    for (int j = 0; j < EG_BATCH; ++j) {
                        if (q + j < q1) {
#pragma unroll
                            for (int t = 0; t < VE; ++t) acc[t] += x[j][t];
                        }
                    }
                }
            }
            store_elems<float, VE>(part_s + threadIdx.x * VE, acc);
            __syncthreads();
            if (g == 0 && c < D) {
                for (int o = 1; o < EG_PIECES; ++o) {
                    float x[VE];
                    load_elems<float, VE>(part_s + (o * G + gl) * VE, x);
#pragma unroll
                    for (int t = 0; t < VE; ++t) acc[t] += x[t];
                }
                embed_grad_store<TG, VE>(grad + (int64_t)run_s[i] * ldg + c, acc, scale, accumulate != 0);
            }
            __syncthreads();
        }
    }
}

// rows that no id names, where there are no ids at all
template <typename TG, int VE>
__global__ void __launch_bounds__(EG_THREADS) embed_grad_zero_kernel(const uint8_t *__restrict__ named, int64_t V, int D, TG *__restrict__ grad, int64_t ldg, int G)
{
    LP_DEP_ENTER();
    embed_zero_rows<TG, VE>(named, V, D, grad, ldg, G, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------------------------------------
// the gradient for few ids, in one launch: a block owns `R` rows of the table, picks the ids that name them out of all ids,
// sorts those by (row, position) in shared memory, sets its other rows to zero and adds up its own.
// ---------------------------------------------------------------------------------------------
constexpr int EGS_MAX_IDS = 8192;  // 13 bits of a key, the row takes the other 13
constexpr int EGS_MAX_ROWS = 8192;

template <typename TD, typename TG, int VE>
__global__ void __launch_bounds__(EG_THREADS) embed_grad_few_kernel(const int *__restrict__ ids, int N, int64_t V, int padding, int R, const TD *__restrict__ dout, int64_t ldd,
                                                                    int D, float scale, TG *__restrict__ grad, int64_t ldg, int accumulate, int G, int *__restrict__ err)
{
    LP_DEP_ENTER();
    extern __shared__ uint32_t list[];                // (row - r0) << 13 | position
    __shared__ uint32_t named[EGS_MAX_ROWS / 32];
    constexpr int PU = PIECES_PER_LANE<VE>, E = PU * VE;
    __shared__ __align__(16) float head[EG_THREADS * E], tail[EG_THREADS * E];
    __shared__ int count_s;
    const int64_t r0 = (int64_t)blockIdx.x * R, r1 = min(r0 + R, V);
    for (int i = threadIdx.x; i < (R + 31) / 32; i += EG_THREADS) named[i] = 0;
    if (threadIdx.x == 0) count_s = 0;
    __syncthreads();
    constexpr int U = 4;
    for (int i0 = threadIdx.x; i0 < N; i0 += U * EG_THREADS) {
        int id[U];
#pragma unroll
        for (int u = 0; u < U; ++u) id[u] = i0 + u * EG_THREADS < N ? ids[i0 + u * EG_THREADS] : -1;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * EG_THREADS;
            if (i >= N) continue;
            const uint32_t key = embed_key(id[u], V, padding);
            if (key == (uint32_t)V) {
                if (blockIdx.x == 0 && (id[u] != padding || padding == LP_NO_PADDING)) atomicOr(err, 1);
            } else if (key >= r0 && key < r1) {
                const int row = (int)(key - r0);
                list[atomicAdd(&count_s, 1)] = (uint32_t)row << 13 | (uint32_t)i;
                atomicOr(&named[row >> 5], 1u << (row & 31));
            }
        }
    }
    __syncthreads();
    const int M = count_s;
    const int gl = threadIdx.x & (G - 1), g = threadIdx.x / G, groups = EG_THREADS / G;
    if (!accumulate) {
        float z[VE];
#pragma unroll
        for (int t = 0; t < VE; ++t) z[t] = 0.f;
        for (int64_t v = r0 + g; v < r1; v += groups) {
            const int row = (int)(v - r0);
            if ((named[row >> 5] >> (row & 31)) & 1u) continue;
            for (int c = gl * VE; c < D; c += G * VE) store_elems<TG, VE>(grad + v * ldg + c, z);
        }
    }
    if (M == 0) return;
    int P = 2;
    while (P < M) P <<= 1;
    for (int i = M + threadIdx.x; i < P; i += EG_THREADS) list[i] = 0xFFFFFFFFu;
    __syncthreads();
    for (int k = 2; k <= P; k <<= 1) {
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int i = threadIdx.x; i < P / 2; i += EG_THREADS) {
                const int a = 2 * i - (i & (j - 1)), b = a + j;  // pairs j apart; ascending where bit k of a is clear
                const uint32_t x = list[a], y = list[b];
                if ((x > y) == ((a & k) == 0)) { list[a] = y; list[b] = x; }
            }
            __syncthreads();
        }
    }
    // the sorted list is cut into pieces, one group of lanes each; runs that cross pieces are joined through shared memory
    const int per = (M + EG_PIECES - 1) / EG_PIECES, a0 = g < EG_PIECES ? min(M, g * per) : M, a1 = min(M, a0 + per);
    const uint32_t none = 0xFFFFFFFFu;
    const uint32_t before = a0 > 0 && a0 < a1 ? list[a0 - 1] >> 13 : none, after = a1 < M && a0 < a1 ? list[a1] >> 13 : none;
    auto keep = [&](float *to, const float *acc) {
#pragma unroll
        for (int t = 0; t < E; ++t) to[threadIdx.x * E + t] = acc[t];
    };
    for (int c0 = 0; c0 < D; c0 += PU * G * VE) {
        const int c = c0 + gl * VE;
        auto finish = [&](uint32_t row, const float *acc) {
#pragma unroll
            for (int u = 0; u < PU; ++u)
                if (c + u * G * VE < D) embed_grad_store<TG, VE>(grad + (r0 + row) * ldg + c + u * G * VE, acc + u * VE, scale, accumulate != 0);
        };
        uint32_t open = none;  // the run that began here and goes on
        if (a0 < a1 && c < D) {
            uint32_t cur = list[a0] >> 13;
            bool from_before = before == cur;
            float acc[E];
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] = 0.f;
            for (int b = a0; b < a1; b += EG_BATCH) {
                uint32_t k[EG_BATCH];
                RawAligned<TD, VE> x[EG_BATCH][PU];
#pragma unroll
                for (int j = 0; j < EG_BATCH; ++j) {
                    k[j] = b + j < a1 ? list[b + j] : none;
                    if (b + j < a1) {
#pragma unroll
                        for (int u = 0; u < PU; ++u)
                            if (c + u * G * VE < D) x[j][u].load(dout + (int64_t)(k[j] & 8191u) * ldd + c + u * G * VE);
                    }
                }
#pragma unroll
                for (int j = 0; j < EG_BATCH; ++j) {
                    if (b + j < a1) {
                        if ((k[j] >> 13) != cur) {
                            if (from_before) keep(head, acc);
                            else finish(cur, acc);
                            from_before = false;
                            cur = k[j] >> 13;
#pragma unroll
                            for (int t = 0; t < E; ++t) acc[t] = 0.f;
                        }
#pragma unroll
                        for (int u = 0; u < PU; ++u)
                            if (c + u * G * VE < D) x[j][u].add_to(acc + u * VE);
                    }
                }
            }
            if (from_before) keep(head, acc);
            else if (after == cur) { keep(tail, acc); open = cur; }
            else finish(cur, acc);
        }
        __syncthreads();
        if (open != none) {
            float acc[E];
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] = tail[threadIdx.x * E + t];
            for (int o = g + 1; o < EG_PIECES && o * per < M && (list[o * per] >> 13) == open; ++o) {
#pragma unroll
                for (int t = 0; t < E; ++t) acc[t] += head[(o * G + gl) * E + t];
            }
            finish(open, acc);
        }
        __syncthreads();
    }
}

// the list is sorted as a power of two of entries
static size_t few_bytes(int64_t N)
{
    size_t n = 2;
    while ((int64_t)n < N) n <<= 1;
    return n * sizeof(uint32_t);
}

// One launch for few ids (768 ids, 2,000 rows: 5.5 us against 31 for the sort; 8,192 ids: 15 against 31, all of one row 180
// against 27).  Where a block's range of rows is wide, ids that lie together land in few blocks (8,192 ids inside 5,000 of
// 2.9 M rows: 300 us against 150; 2,048: 137 against 150), so the limit is lower there.
static int few_rows(int64_t V) { return (int)std::min<int64_t>(EGS_MAX_ROWS, std::max<int64_t>(4, ceil_div64(V, 148 * 4))); }
static bool embed_grad_is_few(int64_t N, int64_t V) { return N > 0 && N <= (few_rows(V) <= 1024 ? EGS_MAX_IDS : EGS_MAX_IDS / 4); }

constexpr int64_t EG_CLEAR_BYTES = (int64_t)64 << 20;

struct EmbedGradScratch {
    EmbedSort sort;
    float *head = nullptr, *tail = nullptr;
    size_t clear_bytes = 0;  // from sort.named on
};

template <typename TD, typename TG, int VE>
static void embed_grad_rows(Exec &ex, const TD *dout, int64_t ldd, const int *ids, int64_t N, int padding, float scale, int64_t V, int D, TG *grad, int64_t ldg,
                            int accumulate, const EmbedGradScratch &sc, int *err)
{
    const EmbedSort &s = sc.sort;
    const int G = lanes_per_row((D + VE - 1) / VE);
    const int64_t groups = EG_THREADS / G;
    const int R = few_rows(V);
    const bool few = embed_grad_is_few(N, V);
    // A large dense gradient is cleared as a whole first where the rows without ids are nearly all of it and stores of a row are slow
    // or all that there is to do.  Few ids: 937,500 x 320 floats, 550 ids 201 -> 178 us, 1,087,079 x 46 BF16, 819 ids 86 -> 25, but with
    // a 53rd of 218,261 rows named 30 -> 35 and a 9th of 72,765 40 -> 57, since there the blocks' own sums hide the zeros.  Sorted ids,
    // pieces of four bytes: 1,654,733 x 37 floats, 227,613 ids 147 -> 127, but pieces of 16 bytes: 701,850 x 64, 96,035 ids 71 -> 82.
    const int64_t grad_bytes = V * D * (int64_t)sizeof(TG);
    const bool clear = !accumulate && N > 0 && ldg == D && grad_bytes >= EG_CLEAR_BYTES && (few ? 64 * N <= V : VE * sizeof(TG) <= 4 && 4 * N <= V);
    if (clear) cudaMemsetAsync(grad, 0, (size_t)grad_bytes, ex.st);
    if (few) {
        if (few_bytes(N) > 8192)  // beside the static arrays it may pass the default limit; if refused, the launch reports the error
            cudaFuncSetAttribute(embed_grad_few_kernel<TD, TG, VE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_bytes(EGS_MAX_IDS));
        launch_dep(embed_grad_few_kernel<TD, TG, VE>, dim3((unsigned)ceil_div64(V, R)), dim3(EG_THREADS), few_bytes(N), ex.st, ids, (int)N, V, padding, R, dout, ldd, D, scale, grad, ldg,
                   accumulate || clear, G, err);
        ex.launches += 1;
        return;
    }
    cudaMemsetAsync(s.named, 0, sc.clear_bytes, ex.st);
    if (N == 0) {
        launch_dep(embed_grad_zero_kernel<TG, VE>, dim3((unsigned)std::min<int64_t>(ceil_div64(V, 256), 148 * 8)), dim3(EG_THREADS), 0, ex.st, s.named, V, D, grad, ldg, G);
        ex.launches += 1;
        return;
    }
    launch_dep(embed_hist_kernel, dim3(s.tiles), dim3(EG_THREADS), 0, ex.st, ids, N, V, padding, s, err);
    for (int p = 0; p < s.passes; ++p)
        launch_dep(embed_sort_kernel, dim3(s.tiles), dim3(EG_THREADS), 0, ex.st, ids, N, V, padding, s, p, err);
    uint8_t *named = accumulate || clear ? nullptr : s.named;
    const int zero_blocks = named ? (int)std::min<int64_t>(ceil_div64(V, 256), 148 * 8) : 0;
    const uint32_t *keys = s.keys[(s.passes - 1) & 1], *vals = s.vals[(s.passes - 1) & 1];
    const int64_t spans = ceil_div64(N, EG_SPAN), sums = ceil_div64(spans, groups / EG_PIECES), joins = ceil_div64(spans, EG_JOIN);
    // few blocks share out the columns of wide rows as well (13,413 ids, rows of 450 floats: sums 40 -> 14 us, joins 16 -> 8)
    auto split = [&](int64_t blocks, int columns) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div64(D, columns), 148 * 4 / blocks)); };
    launch_dep(embed_grad_sum_kernel<TD, TG, VE>, dim3((unsigned)sums, split(sums, PIECES_PER_LANE<VE> * G * VE)), dim3(EG_THREADS), 0, ex.st, keys, vals, N, V, dout, ldd, D, scale, grad,
               ldg, accumulate, sc.head, sc.tail, named, G);
    const unsigned ways = split(joins, G * VE);
    launch_dep(embed_grad_join_kernel<TG, VE>, dim3((unsigned)joins + ceil_div64(zero_blocks, ways), ways), dim3(EG_THREADS), 0, ex.st, keys, N, V, D, scale, grad, ldg, accumulate, sc.head,
               sc.tail, named, (int)joins, G);
    ex.launches += 3 + s.passes;
}

template <typename TD, typename TG>
static void embed_grad_launch(Exec &ex, const TD *dout, int64_t ldd, const int *ids, int64_t N, int padding, float scale, int64_t V, int D, TG *grad, int64_t ldg,
                              int accumulate, const EmbedGradScratch &s, int *err)
{
    constexpr int most = sizeof(TD) == 4 ? 4 : 8;
    const int ve = std::min(elems_per_piece(dout, ldd, D, sizeof(TD), most), elems_per_piece(grad, ldg, D, sizeof(TG), most));
    if (ve == 8) { if constexpr (most == 8) embed_grad_rows<TD, TG, 8>(ex, dout, ldd, ids, N, padding, scale, V, D, grad, ldg, accumulate, s, err); }
    else if (ve == 4) embed_grad_rows<TD, TG, 4>(ex, dout, ldd, ids, N, padding, scale, V, D, grad, ldg, accumulate, s, err);
    else if (ve == 2) embed_grad_rows<TD, TG, 2>(ex, dout, ldd, ids, N, padding, scale, V, D, grad, ldg, accumulate, s, err);
    else embed_grad_rows<TD, TG, 1>(ex, dout, ldd, ids, N, padding, scale, V, D, grad, ldg, accumulate, s, err);
}
