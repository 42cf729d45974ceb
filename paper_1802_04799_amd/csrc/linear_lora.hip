// Projection of rows with a low-rank adapter chosen row by row:
//   y = act(x W^T + bias + scale_i (x A_i^T) B_i^T + residual),  i = adapter[row]
//
// Two launches.  The first makes the adapters' middle vectors h = scale_i A_i x.  The second is a matrix product whose
// reduction goes on, after the c channels, over the rank: the same accumulators take B_i h.  With few tiles the first launch makes
// h and the product in parts of the reduction, the second adds both up.  Many rows are bound by the matrix cores and what feeds
// them (8192 rows 4096 -> 4096 in bf16: 222 us without adapters, 1.24 PFLOP/s, 251 with 16 of rank 32), few by the weights' bytes and
// the two launches (64 rows 4096 -> 4096: 14.9 us without adapters, 19.8 with 32 of rank 16).
//
// Both types are the same kernels in bytes: a lane's operand of a 16x16 tile is 16 bytes, 8 bf16 of one
// v_mfma_f32_16x16x32_bf16 or 4 fp32 of four v_mfma_f32_16x16x4_f32, whose order of the reduction is that of the loads.
// Channels are the tile's rows and tokens its columns, so that a lane holds four adjacent channels of one token: what
// depends on the token (its adapter) is a select per lane.
//
// h lies in the workspace as the product's operands, 64 bytes for 16 ranks of a row.  In bf16 that is h in two parts,
// h = hi + lo with an error of 2^-17 of h, hi of 16 ranks and lo of 16 ranks as one MFMA of 32 against B twice: the middle
// vector costs no digits.
//
// Rows of a tile with different adapters: a pass per adapter in use, whose sums the tokens that have the adapter take and the
// others do not; blocks of 16 tokens without it are skipped.  No row is multiplied with another's adapter, not by zero either, so
// what an adapter holds (infinities, NaN) reaches no other row, and a row's bits do not depend on the rows beside it.  Of its own
// adapter an infinity in B meets both parts of h in bf16, of which one may be zero or of the other sign: a NaN then.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "tvg_device.h"
#include "tvg_internal.h"

namespace tvg {

namespace {

struct LoraArgs {
    const void *x, *w, *a, *b;
    const int32_t *adapter;
    const float *scale, *bias;
    const void *residual;
    void *y;
    unsigned char *h;                      // [rows][rblocks][64 bytes]
    float *parts;                          // [splits][rows][parts_row]
    int *order;                            // [rows]: the rows by adapter, or NULL
    int rows, c, k, adapters, rank, rblocks;
    int slots, shrink_groups;              // workgroups that share the adapters of a tile; all that make h
    int splits, chunks_per_split, parts_row;
    int act, wide_rows, wide_rank, wide_y, wide_y4;        // 16-byte rows of c, of rank, of y and the residual; groups of four of y
    int tiles_n;                           // channel tiles
    int tiles;
};

template <typename T> constexpr int kPer16 = 16 / (int)sizeof(T);      // elements of an operand

__device__ __forceinline__ void mma(const uint4v &a, const uint4v &b, float4v &acc, bf16_t)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, a), __builtin_bit_cast(bf16x8v, b), acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(const uint4v &a, const uint4v &b, float4v &acc, float)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), acc, 0, 0, 0);
}

// All pairs of MB blocks of channels and NB of tokens.  fp32 goes through the four products of a pair in four rounds, so that
// no MFMA waits for the one before it.
template <int MB, int NB> __device__ __forceinline__ void mma_all(const uint4v (&w)[MB], const uint4v (&x)[NB], float4v (&acc)[MB][NB], bf16_t)
{
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int m = 0; m < MB; ++m) mma(w[m], x[n], acc[m][n], bf16_t());
}
template <int MB, int NB> __device__ __forceinline__ void mma_all(const uint4v (&w)[MB], const uint4v (&x)[NB], float4v (&acc)[MB][NB], float)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int m = 0; m < MB; ++m)
                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[m][i]), __uint_as_float(x[n][i]), acc[m][n], 0, 0, 0);
}

// 16 bytes at any element (the hardware takes them as one access, a little slower where they lie across lines).
template <typename T> __device__ __forceinline__ uint4v load16(const T *p)
{
    uint4v v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
// 16 bytes of row p from element k on, zeros from element `end` on.
template <typename T> __device__ __forceinline__ uint4v load16(const T *p, int k, int end)
{
    if (k + kPer16<T> <= end) return load16(p + k);
    T v[kPer16<T>];
#pragma unroll
    for (int i = 0; i < kPer16<T>; ++i) v[i] = k + i < end ? p[k + i] : (T)0;
    return __builtin_bit_cast(uint4v, v);
}

// 16 bytes per lane from a buffer straight into LDS at `lds` + 16 lane.  In assembly because the compiler waits for all loads
// in flight before any LDS read that follows its own form; whoever reads the bytes waits with wait_loads.  (M0 is an output,
// so that the compiler knows that it has changed.  Five wait states: a vector instruction may have written an SGPR just before.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, const uint4v &rsrc, uint32_t uniform_offset)
{
    uint32_t m0;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds"
                 : "={m0}"(m0) : "s"(lds), "v"(offset), "s"(rsrc), "s"(uniform_offset) : "memory");
}

// until at most N younger memory operations are in flight
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

// until no LDS operation is in flight
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

constexpr uint32_t kBeyond = 0x80000000u;  // an offset outside of every buffer: a load returns zeros

// The product of 16 MB rows of w and 16 NB rows of x over a part of the reduction, by one wave: 128 bytes of every row at a
// time come straight into LDS of its own, DEPTH such chunks in flight, and no barrier.  (Loads in the operands' own layout,
// one row per lane, take a lookup of the cache per 16 bytes and reach 30 GB/s a CU; these take one per 128 bytes.)
template <typename T, int MB, int NB, int DEPTH> struct WaveProduct {
    static constexpr int kLoads = 2 * (MB + NB), kBytes = DEPTH * kLoads * 1024;
    static_assert((DEPTH - 1) * kLoads < 64, "the counter of loads in flight");
    uint32_t from[kLoads], row_bytes, end_bytes, piece;
    uint4v xbuf, wbuf;
    uint32_t lds;                          // address of the wave's part
    const unsigned char *at;

    // x, w: the first row of each, of `xrows` and `wrows` there are
    __device__ __forceinline__ void start(const void *x, int xrows, const void *w, int wrows, uint32_t row_bytes_, unsigned char *part, int lane)
    {
        row_bytes = row_bytes_;
        xbuf = raw_buffer(x, (uint32_t)min(xrows, 16 * NB) * row_bytes);
        wbuf = raw_buffer(w, (uint32_t)min(wrows, 16 * MB) * row_bytes);
        at = part;
        lds = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char *)part);
        const int lrow = lane >> 3;
        piece = ((lane & 7) ^ lrow) * 16;  // pieces permuted against bank conflicts
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = (i < 2 * NB ? i : i - 2 * NB) * 8 + lrow;
            from[i] = row < (i < 2 * NB ? xrows : wrows) ? row * row_bytes + piece : kBeyond;
        }
    }
    __device__ __forceinline__ void fetch(int chunk, int slot)
    {
        const uint32_t k = (uint32_t)chunk * 128;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            load_to_lds(lds + (slot * kLoads + i) * 1024, k + piece < end_bytes ? from[i] : kBeyond, i < 2 * NB ? xbuf : wbuf,
                        k < end_bytes ? k : 0);
    }
    // chunks first, first + step, ... below `chunks`
    __device__ __forceinline__ void run(int first, int step, int chunks, float4v (&acc)[MB][NB], int lane)
    {
        const int rsel = lane & 15, quad = lane >> 4;
        end_bytes = min(row_bytes, (uint32_t)chunks * 128);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) fetch(first + d * step, d);
        int slot = 0;
        for (int c = first; c < chunks; c += step) {
            wait_loads<(DEPTH - 1) * kLoads>();
            const unsigned char *p = at + slot * kLoads * 1024;
            uint4v x[2][NB], w[2][MB];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int o = rsel * 128 + (((s * 4 + quad) ^ (rsel & 7)) << 4);
#pragma unroll
                for (int n = 0; n < NB; ++n) x[s][n] = *reinterpret_cast<const uint4v *>(p + n * 2048 + o);
#pragma unroll
                for (int m = 0; m < MB; ++m) w[s][m] = *reinterpret_cast<const uint4v *>(p + (NB + m) * 2048 + o);
            }
            wait_reads();
            fetch(c + DEPTH * step, slot);
#pragma unroll
            for (int s = 0; s < 2; ++s) mma_all(w[s], x[s], acc, T());
            slot = slot + 1 == DEPTH ? 0 : slot + 1;
        }
        wait_loads<0>();                   // (the part is the caller's again)
    }
};
// Waves per workgroup, and as many chunks in flight as the LDS holds.
constexpr int product_waves(int mb, int nb) { return mb + nb <= 4 ? 8 : 4; }
constexpr int kAllLds = 152, kHalfLds = 76;                // KB that a workgroup takes: for one or two of them a CU
constexpr int product_depth(int mb, int nb, int waves, int kb)
{
    const int chunks = kb / waves / (2 * (mb + nb));
    return chunks < 1 ? 1 : chunks;
}

// The same for WIDE rows (whole 16-byte pieces) through LDS at `part`, and for any others.
template <typename T, int MB, int NB, int W, bool WIDE, int KB>
__device__ __forceinline__ void wave_product(const T *x0, int xrows, const T *w0, int wrows, int c, int first, int chunks, unsigned char *part,
                                             int lane, float4v (&acc)[MB][NB])
{
    if constexpr (WIDE) {
        WaveProduct<T, MB, NB, product_depth(MB, NB, W, KB)> p;
        p.start(x0, xrows, w0, wrows, (uint32_t)c * sizeof(T), part, lane);
        p.run(first, W, chunks, acc, lane);
    } else {
        // (a row of x beyond the last one is the last one again, a row of w zeros)
        constexpr int E = kPer16<T>;
        const int rsel = lane & 15, quad = lane >> 4;
        const auto chunk = [&](int k, bool whole) {
            uint4v xv[2][NB], wv[2][MB];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int at = k + s * 4 * E + quad * E;
#pragma unroll
                for (int m = 0; m < MB; ++m) {
                    const int r = m * 16 + rsel;
                    wv[s][m] = uint4v{0, 0, 0, 0};
                    if (r < wrows) wv[s][m] = whole ? load16(w0 + (size_t)r * c + at) : load16(w0 + (size_t)r * c, at, c);
                }
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const T *x = x0 + (size_t)min(n * 16 + rsel, xrows - 1) * c;
                    xv[s][n] = whole ? load16(x + at) : load16(x, at, c);
                }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) mma_all(wv[s], xv[s], acc, T());
        };
        int i = first;
        for (; i < chunks && (i + 1) * 8 * E <= c; i += W) chunk(i * 8 * E, true);
        if (i < chunks) chunk(i * 8 * E, false);
    }
}
template <typename T, int MB, int NB, int W, bool WIDE, int KB>
constexpr int kPartBytes = WIDE ? WaveProduct<T, MB, NB, product_depth(MB, NB, W, KB)>::kBytes : MB * NB * 1024;

template <int MB, int NB> __device__ __forceinline__ void clear(float4v (&acc)[MB][NB])
{
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[m][n] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
}

// A wave's accumulators to its part of LDS, and block e of all waves' sums back.
template <int MB, int NB> __device__ __forceinline__ void put_sums(unsigned char *part, int lane, const float4v (&acc)[MB][NB])
{
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n) reinterpret_cast<float4v *>(part)[(m * NB + n) * 64 + lane] = acc[m][n];
}
template <int W> __device__ __forceinline__ float4v get_sum(const unsigned char *lds, int part_bytes, int e, int lane)
{
    float4v t = reinterpret_cast<const float4v *>(lds)[e * 64 + lane];
#pragma unroll
    for (int v = 1; v < W; ++v) t += reinterpret_cast<const float4v *>(lds + v * part_bytes)[e * 64 + lane];
    return t;
}

// ---------------------------------------------------------------------------------------
// h = A_i x
// ---------------------------------------------------------------------------------------

// A token's adapter, -1 for none.
__device__ __forceinline__ int adapter_of(const LoraArgs &a, int row)
{
    const int i = row < a.rows ? a.adapter[row] : -1;
    return i >= 0 && i < a.adapters ? i : -1;
}

// The adapters of 64 N rows (a lane has every 64th) in the order of their first row: *found of them go to list.
template <int N> __device__ __forceinline__ int distinct_adapters(const int (&mine)[N], int lane, int *list)
{
    int found = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        int left = mine[n];
        uint64_t pending = __ballot(left >= 0);
        while (pending) {
            const int i = __builtin_amdgcn_readlane(left, __builtin_ctzll(pending));
            bool listed = false;
#pragma unroll
            for (int b = 0; b < n; ++b) listed = listed || __ballot(mine[b] == i) != 0;
            if (!listed) {
                if (lane == 0) list[found] = i;
                ++found;
            }
            pending &= ~__ballot(left == i);
        }
    }
    return found;
}

constexpr float kLargestBf16 = 0x1.FEp127f;

// h of NB blocks of 16 tokens and JB blocks of 16 ranks; the waves take 128 bytes of the reduction in turn and add up through
// LDS.  Adapters of the tile: every slots-th of them.  Bound by reading x, once per adapter of the tile: 8192 rows of 4096 (67 MB)
// with 16 adapters of rank 32, eight requests, 28 us, 2.4 TB/s.  h leaves in bf16 as two numbers, whose sum has an error of 2^-17.
template <typename T, int NB, int JB, int W, bool WIDE, int KB> __device__ __forceinline__ void shrink_tile(const LoraArgs &a, int b, unsigned char *lds)
{
    constexpr int kPart = kPartBytes<T, JB, NB, W, WIDE, KB>;
    static_assert(kPart >= NB * JB * 1024, "the sums lie where the chunks were");
    int *list = reinterpret_cast<int *>(lds + W * kPart), *count = list + 16 * NB;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rsel = lane & 15, quad = lane >> 4;
    const int jgroups = (a.rblocks + JB - 1) / JB;
    const int slot = b % a.slots;
    b /= a.slots;
    const int j0 = b % jgroups * JB, row0 = b / jgroups * 16 * NB;
    if (wave == 0) {
        const int mine[1] = {lane < 16 * NB ? adapter_of(a, row0 + lane) : -1};
        const int found = distinct_adapters<1>(mine, lane, list);
        if (lane == 0) *count = found;
    }
    __syncthreads();
    const T *x0 = static_cast<const T *>(a.x) + (size_t)row0 * a.c;
    unsigned char *part = lds + wave * kPart;
    for (int at = slot; at < *count; at += a.slots) {
        const int i = __builtin_amdgcn_readfirstlane(list[at]);
        const T *A = static_cast<const T *>(a.a) + ((size_t)i * a.rank + j0 * 16) * a.c;
        float4v acc[JB][NB];
        clear(acc);
        wave_product<T, JB, NB, W, WIDE, KB>(x0, a.rows - row0, A, min(a.rank - j0 * 16, 16 * JB), a.c, wave,
                                         (a.c + 8 * kPer16<T> - 1) / (8 * kPer16<T>), part, lane, acc);
        put_sums(part, lane, acc);
        __syncthreads();
        const float scale = a.scale ? a.scale[i] : 1.0f;
        for (int e = wave; e < NB * JB; e += W) {
            const int row = row0 + e % NB * 16 + rsel, j = j0 + e / NB;
            if (j >= a.rblocks || adapter_of(a, row) != i) continue;
            float4v h = get_sum<W>(lds, kPart, e, lane) * scale;
            // (beyond the rank A's rows are zeros, which an infinity of x or of the scale makes a NaN)
#pragma unroll
            for (int v = 0; v < 4; ++v) h[v] = j * 16 + quad * 4 + v < a.rank ? h[v] : 0.0f;
            unsigned char *to = a.h + ((size_t)row * a.rblocks + j) * 64;
            if constexpr (sizeof(T) == 4) *reinterpret_cast<float4v *>(to + quad * 16) = h;
            else {
                float f[4], lo[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    // (a finite number stays one: what bf16 would round to infinity has its largest number as upper part)
                    f[v] = __builtin_amdgcn_fmed3f(h[v], -kLargestBf16, kLargestBf16);
                    f[v] = fabsf(h[v]) < INFINITY ? f[v] : h[v];
                    const float d = h[v] - bf16_to_f32(f32_to_bf16(f[v]));
                    lo[v] = d == d ? d : 0.0f;             // (of an infinity the upper part is all)
                }
                *reinterpret_cast<uint2v *>(to + quad * 8) = Group4<bf16_t>::pack(f);
                *reinterpret_cast<uint2v *>(to + 32 + quad * 8) = Group4<bf16_t>::pack(lo);
            }
        }
        __syncthreads();
    }
}

// The rows in the order of their adapters (modulo kBins, rows without one last), for a product whose tiles then have few
// adapters each: 1200 rows of 150 requests with 24 adapters of rank 64, 2048 -> 8192, took 148 us in their own order and 97 in
// this one.  The order of rows of an adapter is left to chance: a row's result does not depend on its place.
constexpr int kBins = 2048, kBinsPerLane = 5;

// bins[bin] += 1 for every lane with `ok`; what it was before, every lane one more than the last.  Lanes of a run add up first:
// atomics of a wave on one address take their turns, 4096 rows of eight adapters 4 us.
__device__ __forceinline__ int count_up(int *bins, int bin, bool ok, int lane)
{
    uint64_t pending = __ballot(ok);
    int before = 0;
    for (int round = 0; round < 4 && pending; ++round) {
        const int first = __builtin_ctzll(pending), b = __builtin_amdgcn_readlane(bin, first);
        const uint64_t same = __ballot(ok && bin == b) & pending;
        int start = 0;
        if (lane == first) start = atomicAdd(&bins[b], __popcll(same));
        start = __builtin_amdgcn_readlane(start, first);
        if ((same >> lane) & 1) before = start + __popcll(same & ((1ull << lane) - 1));
        pending &= ~same;
    }
    if ((pending >> lane) & 1) before = atomicAdd(&bins[bin], 1);
    return before;
}

static_assert(512 * kBinsPerLane > kBins, "a lane for every bin");
template <int THREADS> constexpr size_t kOrderBytes = (THREADS * kBinsPerLane + THREADS / 64) * sizeof(int);
template <int THREADS> __device__ __forceinline__ void order_rows(const LoraArgs &a, unsigned char *lds)
{
    int *bins = reinterpret_cast<int *>(lds), *sums = bins + THREADS * kBinsPerLane;
    const int tid = threadIdx.x;
    // eight rows a lane at a time: their loads are under way together
    constexpr int kRows = 8;
    const auto bins_of = [&](int r0, int (&bin)[kRows]) {
#pragma unroll
        for (int u = 0; u < kRows; ++u) bin[u] = a.adapter[min(r0 + u * THREADS + tid, a.rows - 1)];
#pragma unroll
        for (int u = 0; u < kRows; ++u) bin[u] = bin[u] < 0 || bin[u] >= a.adapters ? kBins : bin[u] % kBins;
    };
    for (int i = tid; i < THREADS * kBinsPerLane; i += THREADS) bins[i] = 0;
    __syncthreads();
    int bin[kRows];
    for (int r0 = 0; r0 < a.rows; r0 += kRows * THREADS) {
        bins_of(r0, bin);
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            count_up(bins, bin[u], r0 + u * THREADS + tid < a.rows, tid & 63);
    }
    __syncthreads();
    int mine[kBinsPerLane], total = 0;
#pragma unroll
    for (int i = 0; i < kBinsPerLane; ++i) {
        mine[i] = total;
        total += bins[tid * kBinsPerLane + i];
    }
    // sums of the lanes before: within the wave, then of the waves
    int upto = total;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(upto, d);
        upto += (tid & 63) >= d ? v : 0;
    }
    if ((tid & 63) == 63) sums[tid >> 6] = upto;
    __syncthreads();
    for (int w = 0; w < tid >> 6; ++w) upto += sums[w];
    const int before = upto - total;
#pragma unroll
    for (int i = 0; i < kBinsPerLane; ++i) bins[tid * kBinsPerLane + i] = before + mine[i];
    __syncthreads();
    for (int r0 = 0; r0 < a.rows; r0 += kRows * THREADS) {
        if (a.rows > kRows * THREADS) bins_of(r0, bin);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int r = r0 + u * THREADS + tid;
            const int at = count_up(bins, bin[u], r < a.rows, tid & 63);
            if (r < a.rows) a.order[at] = r;
        }
    }
}

// The first workgroup orders the rows where that is wanted, the others make h.  Two a CU, since with it they are one more than
// the CUs where tiles are as many.
constexpr int kShrinkWaves = 8;
template <typename T, int NB, int JB, bool WIDE> __global__ __launch_bounds__(64 * kShrinkWaves, 2) void lora_shrink_kernel(LoraArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    if (a.order && blockIdx.x == 0) {
        order_rows<64 * kShrinkWaves>(a, lds);
        return;
    }
    const uint32_t b = blockIdx.y * gridDim.x + blockIdx.x - (a.order ? 1 : 0);
    if (b >= (uint32_t)a.shrink_groups) return;
    shrink_tile<T, NB, JB, kShrinkWaves, WIDE, kHalfLds>(a, b, lds);
}

// ---------------------------------------------------------------------------------------
// the product
// ---------------------------------------------------------------------------------------

// A lane's operand of h: block j of 16 ranks of a token.
__device__ __forceinline__ uint4v load_h(const LoraArgs &a, int row, int j, int quad)
{
    return *reinterpret_cast<const uint4v *>(a.h + ((size_t)row * a.rblocks + j) * 64 + quad * 16);
}

// ... and of B: block j of 16 ranks of a channel.
template <typename T> __device__ __forceinline__ uint4v load_b(const LoraArgs &a, const T *B, int channel, int j, int quad)
{
    if (channel >= a.k) return uint4v{0, 0, 0, 0};
    const int r = j * 16 + (sizeof(T) == 2 ? (quad & 1) * 8 : quad * 4);
    return load16(B + (size_t)channel * a.rank, r, a.rank);
}

// Adds a block of 16 ranks of an adapter to the accumulators of the tokens that have it.
template <typename T, int MB, int NB, typename M, typename H>
__device__ __forceinline__ void multiply_adapter(M &&has_it, const uint4v (&bv)[MB], H &&h, float4v (&acc)[MB][NB])
{
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const bool own = has_it(n);
        if (__ballot(own) == 0) continue;
        const uint4v hv = h(n);
#pragma unroll
        for (int m = 0; m < MB; ++m) {
            float4v s = acc[m][n];
            mma(bv[m], hv, s, T());
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[m][n][v] = own ? s[v] : acc[m][n][v];
        }
    }
}

template <typename T> __device__ __forceinline__ float lora_act(float t, int act)
{
    if (act == TVG_ACT_RELU) return t < 0.0f ? 0.0f : t;               // (a NaN stays one)
    if (act == TVG_ACT_SILU) return t * sigmoid<sizeof(T) == 4>(t);
    return t;
}

// Stores a wave's accumulators through LDS of its own, with the tail: whole rows of the tile's channels leave as 16-byte
// stores, or element by element where rows of y do not allow it (row_of: the rows of the wave's tokens).  Two blocks of 16 tokens at a time, in loops that stay
// loops: code that runs once a tile is fetched once a tile.
constexpr int kStoreTokens = 32;
template <int MB> constexpr int kStoreRow = 16 * MB + 4;   // floats; the four keep rows on different banks
template <int MB> constexpr int kStoreBytes = kStoreTokens * kStoreRow<MB> * 4;
template <typename T, int MB, int NB>
__device__ __forceinline__ void store_rows(const LoraArgs &a, int channel0, const int *row_of, int lane, const float4v (&acc)[MB][NB], float *stage)
{
    static_assert(NB % 2 == 0, "two blocks of tokens at a time");
    constexpr int kRow = kStoreRow<MB>, E = kPer16<T>;
    const int rsel = lane & 15, quad = lane >> 4;
    const T *res = static_cast<const T *>(a.residual);
    T *y = static_cast<T *>(a.y);
    constexpr int kLanes = 16 * MB / E, kTokens = 64 / kLanes;         // lanes per token, tokens per store
    constexpr int kLanes1 = MB >= 4 ? 64 : 16 * MB, kTokens1 = 64 / kLanes1;
    const int c16 = channel0 + lane % kLanes * E, c1 = channel0 + lane % kLanes1;
    const bool wide = a.wide_y != 0;
    float bias[E];
#pragma unroll
    for (int v = 0; v < E; ++v) bias[v] = a.bias && wide && c16 < a.k ? a.bias[c16 + v] : 0.0f;
    if (!wide && a.bias && c1 < a.k) bias[0] = a.bias[c1];
#pragma unroll
    for (int n = 0; n < NB; n += 2) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int m = 0; m < MB; ++m)
                *reinterpret_cast<float4v *>(stage + (i * 16 + rsel) * kRow + m * 16 + quad * 4) = acc[m][n + i];
        __builtin_amdgcn_wave_barrier();
        if (wide) {
#pragma unroll 1
            for (int t = lane / kLanes; t < kStoreTokens; t += kTokens) {
                const int row = row_of[n * 16 + t];
                if (row >= a.rows || c16 >= a.k) break;
                const size_t at = (size_t)row * a.k + c16;
                float f[E];
#pragma unroll
                for (int v = 0; v < E; v += 4) {
                    const float4v q = *reinterpret_cast<const float4v *>(stage + t * kRow + lane % kLanes * E + v);
#pragma unroll
                    for (int u = 0; u < 4; ++u) f[v + u] = q[u] + bias[v + u];
                }
                if (res) {
                    const uint4v r = *reinterpret_cast<const uint4v *>(res + at);
#pragma unroll
                    for (int v = 0; v < E; ++v) {
                        if constexpr (sizeof(T) == 2) f[v] += __uint_as_float(v & 1 ? r[v / 2] & 0xFFFF0000u : r[v / 2] << 16);
                        else f[v] += __uint_as_float(r[v]);
                    }
                }
                if (a.act != TVG_ACT_NONE) {
#pragma unroll
                    for (int v = 0; v < E; ++v) f[v] = lora_act<T>(f[v], a.act);
                }
                uint4v out;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    if constexpr (sizeof(T) == 2) out[v] = f32x2_to_bf16x2(f[2 * v], f[2 * v + 1]);
                    else out[v] = __float_as_uint(f[v]);
                }
                *reinterpret_cast<uint4v *>(y + at) = out;
            }
        } else {
#pragma unroll 1
            for (int t = lane / kLanes1; t < kStoreTokens; t += kTokens1) {
                const int row = row_of[n * 16 + t];
                if (row >= a.rows || c1 >= a.k) break;
                const size_t at = (size_t)row * a.k + c1;
                float f = stage[t * kRow + lane % kLanes1] + bias[0];
                if (res) f += Elem<T>::load(res + at, 0);
                Elem<T>::store(y + at, 0, lora_act<T>(f, a.act));
            }
        }
    }
}

// The adapters' part of 16 MB channels x 16 NB tokens (16 NB <= 64), operands straight from memory, those of the next block of
// ranks under way while this one's are multiplied.  Of the blocks of all adapters the wave takes every W-th (W a power of two).
// mine: the adapter of token row0 + lane, -1 for none; start: the wave that takes the first block of that adapter.  Returns
// whether this wave took any.
template <typename T, int MB, int NB, int W>
__device__ __forceinline__ bool add_adapters(const LoraArgs &a, int mine, int channel0, int row0, int lane, int wave, int &start, float4v (&acc)[MB][NB])
{
    const int rsel = lane & 15, quad = lane >> 4;
    uint64_t pending = __ballot(mine >= 0), have = 0;
    int i = 0, j = wave, before = 0;                       // before: blocks of the adapters before this one
    const auto adapter = [&] {
        i = __builtin_amdgcn_readlane(mine, __builtin_ctzll(pending));
        have = __ballot(mine == i);
        start = mine == i ? before & (W - 1) : start;
    };
    const auto settle = [&] {                              // to the block j of adapter i, which may be a later one's
        while (pending && j >= a.rblocks) {
            j -= a.rblocks;
            before += a.rblocks;
            pending &= ~have;
            if (pending) adapter();
        }
    };
    uint4v bv[MB], hv[NB];
    const auto load = [&] {
        const T *B = static_cast<const T *>(a.b) + (size_t)i * a.k * a.rank;
#pragma unroll
        for (int m = 0; m < MB; ++m) bv[m] = load_b(a, B, channel0 + m * 16 + rsel, j, quad);
#pragma unroll
        for (int n = 0; n < NB; ++n) hv[n] = load_h(a, min(row0 + n * 16 + rsel, a.rows - 1), j, quad);
    };
    start = 0;
    if (!pending) return false;
    adapter();
    settle();
    if (!pending) return false;
    load();
    while (pending) {
        uint4v b[MB], h[NB];
#pragma unroll
        for (int m = 0; m < MB; ++m) b[m] = bv[m];
#pragma unroll
        for (int n = 0; n < NB; ++n) h[n] = hv[n];
        const uint64_t own = have;
        j += W;
        settle();
        if (pending) load();
        multiply_adapter<T>([&](int n) { return ((own >> (n * 16 + rsel)) & 1) != 0; }, b, [&](int n) { return h[n]; }, acc);
    }
    return true;
}

// Block e of the waves' sums of an adapter, that of its first block (`start`) first: the order of a row's sum is its own, not that of
// the adapters beside it.
template <int W> __device__ __forceinline__ float4v get_adapter_sum(const unsigned char *lds, int part_bytes, int e, int lane, int start, int rblocks)
{
    float4v t = reinterpret_cast<const float4v *>(lds + start * part_bytes)[e * 64 + lane];
    for (int q = 1; q < min(W, rblocks); ++q) t += reinterpret_cast<const float4v *>(lds + ((start + q) & (W - 1)) * part_bytes)[e * 64 + lane];
    return t;
}

// The tail of a lane's four channels of a token.
template <typename T> __device__ __forceinline__ void store4(const LoraArgs &a, int row, int ch, const float4v &t)
{
    if (row >= a.rows || ch >= a.k) return;
    const T *res = static_cast<const T *>(a.residual);
    T *y = static_cast<T *>(a.y);
    const size_t at = (size_t)row * a.k + ch;
    float f[4];
    if (a.wide_y4) {
        typedef typename Group4<T>::vec gvec;
        float r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (res) Group4<T>::unpack(*reinterpret_cast<const gvec *>(res + at), r);
#pragma unroll
        for (int v = 0; v < 4; ++v) f[v] = lora_act<T>(t[v] + (a.bias ? a.bias[ch + v] : 0.0f) + r[v], a.act);
        *reinterpret_cast<gvec *>(y + at) = Group4<T>::pack(f);
        return;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (ch + v < a.k) {
            f[v] = t[v] + (a.bias ? a.bias[ch + v] : 0.0f) + (res ? Elem<T>::load(res + at, v) : 0.0f);
            Elem<T>::store(y + at, v, lora_act<T>(f[v], a.act));
        }
}

// Rows of x, w and a of c elements, behind each other as rows of `pieces` 16 bytes, zeros behind the last element: a copy, 13 us
// for 1200 rows of 2001 and 2000 of w (bf16, launch included).
template <typename T> __global__ __launch_bounds__(256) void lora_pack_kernel(LoraArgs a, uint32_t rows, uint32_t pieces, T *to)
{
    const uint32_t at = blockIdx.x * 256u + threadIdx.x, row = at / pieces, piece = at - row * pieces;
    if (row >= rows) return;
    const uint32_t xw = (uint32_t)a.rows + a.k;
    const T *from = row < (uint32_t)a.rows ? static_cast<const T *>(a.x) + (size_t)row * a.c
                    : row < xw             ? static_cast<const T *>(a.w) + (size_t)(row - a.rows) * a.c
                                           : static_cast<const T *>(a.a) + (size_t)(row - xw) * a.c;
    *reinterpret_cast<uint4v *>(to + (size_t)at * kPer16<T>) = load16(from, (int)piece * kPer16<T>, a.c);
}

// A workgroup has 16 NB tokens x 16 MB channels and its waves split the reduction, without a barrier; then they take the
// adapters' blocks of ranks in turn, and add up through LDS.  kParts: the product is there already, in parts of the reduction, whose
// reading is all of it (64 rows 4096 -> 4096, traced: 4.0 us without adapters, 6.8 with 32).  kAnyRows: rows at any element, operands straight from
// memory, 30 GB/s a CU (1200 rows 2001 -> 2000 in bf16 155 us): left for tensors that begin between 16-byte pieces and for short rows.
enum { kAnyRows = 0, kParts = 2 };
constexpr size_t waves_lds(int mb, int nb, int w) { return (size_t)w * mb * nb * 1024 * (w * mb * nb <= 32 ? 2 : 1); }
template <typename T, int MB, int NB, int W, int MODE> __global__ __launch_bounds__(64 * W, 2) void linear_lora_waves_kernel(LoraArgs a)
{
    constexpr int kPart = MB * NB * 1024;
    extern __shared__ __align__(16) unsigned char lds[];
    const int tile = xcd_remap(blockIdx.x, a.tiles);
    const int tm = tile / a.tiles_n, tn = tile - tm * a.tiles_n;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rsel = lane & 15, quad = lane >> 4;
    const int row0 = tm * 16 * NB, ch0 = tn * 16 * MB;
    const int mine = a.adapters > 0 && lane < 16 * NB ? adapter_of(a, row0 + lane) : -1;
    float4v acc[MB][NB];
    clear(acc);
    unsigned char *part = lds + wave * kPart;
    if constexpr (MODE == kParts) {
        for (int s = wave; s < a.splits; s += W)
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const int row = row0 + n * 16 + rsel;
                    if (row < a.rows)
                        acc[m][n] += *reinterpret_cast<const float4v *>(a.parts + ((size_t)s * a.rows + row) * a.parts_row + ch0 + m * 16 + quad * 4);
                }
    } else {
        wave_product<T, MB, NB, W, false, kAllLds>(static_cast<const T *>(a.x) + (size_t)row0 * a.c, a.rows - row0,
                                                      static_cast<const T *>(a.w) + (size_t)ch0 * a.c, a.k - ch0, a.c, wave,
                                                      (a.c + 8 * kPer16<T> - 1) / (8 * kPer16<T>), part, lane, acc);
    }
    // The adapters' sums lie apart from the product's, beside them where 64 KB hold both, else in their place later: which wave has
    // them depends on the adapters of the other rows.
    constexpr size_t kMore = waves_lds(MB, NB, W) / 2;
    constexpr bool kBeside = kMore == (size_t)W * kPart;
    float4v more[MB][NB];
    clear(more);
    int start = 0;
    const bool any = a.adapters > 0 && add_adapters<T, MB, NB, W>(a, mine, ch0, row0, lane, wave, start, more);
    put_sums(part, lane, acc);
    if (kBeside && any) put_sums(part + kMore, lane, more);
    __syncthreads();
    constexpr int kMine = (MB * NB + W - 1) / W;           // blocks of 16 x 16 that a wave stores
    float4v t[kMine];
#pragma unroll
    for (int u = 0; u < kMine; ++u)
        if (wave + u * W < MB * NB) t[u] = get_sum<W>(lds, kPart, wave + u * W, lane);
    if (!kBeside && a.adapters > 0) {
        __syncthreads();
        if (any) put_sums(part, lane, more);
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kMine; ++u) {
        const int e = wave + u * W, token = e % NB * 16 + rsel;
        if (e >= MB * NB) break;
        const int adapter = __shfl(mine, token), first = __shfl(start, token);
        if (adapter >= 0) t[u] += get_adapter_sum<W>(lds + (kBeside ? kMore : 0), kPart, e, lane, first, a.rblocks);
        store4<T>(a, row0 + token, ch0 + e / NB * 16 + quad * 4, t[u]);
    }
}

// Few rows: the first workgroups make h, the others parts of the product, 16 NB tokens x 16 MB channels over a part of the
// reduction, which the next launch adds up.  64 rows 4096 -> 4096 in bf16, traced: 12.1 us for the weights' 34 MB (2.8 TB/s; 13.3 beside
// h of 32 adapters); one row 1024 -> 1024 4.2 us, a launch's latency.
template <typename T, int MB, int NB, bool WIDE> __global__ __launch_bounds__(64 * product_waves(MB, NB), 2) void lora_parts_kernel(LoraArgs a)
{
    constexpr int W = product_waves(MB, NB), kPart = kPartBytes<T, MB, NB, W, WIDE, kAllLds>;
    extern __shared__ __align__(16) unsigned char lds[];
    if ((int)blockIdx.x < a.shrink_groups) {
        shrink_tile<T, 1, 1, W, WIDE, kAllLds>(a, blockIdx.x, lds);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rsel = lane & 15, quad = lane >> 4;
    const int tiles_m = (a.rows + 16 * NB - 1) / (16 * NB);
    int b = xcd_remap(blockIdx.x - a.shrink_groups, a.tiles);          // (row tiles that share w follow each other)
    const int row0 = b % tiles_m * 16 * NB;
    b /= tiles_m;
    const int ch0 = b % a.tiles_n * 16 * MB, split = b / a.tiles_n;
    float4v acc[MB][NB];
    clear(acc);
    unsigned char *part = lds + wave * kPart;
    const int chunks = (a.c + 8 * kPer16<T> - 1) / (8 * kPer16<T>);
    wave_product<T, MB, NB, W, WIDE, kAllLds>(static_cast<const T *>(a.x) + (size_t)row0 * a.c, a.rows - row0,
                                     static_cast<const T *>(a.w) + (size_t)ch0 * a.c, a.k - ch0, a.c, split * a.chunks_per_split + wave,
                                     min(chunks, (split + 1) * a.chunks_per_split), part, lane, acc);
    put_sums(part, lane, acc);
    __syncthreads();
    for (int e = wave; e < MB * NB; e += W) {
        const int row = row0 + e % NB * 16 + rsel, ch = ch0 + e / NB * 16 + quad * 4;
        const float4v t = get_sum<W>(lds, kPart, e, lane);
        if (row < a.rows) *reinterpret_cast<float4v *>(a.parts + ((size_t)split * a.rows + row) * a.parts_row + ch) = t;
    }
}

template <typename K> bool allow_lds(K kernel, size_t bytes)
{
    return bytes <= 64 * 1024 || hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                     (int)bytes) == hipSuccess;
}

template <typename T, int MB, int NB, int W, int MODE> tvg_status launch_waves(LoraArgs a, hipStream_t stream)
{
    const auto kernel = linear_lora_waves_kernel<T, MB, NB, W, MODE>;
    constexpr size_t kLds = waves_lds(MB, NB, W);
    static const bool ok = allow_lds(kernel, kLds);
    if (!ok) return TVG_ERR_LAUNCH;
    a.tiles_n = (a.k + 16 * MB - 1) / (16 * MB);
    a.tiles = (a.rows + 16 * NB - 1) / (16 * NB) * a.tiles_n;
    hipLaunchKernelGGL(kernel, dim3(a.tiles), dim3(64 * W), kLds, stream, a);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

template <typename T, int MB, int NB, bool WIDE> tvg_status launch_parts(LoraArgs a, hipStream_t stream)
{
    const auto kernel = lora_parts_kernel<T, MB, NB, WIDE>;
    constexpr int W = product_waves(MB, NB);
    constexpr size_t kLds = std::max((size_t)W * kPartBytes<T, MB, NB, W, WIDE, kAllLds>, (size_t)W * kPartBytes<T, 1, 1, W, WIDE, kAllLds> + 17 * sizeof(int));
    static const bool ok = allow_lds(kernel, kLds);
    if (!ok) return TVG_ERR_LAUNCH;
    a.tiles_n = (a.k + 16 * MB - 1) / (16 * MB);
    a.tiles = (a.rows + 16 * NB - 1) / (16 * NB) * a.tiles_n * a.splits;
    a.shrink_groups = a.adapters > 0 ? (a.rows + 15) / 16 * a.rblocks * a.slots : 0;
    hipLaunchKernelGGL(kernel, dim3(a.shrink_groups + a.tiles), dim3(64 * W), kLds, stream, a);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

// f(0), f(1), ... as types, so that each is a constant
template <typename F, int... I> __device__ __forceinline__ void for_constants(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>()), ...);
}

constexpr int kSlice = 64;                 // bytes of the reduction per step of the kernel below

// Byte of a 16-byte piece (0..3) of a row's slice: two rows share 128 bytes, pieces permuted against bank conflicts.
__device__ __forceinline__ int slice_at(int row, int piece)
{
    const int pair = row >> 1;
    return pair * 128 + (((((row & 1) << 2) | piece) ^ (pair & 7)) << 4);
}

// Rows of whole 16-byte pieces: TM tokens x TN channels, WR x WC waves.  Both operands' slices come straight from memory
// into a ring of RING steps in LDS, RING - 1 steps ahead; a wave reads the operands of the next step while it multiplies those
// of this one, with one barrier a step.  Clocks a step, of which the matrix instructions take: 256 x 256 bf16 1360 and 1024 (two
// waves a SIMD, all of whose registers it takes), 64 x 64 bf16 260 and 64 (what comes from the caches bounds it: 8 KB a step), 64 x 64
// fp32 690 and 512.  Beside the steps: 2 us until the first slices are there, 1 to 5 us of stores, which all tiles do together.
template <typename T, int TM, int TN, int WR, int WC, int RING> __global__ __launch_bounds__(64 * WR * WC, 2) void linear_lora_tile_kernel(LoraArgs a)
{
    constexpr int W = WR * WC, kLoads = (TM + TN) / 16 / W, kLoadsX = TM / 16 / W;
    constexpr int NB = TM / WR / 16, MB = TN / WC / 16;                // blocks of 16 tokens, of 16 channels, per wave
    constexpr int kStage = (TM + TN) * kSlice;
    static_assert(kLoads * W * 16 == TM + TN && kLoadsX * W * 16 == TM, "every wave loads whole rows of one operand");
    static_assert(MB <= 4 && W * kStoreBytes<MB> <= RING * kStage, "the stores' rows lie where the ring was");
    extern __shared__ __align__(1024) unsigned char lds[];
    int *row_of = reinterpret_cast<int *>(lds + RING * kStage), *ids = row_of + TM, *list = ids + TM;
    const int tile = xcd_remap(blockIdx.x, a.tiles);
    int tm, tn;
    {
        // groups of four rows of tiles, column by column: what runs together shares rows and columns
        const int group = tile / (4 * a.tiles_n), in = tile - group * 4 * a.tiles_n;
        const int high = min(4, a.tiles / a.tiles_n - group * 4);
        tn = in / high;
        tm = group * 4 + in - tn * high;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rsel = lane & 15, quad = lane >> 4;
    const int row0 = tm * TM, ch0 = tn * TN, wr = wave / WC * (TM / WR), wc = wave % WC * (TN / WC);
    const uint32_t row_bytes = (uint32_t)a.c * sizeof(T);
    // (rows in order of their adapters: anywhere in x, whose bytes 32 bits count then)
    const int base = a.order ? 0 : row0, reach = a.order ? a.rows : min(TM, a.rows - row0);
    const uint4v xbuf = raw_buffer(static_cast<const T *>(a.x) + (size_t)base * a.c, (uint32_t)reach * row_bytes);
    const uint4v wbuf = raw_buffer(static_cast<const T *>(a.w) + (size_t)ch0 * a.c, (uint32_t)min(TN, a.k - ch0) * row_bytes);
    // a load: 16 rows of an operand; where a lane's 16 bytes come from
    uint32_t from[kLoads];
    const uint32_t pair = lane >> 3, slot = (lane & 7) ^ (pair & 7), lrow = pair * 2 + (slot >> 2), piece = slot & 3;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int block = i < kLoadsX ? i * W + wave : (i - kLoadsX) * W + wave;
        const int row = block * 16 + lrow, end = i < kLoadsX ? min(TM, a.rows - row0) : min(TN, a.k - ch0);
        const uint32_t at = i < kLoadsX && a.order && row < end ? a.order[row0 + row] : row;
        from[i] = row < end ? at * row_bytes + piece * 16 : kBeyond;
    }
    const int whole = (int)(row_bytes / kSlice), steps = (int)((row_bytes + kSlice - 1) / kSlice);
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char *)lds);
    const int turns = (steps + 1) & ~1;                    // (an odd step more: zeros)
    int adapters = 0, blocks = 0, fetched = 0;             // of the tile; blocks of ranks in the ring, the next one
    const auto fetch = [&](int s) {                        // a whole slice of the channels
        const uint32_t to = lds0 + (s & (RING - 1)) * kStage + wave * 1024;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_to_lds(to + i * W * 1024, from[i], i < kLoadsX ? xbuf : wbuf, s * kSlice);
    };
    // 16 bytes a lane of a row of B at any element: through registers.  (It waits for all loads: such a step has fewer than
    // kLoads in flight, or none of B where all channels of the wave lie beyond the last.)
    const auto copy_b = [&](int i, int row, int r0, int to) {
        const T *from_b = static_cast<const T *>(a.b) + ((size_t)i * a.k + ch0 + row) * a.rank + r0;
        T *to_b = reinterpret_cast<T *>(lds + to + lane * 16);
#pragma unroll 1
        for (int e = 0; e < kPer16<T>; ++e) to_b[e] = ch0 + row < a.k && r0 + e < a.rank ? from_b[e] : (T)0;
        wait_loads<0>();
        wait_reads();
    };
    // Tiles of several adapters: a step of the ring is a block of 16 ranks of h and of B of the next kBGroup adapters.
    constexpr int kBRow = sizeof(T) == 2 && TN > 64 ? 32 : 64;         // bytes of a row of B (bf16, 64: its 16 ranks twice)
    constexpr int kBLoads = TN * kBRow / 1024 / W, kBStage = TN * kBRow, kBGroup = (kLoads - kLoadsX) / kBLoads;
    static_assert(kBLoads * W * 1024 == kBStage && kBGroup * kBLoads == kLoads - kLoadsX, "as many loads a step as the product has");
    int next_at = 0, next_block = 0;
    const auto fetch_h = [&](uint32_t to, int j, bool any) {
        const uint4v hbuf = raw_buffer(a.h + (size_t)base * a.rblocks * 64, (uint32_t)reach * a.rblocks * 64);
#pragma unroll
        for (int n = 0; n < kLoadsX; ++n) {
            const int row = (n * W + wave) * 16 + lrow;
            const uint32_t at = ((row_of[row] - base) * a.rblocks + j) * 64 + piece * 16;
            load_to_lds(to + n * W * 1024, any && row0 + row < a.rows ? at : kBeyond, hbuf, 0);
        }
    };
    const auto fetch_b = [&](int to, int at) {
        const bool any = next_block < a.rblocks && at < adapters;
        const int i = any ? __builtin_amdgcn_readfirstlane(list[at]) : 0;
        const uint4v bbuf = raw_buffer(static_cast<const T *>(a.b) + ((size_t)i * a.k + ch0) * a.rank,
                                       (uint32_t)min(TN, a.k - ch0) * a.rank * (uint32_t)sizeof(T));
#pragma unroll
        for (int l = 0; l < kBLoads; ++l) {
            const int row = ((l * W + wave) * 1024 + lane * 16) / kBRow;
            const uint32_t r = sizeof(T) == 2 ? next_block * 32 + (lane & 1) * 16 : next_block * 64 + (lane & 3) * 16;
            const bool ok = any && ch0 + row < a.k && r < a.rank * sizeof(T);
            if (a.wide_rank || !any) load_to_lds(lds0 + to + l * W * 1024, ok ? row * a.rank * (uint32_t)sizeof(T) + r : kBeyond, bbuf, 0);
            else copy_b(i, row, (int)(r / sizeof(T)), to + l * W * 1024);
        }
    };
    const auto fetch_any = [&](int s) {
        const uint32_t to = lds0 + (s & (RING - 1)) * kStage + wave * 1024;
        if (s < turns) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const uint32_t at = s * kSlice + piece * 16 < row_bytes ? from[i] : kBeyond;
                load_to_lds(to + i * W * 1024, at, i < kLoadsX ? xbuf : wbuf, s >= steps ? 0 : s * kSlice);
            }
            return;
        }
        if (adapters > 0 && blocks == 0) {
            fetch_h(to, next_block, next_block < a.rblocks);
#pragma unroll
            for (int q = 0; q < kBGroup; ++q) fetch_b((s & (RING - 1)) * kStage + TM * kSlice + q * kBStage + wave * 1024, next_at + q);
            next_at += kBGroup;
            if (next_at >= adapters) {
                next_at = 0;
                ++next_block;
            }
            return;
        }
        // a block of 16 ranks of the only adapter: h of the tokens, and B, whose 16 ranks bf16 takes twice
        const bool any = fetched < blocks;
        const int i = any ? __builtin_amdgcn_readfirstlane(list[0]) : 0;
        fetch_h(to, fetched, any);
        const uint4v bbuf = raw_buffer(static_cast<const T *>(a.b) + ((size_t)i * a.k + ch0) * a.rank,
                                       (uint32_t)min(TN, a.k - ch0) * a.rank * (uint32_t)sizeof(T));
        const uint32_t bpiece = sizeof(T) == 2 ? fetched * 32 + (piece & 1) * 16 : fetched * 64 + piece * 16;
#pragma unroll
        for (int n = kLoadsX; n < kLoads; ++n) {
            const int row = ((n - kLoadsX) * W + wave) * 16 + lrow;
            const bool ok = any && ch0 + row < a.k && bpiece < a.rank * sizeof(T);
            if (a.wide_rank || !any) load_to_lds(to + n * W * 1024, ok ? row * a.rank * (uint32_t)sizeof(T) + bpiece : kBeyond, bbuf, 0);
            else copy_b(i, row, (int)(bpiece / sizeof(T)), (int)(to - lds0) + n * W * 1024);
        }
        ++fetched;
    };
    float4v acc[MB][NB];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[m][n] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    uint4v xv[2][NB], wv[2][MB];
    const int xat = slice_at(wr + rsel, quad), wat = TM * kSlice + slice_at(wc + rsel, quad);
    const auto read = [&](int s, uint4v (&x)[NB], uint4v (&w)[MB]) {
        const unsigned char *p = lds + (s & (RING - 1)) * kStage;
#pragma unroll
        for (int n = 0; n < NB; ++n) x[n] = *reinterpret_cast<const uint4v *>(p + xat + n * 16 * kSlice);
#pragma unroll
        for (int m = 0; m < MB; ++m) w[m] = *reinterpret_cast<const uint4v *>(p + wat + m * 16 * kSlice);
    };
    const auto multiply = [&](uint4v (&x)[NB], uint4v (&w)[MB]) { mma_all(w, x, acc, T()); };
    const auto behind = [&] {
        wait_loads<(RING - 3) * kLoads>();                 // the next step has landed, of this wave and behind the barrier of all
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto step = [&](int s, uint4v (&x)[NB], uint4v (&w)[MB], uint4v (&nx)[NB], uint4v (&nw)[MB]) {
        behind();
        fetch(s + RING - 1);                               // (to where step s - 1 was, which all waves have read)
        read(s + 1, nx, nw);
        multiply(x, w);
#pragma unroll
        for (int i = 0; i < NB + MB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int t = threadIdx.x; t < TM; t += 64 * W)
        row_of[t] = row0 + t >= a.rows ? a.rows : a.order ? a.order[row0 + t] : row0 + t;
#pragma unroll 1
    for (int i = 0; i < RING - 1; ++i) {
        if (i == 2 && a.adapters > 0) {
            wait_reads();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (wave == 0) {
                constexpr int N = (TM + 63) / 64;
                int mine[N];
#pragma unroll
                for (int n = 0; n < N; ++n) mine[n] = adapter_of(a, row_of[n * 64 + lane]);
                const int found = distinct_adapters<N>(mine, lane, list);
                const int first = found ? list[0] : -1;
                bool same = true;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    ids[n * 64 + lane] = mine[n];
                    same = same && (mine[n] == first || row0 + n * 64 + lane >= a.rows);
                }
                same = __ballot(same) == ~0ull;
                if (lane == 0) {
                    list[TM] = found;
                    list[TM + 1] = same;
                }
            }
            wait_reads();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            adapters = __builtin_amdgcn_readfirstlane(list[TM]);
            if (__builtin_amdgcn_readfirstlane(list[TM + 1])) blocks = adapters * a.rblocks;
        }
        fetch_any(i);
    }
    wait_loads<(RING - 2) * kLoads>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(0, xv[0], wv[0]);
    int s = 0;
    for (; s + RING < whole; s += 2) {
        step(s, xv[0], wv[0], xv[1], wv[1]);
        step(s + 1, xv[1], wv[1], xv[0], wv[0]);
    }
    const bool mixed = adapters > 0 && blocks == 0;
    constexpr bool kAhead = TM < 256;      // (the largest tile's registers have no room for two steps here)
    // the last slices to fetch, then, where all tokens have the same adapter, its blocks of ranks
#pragma unroll 1
    for (const int end = mixed ? turns : turns + blocks - (RING - 1); s < end; ++s) {
        behind();
        fetch_any(s + RING - 1);
        if constexpr (kAhead) {
            read(s + 1, xv[1], wv[1]);
            multiply(xv[0], wv[0]);
            wait_reads();                  // (the next step's barrier lets other waves write there)
#pragma unroll
            for (int n = 0; n < NB; ++n) xv[0][n] = xv[1][n];
#pragma unroll
            for (int m = 0; m < MB; ++m) wv[0][m] = wv[1][m];
        } else {
            read(s, xv[0], wv[0]);
            wait_reads();
            multiply(xv[0], wv[0]);
        }
    }
    // what is in the ring (zeros where the sum has fewer steps than that)
    if constexpr (!kAhead) {
        if (!mixed) {
            wait_loads<0>();
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll 1
            for (const int end = s + RING - 1; s < end; ++s) {
                read(s, xv[0], wv[0]);
                multiply(xv[0], wv[0]);
            }
        }
    } else if (!mixed)
        for_constants([&](auto d) {
            constexpr int kStep = decltype(d)::value;
            if constexpr (kStep < RING - 2) {
                wait_loads<(RING - 3 - kStep) * kLoads>();
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
                read(s + kStep + 1, xv[(kStep + 1) & 1], wv[(kStep + 1) & 1]);
            }
            multiply(xv[kStep & 1], wv[kStep & 1]);
            __builtin_amdgcn_sched_barrier(0);
        }, std::make_integer_sequence<int, RING - 1>());
    if (mixed) {
        int mine[NB], at = 0, j = 0;
#pragma unroll
        for (int n = 0; n < NB; ++n) mine[n] = ids[wr + n * 16 + rsel];
        const int bat = (wc + rsel) * kBRow + (sizeof(T) == 2 && kBRow == 32 ? quad & 1 : quad) * 16;
#pragma unroll 1
        for (; j < a.rblocks; ++s) {
            behind();
            fetch_any(s + RING - 1);
            const unsigned char *p = lds + (s & (RING - 1)) * kStage;
#pragma unroll
            for (int n = 0; n < NB; ++n) xv[0][n] = *reinterpret_cast<const uint4v *>(p + xat + n * 16 * kSlice);
#pragma unroll 1
            for (int q = 0; q < kBGroup && at < adapters; ++q, ++at) {
                const int i = __builtin_amdgcn_readfirstlane(list[at]);
#pragma unroll
                for (int m = 0; m < MB; ++m) wv[0][m] = *reinterpret_cast<const uint4v *>(p + TM * kSlice + q * kBStage + bat + m * 16 * kBRow);
                multiply_adapter<T>([&](int n) { return mine[n] == i; }, wv[0],
                                    [&](int n) { return xv[0][n]; }, acc);
            }
            wait_reads();
            if (at == adapters) {
                at = 0;
                ++j;
            }
        }
    }
    wait_loads<0>();
    __syncthreads();
    store_rows<T, MB, NB>(a, ch0 + wc, row_of + wr, lane, acc, reinterpret_cast<float *>(lds + wave * kStoreBytes<MB>));
}

template <typename T, int TM, int TN, int WR, int WC, int RING> tvg_status launch_tile(LoraArgs a, hipStream_t stream)
{
    const auto kernel = linear_lora_tile_kernel<T, TM, TN, WR, WC, RING>;
    constexpr size_t kLds = (size_t)RING * (TM + TN) * kSlice + (3 * TM + 2) * sizeof(int);
    static const bool ok = allow_lds(kernel, kLds);
    if (!ok) return TVG_ERR_LAUNCH;
    a.tiles_n = (a.k + TN - 1) / TN;
    a.tiles = (a.rows + TM - 1) / TM * a.tiles_n;
    hipLaunchKernelGGL(kernel, dim3(a.tiles), dim3(64 * WR * WC), kLds, stream, a);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

int rank_blocks(const LoraProblem &p) { return (p.rank + 15) / 16; }

template <typename T, int NB, int JB, bool WIDE> tvg_status launch_shrink(LoraArgs a, hipStream_t stream)
{
    const auto kernel = lora_shrink_kernel<T, NB, JB, WIDE>;
    constexpr int W = kShrinkWaves;
    constexpr size_t kLds = std::max((size_t)W * kPartBytes<T, JB, NB, W, WIDE, kHalfLds> + (16 * NB + 1) * sizeof(int), kOrderBytes<64 * W>);
    static const bool ok = allow_lds(kernel, kLds);
    if (!ok) return TVG_ERR_LAUNCH;
    const int tiles = (a.rows + 16 * NB - 1) / (16 * NB) * ((a.rblocks + JB - 1) / JB);
    // few tiles: their adapters in turn by several workgroups
    a.slots = std::max(1, std::min(std::min(16 * NB, std::min(a.rows, a.adapters)), 2 * kComputeUnits / tiles));
    a.shrink_groups = tiles * a.slots;
    // (a launch has fewer than 2^32 work items in x: 8.4 million rows of rank 256 would pass that, and lose the rows behind)
    const int in_x = std::min(a.shrink_groups, 1 << 22), in_y = (a.shrink_groups + in_x - 1) / in_x;
    hipLaunchKernelGGL(kernel, dim3(in_x + (a.order ? 1 : 0), in_y), dim3(64 * W), kLds, stream, a);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

int tiles_of(const LoraProblem &p, int tokens, int channels)
{
    return (p.rows + tokens - 1) / tokens * ((p.k + channels - 1) / channels);
}

// How the product of few tiles is cut: 16 mb channels x 16 nb tokens, parts of the reduction.
struct PartsPlan {
    int use, mb, nb, splits, chunks_per_split, parts_row, slots;
    size_t h_bytes, bytes;
};

// Up to a round of 64 x 64 tiles (one a CU): measured with 8 to 16 adapters of rank 16, 512 rows 1024 -> 1024 13.4 us in parts
// and 15.2 in the ring's 64 x 64 tiles (bf16; fp32 23.5 and 30.6), 1024 rows, a whole round, 20.8 and 15.1 (fp32 37.0, 33.1).
// Narrower tiles where these and parts of four chunks a wave at least are fewer than half the CUs: 64 rows 1024 -> 1024 12.6 us
// in 32 channels, 13.0 in 64.
PartsPlan plan_parts(const LoraProblem &p, bool wide)
{
    PartsPlan plan{};
    plan.parts_row = (p.k + 63) / 64 * 64;
    plan.h_bytes = p.adapters > 0 ? ((size_t)p.rows * rank_blocks(p) * 64 + 255) & ~(size_t)255 : 0;
    plan.bytes = plan.h_bytes + (p.adapters > 0 ? (size_t)p.rows * sizeof(int) : 0);
    plan.use = tiles_of(p, 64, 64) < kComputeUnits;
    if (!plan.use) return plan;
    const int chunks = (int)(((size_t)p.c * (p.dtype == TVG_BF16 ? 2 : 4) + 127) / 128);
    plan.nb = p.rows <= 16 ? 1 : p.rows <= 32 && wide ? 2 : 4;
    plan.mb = 4;
    const auto most = [&] { return std::max(1, std::min(8, chunks / product_waves(plan.mb, plan.nb))); };
    if (tiles_of(p, 16 * plan.nb, 64) * most() < kComputeUnits / 2 || !wide) plan.mb = plan.nb == 1 ? (wide ? 1 : 4) : 2;
    const int tiles = tiles_of(p, 16 * plan.nb, 16 * plan.mb);
    const int htiles = p.adapters > 0 ? (p.rows + 15) / 16 * rank_blocks(p) : 0;
    plan.slots = htiles > 0 ? std::max(1, std::min(std::min(16, std::min(p.rows, p.adapters)), kComputeUnits / 4 / htiles)) : 0;
    // (what makes h takes a place too)
    const int splits = std::max(1, std::min(most(), (kComputeUnits - htiles * plan.slots) / tiles));
    plan.chunks_per_split = (chunks + splits - 1) / splits;
    plan.splits = (chunks + plan.chunks_per_split - 1) / plan.chunks_per_split;
    plan.bytes = plan.h_bytes + (size_t)plan.splits * p.rows * plan.parts_row * sizeof(float);
    return plan;
}

template <typename T> tvg_status launch_few_tiles(const PartsPlan &plan, bool wide, LoraArgs &a, hipStream_t stream)
{
    a.splits = plan.splits;
    a.slots = plan.slots;
    a.chunks_per_split = plan.chunks_per_split;
    a.parts_row = plan.parts_row;
    a.parts = reinterpret_cast<float *>(a.h + plan.h_bytes);
    tvg_status st;
    if (!wide) st = plan.nb == 1 ? launch_parts<T, 4, 1, false>(a, stream) : launch_parts<T, 2, 4, false>(a, stream);
    else if (plan.nb == 1) st = plan.mb == 1 ? launch_parts<T, 1, 1, true>(a, stream) : launch_parts<T, 4, 1, true>(a, stream);
    else if (plan.nb == 2) st = plan.mb == 2 ? launch_parts<T, 2, 2, true>(a, stream) : launch_parts<T, 4, 2, true>(a, stream);
    else st = plan.mb == 2 ? launch_parts<T, 2, 4, true>(a, stream) : launch_parts<T, 4, 4, true>(a, stream);
    return st != TVG_OK ? st : launch_waves<T, 4, 1, 8, kParts>(a, stream);
}

// The ring's tile, by rounds.  bf16, us per 4096 channels: 256 x 256 95 a round of 256 tiles; 128 x 128 44, two of them a CU, so
// that parts of a round count as such; 64 x 64 for up to two rounds (512 rows 1024 -> 4096 20.0 us, 21.8 in 128 x 128; 1024
// rows 30.9 and 22.1).  fp32, whose matrix rate bounds all, per 1024 channels: 128 x 128 71, 64 x 64 20 a round.
int ring_tile(const LoraProblem &p)
{
    const int t64 = tiles_of(p, 64, 64), t128 = tiles_of(p, 128, 128), t256 = tiles_of(p, 256, 256);
    const auto rounds = [](int t) { return (t + kComputeUnits - 1) / kComputeUnits; };
    if (p.dtype == TVG_F32) return 71 * rounds(t128) <= 20 * rounds(t64) ? 128 : 64;
    if (t64 <= 2 * kComputeUnits) return 64;
    return (int64_t)95 * rounds(t256) * kComputeUnits <= (int64_t)44 * std::max(t128, kComputeUnits) ? 256 : 128;
}

// Rows that are no whole 16-byte pieces are copied to rows that are, where a round of 64 x 64 tiles reads each often enough and a
// row is no shorter than two pieces of 128 bytes.  Copied and read as they are, us: 8192 rows 4097 -> 4096 in bf16 314 and 3168 (fp32
// 1997 and 3260), 1200 rows 2001 -> 2000 49 and 171 (132 and 181), 1200 rows 133 -> 2000 19 and 24 (33 and 34), 1000 rows
// 131 -> 1040, the smallest copied, 17 and 15 (24 and 20).  With fewer tiles where that is as much work as 16 rows 4096 -> 4096, and
// in bf16: 16 rows 4097 -> 4096 28 and 34, 64 rows 29 and 82, 777 rows 1001 -> 515 18 and 28, 64 rows 1001 -> 1024 13 and 12; fp32, whose
// products take longer, 100 rows 4097 -> 4096 98 and 77, 777 rows 1001 -> 515 36 and 32.  Rows of 1000 to 2000 elements cross there: 64 rows
// 1001 -> 1024 13.9 and 12.4, 2001 -> 2048 21.5 and 19.9, 200 rows 17.4 and 20.8, 25 and 57; longer ones do further down, which this leaves (16
// rows 4097 -> 1024 22 and 35, 1 row 18 and 23).  Not where the adapters, of which a call
// may use a few, would be most of the copy.
size_t elem_size(const LoraProblem &p) { return p.dtype == TVG_BF16 ? 2 : 4; }
int packed_c(const LoraProblem &p)
{
    const int e = 16 / (int)elem_size(p);
    return (p.c + e - 1) / e * e;
}
bool packs(const LoraProblem &p)
{
    return packed_c(p) != p.c && p.c * elem_size(p) >= 256 && packed_c(p) * elem_size(p) < 1 << 23 &&
           (int64_t)p.adapters * p.rank <= (int64_t)p.rows + p.k &&
           (tiles_of(p, 64, 64) >= kComputeUnits || (p.dtype == TVG_BF16 && (double)p.rows * p.c * p.k >= 1 << 28));
}
// Workspace in front of the copies.
size_t front_bytes(const LoraProblem &p)
{
    LoraProblem q = p;
    q.c = packed_c(p);
    return (std::max(std::max(plan_parts(p, true).bytes, plan_parts(p, false).bytes), plan_parts(q, true).bytes) + 255) & ~(size_t)255;
}
size_t packed_rows(const LoraProblem &p) { return (size_t)p.rows + p.k + (size_t)p.adapters * p.rank; }

template <typename T> tvg_status launch(const LoraProblem &problem, LoraArgs &a, hipStream_t stream)
{
    LoraProblem p = problem;
    if (packs(p)) {
        const size_t rows = packed_rows(p);
        const uint32_t pieces = (uint32_t)(packed_c(p) / kPer16<T>);
        T *to = reinterpret_cast<T *>(a.h + front_bytes(p));
        hipLaunchKernelGGL((lora_pack_kernel<T>), dim3((unsigned)((rows * pieces + 255) / 256)), dim3(256), 0, stream, a, (uint32_t)rows, pieces, to);
        if (hipGetLastError() != hipSuccess) return TVG_ERR_LAUNCH;
        p.c = a.c = packed_c(p);
        a.x = to;
        a.w = to + (size_t)p.rows * p.c;
        a.a = to + ((size_t)p.rows + p.k) * p.c;
        a.wide_rows = 1;
    }
    const bool wide = a.wide_rows && (size_t)p.c * sizeof(T) < 1 << 23;
    const PartsPlan parts = plan_parts(p, wide);
    if (parts.use) return launch_few_tiles<T>(parts, wide, a, stream);
    if (p.adapters > 0) {
        if (wide && (int64_t)p.rows * std::max((int64_t)p.c * (int64_t)sizeof(T), (int64_t)a.rblocks * 64) < (int64_t)kBeyond)
            a.order = reinterpret_cast<int *>(a.h + parts.h_bytes);
        const tvg_status st = !wide ? launch_shrink<T, 1, 1, false>(a, stream)
                                    : a.rblocks == 1 ? launch_shrink<T, 1, 1, true>(a, stream) : launch_shrink<T, 2, 2, true>(a, stream);
        if (st != TVG_OK) return st;
    }
    if (!wide) return launch_waves<T, 4, 4, 4, kAnyRows>(a, stream);
    switch (ring_tile(p)) {
    case 256:
        if constexpr (sizeof(T) == 2) return launch_tile<T, 256, 256, 2, 4, 4>(a, stream);
        [[fallthrough]];
    case 128: return launch_tile<T, 128, 128, 2, 2, 4>(a, stream);
    default: return launch_tile<T, 64, 64, 2, 2, 8>(a, stream);
    }
}

}  // namespace

size_t linear_lora_workspace(const LoraProblem &p)
{
    if (p.rows == 0) return 0;
    return packs(p) ? front_bytes(p) + packed_rows(p) * packed_c(p) * elem_size(p) : std::max(plan_parts(p, true).bytes, plan_parts(p, false).bytes);
}

tvg_status launch_linear_lora(const LoraProblem &p, const LoraPointers &ptr, hipStream_t stream)
{
    const size_t elem = p.dtype == TVG_BF16 ? 2 : 4;
    const auto aligned = [](const void *q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
    LoraArgs a{};
    a.x = ptr.x; a.w = ptr.w; a.a = ptr.a; a.b = ptr.b; a.adapter = ptr.adapter; a.scale = ptr.scale; a.bias = ptr.bias;
    a.residual = ptr.residual; a.y = ptr.y; a.h = reinterpret_cast<unsigned char *>(ptr.workspace);
    a.rows = p.rows; a.c = p.c; a.k = p.k; a.adapters = p.adapters; a.rank = p.rank; a.act = p.act;
    a.rblocks = rank_blocks(p);
    a.wide_rows = p.c * elem % 16 == 0 && aligned(ptr.x) && aligned(ptr.w) && aligned(ptr.a);
    a.wide_rank = p.rank * elem % 16 == 0 && aligned(ptr.b);
    a.wide_y4 = p.k % 4 == 0 && reinterpret_cast<uintptr_t>(ptr.y) % (4 * elem) == 0 && reinterpret_cast<uintptr_t>(ptr.residual) % (4 * elem) == 0;
    a.wide_y = p.k * elem % 16 == 0 && aligned(ptr.y) && aligned(ptr.residual);
    return p.dtype == TVG_BF16 ? launch<bf16_t>(p, a, stream) : launch<float>(p, a, stream);
}

}  // namespace tvg
