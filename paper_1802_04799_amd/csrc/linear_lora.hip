// Projection of rows with a low-rank adapter chosen row by row:
//   y = act(x W^T + bias + scale_i (x A_i^T) B_i^T + residual),  i = adapter[row]
//
// Two launches.  The first makes the adapters' middle vectors h = A_i x, fp32, in `splits` parts of the reduction that
// the second adds in order.  The second is a matrix product whose reduction goes on, after the c channels, over the rank:
// the same accumulators take B_i h.
//
// Both types are the same kernel in bytes: a lane's operand of a 16x16 tile is 16 bytes, 8 bf16 of one
// v_mfma_f32_16x16x32_bf16 or 4 fp32 of four v_mfma_f32_16x16x4_f32, whose order of the reduction is that of the loads.
// Channels are the tile's rows and tokens its columns, so that a lane holds four adjacent channels of one token: what
// depends on the token (its adapter) is a select per lane.
//
// h for the bf16 product is split into two bf16 parts, h = hi + lo with an error of 2^-17 of h, and a block of 16 ranks is
// one MFMA of 32: hi in the first 16, lo in the others, against B twice.  So the middle vector costs no digits.
//
// Rows of a tile with different adapters: one pass per adapter in use, into accumulators of its own, of which the rows
// that have this adapter take their sums.  Nothing is multiplied by zero, so what an adapter holds (infinities, NaN)
// reaches no other row.
#include <algorithm>
#include <limits.h>

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
    float *h;                              // [splits][rows][16 rblocks]
    int rows, c, k, adapters, rank, rblocks, splits, c_per_split;
    int act, wide_rows, wide_rank, wide_y; // 16-byte accesses of rows of c, of rows of rank, groups of four of y
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

// 16 bytes of row p from element k on, zeros from element `end` on.
template <typename T> __device__ __forceinline__ uint4v load16(const T *p, int k, int end, bool wide)
{
    if (wide && k + kPer16<T> <= end) return *reinterpret_cast<const uint4v *>(p + k);
    T v[kPer16<T>];
#pragma unroll
    for (int i = 0; i < kPer16<T>; ++i) v[i] = k + i < end ? p[k + i] : (T)0;
    return __builtin_bit_cast(uint4v, v);
}

// ---------------------------------------------------------------------------------------
// h = A_i x
// ---------------------------------------------------------------------------------------

constexpr int kShrinkWaves = 4;
constexpr int kShrinkRanks = 4;            // blocks of 16 ranks at a time

// The next adapter index above `last` among the tokens of NB blocks (lanes 16 apart hold the same token).
template <int NB> __device__ __forceinline__ int next_adapter(const int (&mine)[NB], int last)
{
    int next = INT_MAX;
#pragma unroll
    for (int i = 0; i < NB; ++i) next = mine[i] > last ? min(next, mine[i]) : next;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) next = min(next, __shfl_xor(next, d));
    return __builtin_amdgcn_readfirstlane(next);
}

// A token's adapter, -1 for none.
__device__ __forceinline__ int adapter_of(const LoraArgs &a, int row)
{
    const int i = row < a.rows ? a.adapter[row] : -1;
    return i >= 0 && i < a.adapters ? i : -1;
}

// 16 tokens x 16 rblocks ranks x one part of the reduction; the waves split it further and add up through LDS.
template <typename T> __global__ __launch_bounds__(64 * kShrinkWaves) void lora_shrink_kernel(LoraArgs a)
{
    __shared__ float4v parts[kShrinkWaves][kShrinkRanks][64];
    constexpr int E = kPer16<T>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int token = lane & 15, quad = lane >> 4;
    const int split = blockIdx.x % a.splits, row = blockIdx.x / a.splits * 16 + token;
    const int mine[1] = {adapter_of(a, row)};
    const int k0 = split * a.c_per_split, k1 = min(k0 + a.c_per_split, a.c);
    const T *x = static_cast<const T *>(a.x) + (size_t)min(row, a.rows - 1) * a.c;
    for (int i = next_adapter(mine, -1); i != INT_MAX; i = next_adapter(mine, i)) {
        const T *A = static_cast<const T *>(a.a) + (size_t)i * a.rank * a.c;
        for (int j0 = 0; j0 < a.rblocks; j0 += kShrinkRanks) {
            float4v acc[kShrinkRanks];
#pragma unroll
            for (int j = 0; j < kShrinkRanks; ++j) acc[j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
            for (int k = k0 + wave * 4 * E; k < k1; k += kShrinkWaves * 4 * E) {
                const uint4v xv = load16(x, k + quad * E, k1, a.wide_rows);
#pragma unroll
                for (int j = 0; j < kShrinkRanks; ++j) {
                    const int r = (j0 + j) * 16 + token;
                    if (j0 + j >= a.rblocks) continue;
                    const uint4v av = r < a.rank ? load16(A + (size_t)r * a.c, k + quad * E, k1, a.wide_rows) : uint4v{0, 0, 0, 0};
                    mma(av, xv, acc[j], T());
                }
            }
#pragma unroll
            for (int j = 0; j < kShrinkRanks; ++j) parts[wave][j][lane] = acc[j];
            __syncthreads();
            // a wave adds up a block of ranks
            if (j0 + wave < a.rblocks && mine[0] == i) {
                float4v s = parts[0][wave][lane];
#pragma unroll
                for (int v = 1; v < kShrinkWaves; ++v) s += parts[v][wave][lane];
                float *h = a.h + ((size_t)split * a.rows + row) * a.rblocks * 16 + (j0 + wave) * 16 + quad * 4;
                *reinterpret_cast<float4v *>(h) = s;
            }
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------------------------------
// the product
// ---------------------------------------------------------------------------------------

// A lane's operand of h: block j of 16 ranks of a token, scaled.
__device__ __forceinline__ uint4v load_h(const LoraArgs &a, int row, int j, int quad, float scale, float)
{
    float4v s = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < a.splits; ++p)
        s += *reinterpret_cast<const float4v *>(a.h + (((size_t)p * a.rows + row) * a.rblocks + j) * 16 + quad * 4);
    s *= scale;
    return __builtin_bit_cast(uint4v, s);
}
__device__ __forceinline__ uint4v load_h(const LoraArgs &a, int row, int j, int quad, float scale, bf16_t)
{
    float4v s0 = float4v{0.0f, 0.0f, 0.0f, 0.0f}, s1 = s0;
    for (int p = 0; p < a.splits; ++p) {
        const float4v *h = reinterpret_cast<const float4v *>(a.h + (((size_t)p * a.rows + row) * a.rblocks + j) * 16 + (quad & 1) * 8);
        s0 += h[0];
        s1 += h[1];
    }
    s0 *= scale;
    s1 *= scale;
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = s0[i], f[4 + i] = s1[i];
    if (quad >= 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = f[i] - bf16_to_f32(f32_to_bf16(f[i]));
            f[i] = d == d ? d : 0.0f;                      // (of an infinity the upper part is all)
        }
    }
    return uint4v{f32x2_to_bf16x2(f[0], f[1]), f32x2_to_bf16x2(f[2], f[3]), f32x2_to_bf16x2(f[4], f[5]), f32x2_to_bf16x2(f[6], f[7])};
}

// ... and of B: block j of 16 ranks of a channel.
template <typename T> __device__ __forceinline__ uint4v load_b(const LoraArgs &a, const T *B, int channel, int j, int quad)
{
    if (channel >= a.k) return uint4v{0, 0, 0, 0};
    const int r = j * 16 + (sizeof(T) == 2 ? (quad & 1) * 8 : quad * 4);
    return load16(B + (size_t)channel * a.rank, r, a.rank, a.wide_rank);
}

// Adds the adapters' part to a wave's accumulators: MB blocks of 16 channels from channel0, NB blocks of 16 tokens from row0.
template <typename T, int MB, int NB>
__device__ __forceinline__ void add_adapters(const LoraArgs &a, int channel0, int row0, int lane, float4v (&acc)[MB][NB])
{
    const int token = lane & 15, quad = lane >> 4;
    int mine[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) mine[n] = adapter_of(a, row0 + n * 16 + token);
    for (int i = next_adapter(mine, -1); i != INT_MAX; i = next_adapter(mine, i)) {
        const T *B = static_cast<const T *>(a.b) + (size_t)i * a.k * a.rank;
        const float scale = a.scale ? a.scale[i] : 1.0f;
        for (int j = 0; j < a.rblocks; ++j) {
            uint4v bv[MB];
#pragma unroll
            for (int m = 0; m < MB; ++m) bv[m] = load_b(a, B, channel0 + m * 16 + token, j, quad);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                if (__ballot(mine[n] == i) == 0) continue;
                const uint4v hv = load_h(a, min(row0 + n * 16 + token, a.rows - 1), j, quad, scale, T());
#pragma unroll
                for (int m = 0; m < MB; ++m) {
                    float4v s = float4v{0.0f, 0.0f, 0.0f, 0.0f};
                    mma(bv[m], hv, s, T());
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[m][n][v] += mine[n] == i ? s[v] : 0.0f;
                }
            }
        }
    }
}

__device__ __forceinline__ float lora_act(float t, int act)
{
    if (act == TVG_ACT_RELU) return t < 0.0f ? 0.0f : t;               // (a NaN stays one)
    if (act == TVG_ACT_SILU) return t / (1.0f + expf(-t));
    return t;
}

// The tail of a lane's four channels of a token.
template <typename T> __device__ __forceinline__ void store4(const LoraArgs &a, int row, int channel, const float4v &acc)
{
    if (row >= a.rows || channel >= a.k) return;
    const size_t at = (size_t)row * a.k + channel;
    const T *res = static_cast<const T *>(a.residual);
    T *y = static_cast<T *>(a.y);
    if (a.wide_y) {
        float f[4], r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        typedef typename Group4<T>::vec gvec;
        if (res) Group4<T>::unpack(*reinterpret_cast<const gvec *>(res + at), r);
#pragma unroll
        for (int v = 0; v < 4; ++v) f[v] = lora_act(acc[v] + (a.bias ? a.bias[channel + v] : 0.0f) + r[v], a.act);
        *reinterpret_cast<gvec *>(y + at) = Group4<T>::pack(f);
        return;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (channel + v < a.k) {
            const float t = acc[v] + (a.bias ? a.bias[channel + v] : 0.0f) + (res ? Elem<T>::load(res + at, v) : 0.0f);
            Elem<T>::store(y + at, v, lora_act(t, a.act));
        }
}

constexpr int kStep = 128;                 // bytes of the reduction per step

// Byte of a tile's 16-byte piece in LDS: rows of a step, pieces permuted so that 8 rows' reads fall into different banks.
__device__ __forceinline__ int piece_at(int row, int piece) { return row * kStep + ((piece ^ (row & 7)) << 4); }

// Any alignment: 64 tokens x 64 channels, four waves of 32 x 32; rows go through registers into LDS.
template <typename T> __global__ __launch_bounds__(256) void linear_lora_any_kernel(LoraArgs a)
{
    constexpr int E = kPer16<T>, TM = 64, TN = 64, kElems = kStep / (int)sizeof(T);
    __shared__ __align__(16) unsigned char lds[(TM + TN) * kStep];
    const int tile = xcd_remap(blockIdx.x, a.tiles);
    const int tm = tile / a.tiles_n, tn = tile - tm * a.tiles_n;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rsel = lane & 15, quad = lane >> 4;
    const int row0 = tm * TM, ch0 = tn * TN, wr = (wave & 1) * 32, wc = (wave >> 1) * 32;
    float4v acc[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    uint4v raw[4];
    const int piece = threadIdx.x & 7, prow = threadIdx.x >> 3;        // 32 rows a round
    const auto fetch = [&](int k) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = (r & 1) * 32 + prow;
            if (r < 2)
                raw[r] = row0 + row < a.rows ? load16(static_cast<const T *>(a.x) + (size_t)(row0 + row) * a.c, k + piece * E, a.c, a.wide_rows)
                                             : uint4v{0, 0, 0, 0};
            else
                raw[r] = ch0 + row < a.k ? load16(static_cast<const T *>(a.w) + (size_t)(ch0 + row) * a.c, k + piece * E, a.c, a.wide_rows)
                                         : uint4v{0, 0, 0, 0};
        }
    };
    fetch(0);
    for (int k = 0; k < a.c; k += kElems) {
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
            *reinterpret_cast<uint4v *>(lds + (r >> 1) * TM * kStep + piece_at((r & 1) * 32 + prow, piece)) = raw[r];
        __syncthreads();
        if (k + kElems < a.c) fetch(k + kElems);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint4v xv[2], wv[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                xv[i] = *reinterpret_cast<const uint4v *>(lds + piece_at(wr + i * 16 + rsel, s * 4 + quad));
                wv[i] = *reinterpret_cast<const uint4v *>(lds + TM * kStep + piece_at(wc + i * 16 + rsel, s * 4 + quad));
            }
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < 2; ++n) mma(wv[m], xv[n], acc[m][n], T());
        }
    }
    if (a.adapters > 0) add_adapters<T, 2, 2>(a, ch0 + wc, row0 + wr, lane, acc);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n) store4<T>(a, row0 + wr + n * 16 + rsel, ch0 + wc + m * 16 + quad * 4, acc[m][n]);
}

struct LoraPlan {
    int rblocks, splits, c_per_split;
    size_t h_bytes;
};

// Parts of the first launch's reduction: enough workgroups for every CU where rows are few, 512 channels at least.
LoraPlan plan_lora(const LoraProblem &p)
{
    LoraPlan plan;
    plan.rblocks = (p.rank + 15) / 16;
    const int tiles = (p.rows + 15) / 16;
    int splits = std::max(1, std::min(kComputeUnits / std::max(tiles, 1), p.c / 512));
    splits = std::min(splits, 8);
    plan.c_per_split = ((p.c + splits - 1) / splits + 127) / 128 * 128;
    plan.splits = (p.c + plan.c_per_split - 1) / plan.c_per_split;
    plan.h_bytes = (size_t)plan.splits * p.rows * plan.rblocks * 16 * sizeof(float);
    return plan;
}

}  // namespace

size_t linear_lora_workspace(const LoraProblem &p)
{
    return p.rows == 0 || p.adapters == 0 ? 0 : plan_lora(p).h_bytes;
}

tvg_status launch_linear_lora(const LoraProblem &p, const LoraPointers &ptr, hipStream_t stream)
{
    const LoraPlan plan = plan_lora(p);
    const int elem = p.dtype == TVG_BF16 ? 2 : 4;
    const auto aligned = [](const void *q, size_t n) { return reinterpret_cast<uintptr_t>(q) % n == 0; };
    LoraArgs a{};
    a.x = ptr.x; a.w = ptr.w; a.a = ptr.a; a.b = ptr.b; a.adapter = ptr.adapter; a.scale = ptr.scale; a.bias = ptr.bias;
    a.residual = ptr.residual; a.y = ptr.y; a.h = ptr.workspace;
    a.rows = p.rows; a.c = p.c; a.k = p.k; a.adapters = p.adapters; a.rank = p.rank; a.act = p.act;
    a.rblocks = plan.rblocks; a.splits = plan.splits; a.c_per_split = plan.c_per_split;
    a.wide_rows = p.c * (size_t)elem % 16 == 0 && aligned(ptr.x, 16) && aligned(ptr.w, 16) && aligned(ptr.a, 16);
    a.wide_rank = p.rank * (size_t)elem % 16 == 0 && aligned(ptr.b, 16);
    a.wide_y = p.k % 4 == 0 && aligned(ptr.y, 4 * elem) && aligned(ptr.residual, 4 * elem);
    if (p.adapters > 0) {
        const dim3 grid((p.rows + 15) / 16 * plan.splits);
        if (p.dtype == TVG_BF16) hipLaunchKernelGGL((lora_shrink_kernel<bf16_t>), grid, dim3(64 * kShrinkWaves), 0, stream, a);
        else hipLaunchKernelGGL((lora_shrink_kernel<float>), grid, dim3(64 * kShrinkWaves), 0, stream, a);
        if (hipGetLastError() != hipSuccess) return TVG_ERR_LAUNCH;
    }
    a.tiles_n = (p.k + 63) / 64;
    a.tiles = (p.rows + 63) / 64 * a.tiles_n;
    if (p.dtype == TVG_BF16) hipLaunchKernelGGL((linear_lora_any_kernel<bf16_t>), dim3(a.tiles), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((linear_lora_any_kernel<float>), dim3(a.tiles), dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

}  // namespace tvg
