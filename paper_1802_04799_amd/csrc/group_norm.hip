// Group norm with an activation over channels-last maps x [n][p][c], forward and backward.
//
//   mean, var over the p * (c / groups) elements of a group;  xhat = (x - mean) / sqrt(var + eps)
//   z = gamma xhat + beta,  y = act(z)
//   backward, with dz = dy act'(z), S1 = sum_p dz and S2 = sum_p dz xhat per sample and channel:
//   dbeta = sum_n S1, dgamma = sum_n S2, dx = rstd (gamma dz - (a + xhat b) / m)
//   with a, b the sums of gamma S1, gamma S2 over a group's channels and m its elements
//
// Bound by memory: about 10 (forward) or 25 (backward) operations an element.  Where a block of channels of a sample fits a
// workgroup's registers one launch reads it once (32 maps 56x56x256 in bf16, 51 MB read and written: 25 us a call among others, 4.1 TB/s
// of a copy's 5.1; 29 us in a trace, whose calls have gaps and colder caches, as the times of single kernels below).  Else two
// launches: the first leaves partial statistics of row chunks in the workspace, the second joins those of its sample in a fixed
// order and applies them, the last chunk first: it is the one whose rows the caches still hold (64 maps 112x112x256, 411 MB: 74 us
// and 149, 5.5 TB/s over both reads and the write; backward 147 us and 219, 5.6 TB/s over four reads and a write).
// Values are rounded to fewer bits once, as y or dx; statistics, sums, gamma, beta and their gradients are fp32.
//
// A workgroup covers a chunk of rows of one sample and a block of whole groups; a lane covers V adjacent channels (16
// bytes where the channels allow it) of every RP-th row, so that what it needs of a channel stays in registers and groups
// may begin and end anywhere in a vector.
//
// Variances are sums of squared distances from a mean that is known, never differences of large sums: a batch of rows in
// registers has its own mean, and batches, lanes and chunks are joined by
//   mean = mean_a + d n_b / n,  M2 = M2_a + M2_b + d^2 n_a n_b / n,  d = mean_b - mean_a.
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "tvg_device.h"
#include "tvg_internal.h"

namespace tvg {

namespace {

constexpr int kThreads = 256;
constexpr int kTeam = 16;                  // lanes that join the statistics of a group

// V elements of memory: 16 bytes or less.
template <typename T, int V> struct Vec {
    typedef T type __attribute__((ext_vector_type(V)));
    // LAST: the memory is not read again; NT: not soon
    template <bool LAST = false> static __device__ __forceinline__ type load(const T *p)
    {
        if constexpr (LAST) return __builtin_nontemporal_load(reinterpret_cast<const type *>(p));
        else return *reinterpret_cast<const type *>(p);
    }
    static __device__ __forceinline__ void get(const type &r, float *f)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(T) == 2) f[i] = bf16_to_f32(r[i]);
            else f[i] = r[i];
        }
    }
    template <bool NT = false> static __device__ __forceinline__ void store(T *p, const float *f)
    {
        type r;
        if constexpr (sizeof(T) == 2 && V > 1) {
            uint32_t w[V / 2];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) w[i] = f32x2_to_bf16x2(f[2 * i], f[2 * i + 1]);
            __builtin_memcpy(&r, w, sizeof(r));
        } else if constexpr (sizeof(T) == 2) r[0] = f32_to_bf16(f[0]);
        else {
#pragma unroll
            for (int i = 0; i < V; ++i) r[i] = f[i];
        }
        if constexpr (NT) __builtin_nontemporal_store(r, reinterpret_cast<type *>(p));
        else *reinterpret_cast<type *>(p) = r;
    }
};
template <typename T> struct Vec<T, 1> {
    typedef T type;
    template <bool LAST = false> static __device__ __forceinline__ type load(const T *p) { return *p; }
    static __device__ __forceinline__ void get(const type &r, float *f) { f[0] = Elem<T>::load(&r, 0); }
    template <bool NT = false> static __device__ __forceinline__ void store(T *p, const float *f) { Elem<T>::store(p, 0, f[0]); }
};

template <typename T, int ACT> __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == TVG_ACT_RELU) return z < 0.0f ? 0.0f : z;      // (a NaN stays one)
    if constexpr (ACT == TVG_ACT_SILU) return z * sigmoid<sizeof(T) == 4>(z);
    return z;
}

// dy times the activation's derivative at z.  bf16 takes 1 - s by subtraction: an error of |z| 2^-24 of dy in what dgamma, dbeta and
// the group's sums add up, up to z = 17 where s is 1, against the 2^-9 with which dy and x came (both of s and 1 - s from the exponential,
// 56.8 -> 63.3 us for 32 maps 56x56x256; fp32, where it counts, 48.7 -> 49.4 for 16).
template <typename T, int ACT> __device__ __forceinline__ float activate_grad(float dy, float z)
{
    if constexpr (ACT == TVG_ACT_RELU) return z <= 0.0f ? 0.0f : dy;
    if constexpr (ACT == TVG_ACT_SILU) {
        Sigmoid g;
        if constexpr (sizeof(T) == 4) g = sigmoid_and_rest(z);
        else {
            g.s = sigmoid<false>(z);
            g.rest = 1.0f - g.s;
        }
        return dy * fmaf(z * g.s, g.rest, g.s);            // s (1 + z (1 - s))
    }
    return dy;
}

struct NormArgs {
    const void *x, *dy;
    const float *gamma, *beta;
    void *y;                               // dx in the backward pass
    float *mean, *rstd;
    float *part;                           // [n][groups][chunks][2]
    float *chan;                           // backward: [n][chunks][c][2]
    float *dgamma, *dbeta;
    int n, p, c, groups, cpg, block, blocks, rows, chunks;      // channels per block, rows per chunk
    int tiles;                             // n * blocks * chunks
    float eps;
    int act;
    int passing;                           // one launch: results pass the caches by; two: x does when it is read last (results always do)
};

// The part of the problem that a workgroup has.
struct Tile {
    int sample, chunk, c0, width, row0, row1, cols, rp;
};

template <int V> __device__ __forceinline__ Tile tile_of(const NormArgs &a, int t)
{
    Tile r;
    r.chunk = t % a.chunks;
    const int b = t / a.chunks;
    r.c0 = b % a.blocks * a.block;
    r.sample = b / a.blocks;
    r.width = min(a.block, a.c - r.c0);
    r.row0 = r.chunk * a.rows;
    r.row1 = min(r.row0 + a.rows, a.p);
    r.cols = min(r.width / V, kThreads);
    r.rp = kThreads / r.cols;
    return r;
}

// Sum over the lanes of a team; the result in all of them.
template <int TEAM = kTeam> __device__ __forceinline__ float team_sum(float v)
{
#pragma unroll
    for (int d = 1; d < TEAM; d *= 2) v += __shfl_xor(v, d, TEAM);
    return v;
}

// f(i, group) for the channels cc + i of a lane, groups counted from the block's first.
template <int V, bool WHOLE, typename F> __device__ __forceinline__ void for_channels(int cc, int cpg, F &&f)
{
    int c;
    int g = fast_div(cc, cpg, 1.0f / (float)cpg, &c);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        f(i, g);
        if constexpr (!WHOLE) {
            const bool next = ++c == cpg;
            g += next;
            c = next ? 0 : c;
        }
    }
}

// The pairs of a group's chunks k0 to k0 + 63, eight lanes a group: all loads of a lane are under way together.
constexpr int kPairTeam = 8, kPairs = 8, kPairChunks = kPairTeam * kPairs;
__device__ __forceinline__ void load_pairs(const NormArgs &a, int sample, int group, int k0, int tl, float2 (&v)[kPairs])
{
    const float2 *part = reinterpret_cast<const float2 *>(a.part) + ((size_t)sample * a.groups + group) * a.chunks;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const int k = k0 + tl + i * kPairTeam;
        v[i] = k < a.chunks ? part[k] : float2{0.0f, 0.0f};
    }
}

// U rows of a lane's channels joined to its running mean and M2 of `count` rows (rows beyond `left` do not count).
template <typename T, int V, int U, bool FULL>
__device__ __forceinline__ void join_rows(const typename Vec<T, V>::type (&raw)[U], int valid, int count, float (&mean)[V],
                                          float (&m2)[V])
{
    const float n = FULL ? (float)U : (float)valid;
    const float inv = FULL ? 1.0f / U : 1.0f / n;
    const float share = n / (n + (float)count), cross = share * (float)count;
    float sum[V], sq[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = sq[i] = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[V];
        Vec<T, V>::get(raw[u], f);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += FULL || u < valid ? f[i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] *= inv;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[V];
        Vec<T, V>::get(raw[u], f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = f[i] - sum[i];
            sq[i] = FULL || u < valid ? fmaf(d, d, sq[i]) : sq[i];
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float d = sum[i] - mean[i];
        mean[i] = fmaf(d, share, mean[i]);
        m2[i] += fmaf(d, d * cross, sq[i]);                // (of the first rows cross is 0, d the mean, whose square may be infinite)
    }
}

// Statistics of a chunk.  LDS: per entry of a pass the lanes' mean and M2, then per group (elements, mean, M2).  Eight rows in
// flight a lane: 64 maps 112x112x256 74 us, 5.5 TB/s with what the caches hold of a call before.
template <typename T, int V, bool WHOLE> __global__ __launch_bounds__(kThreads) void group_norm_stats_kernel(NormArgs a)
{
    constexpr int U = 8, Q = WHOLE ? 1 : V;                // entries per lane
    extern __shared__ float lds[];
    float *lane_mean = lds, *lane_m2 = lds + kThreads * Q, *group = lds + 2 * kThreads * Q;
    const Tile t = tile_of<V>(a, blockIdx.x);
    const int g0 = t.c0 / a.cpg, ng = t.width / a.cpg;
    int col;
    const int rp = fast_div(threadIdx.x, t.cols, 1.0f / (float)t.cols, &col);
    const T *x = static_cast<const T *>(a.x) + ((size_t)t.sample * a.p) * a.c + t.c0;
    const int each = (t.row1 - t.row0) / t.rp, more = (t.row1 - t.row0) % t.rp;        // rows of a lane
    for (int g = threadIdx.x; g < ng; g += kThreads) group[3 * g] = group[3 * g + 1] = group[3 * g + 2] = 0.0f;
    for (int pass = 0; pass * t.cols * V < t.width; ++pass) {
        const int first = pass * t.cols * V, cc = first + col * V;        // channels of the pass, of this lane
        const int pass_width = min(t.cols * V, t.width - first);
        float mean[V], m2[V];
        int count = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) mean[i] = m2[i] = 0.0f;
        if (rp < t.rp && cc < t.width) {
            typename Vec<T, V>::type raw[U];
            int row = t.row0 + rp;
            for (; row + (U - 1) * t.rp < t.row1; row += U * t.rp) {
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = Vec<T, V>::load(x + (size_t)(row + u * t.rp) * a.c + cc);
                join_rows<T, V, U, true>(raw, U, count, mean, m2);
                count += U;
            }
            if (row < t.row1) {
                const int valid = (t.row1 - row + t.rp - 1) / t.rp;
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = Vec<T, V>::load(x + (size_t)(u < valid ? row + u * t.rp : row) * a.c + cc);
                join_rows<T, V, U, false>(raw, valid, count, mean, m2);
                count += valid;
            }
        }
        __syncthreads();                                   // (the previous pass has been read)
        if constexpr (WHOLE) {                             // the lane's channels are of one group
            float m = 0.0f, q = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) m += mean[i];
            m *= 1.0f / V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = mean[i] - m;
                q += fmaf(d * d, (float)count, m2[i]);
            }
            lane_mean[threadIdx.x] = m;
            lane_m2[threadIdx.x] = q;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                lane_mean[threadIdx.x * V + i] = mean[i];
                lane_m2[threadIdx.x * V + i] = m2[i];
            }
        }
        __syncthreads();
        // a team joins the entries of a group in this pass: rp lanes per column, of known row counts
        constexpr int P = V / Q;                           // channels per entry
        const int team = threadIdx.x / kTeam, tl = threadIdx.x % kTeam, row_entries = t.cols * Q;
        for (int g = first / a.cpg + team; g * a.cpg < first + pass_width; g += kThreads / kTeam) {
            const int lo = max(g * a.cpg, first), hi = min((g + 1) * a.cpg, first + pass_width);
            const int base = (lo - first) / P, w = (hi - lo) / P;
            const int entries = w * t.rp, rows = t.row1 - t.row0;
            const float inv_w = 1.0f / (float)w;
            const auto rows_of = [&](int r) { return each + (r < more); };     // (every rp-th)
            float s = 0.0f;
            for (int e = tl; e < entries; e += kTeam) {
                int c;
                const int r = fast_div(e, w, inv_w, &c);
                s += (float)rows_of(r) * lane_mean[r * row_entries + base + c];
            }
            const float m = team_sum(s) / ((float)rows * (float)w), total = (float)rows * (float)(w * P);
            float q = 0.0f;
            for (int e = tl; e < entries; e += kTeam) {
                int c;
                const int r = fast_div(e, w, inv_w, &c), at = r * row_entries + base + c, n = rows_of(r);
                const float d = lane_mean[at] - m;
                q += n ? fmaf(d * d, (float)(n * P), lane_m2[at]) : 0.0f;
            }
            q = team_sum(q);
            if (tl == 0) {
                float *o = group + 3 * g;
                const float before = o[0], all = before + total, d = m - o[1];
                o[0] = all;
                o[1] += d * (total / all);
                o[2] += q + d * (d * (before * (total / all)));        // (as above)
            }
        }
    }
    __syncthreads();
    for (int g = threadIdx.x; g < ng; g += kThreads) {
        float *o = a.part + (((size_t)t.sample * a.groups + g0 + g) * a.chunks + t.chunk) * 2;
        o[0] = group[3 * g + 1];
        o[1] = group[3 * g + 2];
    }
}

// Mean and 1/sqrt(var + eps) of the tile's groups from the chunks' partial statistics, into LDS.
__device__ __forceinline__ void join_chunks(const NormArgs &a, const Tile &t, int g0, int ng, float *gmean, float *grstd)
{
    const int team = threadIdx.x / kPairTeam, tl = threadIdx.x % kPairTeam;
    const float total = (float)a.p;                        // (in rows: every chunk has cpg channels a row)
    for (int g = team; g < ng; g += kThreads / kPairTeam) {
        float2 v[kPairs];
        const auto rows = [&](int k) { return (float)max(0, min(a.rows, a.p - k * a.rows)); };
        float s = 0.0f, q = 0.0f;
        for (int k0 = 0; k0 < a.chunks; k0 += kPairChunks) {
            load_pairs(a, t.sample, g0 + g, k0, tl, v);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) s += rows(k0 + tl + i * kPairTeam) * v[i].x;
        }
        const float m = team_sum<kPairTeam>(s) / total;
        for (int k0 = 0; k0 < a.chunks; k0 += kPairChunks) {
            if (a.chunks > kPairChunks) load_pairs(a, t.sample, g0 + g, k0, tl, v);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                const float d = v[i].x - m, n = rows(k0 + tl + i * kPairTeam) * (float)a.cpg;
                q += n > 0.0f ? fmaf(d * d, n, v[i].y) : 0.0f;
            }
        }
        q = team_sum<kPairTeam>(q);
        if (tl == 0) {
            const float r = 1.0f / sqrtf(q / (total * (float)a.cpg) + a.eps);
            gmean[g] = m;
            grstd[g] = r;
            if (t.chunk == 0 && a.mean) a.mean[(size_t)t.sample * a.groups + g0 + g] = m;
            if (t.chunk == 0 && a.rstd) a.rstd[(size_t)t.sample * a.groups + g0 + g] = r;
        }
    }
}

// y from the statistics of all chunks, which every workgroup joins for its own groups (a launch between would cost 4 us).
// 64 maps 112x112x256: 149 us, 822 MB at 5.5 TB/s.
template <typename T, int V, int ACT, bool WHOLE, bool PASS> __global__ __launch_bounds__(kThreads) void group_norm_apply_kernel(NormArgs a)
{
    constexpr int U = 4;
    extern __shared__ float lds[];
    const Tile t = tile_of<V>(a, a.tiles - 1 - blockIdx.x);
    const int g0 = t.c0 / a.cpg, ng = t.width / a.cpg;
    float *gmean = lds, *grstd = lds + ng;
    int col;
    const int rp = fast_div(threadIdx.x, t.cols, 1.0f / (float)t.cols, &col);
    const T *x = static_cast<const T *>(a.x) + ((size_t)t.sample * a.p) * a.c + t.c0;
    T *y = static_cast<T *>(a.y) + ((size_t)t.sample * a.p) * a.c + t.c0;
    bool joined = false;
    for (int cc = col * V, pass = 0; pass * t.cols * V < t.width; ++pass, cc += t.cols * V) {
        const bool active = rp < t.rp && cc < t.width;
        // the first rows and the parameters are under way while the chunks are joined
        typename Vec<T, V>::type raw[U];
        float mean[V], mul[V], add[V];
        int row = t.row0 + rp;
        const auto load = [&] {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (row + u * t.rp < t.row1) raw[u] = Vec<T, V>::template load<PASS>(x + (size_t)(row + u * t.rp) * a.c + cc);
        };
        if (active) {
            load();
#pragma unroll
            for (int i = 0; i < V; ++i) {
                mul[i] = a.gamma ? a.gamma[t.c0 + cc + i] : 1.0f;
                add[i] = a.beta ? a.beta[t.c0 + cc + i] : 0.0f;
            }
        }
        if (!joined) {
            join_chunks(a, t, g0, ng, gmean, grstd);
            __syncthreads();
            joined = true;
        }
        if (!active) continue;
        for_channels<V, WHOLE>(cc, a.cpg, [&](int i, int g) {
            mean[i] = gmean[g];
            mul[i] *= grstd[g];
        });
        for (; row < t.row1; row += U * t.rp, load()) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (row + u * t.rp >= t.row1) break;
                float f[V];
                Vec<T, V>::get(raw[u], f);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = activate<T, ACT>(fmaf(f[i] - mean[i], mul[i], add[i]));
                Vec<T, V>::template store<true>(y + (size_t)(row + u * t.rp) * a.c + cc, f);
            }
        }
    }
}

// What a lane of the backward pass needs of its channels: with d = x - mean, z = mul d + add, S2 = rstd sum dz d, and
// dx = mul dz - (rstd a + rstd^2 b d).
template <int V, bool WHOLE> struct Channels {
    float mean[V], rstd[V], mul[V], add[V];
    __device__ __forceinline__ void load(const NormArgs &a, const Tile &t, int g0, int cc)
    {
        const size_t at = (size_t)t.sample * a.groups + g0;
        for_channels<V, WHOLE>(cc, a.cpg, [&](int i, int g) {
            if (!WHOLE || i == 0) {
                mean[i] = a.mean[at + g];
                rstd[i] = a.rstd[at + g];
            } else {
                mean[i] = mean[0];
                rstd[i] = rstd[0];
            }
            mul[i] = a.gamma ? a.gamma[t.c0 + cc + i] : 1.0f;
            add[i] = a.beta ? a.beta[t.c0 + cc + i] : 0.0f;
        });
#pragma unroll
        for (int i = 0; i < V; ++i) mul[i] *= rstd[i];
    }
};

// S1 and S2 of a chunk's rows per channel, and gamma's sums of them per group.  64 maps 112x112x256: 147 us, 822 MB at 5.6 TB/s.
template <typename T, int V, int ACT, bool WHOLE> __global__ __launch_bounds__(kThreads) void group_norm_grad_sums_kernel(NormArgs a)
{
    constexpr int U = 4;
    extern __shared__ float lds[];
    float *lane1 = lds, *lane2 = lds + kThreads * V, *group = lds + 2 * kThreads * V;
    const Tile t = tile_of<V>(a, blockIdx.x);
    const int g0 = t.c0 / a.cpg, ng = t.width / a.cpg;
    int col;
    const int rp = fast_div(threadIdx.x, t.cols, 1.0f / (float)t.cols, &col);
    const size_t at0 = ((size_t)t.sample * a.p) * a.c + t.c0;
    const T *x = static_cast<const T *>(a.x) + at0, *dy = static_cast<const T *>(a.dy) + at0;
    for (int g = threadIdx.x; g < ng; g += kThreads) group[2 * g] = group[2 * g + 1] = 0.0f;
    for (int pass = 0; pass * t.cols * V < t.width; ++pass) {
        const int first = pass * t.cols * V, cc = first + col * V;
        const int pass_width = min(t.cols * V, t.width - first);
        float s1[V], s2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s1[i] = s2[i] = 0.0f;
        if (rp < t.rp && cc < t.width) {
            int row = t.row0 + rp;
            typename Vec<T, V>::type rx[U], rd[U];
            const auto load = [&] {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (row + u * t.rp < t.row1) {
                        const size_t at = (size_t)(row + u * t.rp) * a.c + cc;
                        rx[u] = Vec<T, V>::load(x + at);
                        rd[u] = Vec<T, V>::load(dy + at);
                    }
            };
            load();
            Channels<V, WHOLE> k;
            k.load(a, t, g0, cc);
            for (; row < t.row1; row += U * t.rp, load()) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (row + u * t.rp >= t.row1) break;
                    float fx[V], fd[V];
                    Vec<T, V>::get(rx[u], fx);
                    Vec<T, V>::get(rd[u], fd);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float d = fx[i] - k.mean[i];
                        const float dz = activate_grad<T, ACT>(fd[i], fmaf(d, k.mul[i], k.add[i]));
                        s1[i] += dz;
                        s2[i] = fmaf(dz, d, s2[i]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) s2[i] *= k.rstd[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lane1[threadIdx.x * V + i] = s1[i];
            lane2[threadIdx.x * V + i] = s2[i];
        }
        __syncthreads();
        // per channel, into the first row of lanes and the workspace
        for (int c = threadIdx.x; c < pass_width; c += kThreads) {
            float v1 = 0.0f, v2 = 0.0f;
#pragma unroll 8
            for (int r = 0; r < t.rp; ++r) {
                v1 += lane1[r * t.cols * V + c];
                v2 += lane2[r * t.cols * V + c];
            }
            float *o = a.chan + (((size_t)t.sample * a.chunks + t.chunk) * a.c + t.c0 + first + c) * 2;
            o[0] = v1;
            o[1] = v2;
            const float gm = a.gamma ? a.gamma[t.c0 + first + c] : 1.0f;
            lane1[c] = v1 * gm;
            lane2[c] = v2 * gm;
        }
        __syncthreads();
        const int team = threadIdx.x / kTeam, tl = threadIdx.x % kTeam;
        for (int g = first / a.cpg + team; g * a.cpg < first + pass_width; g += kThreads / kTeam) {
            const int lo = max(g * a.cpg, first), hi = min((g + 1) * a.cpg, first + pass_width);
            float v1 = 0.0f, v2 = 0.0f;
            for (int c = lo + tl; c < hi; c += kTeam) {
                v1 += lane1[c - first];
                v2 += lane2[c - first];
            }
            v1 = team_sum(v1);
            v2 = team_sum(v2);
            if (tl == 0) {
                group[2 * g] += v1;
                group[2 * g + 1] += v2;
            }
        }
    }
    __syncthreads();
    for (int g = threadIdx.x; g < ng; g += kThreads) {
        float *o = a.part + (((size_t)t.sample * a.groups + g0 + g) * a.chunks + t.chunk) * 2;
        o[0] = group[2 * g];
        o[1] = group[2 * g + 1];
    }
}

constexpr int kReduceChannels = 16;        // channels of a workgroup that adds up dgamma and dbeta

// dgamma and dbeta of kReduceChannels channels: the sums of all samples' chunks.
__device__ __forceinline__ void reduce_channels(const NormArgs &a, int rows, int c0, float *lds)
{
    const int lc = threadIdx.x % kReduceChannels, lr = threadIdx.x / kReduceChannels, c = c0 + lc;
    constexpr int kLanes = kThreads / kReduceChannels;
    float v1 = 0.0f, v2 = 0.0f;
    if (c < a.c)
#pragma unroll 8
        for (int r = lr; r < rows; r += kLanes) {
            const float2 v = reinterpret_cast<const float2 *>(a.chan)[(size_t)r * a.c + c];
            v1 += v.x;
            v2 += v.y;
        }
    lds[threadIdx.x] = v1;
    lds[kThreads + threadIdx.x] = v2;
    __syncthreads();
    if (lr == 0 && c < a.c) {
        for (int r = 1; r < kLanes; ++r) {
            v1 += lds[r * kReduceChannels + lc];
            v2 += lds[kThreads + r * kReduceChannels + lc];
        }
        if (a.dbeta) a.dbeta[c] = v1;
        if (a.dgamma) a.dgamma[c] = v2;
    }
}

// The first workgroups add up dgamma and dbeta, the others write dx: z and its derivative again from x, cheaper than a stored dz.
// 64 maps 112x112x256: 219 us, 1233 MB at 5.6 TB/s.
template <typename T, int V, int ACT, bool WHOLE, bool PASS>
__global__ __launch_bounds__(kThreads) void group_norm_grad_apply_kernel(NormArgs a, int reducers)
{
    constexpr int U = 4;
    extern __shared__ float lds[];
    if ((int)blockIdx.x < reducers) {
        reduce_channels(a, a.n * a.chunks, blockIdx.x * kReduceChannels, lds);
        return;
    }
    const Tile t = tile_of<V>(a, a.tiles - 1 - (blockIdx.x - reducers));
    const int g0 = t.c0 / a.cpg, ng = t.width / a.cpg;
    float *ga = lds, *gb = lds + ng;
    int col;
    const int rp = fast_div(threadIdx.x, t.cols, 1.0f / (float)t.cols, &col);
    const size_t at0 = ((size_t)t.sample * a.p) * a.c + t.c0;
    const T *x = static_cast<const T *>(a.x) + at0, *dy = static_cast<const T *>(a.dy) + at0;
    T *dx = static_cast<T *>(a.y) + at0;
    bool joined = false;
    for (int cc = col * V, pass = 0; pass * t.cols * V < t.width; ++pass, cc += t.cols * V) {
        const bool active = rp < t.rp && cc < t.width;
        typename Vec<T, V>::type rx[U], rd[U];
        int row = t.row0 + rp;
        const auto load = [&] {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (row + u * t.rp < t.row1) {
                    const size_t at = (size_t)(row + u * t.rp) * a.c + cc;
                    rx[u] = Vec<T, V>::template load<PASS>(x + at);
                    rd[u] = Vec<T, V>::template load<PASS>(dy + at);
                }
        };
        Channels<V, WHOLE> k;
        if (active) {
            load();
            k.load(a, t, g0, cc);
        }
        if (!joined) {
            const int team = threadIdx.x / kPairTeam, tl = threadIdx.x % kPairTeam;
            const float inv = 1.0f / ((float)a.p * (float)a.cpg);
            for (int g = team; g < ng; g += kThreads / kPairTeam) {
                float v1 = 0.0f, v2 = 0.0f;
                for (int k0 = 0; k0 < a.chunks; k0 += kPairChunks) {
                    float2 v[kPairs];
                    load_pairs(a, t.sample, g0 + g, k0, tl, v);
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        v1 += v[i].x;
                        v2 += v[i].y;
                    }
                }
                v1 = team_sum<kPairTeam>(v1);
                v2 = team_sum<kPairTeam>(v2);
                if (tl == 0) {
                    ga[g] = v1 * inv;
                    gb[g] = v2 * inv;
                }
            }
            __syncthreads();
            joined = true;
        }
        if (!active) continue;
        float sa[V], sb[V];
        for_channels<V, WHOLE>(cc, a.cpg, [&](int i, int g) {
            sa[i] = ga[g] * k.rstd[i];
            sb[i] = gb[g] * k.rstd[i] * k.rstd[i];             // (rstd^2 alone may be infinite)
        });
        for (; row < t.row1; row += U * t.rp, load()) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (row + u * t.rp >= t.row1) break;
                float fx[V], fd[V];
                Vec<T, V>::get(rx[u], fx);
                Vec<T, V>::get(rd[u], fd);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = fx[i] - k.mean[i];
                    const float dz = activate_grad<T, ACT>(fd[i], fmaf(d, k.mul[i], k.add[i]));
                    fx[i] = fmaf(dz, k.mul[i], -fmaf(d, sb[i], sa[i]));
                }
                Vec<T, V>::template store<true>(dx + (size_t)(row + u * t.rp) * a.c + cc, fx);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------
// One launch, where a sample's block of channels fits the registers of a workgroup: NV vectors a lane, read once.
// Mean first, then the squared distances from it, both over the workgroup's LDS.  Bound by latency where it is small (one map
// 7x7x512 5.3 us: a launch, a read, two sums over LDS), by reading and writing in turn where it is large (51 MB 29 us).
// ---------------------------------------------------------------------------------------

// Sums over the channels and lanes of every group, given a value per channel and lane in LDS ([rp][width]); f(group, sum) by
// one lane of the group's team.
template <typename F>
__device__ __forceinline__ void sum_groups(const float *values, int width, int rp, int cpg, int ng, int team, int threads, F &&f)
{
    const int tl = threadIdx.x & (team - 1);
    const float inv = 1.0f / (float)cpg;
    for (int g = threadIdx.x / team; g < ng; g += threads / team) {
        float s = 0.0f;
        for (int e = tl; e < rp * cpg; e += team) {
            int c;
            const int r = fast_div(e, cpg, inv, &c);
            s += values[r * width + g * cpg + c];
        }
        for (int d = 1; d < team; d *= 2) s += __shfl_xor(s, d);
        if (tl == 0) f(g, s);
    }
}

template <typename T, int V, int NV, int THREADS, bool WHOLE> __global__ __launch_bounds__(THREADS) void group_norm_once_kernel(NormArgs a, int team)
{
    constexpr int Q = WHOLE ? 1 : V;                       // entries per lane
    extern __shared__ float lds[];
    const int b = xcd_remap(blockIdx.x, a.tiles);          // (neighbouring blocks share lines of memory)
    const int sample = b / a.blocks, c0 = (b - sample * a.blocks) * a.block, width = min(a.block, a.c - c0);
    const int cols = width / V, ng = width / a.cpg;
    int col;
    const int rp = THREADS / cols, lane_row = fast_div(threadIdx.x, cols, 1.0f / (float)cols, &col);
    const bool active = lane_row < rp;
    const int cc = col * V;
    float *values = lds, *gmean = lds + THREADS * Q, *grstd = gmean + ng;
    const size_t at0 = ((size_t)sample * a.p) * a.c + c0 + cc;
    const T *x = static_cast<const T *>(a.x) + at0;
    T *y = static_cast<T *>(a.y) + at0;
    typename Vec<T, V>::type raw[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int row = lane_row + u * rp;
        if (active && row < a.p) raw[u] = Vec<T, V>::load(x + (size_t)row * a.c);
    }
    float mul[V], add[V], sum[V], mean[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        mul[i] = a.gamma ? a.gamma[c0 + cc + i] : 1.0f;
        add[i] = a.beta ? a.beta[c0 + cc + i] : 0.0f;
        sum[i] = 0.0f;
    }
    const auto put = [&] {                                 // the lane's sums to LDS
        if (!active) return;
        if constexpr (WHOLE) {
#pragma unroll
            for (int d = 1; d < V; d *= 2)
#pragma unroll
                for (int i = 0; i < V; i += 2 * d) sum[i] += sum[i + d];
            values[lane_row * cols + col] = sum[0];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) values[lane_row * width + cc + i] = sum[i];
        }
    };
#pragma unroll
    for (int u = 0; u < NV; ++u)
        if (active && lane_row + u * rp < a.p) {
            float f[V];
            Vec<T, V>::get(raw[u], f);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += f[i];
        }
    put();
    __syncthreads();
    const float count = (float)a.p * (float)a.cpg;
    constexpr int P = V / Q;                               // channels per entry
    sum_groups(values, width / P, rp, a.cpg / P, ng, team, THREADS, [&](int g, float s) { gmean[g] = s / count; });
    __syncthreads();
    if (active) for_channels<V, WHOLE>(cc, a.cpg, [&](int i, int g) { mean[i] = gmean[g]; });
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u)
        if (active && lane_row + u * rp < a.p) {
            float f[V];
            Vec<T, V>::get(raw[u], f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = f[i] - mean[i];
                sum[i] = fmaf(d, d, sum[i]);
            }
        }
    put();
    __syncthreads();
    const size_t stat = (size_t)sample * a.groups + c0 / a.cpg;
    sum_groups(values, width / P, rp, a.cpg / P, ng, team, THREADS, [&](int g, float s) {
        const float r = 1.0f / sqrtf(s / count + a.eps);
        grstd[g] = r;
        if (a.mean) a.mean[stat + g] = gmean[g];
        if (a.rstd) a.rstd[stat + g] = r;
    });
    __syncthreads();
    if (!active) return;
    for_channels<V, WHOLE>(cc, a.cpg, [&](int i, int g) { mul[i] *= grstd[g]; });
    const auto write_as = [&](auto act, auto pass) {
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int row = lane_row + u * rp;
            if (row >= a.p) break;
            float f[V];
            Vec<T, V>::get(raw[u], f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = activate<T, decltype(act)::value>(fmaf(f[i] - mean[i], mul[i], add[i]));
            Vec<T, V>::template store<decltype(pass)::value>(y + (size_t)row * a.c, f);
        }
    };
    const auto write = [&](auto act) {
        if (a.passing) write_as(act, std::true_type());
        else write_as(act, std::false_type());
    };
    if (a.act == TVG_ACT_SILU) write(std::integral_constant<int, TVG_ACT_SILU>());
    else if (a.act == TVG_ACT_RELU) write(std::integral_constant<int, TVG_ACT_RELU>());
    else write(std::integral_constant<int, TVG_ACT_NONE>());
}

template <typename T, int V, bool WHOLE> tvg_status launch_once(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    const int ng = a.block / a.cpg;
    int team = 64;
    while (team > 1 && ng * team > plan.threads) team /= 2;
    const size_t lds = ((size_t)plan.threads * V + 2 * ng) * sizeof(float);
    if (plan.threads == 256) hipLaunchKernelGGL((group_norm_once_kernel<T, V, 4, 256, WHOLE>), dim3(a.tiles), dim3(256), lds, stream, a, team);
    else if (plan.threads == 512) hipLaunchKernelGGL((group_norm_once_kernel<T, V, 8, 512, WHOLE>), dim3(a.tiles), dim3(512), lds, stream, a, team);
    else hipLaunchKernelGGL((group_norm_once_kernel<T, V, 16, 1024, WHOLE>), dim3(a.tiles), dim3(1024), lds, stream, a, team);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

// The same for the backward pass: x and dy in registers.  The sums of a sample's channels go to the workspace ([n][c][2]), or,
// of the only sample, to dgamma and dbeta.  2 maps 14x14x256 in fp32: 6.7 us and 1.6 of the launch that adds up the samples.
constexpr int kSumParts = 16;
template <typename T, int V, int NV, int THREADS, bool WHOLE> __global__ __launch_bounds__(THREADS) void group_norm_grad_once_kernel(NormArgs a)
{
    extern __shared__ float lds[];
    const int b = xcd_remap(blockIdx.x, a.tiles);
    Tile t;
    t.sample = b / a.blocks;
    t.c0 = (b - t.sample * a.blocks) * a.block;
    const int width = min(a.block, a.c - t.c0), cols = width / V, ng = width / a.cpg, g0 = t.c0 / a.cpg;
    int col;
    const int rp = THREADS / cols, lane_row = fast_div(threadIdx.x, cols, 1.0f / (float)cols, &col);
    const bool active = lane_row < rp;
    const int cc = col * V;
    float *values = lds, *parts = lds + THREADS * V, *sums = parts + kSumParts * width, *group = sums + 2 * width;
    const size_t at0 = ((size_t)t.sample * a.p) * a.c + t.c0 + cc;
    const T *x = static_cast<const T *>(a.x) + at0, *dy = static_cast<const T *>(a.dy) + at0;
    T *dx = static_cast<T *>(a.y) + at0;
    typename Vec<T, V>::type rx[NV], rd[NV];
    Channels<V, WHOLE> k;
    if (active) {
#pragma unroll
        for (int u = 0; u < NV; ++u)
            if (lane_row + u * rp < a.p) {
                rx[u] = Vec<T, V>::load(x + (size_t)(lane_row + u * rp) * a.c);
                rd[u] = Vec<T, V>::load(dy + (size_t)(lane_row + u * rp) * a.c);
            }
        k.load(a, t, g0, cc);
    }
    const auto rows = [&](auto act, auto &&f) {            // f(u, x, dz of i, which also gives d) of the lane's rows
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            if (lane_row + u * rp >= a.p) break;
            float fx[V], fd[V];
            Vec<T, V>::get(rx[u], fx);
            Vec<T, V>::get(rd[u], fd);
            f(u, fx, [&](int i, float &d) {
                d = fx[i] - k.mean[i];
                return activate_grad<T, decltype(act)::value>(fd[i], fmaf(d, k.mul[i], k.add[i]));
            });
        }
    };
    const auto with_act = [&](auto &&f) {
        if (a.act == TVG_ACT_SILU) f(std::integral_constant<int, TVG_ACT_SILU>());
        else if (a.act == TVG_ACT_RELU) f(std::integral_constant<int, TVG_ACT_RELU>());
        else f(std::integral_constant<int, TVG_ACT_NONE>());
    };
    float s[2][V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[0][i] = s[1][i] = 0.0f;
    if (active)
        with_act([&](auto act) {
            rows(act, [&](int, float (&)[V], auto &&dz_of) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float d;
                    const float dz = dz_of(i, d);
                    s[0][i] += dz;
                    s[1][i] = fmaf(dz, d, s[1][i]);
                }
            });
#pragma unroll
            for (int i = 0; i < V; ++i) s[1][i] *= k.rstd[i];
        });
    const int lanes = min(kSumParts, rp);
    int c;
    const int part = fast_div(threadIdx.x, width, 1.0f / (float)width, &c);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (active) {
#pragma unroll
            for (int i = 0; i < V; ++i) values[lane_row * width + cc + i] = s[q][i];
        }
        __syncthreads();
        // a channel's lanes by `lanes` threads, then those
        const int stride = max(1, min(lanes, THREADS / width));
        for (int c1 = c, p1 = part; c1 < width && p1 < stride; c1 += width <= THREADS ? width : THREADS) {
            float v = 0.0f;
#pragma unroll 4
            for (int r = p1; r < rp; r += stride) v += values[r * width + c1];
            parts[p1 * width + c1] = v;
        }
        __syncthreads();
        for (int c1 = threadIdx.x; c1 < width; c1 += THREADS) {
            float v = 0.0f;
            for (int r = 0; r < stride; ++r) v += parts[r * width + c1];
            sums[q * width + c1] = v;
        }
        __syncthreads();
    }
    for (int c1 = threadIdx.x; c1 < width; c1 += THREADS) {
        const float v1 = sums[c1], v2 = sums[width + c1];
        if (a.n > 1) {
            reinterpret_cast<float2 *>(a.chan)[(size_t)t.sample * a.c + t.c0 + c1] = float2{v1, v2};
        } else {
            if (a.dbeta) a.dbeta[t.c0 + c1] = v1;
            if (a.dgamma) a.dgamma[t.c0 + c1] = v2;
        }
    }
    {
        const int team = threadIdx.x / kPairTeam, tl = threadIdx.x % kPairTeam;
        const float inv = 1.0f / ((float)a.p * (float)a.cpg);
        for (int g = team; g < ng; g += THREADS / kPairTeam) {
            float v1 = 0.0f, v2 = 0.0f;
            for (int i = tl; i < a.cpg; i += kPairTeam) {
                const int c1 = g * a.cpg + i;
                const float gm = a.gamma ? a.gamma[t.c0 + c1] : 1.0f;
                v1 = fmaf(gm, sums[c1], v1);
                v2 = fmaf(gm, sums[width + c1], v2);
            }
            v1 = team_sum<kPairTeam>(v1);
            v2 = team_sum<kPairTeam>(v2);
            if (tl == 0) {
                group[2 * g] = v1 * inv;
                group[2 * g + 1] = v2 * inv;
            }
        }
    }
    __syncthreads();
    if (!active) return;
    float sa[V], sb[V];
    for_channels<V, WHOLE>(cc, a.cpg, [&](int i, int g) {
        sa[i] = group[2 * g] * k.rstd[i];
        sb[i] = group[2 * g + 1] * k.rstd[i] * k.rstd[i];  // (rstd^2 alone may be infinite)
    });
    const auto write = [&](auto act, auto pass) {
        rows(act, [&](int u, float (&fx)[V], auto &&dz_of) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float d;
                const float dz = dz_of(i, d);
                fx[i] = fmaf(dz, k.mul[i], -fmaf(d, sb[i], sa[i]));
            }
            Vec<T, V>::template store<decltype(pass)::value>(dx + (size_t)(lane_row + u * rp) * a.c, fx);
        });
    };
    with_act([&](auto act) {
        if (a.passing) write(act, std::true_type());
        else write(act, std::false_type());
    });
}

__global__ __launch_bounds__(kThreads) void group_norm_reduce_kernel(NormArgs a, int rows)
{
    __shared__ float lds[2 * kThreads];
    reduce_channels(a, rows, blockIdx.x * kReduceChannels, lds);
}

template <typename T, int V, bool WHOLE> tvg_status launch_grad_once(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    const size_t lds = ((size_t)plan.threads * V + (kSumParts + 2) * a.block + 2 * (a.block / a.cpg)) * sizeof(float);
    if (plan.threads == 256) hipLaunchKernelGGL((group_norm_grad_once_kernel<T, V, 2, 256, WHOLE>), dim3(a.tiles), dim3(256), lds, stream, a);
    else if (plan.threads == 512) hipLaunchKernelGGL((group_norm_grad_once_kernel<T, V, 4, 512, WHOLE>), dim3(a.tiles), dim3(512), lds, stream, a);
    else hipLaunchKernelGGL((group_norm_grad_once_kernel<T, V, 8, 1024, WHOLE>), dim3(a.tiles), dim3(1024), lds, stream, a);
    if (a.n > 1 && (a.dgamma || a.dbeta))
        hipLaunchKernelGGL(group_norm_reduce_kernel, dim3((a.c + kReduceChannels - 1) / kReduceChannels), dim3(kThreads), 0, stream, a, a.n);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

// Whether a lane's channels are always of one group.
template <int V> bool whole_vectors(const NormArgs &a) { return a.cpg % V == 0; }

template <typename T, int V, int ACT, bool WHOLE> void launch_apply(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    if constexpr (V * sizeof(T) == 16)
        if (a.passing) {
            hipLaunchKernelGGL((group_norm_apply_kernel<T, V, ACT, WHOLE, true>), dim3(a.tiles), dim3(kThreads), plan.lds_apply, stream, a);
            return;
        }
    hipLaunchKernelGGL((group_norm_apply_kernel<T, V, ACT, WHOLE, false>), dim3(a.tiles), dim3(kThreads), plan.lds_apply, stream, a);
}

template <typename T, int V, bool WHOLE> tvg_status launch_forward(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    if (plan.once) return launch_once<T, V, WHOLE>(a, plan, stream);
    hipLaunchKernelGGL((group_norm_stats_kernel<T, V, WHOLE>), dim3(a.tiles), dim3(kThreads), plan.lds_stats, stream, a);
    if (a.act == TVG_ACT_SILU) launch_apply<T, V, TVG_ACT_SILU, WHOLE>(a, plan, stream);
    else if (a.act == TVG_ACT_RELU) launch_apply<T, V, TVG_ACT_RELU, WHOLE>(a, plan, stream);
    else launch_apply<T, V, TVG_ACT_NONE, WHOLE>(a, plan, stream);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}
template <typename T, int V> tvg_status launch_forward(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    return whole_vectors<V>(a) ? launch_forward<T, V, true>(a, plan, stream) : launch_forward<T, V, false>(a, plan, stream);
}

template <typename T, int V, int ACT, bool WHOLE> tvg_status launch_grad(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    const int reducers = a.dgamma || a.dbeta ? (a.c + kReduceChannels - 1) / kReduceChannels : 0;
    hipLaunchKernelGGL((group_norm_grad_sums_kernel<T, V, ACT, WHOLE>), dim3(a.tiles), dim3(kThreads), plan.lds_stats, stream, a);
    if constexpr (V * sizeof(T) == 16)
        if (a.passing) {
            hipLaunchKernelGGL((group_norm_grad_apply_kernel<T, V, ACT, WHOLE, true>), dim3(a.tiles + reducers), dim3(kThreads), plan.lds_apply, stream, a, reducers);
            return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
        }
    hipLaunchKernelGGL((group_norm_grad_apply_kernel<T, V, ACT, WHOLE, false>), dim3(a.tiles + reducers), dim3(kThreads), plan.lds_apply, stream, a, reducers);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

template <typename T, int V, bool WHOLE> tvg_status launch_backward(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    if (plan.once) return launch_grad_once<T, V, WHOLE>(a, plan, stream);
    if (a.act == TVG_ACT_SILU) return launch_grad<T, V, TVG_ACT_SILU, WHOLE>(a, plan, stream);
    if (a.act == TVG_ACT_RELU) return launch_grad<T, V, TVG_ACT_RELU, WHOLE>(a, plan, stream);
    return launch_grad<T, V, TVG_ACT_NONE, WHOLE>(a, plan, stream);
}
template <typename T, int V> tvg_status launch_backward(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    return whole_vectors<V>(a) ? launch_backward<T, V, true>(a, plan, stream) : launch_backward<T, V, false>(a, plan, stream);
}

int gcd(int a, int b)
{
    while (b) {
        const int r = a % b;
        a = b;
        b = r;
    }
    return a;
}

// Elements per access that the row length and these addresses allow.
int vector_width(const NormProblem &p, std::initializer_list<const void *> pointers)
{
    const int size = p.dtype == TVG_BF16 ? 2 : 4;
    int v = 16 / size;
    while (v > 1 && p.c % v != 0) v /= 2;
    for (const void *q : pointers)
        while (v > 1 && reinterpret_cast<uintptr_t>(q) % ((uintptr_t)v * size) != 0) v /= 2;
    return v;
}

// Results that pass the caches by leave them to x.  64 maps 112x112x256: 261 us, stores that do 242, loads of the second launch too
// 224 (backward 417, 398, 368); 8 maps 64x64x320, which the L2 caches (32 MB) keep, 24.5, 23.5, 24.4.  Of one launch's blocks only
// whole lines do: 64 maps 28x28x512 in blocks of 256 bytes 29.3 us and 27.1, 64 maps 56x56x256 in blocks of 80 bytes 65 and 115.
bool passing(const NormProblem &p, const NormPlan &plan)
{
    const int64_t size = p.dtype == TVG_BF16 ? 2 : 4;
    if (plan.once) return plan.block * size % 128 == 0 && p.c * size % 128 == 0;
    return (int64_t)p.n * p.p * p.c * size > (32 << 20);
}

NormArgs make_args(const NormProblem &p, const NormPlan &plan)
{
    NormArgs a{};
    a.n = p.n; a.p = p.p; a.c = p.c; a.groups = p.groups; a.cpg = p.c / p.groups;
    a.block = plan.block; a.blocks = plan.blocks; a.rows = plan.rows; a.chunks = plan.chunks;
    a.tiles = p.n * plan.blocks * plan.chunks;
    a.eps = p.eps;
    a.act = p.act;
    a.passing = passing(p, plan);
    return a;
}

}  // namespace

// The plan of one launch, if a block of channels fits a workgroup's registers: blocks for a workgroup a CU, 64 bytes of a row
// at least where that fits, 32 at least.  Two launches took 16.8 us for one map 7x7x512 where one takes 5.3, and 50 us for 32 maps
// 56x56x256 where one takes 29; gradients of 2 maps 14x14x256 (fp32) 10.1 and 9.5.
static bool plan_once(const NormProblem &p, int vector, bool backward, NormPlan *plan)
{
    const int cpg = p.c / p.groups, size = p.dtype == TVG_BF16 ? 2 : 4;
    const int unit = cpg / gcd(cpg, vector) * vector;                  // divides c: so do both
    static const int kLanes[3] = {256, 512, 1024}, kVectors[2][3] = {{4, 8, 16}, {2, 4, 8}};
    const auto fits = [&](int width, int k) {
        const int cols = width / vector;
        // (LDS: 32 KB of sums, and of the backward pass 20 floats a channel)
        return cols <= kLanes[k] && width / cpg <= 2048 && (!backward || width <= 384) &&
               ((int64_t)p.p + kLanes[k] / cols - 1) / (kLanes[k] / cols) <= kVectors[backward][k];
    };
    int64_t units = std::max<int64_t>((int64_t)p.n * p.c / kComputeUnits / unit, (64 / size + unit - 1) / unit);
    units = std::min<int64_t>(units, p.c / unit);
    while (units > 1 && !fits((int)units * unit, 2)) --units;
    const int width = (int)units * unit;
    // Few workgroups with much each: the two launches spread it.  One launch and two, us: 4 maps 28x28x256 (50 KB a workgroup) 8.6
    // and 11.6, one map 40x40x512 (100 KB) 13.7 and 13.2, one map 56x56x256 (200 KB) 17.8 and 13.2; gradients of one map 20x20x512
    // (25 KB) 9.7 and 13.3, of 4 maps 28x28x256 15.8 and 13.8.
    if ((int64_t)p.n * ((p.c + width - 1) / width) < kComputeUnits / 2 && (int64_t)p.p * width * size > (backward ? 32 : 64) * 1024) return false;
    if (!fits(width, 2) || (width * size < (backward ? 64 : 32) && width < p.c)) return false;
    int k = 0;
    while (!fits(width, k)) ++k;
    plan->once = true;
    plan->threads = kLanes[k];
    plan->block = width;
    plan->blocks = (p.c + width - 1) / width;
    plan->rows = p.p;
    plan->chunks = 1;
    plan->part_floats = 0;
    plan->chan_floats = backward && p.n > 1 ? (size_t)p.n * p.c * 2 : 0;
    return true;
}


// Row chunks: two workgroups a CU with four vectors a lane at least, or one with two.  Every workgroup of the second launch joins
// the statistics of its sample's chunks, 64 of them in one round of loads: more only where a chunk would have more than 48 KB
// (one map 300x300x64: 64 chunks 32 us, 240 23 us; one map 56x56x256: 64 chunks 13.4 us, 196 15.1 us).  8 maps 64x64x320: two
// workgroups a CU 24.3 us, four 31.5, eight 44.
static void plan_group_norm(const NormProblem &p, int vector, bool backward, NormPlan *plan)
{
    const int cpg = p.c / p.groups;
    plan->once = false;
    plan->vector = vector;
    if (plan_once(p, vector, backward, plan)) return;
    // a block of whole groups and whole vectors, as wide as one pass of the workgroup
    const int64_t unit = (int64_t)cpg * vector / gcd(cpg, vector);
    const int64_t widest = (int64_t)kThreads * vector;
    plan->vector = vector;
    plan->block = unit >= p.c ? p.c : p.c <= widest ? p.c : (int)(unit * std::max<int64_t>(1, widest / unit));
    plan->blocks = (p.c + plan->block - 1) / plan->block;
    const int cols = std::min(plan->block / vector, kThreads), rp = kThreads / cols;
    const int64_t others = (int64_t)p.n * plan->blocks, sample = (int64_t)p.p * p.c * (p.dtype == TVG_BF16 ? 2 : 4) * (backward ? 2 : 1);
    const int64_t most = std::min<int64_t>(256, std::max<int64_t>(kPairChunks, sample / (48 * 1024)));
    const auto chunks_of = [&](int per_cu, int rows) {
        return std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(per_cu * kComputeUnits / others, most), p.p / (rows * rp)));
    };
    const int64_t chunks = std::max(chunks_of(2, 4), chunks_of(1, 2));
    plan->rows = (int)((p.p + chunks - 1) / chunks);
    plan->chunks = (p.p + plan->rows - 1) / plan->rows;
    const int groups = plan->block / cpg;
    plan->lds_stats = (size_t)(2 * kThreads * vector + 3 * groups) * sizeof(float);
    plan->lds_apply = std::max<size_t>((size_t)2 * groups, 2 * kThreads) * sizeof(float);
    plan->part_floats = (size_t)p.n * p.groups * plan->chunks * 2;
    plan->chan_floats = (size_t)p.n * plan->chunks * p.c * 2;
}

// The workspace holds what any alignment of the tensors needs.
size_t group_norm_workspace(const NormProblem &p, bool backward)
{
    size_t bytes = 0;
    NormPlan plan;
    for (int v = vector_width(p, {}); v >= 1; v /= 2) {
        plan_group_norm(p, v, backward, &plan);
        bytes = std::max(bytes, (plan.part_floats + (backward ? plan.chan_floats : 0)) * sizeof(float));
    }
    return bytes;
}

tvg_status launch_group_norm(const NormProblem &p, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                             float *rstd, float *workspace, hipStream_t stream)
{
    NormPlan plan;
    plan_group_norm(p, vector_width(p, {x, y}), false, &plan);
    NormArgs a = make_args(p, plan);
    a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.mean = mean; a.rstd = rstd; a.part = workspace;
    if (p.dtype == TVG_BF16) {
        if (plan.vector == 8) return launch_forward<bf16_t, 8>(a, plan, stream);
        if (plan.vector == 4) return launch_forward<bf16_t, 4>(a, plan, stream);
        if (plan.vector == 2) return launch_forward<bf16_t, 2>(a, plan, stream);
        return launch_forward<bf16_t, 1>(a, plan, stream);
    }
    if (plan.vector == 4) return launch_forward<float, 4>(a, plan, stream);
    if (plan.vector == 2) return launch_forward<float, 2>(a, plan, stream);
    return launch_forward<float, 1>(a, plan, stream);
}

tvg_status launch_group_norm_backward(const NormProblem &p, const void *x, const void *dy, const float *mean, const float *rstd,
                                      const float *gamma, const float *beta, void *dx, float *dgamma, float *dbeta,
                                      float *workspace, hipStream_t stream)
{
    NormPlan plan;
    plan_group_norm(p, vector_width(p, {x, dy, dx}), true, &plan);
    NormArgs a = make_args(p, plan);
    a.x = x; a.dy = dy; a.gamma = gamma; a.beta = beta; a.y = dx; a.dgamma = dgamma; a.dbeta = dbeta;
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
    a.chan = workspace;                    // (first: read as pairs)
    a.part = workspace + plan.chan_floats;
    if (p.dtype == TVG_BF16) {
        if (plan.vector == 8) return launch_backward<bf16_t, 8>(a, plan, stream);
        if (plan.vector == 4) return launch_backward<bf16_t, 4>(a, plan, stream);
        if (plan.vector == 2) return launch_backward<bf16_t, 2>(a, plan, stream);
        return launch_backward<bf16_t, 1>(a, plan, stream);
    }
    if (plan.vector == 4) return launch_backward<float, 4>(a, plan, stream);
    if (plan.vector == 2) return launch_backward<float, 2>(a, plan, stream);
    return launch_backward<float, 1>(a, plan, stream);
}

}  // namespace tvg
