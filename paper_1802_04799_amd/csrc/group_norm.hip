// Group norm with an activation over channels-last maps x [n][p][c], forward and backward.
//
//   mean, var over the p * (c / groups) elements of a group;  xhat = (x - mean) / sqrt(var + eps)
//   z = gamma xhat + beta,  y = act(z)
//   backward, with dz = dy act'(z), S1 = sum_p dz and S2 = sum_p dz xhat per sample and channel:
//   dbeta = sum_n S1, dgamma = sum_n S2, dx = rstd (gamma dz - (a + xhat b) / m)
//   with a, b the sums of gamma S1, gamma S2 over a group's channels and m its elements
//
// Bound by memory: about 10 (forward) or 25 (backward) operations an element.  Two launches: the first leaves partial
// statistics of row chunks in the workspace, the second joins those of its sample in a fixed order and applies them.
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

#include "tvg_device.h"
#include "tvg_internal.h"

namespace tvg {

namespace {

constexpr int kThreads = 256;
constexpr int kTeam = 16;                  // lanes that join the statistics of a group

// V elements of memory: 16 bytes or less.
template <typename T, int V> struct Vec {
    typedef T type __attribute__((ext_vector_type(V)));
    static __device__ __forceinline__ type load(const T *p) { return *reinterpret_cast<const type *>(p); }
    static __device__ __forceinline__ void get(const type &r, float *f)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(T) == 2) f[i] = bf16_to_f32(r[i]);
            else f[i] = r[i];
        }
    }
    static __device__ __forceinline__ void store(T *p, const float *f)
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
        *reinterpret_cast<type *>(p) = r;
    }
};
template <typename T> struct Vec<T, 1> {
    typedef T type;
    static __device__ __forceinline__ type load(const T *p) { return *p; }
    static __device__ __forceinline__ void get(const type &r, float *f) { f[0] = Elem<T>::load(&r, 0); }
    static __device__ __forceinline__ void store(T *p, const float *f) { Elem<T>::store(p, 0, f[0]); }
};

template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == TVG_ACT_RELU) return z < 0.0f ? 0.0f : z;      // (a NaN stays one)
    if constexpr (ACT == TVG_ACT_SILU) return z * sigmoid(z);
    return z;
}

// dy times the activation's derivative at z
template <int ACT> __device__ __forceinline__ float activate_grad(float dy, float z)
{
    if constexpr (ACT == TVG_ACT_RELU) return z <= 0.0f ? 0.0f : dy;
    if constexpr (ACT == TVG_ACT_SILU) {
        const float s = sigmoid(z);
        return dy * (s * fmaf(z, 1.0f - s, 1.0f));
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
__device__ __forceinline__ float team_sum(float v)
{
#pragma unroll
    for (int d = 1; d < kTeam; d *= 2) v += __shfl_xor(v, d, kTeam);
    return v;
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
        m2[i] += fmaf(d * d, cross, sq[i]);
    }
}

// LDS: per channel of a pass the lanes' (mean, M2, rows), then per group (elements, mean, M2).
template <typename T, int V> __global__ __launch_bounds__(kThreads) void group_norm_stats_kernel(NormArgs a)
{
    constexpr int U = 8;
    extern __shared__ float lds[];
    float *lane_mean = lds, *lane_m2 = lds + kThreads * V, *group = lds + 2 * kThreads * V;
    const Tile t = tile_of<V>(a, blockIdx.x);
    const int g0 = t.c0 / a.cpg, ng = t.width / a.cpg;
    const int col = threadIdx.x % t.cols, rp = threadIdx.x / t.cols;
    const T *x = static_cast<const T *>(a.x) + ((size_t)t.sample * a.p) * a.c + t.c0;
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
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lane_mean[threadIdx.x * V + i] = mean[i];
            lane_m2[threadIdx.x * V + i] = m2[i];
        }
        __syncthreads();
        // a team joins the entries of a group's channels in this pass: rp lanes per channel, of known row counts
        const int team = threadIdx.x / kTeam, tl = threadIdx.x % kTeam;
        for (int g = first / a.cpg + team; g * a.cpg < first + pass_width; g += kThreads / kTeam) {
            const int lo = max(g * a.cpg, first), hi = min((g + 1) * a.cpg, first + pass_width), w = hi - lo;
            const int entries = w * t.rp, rows = t.row1 - t.row0;
            float s = 0.0f;
            for (int e = tl; e < entries; e += kTeam) {
                const int r = e / w, at = r * t.cols * V + lo - first + e - r * w;
                const int n = r < rows ? (rows - r + t.rp - 1) / t.rp : 0;
                s += (float)n * lane_mean[at];
            }
            const float total = (float)rows * (float)w, m = team_sum(s) / total;
            float q = 0.0f;
            for (int e = tl; e < entries; e += kTeam) {
                const int r = e / w, at = r * t.cols * V + lo - first + e - r * w;
                const int n = r < rows ? (rows - r + t.rp - 1) / t.rp : 0;
                const float d = lane_mean[at] - m;
                q += n ? fmaf(d * d, (float)n, lane_m2[at]) : 0.0f;
            }
            q = team_sum(q);
            if (tl == 0) {
                float *o = group + 3 * g;
                const float before = o[0], all = before + total, d = m - o[1];
                o[0] = all;
                o[1] += d * (total / all);
                o[2] += q + d * d * (before * (total / all));
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
    const int team = threadIdx.x / kTeam, tl = threadIdx.x % kTeam;
    const float total = (float)a.p;                        // (in rows: every chunk has cpg channels a row)
    for (int g = team; g < ng; g += kThreads / kTeam) {
        const float *part = a.part + ((size_t)t.sample * a.groups + g0 + g) * a.chunks * 2;
        float s = 0.0f;
        for (int k = tl; k < a.chunks; k += kTeam) s += (float)min(a.rows, a.p - k * a.rows) * part[2 * k];
        const float m = team_sum(s) / total;
        float q = 0.0f;
        for (int k = tl; k < a.chunks; k += kTeam) {
            const float d = part[2 * k] - m;
            q += fmaf(d * d, (float)min(a.rows, a.p - k * a.rows) * (float)a.cpg, part[2 * k + 1]);
        }
        q = team_sum(q);
        if (tl == 0) {
            const float r = 1.0f / sqrtf(q / (total * (float)a.cpg) + a.eps);
            gmean[g] = m;
            grstd[g] = r;
            if (t.chunk == 0 && a.mean) a.mean[(size_t)t.sample * a.groups + g0 + g] = m;
            if (t.chunk == 0 && a.rstd) a.rstd[(size_t)t.sample * a.groups + g0 + g] = r;
        }
    }
}

template <typename T, int V, int ACT> __global__ __launch_bounds__(kThreads) void group_norm_apply_kernel(NormArgs a)
{
    constexpr int U = 4;
    extern __shared__ float lds[];
    const Tile t = tile_of<V>(a, blockIdx.x);
    const int g0 = t.c0 / a.cpg, ng = t.width / a.cpg;
    float *gmean = lds, *grstd = lds + ng;
    join_chunks(a, t, g0, ng, gmean, grstd);
    __syncthreads();
    const int col = threadIdx.x % t.cols, rp = threadIdx.x / t.cols;
    if (rp >= t.rp) return;
    const T *x = static_cast<const T *>(a.x) + ((size_t)t.sample * a.p) * a.c + t.c0;
    T *y = static_cast<T *>(a.y) + ((size_t)t.sample * a.p) * a.c + t.c0;
    for (int cc = col * V; cc < t.width; cc += t.cols * V) {
        float mean[V], mul[V], add[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = (cc + i) / a.cpg;
            mean[i] = gmean[g];
            mul[i] = grstd[g] * (a.gamma ? a.gamma[t.c0 + cc + i] : 1.0f);
            add[i] = a.beta ? a.beta[t.c0 + cc + i] : 0.0f;
        }
        for (int row = t.row0 + rp; row < t.row1; row += U * t.rp) {
            typename Vec<T, V>::type raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                raw[u] = Vec<T, V>::load(x + (size_t)(row + u * t.rp < t.row1 ? row + u * t.rp : row) * a.c + cc);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[V];
                Vec<T, V>::get(raw[u], f);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = activate<ACT>(fmaf(f[i] - mean[i], mul[i], add[i]));
                if (row + u * t.rp < t.row1) Vec<T, V>::store(y + (size_t)(row + u * t.rp) * a.c + cc, f);
            }
        }
    }
}

// What a lane of the backward pass needs of its channels.
template <int V> struct Channels {
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ __forceinline__ void load(const NormArgs &a, const Tile &t, int cc)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = t.c0 + cc + i, g = c / a.cpg;
            mean[i] = a.mean[(size_t)t.sample * a.groups + g];
            rstd[i] = a.rstd[(size_t)t.sample * a.groups + g];
            gamma[i] = a.gamma ? a.gamma[c] : 1.0f;
            beta[i] = a.beta ? a.beta[c] : 0.0f;
        }
    }
};

template <typename T, int V, int ACT> __global__ __launch_bounds__(kThreads) void group_norm_grad_sums_kernel(NormArgs a)
{
    constexpr int U = 4;
    extern __shared__ float lds[];
    float *lane1 = lds, *lane2 = lds + kThreads * V, *group = lds + 2 * kThreads * V;
    const Tile t = tile_of<V>(a, blockIdx.x);
    const int g0 = t.c0 / a.cpg, ng = t.width / a.cpg;
    const int col = threadIdx.x % t.cols, rp = threadIdx.x / t.cols;
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
            Channels<V> k;
            k.load(a, t, cc);
            for (int row = t.row0 + rp; row < t.row1; row += U * t.rp) {
                typename Vec<T, V>::type rx[U], rd[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const size_t at = (size_t)(row + u * t.rp < t.row1 ? row + u * t.rp : row) * a.c + cc;
                    rx[u] = Vec<T, V>::load(x + at);
                    rd[u] = Vec<T, V>::load(dy + at);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (row + u * t.rp >= t.row1) break;
                    float fx[V], fd[V];
                    Vec<T, V>::get(rx[u], fx);
                    Vec<T, V>::get(rd[u], fd);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float xhat = (fx[i] - k.mean[i]) * k.rstd[i];
                        const float dz = activate_grad<ACT>(fd[i], fmaf(xhat, k.gamma[i], k.beta[i]));
                        s1[i] += dz;
                        s2[i] = fmaf(dz, xhat, s2[i]);
                    }
                }
            }
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
__device__ __forceinline__ void reduce_channels(const NormArgs &a, int c0, float *lds)
{
    const int lc = threadIdx.x % kReduceChannels, lr = threadIdx.x / kReduceChannels, c = c0 + lc;
    constexpr int kLanes = kThreads / kReduceChannels;
    float v1 = 0.0f, v2 = 0.0f;
    if (c < a.c)
#pragma unroll 8
        for (int r = lr; r < a.n * a.chunks; r += kLanes) {
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

// The first workgroups add up dgamma and dbeta, the others write dx.
template <typename T, int V, int ACT> __global__ __launch_bounds__(kThreads) void group_norm_grad_apply_kernel(NormArgs a, int reducers)
{
    constexpr int U = 4;
    extern __shared__ float lds[];
    if ((int)blockIdx.x < reducers) {
        reduce_channels(a, blockIdx.x * kReduceChannels, lds);
        return;
    }
    const Tile t = tile_of<V>(a, blockIdx.x - reducers);
    const int g0 = t.c0 / a.cpg, ng = t.width / a.cpg;
    float *ga = lds, *gb = lds + ng;
    {
        const int team = threadIdx.x / kTeam, tl = threadIdx.x % kTeam;
        const float inv = 1.0f / ((float)a.p * (float)a.cpg);
        for (int g = team; g < ng; g += kThreads / kTeam) {
            const float *part = a.part + ((size_t)t.sample * a.groups + g0 + g) * a.chunks * 2;
            float v1 = 0.0f, v2 = 0.0f;
            for (int k = tl; k < a.chunks; k += kTeam) {
                v1 += part[2 * k];
                v2 += part[2 * k + 1];
            }
            v1 = team_sum(v1);
            v2 = team_sum(v2);
            if (tl == 0) {
                ga[g] = v1 * inv;
                gb[g] = v2 * inv;
            }
        }
    }
    __syncthreads();
    const int col = threadIdx.x % t.cols, rp = threadIdx.x / t.cols;
    if (rp >= t.rp) return;
    const size_t at0 = ((size_t)t.sample * a.p) * a.c + t.c0;
    const T *x = static_cast<const T *>(a.x) + at0, *dy = static_cast<const T *>(a.dy) + at0;
    T *dx = static_cast<T *>(a.y) + at0;
    for (int cc = col * V; cc < t.width; cc += t.cols * V) {
        Channels<V> k;
        k.load(a, t, cc);
        float sa[V], sb[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            sa[i] = ga[(cc + i) / a.cpg];
            sb[i] = gb[(cc + i) / a.cpg];
        }
        for (int row = t.row0 + rp; row < t.row1; row += U * t.rp) {
            typename Vec<T, V>::type rx[U], rd[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const size_t at = (size_t)(row + u * t.rp < t.row1 ? row + u * t.rp : row) * a.c + cc;
                rx[u] = Vec<T, V>::load(x + at);
                rd[u] = Vec<T, V>::load(dy + at);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float fx[V], fd[V];
                Vec<T, V>::get(rx[u], fx);
                Vec<T, V>::get(rd[u], fd);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xhat = (fx[i] - k.mean[i]) * k.rstd[i];
                    const float dz = activate_grad<ACT>(fd[i], fmaf(xhat, k.gamma[i], k.beta[i]));
                    fx[i] = k.rstd[i] * (fmaf(k.gamma[i], dz, -sa[i]) - xhat * sb[i]);
                }
                if (row + u * t.rp < t.row1) Vec<T, V>::store(dx + (size_t)(row + u * t.rp) * a.c + cc, fx);
            }
        }
    }
}

template <typename T, int V> tvg_status launch_forward(const NormArgs &a, int act, const NormPlan &plan, hipStream_t stream)
{
    const dim3 grid(a.tiles), threads(kThreads);
    hipLaunchKernelGGL((group_norm_stats_kernel<T, V>), grid, threads, plan.lds_stats, stream, a);
    if (act == TVG_ACT_SILU) hipLaunchKernelGGL((group_norm_apply_kernel<T, V, TVG_ACT_SILU>), grid, threads, plan.lds_apply, stream, a);
    else if (act == TVG_ACT_RELU) hipLaunchKernelGGL((group_norm_apply_kernel<T, V, TVG_ACT_RELU>), grid, threads, plan.lds_apply, stream, a);
    else hipLaunchKernelGGL((group_norm_apply_kernel<T, V, TVG_ACT_NONE>), grid, threads, plan.lds_apply, stream, a);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
}

template <typename T, int V, int ACT> void launch_grad(const NormArgs &a, const NormPlan &plan, hipStream_t stream)
{
    const int reducers = a.dgamma || a.dbeta ? (a.c + kReduceChannels - 1) / kReduceChannels : 0;
    hipLaunchKernelGGL((group_norm_grad_sums_kernel<T, V, ACT>), dim3(a.tiles), dim3(kThreads), plan.lds_stats, stream, a);
    hipLaunchKernelGGL((group_norm_grad_apply_kernel<T, V, ACT>), dim3(a.tiles + reducers), dim3(kThreads), plan.lds_apply, stream, a, reducers);
}

template <typename T, int V> tvg_status launch_backward(const NormArgs &a, int act, const NormPlan &plan, hipStream_t stream)
{
    if (act == TVG_ACT_SILU) launch_grad<T, V, TVG_ACT_SILU>(a, plan, stream);
    else if (act == TVG_ACT_RELU) launch_grad<T, V, TVG_ACT_RELU>(a, plan, stream);
    else launch_grad<T, V, TVG_ACT_NONE>(a, plan, stream);
    return hipGetLastError() == hipSuccess ? TVG_OK : TVG_ERR_LAUNCH;
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

NormArgs make_args(const NormProblem &p, const NormPlan &plan)
{
    NormArgs a{};
    a.n = p.n; a.p = p.p; a.c = p.c; a.groups = p.groups; a.cpg = p.c / p.groups;
    a.block = plan.block; a.blocks = plan.blocks; a.rows = plan.rows; a.chunks = plan.chunks;
    a.tiles = p.n * plan.blocks * plan.chunks;
    a.eps = p.eps;
    return a;
}

}  // namespace

// Row chunks: as many workgroups as keep every CU busy, with eight vectors a lane at least and 64 chunks of a sample at
// most, whose statistics every workgroup of the second launch joins.
void plan_group_norm(const NormProblem &p, int vector, NormPlan *plan)
{
    const int cpg = p.c / p.groups;
    // a block of whole groups and whole vectors, as wide as one pass of the workgroup
    const int64_t unit = (int64_t)cpg * vector / gcd(cpg, vector);
    const int64_t most = (int64_t)kThreads * vector;
    plan->vector = vector;
    plan->block = unit >= p.c ? p.c : p.c <= most ? p.c : (int)(unit * std::max<int64_t>(1, most / unit));
    plan->blocks = (p.c + plan->block - 1) / plan->block;
    const int cols = std::min(plan->block / vector, kThreads), rp = kThreads / cols;
    const int64_t want = std::max<int64_t>(1, 8 * kComputeUnits / ((int64_t)p.n * plan->blocks));
    int64_t chunks = std::min<int64_t>(std::min<int64_t>(want, 64), std::max<int64_t>(1, p.p / (8 * rp)));
    plan->rows = (int)((p.p + chunks - 1) / chunks);
    plan->chunks = (p.p + plan->rows - 1) / plan->rows;
    const int groups = plan->block / cpg;
    plan->lds_stats = (size_t)(2 * kThreads * vector + 3 * groups) * sizeof(float);
    plan->lds_apply = std::max<size_t>((size_t)2 * groups, 2 * kThreads) * sizeof(float);
    plan->part_floats = (size_t)p.n * p.groups * plan->chunks * 2;
    plan->chan_floats = (size_t)p.n * plan->chunks * p.c * 2;
}

// The workspace holds what any alignment of the tensors needs.
static NormPlan widest_plan(const NormProblem &p, bool backward, size_t *bytes)
{
    NormPlan plan;
    *bytes = 0;
    for (int v = vector_width(p, {}); v >= 1; v /= 2) {
        plan_group_norm(p, v, &plan);
        *bytes = std::max(*bytes, (plan.part_floats + (backward ? plan.chan_floats : 0)) * sizeof(float));
    }
    return plan;
}

size_t group_norm_workspace(const NormProblem &p, bool backward)
{
    size_t bytes;
    widest_plan(p, backward, &bytes);
    return bytes;
}

tvg_status launch_group_norm(const NormProblem &p, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                             float *rstd, float *workspace, hipStream_t stream)
{
    NormPlan plan;
    plan_group_norm(p, vector_width(p, {x, y}), &plan);
    NormArgs a = make_args(p, plan);
    a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.mean = mean; a.rstd = rstd; a.part = workspace;
    if (p.dtype == TVG_BF16) {
        if (plan.vector == 8) return launch_forward<bf16_t, 8>(a, p.act, plan, stream);
        if (plan.vector == 4) return launch_forward<bf16_t, 4>(a, p.act, plan, stream);
        if (plan.vector == 2) return launch_forward<bf16_t, 2>(a, p.act, plan, stream);
        return launch_forward<bf16_t, 1>(a, p.act, plan, stream);
    }
    if (plan.vector == 4) return launch_forward<float, 4>(a, p.act, plan, stream);
    if (plan.vector == 2) return launch_forward<float, 2>(a, p.act, plan, stream);
    return launch_forward<float, 1>(a, p.act, plan, stream);
}

tvg_status launch_group_norm_backward(const NormProblem &p, const void *x, const void *dy, const float *mean, const float *rstd,
                                      const float *gamma, const float *beta, void *dx, float *dgamma, float *dbeta,
                                      float *workspace, hipStream_t stream)
{
    NormPlan plan;
    plan_group_norm(p, vector_width(p, {x, dy, dx}), &plan);
    NormArgs a = make_args(p, plan);
    a.x = x; a.dy = dy; a.gamma = gamma; a.beta = beta; a.y = dx; a.dgamma = dgamma; a.dbeta = dbeta;
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
    a.chan = workspace;                    // (first: read as pairs)
    a.part = workspace + plan.chan_floats;
    if (p.dtype == TVG_BF16) {
        if (plan.vector == 8) return launch_backward<bf16_t, 8>(a, p.act, plan, stream);
        if (plan.vector == 4) return launch_backward<bf16_t, 4>(a, p.act, plan, stream);
        if (plan.vector == 2) return launch_backward<bf16_t, 2>(a, p.act, plan, stream);
        return launch_backward<bf16_t, 1>(a, p.act, plan, stream);
    }
    if (plan.vector == 4) return launch_backward<float, 4>(a, p.act, plan, stream);
    if (plan.vector == 2) return launch_backward<float, 2>(a, p.act, plan, stream);
    return launch_backward<float, 1>(a, p.act, plan, stream);
}

}  // namespace tvg
