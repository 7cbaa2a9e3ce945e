// Group norm with an activation, channels last:
//
//   y[b, s, c] = act((x[b, s, c] - mean[b, g]) / sqrt(var[b, g] + eps) * weight[c] + bias[c]),   g = c / (C / groups)
//
// mean and var (biased) over the S rows and the C / groups channels of a group.  Every few rows of a channel are summed up, then their
// squared deviations from their own mean, and parts are joined by count, mean and sum of squared deviations: channels far from zero
// and rows unlike the others lose nothing (differences to a value picked beforehand do, where that value is such a row's).  Deviations
// beyond 1.8e19, whose squares fp32 does not hold, make the variance infinite.
#include <algorithm>

#include "elem.h"
#include "wave_reduce.h"

namespace dvdq {

namespace {

struct Moments { float mean, m2; };   // of a part of a group: mean, sum of squared deviations from it

struct GnArgs {
    const void *x;
    void *y;
    const void *weight, *bias;
    int64_t x_batch, x_row, y_batch, y_row;   // elements between batches, rows
    int64_t S;
    int C, groups, cpg;
    int cols, rows_at_once;                   // pieces of a row; rows a workgroup takes at once
    int64_t slab_rows;                        // rows of a part
    int slabs;
    float eps;
    Moments *parts;                           // [B][groups][slabs]
    float2 *stats;                            // [B][groups]: mean, 1 / sqrt(var + eps)
};

// Joins the moments of `nb` values to those of `n`, for every channel of a piece.
template <int V>
static __device__ __forceinline__ void join(float n, float (&mean)[V], float (&m2)[V], float nb, const float (&meanb)[V], const float (&m2b)[V]) {
    const float share = nb / (n + nb), weight = n * share;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float d = meanb[i] - mean[i];
        mean[i] = fmaf(d, share, mean[i]);
        m2[i] += fmaf(d * d, weight, m2b[i]);
    }
}

// Bound by memory and, where a slab is a few dozen rows, by what stands behind it: the moments of a slab's threads, channels and groups meet in
// LDS.  475200 x 512 in 16 bits, 487 MB read in 98 us (5.0 TB/s; a sum on this card reads at 5.9).  Slabs of 8 rows a thread at least and
// 2048 of them at most: with 4 rows a thread 32760 x 512 takes 38 us in place of 30 (all three launches), with 16 rows 8000 x 512 23 in place of 18;
// with 1024 slabs 475200 x 512 306 in place of 296.
constexpr int kBatch = 4;   // rows of a thread that are in registers at a time

// WHOLE: a piece lies within one group (C / groups a multiple of it), and a thread joins its channels before it meets the others;
// otherwise channels are joined first.
template <typename E, bool WHOLE>
__global__ __launch_bounds__(1024) void gn_parts(GnArgs a) {
    using Raw = typename E::Raw;
    constexpr int V = E::kVec;
    extern __shared__ float lds[];                      // WHOLE: [rows_at_once][cols] moments, else [rows_at_once][2][cols * V]
    const int b = blockIdx.y, slab = blockIdx.x;
    const int64_t s0 = slab * a.slab_rows;
    const int rows = (int)min(a.S - s0, a.slab_rows);
    const int width = a.cols * V;
    const int r = threadIdx.x / a.cols, col = threadIdx.x - r * a.cols, c0 = col * V, n = min(V, a.C - c0);
    const int64_t step = a.rows_at_once * a.x_row;
    const auto rows_of = [&](int i) { return max(0, (rows - i + a.rows_at_once - 1) / a.rows_at_once); };   // of the i-th row of threads
    if (r < a.rows_at_once) {
        const Raw *x = static_cast<const Raw *>(a.x) + (b * a.x_batch + (s0 + r) * a.x_row + c0);
        const int mine = rows_of(r);
        float mean[V] = {}, m2[V] = {};
        for (int i0 = 0; i0 < mine; i0 += kBatch) {
            const int nb = min(kBatch, mine - i0);
            Piece<E> p[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i < nb) p[i] = load_piece<E>(x + i * step, n);
                else p[i] = Piece<E>{};
            x += kBatch * step;
            // (differences to the first row: a constant channel has no deviations at all, whatever the rounding of 1 / nb)
            float mb[V] = {}, qb[V] = {};
#pragma unroll
            for (int i = 1; i < kBatch; ++i)
                if (i < nb) {
#pragma unroll
                    for (int j = 0; j < V; ++j) mb[j] += E::to_f32(p[i].e[j]) - E::to_f32(p[0].e[j]);
                }
            const float inv = 1.0f / (float)nb;
#pragma unroll
            for (int j = 0; j < V; ++j) mb[j] = fmaf(mb[j], inv, E::to_f32(p[0].e[j]));
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i < nb) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float d = E::to_f32(p[i].e[j]) - mb[j];
                        qb[j] = fmaf(d, d, qb[j]);
                    }
                }
            if (i0 > 0) {
                join<V>((float)i0, mean, m2, (float)nb, mb, qb);
            } else {                                     // (there is nothing to join: a mean of 0 is no value's, and its difference may be beyond fp32 squared)
#pragma unroll
                for (int j = 0; j < V; ++j) mean[j] = mb[j], m2[j] = qb[j];
            }
        }
        if constexpr (WHOLE) {
            float sum = 0.0f, m = 0.0f;
#pragma unroll
            for (int j = 1; j < V; ++j) sum += mean[j] - mean[0];
            const float all = fmaf(sum, 1.0f / V, mean[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) m += fmaf((mean[j] - all) * (mean[j] - all), (float)mine, m2[j]);
            reinterpret_cast<Moments *>(lds)[r * a.cols + col] = {all, m};
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                lds[(2 * r) * width + c0 + j] = mean[j];
                lds[(2 * r + 1) * width + c0 + j] = m2[j];
            }
        }
    }
    __syncthreads();
    if constexpr (!WHOLE) {
        // per channel: mean and squared deviations over the slab, in the first two rows of lds
        const int filled = min(a.rows_at_once, rows);   // rows of threads that have any
        for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
            const float first = lds[c];
            float sum = 0.0f, m2 = 0.0f;
            for (int i = 1; i < filled; ++i) sum = fmaf((float)rows_of(i), lds[2 * i * width + c] - first, sum);
            const float mean = first + sum / (float)rows;
            for (int i = 0; i < filled; ++i) {
                const float d = lds[2 * i * width + c] - mean;
                m2 += fmaf((float)rows_of(i), d * d, lds[(2 * i + 1) * width + c]);
            }
            lds[c] = mean;
            lds[width + c] = m2;
        }
        __syncthreads();
    }
    // The groups, `lanes` lanes (a power of two) for each: entries e of a group are pieces of rows of threads, or channels.
    const int per_row = a.cpg / V, entries = WHOLE ? a.rows_at_once * per_row : a.cpg;
    const int lanes = entries >= 64 ? 64 : 1 << (32 - __builtin_clz(max(entries, 2) - 1)), l = threadIdx.x & (lanes - 1);
    const auto total = [&](float v) {
        for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o);
        return v;
    };
    for (int g0 = 0; g0 < a.groups; g0 += blockDim.x / lanes) {
        const int g = g0 + threadIdx.x / lanes;
        if (g0 + (int)(threadIdx.x & ~63) / lanes >= a.groups) continue;   // (of whole waves only: the lanes of a wave meet in total())
        const auto entry = [&](int e, float &weight) {
            if constexpr (WHOLE) {
                const int i = e / per_row;
                weight = (float)rows_of(i) * V;
                return reinterpret_cast<const Moments *>(lds)[i * a.cols + g * per_row + (e - i * per_row)];
            } else {
                weight = (float)rows;
                return Moments{lds[g * a.cpg + e], lds[width + g * a.cpg + e]};
            }
        };
        const bool valid = g < a.groups;
        float w, sum = 0.0f, m2 = 0.0f;
        const float first = valid ? entry(0, w).mean : 0.0f;   // (the first row of threads has rows in every slab)
        if (valid)
            for (int e = l; e < entries; e += lanes) {
                const float m = entry(e, w).mean;
                if (w > 0.0f) sum = fmaf(w, m - first, sum);
            }
        const float mean = first + total(sum) / ((float)rows * (float)a.cpg);
        if (valid)
            for (int e = l; e < entries; e += lanes) {
                const Moments m = entry(e, w);
                const float d = m.mean - mean;
                if (w > 0.0f) m2 += fmaf(w * d, d, m.m2);
            }
        m2 = total(m2);
        if (valid && l == 0) a.parts[((int64_t)b * a.groups + g) * a.slabs + slab] = {mean, m2};
    }
}

// The sum over a workgroup, the same in every thread.  `lds`: a word per wave, free on entry; free again behind the next barrier.
template <typename T>
static __device__ __forceinline__ T block_sum(T v, T *lds) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    T sum = lds[0];
    for (int i = 1; i < (int)(blockDim.x >> 6); ++i) sum += lds[i];
    return sum;
}

// A workgroup joins the parts of one group of one batch, all of them in registers (kMaxSlabs).
constexpr int kMaxSlabs = 2048, kPerThread = kMaxSlabs / 256;
__global__ __launch_bounds__(256) void gn_join(GnArgs a) {
    __shared__ double lds[2][4];
    const int g = blockIdx.x, b = blockIdx.y;
    const Moments *p = a.parts + ((int64_t)b * a.groups + g) * a.slabs;
    Moments m[kPerThread];
    double rows[kPerThread], sum = 0.0, m2 = 0.0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const int slab = threadIdx.x + 256 * i;
        if (slab < a.slabs) m[i] = p[slab];
        else m[i] = {};
        rows[i] = slab < a.slabs ? (double)min(a.S - slab * a.slab_rows, a.slab_rows) : 0.0;
    }
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
        if (rows[i] > 0.0) sum += rows[i] * m[i].mean;
    const double mean = block_sum(sum, lds[0]) / (double)a.S;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const double d = (double)m[i].mean - mean;
        if (rows[i] > 0.0) m2 += m[i].m2 + rows[i] * a.cpg * d * d;
    }
    const double var = block_sum(m2, lds[1]) / ((double)a.S * a.cpg);
    if (threadIdx.x == 0) a.stats[b * a.groups + g] = make_float2((float)mean, (float)(1.0 / sqrt(var + (double)a.eps)));
}

// A whole group in a workgroup's registers: read once, written once, one launch.  V: elements of a piece of a row of the group.  Taken
// where a group is at most 8192 pieces: 1560 x 512 in 32 groups, 3.2 MB, 8.9 us a call, most of it the launch (three launches 19).
constexpr int kUnits = 8;
template <typename E, int ACT, int V>
__global__ __launch_bounds__(1024) void gn_whole(GnArgs a) {
    using Raw = typename E::Raw;
    __shared__ double sums[16];
    __shared__ float squares[16];
    const int g = blockIdx.x, b = blockIdx.y, threads = blockDim.x;
    const int per_row = a.cpg / V, total = (int)a.S * per_row;
    const Raw *x = static_cast<const Raw *>(a.x) + b * a.x_batch + g * a.cpg;
    Raw *y = static_cast<Raw *>(a.y) + b * a.y_batch + g * a.cpg;
    const int row0 = threadIdx.x / per_row, c0 = threadIdx.x - row0 * per_row, d_row = threads / per_row, d_c = threads - d_row * per_row;
    Piece<E, V> p[kUnits];
    {
        int row = row0, c = c0;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            if ((int)threadIdx.x + i * threads < total) p[i] = load_piece<E, V>(x + row * a.x_row + c * V, V);
            else p[i] = Piece<E, V>{};
            row += d_row, c += d_c;
            if (c >= per_row) c -= per_row, ++row;
        }
    }
    // a thread's own mean and squared deviations, joined by count: one value that is nothing like the others costs its own thread's few
    // their last places, not the whole group (as differences to the group's first value would)
    int pieces = 0;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) pieces += (int)threadIdx.x + i * threads < total;
    const float first = E::to_f32(p[0].e[0]), n = (float)(pieces * V);
    const double share = 1.0 / (double)((int)a.S * a.cpg);   // of a value (done by the time the values are there)
    float own = 0.0f, m2 = 0.0f;
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
        if (i < pieces) {
#pragma unroll
            for (int j = 0; j < V; ++j) own += E::to_f32(p[i].e[j]) - first;
        }
    if (pieces) own = fmaf(own, __builtin_amdgcn_rcpf(n), first);
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
        if (i < pieces) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = E::to_f32(p[i].e[j]) - own;
                m2 = fmaf(d, d, m2);
            }
        }
    const float mean = (float)(block_sum((double)n * own, sums) * share);   // (64 bits: exact where all are equal)
    if (pieces) m2 = fmaf(n * (own - mean), own - mean, m2);
    const float rstd = (float)rsqrt((double)block_sum(m2, squares) * share + (double)a.eps);
    int row = row0, c = c0;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        if ((int)threadIdx.x + i * threads < total) {
            const int ch = g * a.cpg + c * V;
            Piece<E, V> w, bias;
            if (a.weight) w = load_piece<E, V>(static_cast<const Raw *>(a.weight) + ch, V);
            if (a.bias) bias = load_piece<E, V>(static_cast<const Raw *>(a.bias) + ch, V);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float scale = a.weight ? rstd * E::to_f32(w.e[j]) : rstd, shift = a.bias ? E::to_f32(bias.e[j]) : 0.0f;
                p[i].e[j] = E::from_f32(activate<ACT>(fmaf(E::to_f32(p[i].e[j]) - mean, scale, shift)));
            }
            store_piece<E, V>(y + row * a.y_row + c * V, p[i], V);
        }
        row += d_row, c += d_c;
        if (c >= per_row) c -= per_row, ++row;
    }
}

// Normalizes.  475200 x 512 in 16 bits, 973 MB in 188 us (5.2 TB/s; a copy on this card 5.9).  The statistics need all of x first, so it is
// read twice where it does not fit on the chip; backwards, so that what the first reading left in the caches is read first.
template <typename E, int ACT, bool STREAM>
__global__ __launch_bounds__(1024) void gn_apply(GnArgs a) {
    using Raw = typename E::Raw;
    constexpr int V = E::kVec, kRows = 4;                // rows of a thread that are on their way at a time
    const int b = gridDim.y - 1 - blockIdx.y, slab = gridDim.x - 1 - blockIdx.x;   // backwards: what was read last is still in the caches
    const int r = threadIdx.x / a.cols, col = threadIdx.x - r * a.cols, c0 = col * V, n = min(V, a.C - c0);
    if (r >= a.rows_at_once) return;
    float mean[V], scale[V], shift[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = min(c0 + i, a.C - 1);
        const float2 st = a.stats[b * a.groups + c / a.cpg];
        mean[i] = st.x;
        scale[i] = st.y * (a.weight ? E::to_f32(static_cast<const Raw *>(a.weight)[c]) : 1.0f);
        shift[i] = a.bias ? E::to_f32(static_cast<const Raw *>(a.bias)[c]) : 0.0f;
    }
    const int64_t s0 = slab * a.slab_rows;
    const int rows = (int)min(a.S - s0, a.slab_rows), mine = (rows - r + a.rows_at_once - 1) / a.rows_at_once;
    const int64_t x_step = a.rows_at_once * a.x_row, y_step = a.rows_at_once * a.y_row;
    const Raw *x = static_cast<const Raw *>(a.x) + (b * a.x_batch + (s0 + r) * a.x_row + c0);
    Raw *y = static_cast<Raw *>(a.y) + (b * a.y_batch + (s0 + r) * a.y_row + c0);
    for (int i0 = 0; i0 < mine; i0 += kRows, x += kRows * x_step, y += kRows * y_step) {
        Piece<E> p[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (i0 + i < mine) p[i] = load_piece<E>(x + i * x_step, n);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (i0 + i >= mine) break;
#pragma unroll
            for (int j = 0; j < V; ++j) p[i].e[j] = E::from_f32(activate<ACT>(fmaf(E::to_f32(p[i].e[j]) - mean[j], scale[j], shift[j])));
            store_piece<E, V, STREAM>(y + i * y_step, p[i], n);
        }
    }
}

struct Plan { int cols, rows_at_once, threads, slabs; int64_t slab_rows; size_t parts_bytes, stats_bytes; };

Plan plan(int64_t B, int64_t S, int64_t C, int64_t groups, int vec) {
    Plan p;
    p.cols = (int)((C + vec - 1) / vec);
    p.threads = p.cols <= 256 ? 256 : (p.cols + 63) / 64 * 64;
    p.rows_at_once = p.threads / p.cols;
    const int64_t want = max((int64_t)1, (int64_t)2048 / B);                              // workgroups to fill the chip
    p.slab_rows = max((S + want - 1) / want, (int64_t)8 * p.rows_at_once);
    p.slab_rows = (p.slab_rows + p.rows_at_once - 1) / p.rows_at_once * p.rows_at_once;
    p.slabs = (int)((S + p.slab_rows - 1) / p.slab_rows);   // at most kMaxSlabs
    p.parts_bytes = ((size_t)B * p.slabs * groups * sizeof(Moments) + 255) / 256 * 256;
    p.stats_bytes = ((size_t)B * groups * sizeof(float2) + 255) / 256 * 256;
    return p;
}

}  // namespace

size_t group_norm_workspace_bytes(int64_t B, int64_t S, int64_t C, int64_t groups) {
    size_t most = 0;
    for (int vec : {4, 8}) {
        const Plan p = plan(B, S, C, groups, vec);
        most = max(most, p.parts_bytes + p.stats_bytes);
    }
    return most;
}

int launch_group_norm(const void *x, int64_t B, int64_t S, int64_t C, int64_t x_batch, int64_t x_row, int64_t groups, const void *weight,
                      const void *bias, float eps, int act, int dtype, void *y, int64_t y_batch, int64_t y_row, void *workspace,
                      hipStream_t stream) {
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        const Plan p = plan(B, S, C, groups, E::kVec);
        GnArgs a = {};
        a.x = x, a.y = y, a.weight = weight, a.bias = bias;
        a.x_batch = x_batch, a.x_row = x_row, a.y_batch = y_batch, a.y_row = y_row;
        a.S = S, a.C = (int)C, a.groups = (int)groups, a.cpg = (int)(C / groups);
        a.cols = p.cols, a.rows_at_once = p.rows_at_once, a.slab_rows = p.slab_rows, a.slabs = p.slabs;
        a.eps = eps;
        a.parts = static_cast<Moments *>(workspace);
        a.stats = reinterpret_cast<float2 *>(static_cast<uint8_t *>(workspace) + p.parts_bytes);
        const bool silu = act == DVDQ_ACT_SILU;
        const auto one_launch = [&](auto width) {
            constexpr int V = decltype(width)::value;
            const int64_t total = S * (a.cpg / V);
            if (a.cpg % V != 0 || total > 1024 * kUnits) return false;
            const int threads = (int)std::clamp((total + 127) / 128 * 64, (int64_t)64, (int64_t)1024);   // two pieces a thread, up to 16 waves
            const auto kernel = silu ? gn_whole<E, DVDQ_ACT_SILU, V> : gn_whole<E, DVDQ_ACT_NONE, V>;
            kernel<<<dim3((unsigned)groups, (unsigned)B), threads, 0, stream>>>(a);
            return true;
        };
        if (one_launch(std::integral_constant<int, E::kVec>()) || (E::kVec > 4 && one_launch(std::integral_constant<int, 4>())) ||
            one_launch(std::integral_constant<int, 2>()) || one_launch(std::integral_constant<int, 1>()))
            return check_launch();
        const dim3 grid(p.slabs, (unsigned)B);
        if (a.cpg % E::kVec == 0)
            gn_parts<E, true><<<grid, p.threads, (size_t)p.rows_at_once * p.cols * sizeof(Moments), stream>>>(a);
        else
            gn_parts<E, false><<<grid, p.threads, (size_t)p.rows_at_once * 2 * p.cols * E::kVec * sizeof(float), stream>>>(a);
        gn_join<<<dim3((unsigned)groups, (unsigned)B), 256, 0, stream>>>(a);
        // Streaming stores for outputs beyond an XCD's L2, which also leave x in the caches for the rows that are still to be read.
        const bool stream_out = (int64_t)B * S * C * (int64_t)sizeof(typename E::Raw) >= (4 << 20);
        const auto apply = silu ? (stream_out ? gn_apply<E, DVDQ_ACT_SILU, true> : gn_apply<E, DVDQ_ACT_SILU, false>)
                                : (stream_out ? gn_apply<E, DVDQ_ACT_NONE, true> : gn_apply<E, DVDQ_ACT_NONE, false>);
        apply<<<grid, p.threads, 0, stream>>>(a);
        return check_launch();
    });
}

}  // namespace dvdq
