// Rotary positions of queries and keys, and the table of cosines and sines they read.
//
//   (a, b) -> (a c - b s, a s + b c),   (c, s) = table[position(token, axis(j)), j]
//
// for every pair j of a head: elements 2j and 2j+1 (interleaved) or j and j + R/2 (halves) of the first R elements; the rest of the
// head is copied.  Products and sums in fp32, one rounding to the tensors' type.
#include <algorithm>

#include "elem.h"

namespace dvdq {

namespace {

constexpr int kMaxAxes = 4;
constexpr int kThreads = 256, kHeadsPerThread = 6;

struct RopeKernelArgs {
    const void *in[2];
    void *out[2];
    int64_t in_stride[2][3], out_stride[2][3];   // elements between batches, tokens, heads
    int q_heads, heads;                          // query heads; all heads, queries first
    uint32_t tokens, T;                          // B * T, T
    int D, R;
    const float2 *table;
    int n_pos;
    const int32_t *positions;
    uint32_t pos_batch;                          // positions between batches (0: the same for all)
    int n_axes;
    int bound[kMaxAxes - 1];                     // first pair of axes 1, 2, 3 (R/2 where there is none)
    int inverse;
    int rot_units, units;                        // pieces per head that are rotated; those and the copied ones, as many as a workgroup takes
    int heads_at_once, tokens_per_block, heads_per_block;
};

// A thread owns one piece of the head (16 bytes of each half of the pairs, or 16 bytes of interleaved pairs) for one token, and
// goes through heads: the token's cosines and sines are read once and stay in registers.  Neighbouring threads hold neighbouring
// pieces, so a wave reads and writes whole heads.  Up to six heads of a thread are in flight at a time.
// Bound by memory: 118800 tokens x 48 heads of 128 in 16 bits, 2.9 GB in and out, in 490 us (6.0 TB/s; a copy on the same card 5.9),
// 32760 x 24 in 75 (5.4).  What it took: cosines and sines in 16-byte loads where a piece lies within one axis (780 -> 637 us, one by
// one), streaming stores (-> 532), six heads a thread (-> 490).
template <typename E, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeKernelArgs a) {
    using Raw = typename E::Raw;
    constexpr int V = E::kVec, PAIRS = INTERLEAVED ? V / 2 : V, BATCH = kHeadsPerThread;
    const int per_token = a.units * a.heads_at_once;
    const int lt = (int)threadIdx.x / per_token, rem = (int)threadIdx.x - lt * per_token;
    const uint32_t token = blockIdx.x * (uint32_t)a.tokens_per_block + lt;
    if (lt >= a.tokens_per_block || token >= a.tokens) return;
    const int hs = rem / a.units, u = rem - hs * a.units + (int)blockIdx.z * kThreads;
    const uint32_t b = token / a.T, t = token - b * a.T;
    const int h_end = min(a.heads, ((int)blockIdx.y + 1) * a.heads_per_block);
    const int half = a.R / 2;
    const bool rotated = u < a.rot_units;
    if (!rotated && a.R + (u - a.rot_units) * V >= a.D) return;   // (of a second workgroup's pieces)

    // where the piece lies in a head, and how many elements (of each half) of it there are
    const int j0 = u * PAIRS;                                  // first pair
    const int e0 = rotated ? (INTERLEAVED ? 2 * j0 : j0) : a.R + (u - a.rot_units) * V;
    const int n = rotated ? (INTERLEAVED ? min(V, a.R - e0) : min(V, half - j0)) : min(V, a.D - e0);

    float c[PAIRS], s[PAIRS];
    uint32_t keep = 0;                                         // pairs of a negative position: as they are
    if (rotated) {
        const int np = INTERLEAVED ? n / 2 : n;
        const int32_t *pos = a.positions + ((uint64_t)b * a.pos_batch + (uint64_t)t * a.n_axes);
        int p[kMaxAxes];
#pragma unroll
        for (int i = 0; i < kMaxAxes; ++i) p[i] = i < a.n_axes ? pos[i] : 0;
        const auto axis_of = [&](int j) { return j < a.bound[0] ? 0 : j < a.bound[1] ? 1 : j < a.bound[2] ? 2 : 3; };
        const int axis = axis_of(j0), one = axis == 0 ? p[0] : axis == 1 ? p[1] : axis == 2 ? p[2] : p[3];
        if (np == PAIRS && axis == axis_of(j0 + PAIRS - 1) && one >= 0 && one < a.n_pos) {
            struct __attribute__((packed, aligned(8))) Row { float2 v[PAIRS]; };
            const Row row = *reinterpret_cast<const Row *>(a.table + (int64_t)one * half + j0);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                c[i] = row.v[i].x;
                s[i] = a.inverse ? -row.v[i].y : row.v[i].y;
            }
        } else
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const int j = j0 + i;
            const int pi = j < a.bound[0] ? p[0] : j < a.bound[1] ? p[1] : j < a.bound[2] ? p[2] : p[3];
            float2 cs = make_float2(1.0f, 0.0f);
            if (i < np) {
                if (pi < 0) keep |= 1u << i;
                else if (pi < a.n_pos) cs = a.table[(int64_t)pi * half + j];
                else cs = make_float2(__builtin_nanf(""), __builtin_nanf(""));   // not in the table
            }
            c[i] = cs.x;
            s[i] = a.inverse ? -cs.y : cs.y;
        }
    }

    for (int h0 = (int)blockIdx.y * a.heads_per_block + hs; h0 < h_end; h0 += BATCH * a.heads_at_once) {
        Piece<E> lo[BATCH], hi[BATCH];
        Raw *dst[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int h = h0 + i * a.heads_at_once;
            if (h < h_end) {
                const int w = h >= a.q_heads;
                const int hh = w ? h - a.q_heads : h;
                const Raw *src = static_cast<const Raw *>(a.in[w]) + (b * a.in_stride[w][0] + t * a.in_stride[w][1] + hh * a.in_stride[w][2]) + e0;
                dst[i] = static_cast<Raw *>(a.out[w]) + (b * a.out_stride[w][0] + t * a.out_stride[w][1] + hh * a.out_stride[w][2]) + e0;
                lo[i] = load_piece<E>(src, n);
                if (!INTERLEAVED && rotated) hi[i] = load_piece<E>(src + half, n);
            }
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int h = h0 + i * a.heads_at_once;
            if (h >= h_end) continue;
            if (rotated) {
#pragma unroll
                for (int k = 0; k < PAIRS; ++k) {
                    Raw &ra = INTERLEAVED ? lo[i].e[2 * k] : lo[i].e[k];
                    Raw &rb = INTERLEAVED ? lo[i].e[2 * k + 1] : hi[i].e[k];
                    const float x = E::to_f32(ra), y = E::to_f32(rb);
                    if (!(keep >> k & 1)) {
                        ra = E::from_f32(fmaf(x, c[k], -(y * s[k])));
                        rb = E::from_f32(fmaf(x, s[k], y * c[k]));
                    }
                }
            }
            store_piece<E, V, STREAM>(dst[i], lo[i], n);
            if (!INTERLEAVED && rotated) store_piece<E, V, STREAM>(dst[i] + half, hi[i], n);
        }
    }
}

// One thread per pair of a position; the angle and its cosine and sine in 64 bits, rounded once.
__global__ __launch_bounds__(kThreads) void rope_table_kernel(const double *freq, int half, int64_t total, double magnitude, float2 *table) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= total) return;
    const int64_t p = i / half;
    double s, c;
    sincos((double)p * freq[i - p * half], &s, &c);
    table[i] = make_float2((float)(magnitude * c), (float)(magnitude * s));
}

}  // namespace

int launch_rope_table(const double *freq, int64_t n_pos, int64_t half, double magnitude, float *table, hipStream_t stream) {
    const int64_t total = n_pos * half;
    rope_table_kernel<<<dim3((unsigned)((total + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(freq, (int)half, total, magnitude,
                                                                                                      reinterpret_cast<float2 *>(table));
    return check_launch();
}

int launch_rope(const dvdq_rope_heads *q, const dvdq_rope_heads *k, int64_t B, int64_t T, int64_t D, const float *table, int64_t n_pos,
                int64_t R, const int32_t *positions, int64_t pos_batch, int n_axes, const int32_t *sections, bool interleaved, bool inverse,
                int dtype, hipStream_t stream) {
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        RopeKernelArgs a = {};
        bool in_place = true;
        for (int w = 0; w < (k ? 2 : 1); ++w) {
            const dvdq_rope_heads *h = w ? k : q;
            a.in[w] = h->in;
            a.out[w] = h->out;
            in_place = in_place && h->in == h->out;
            for (int i = 0; i < 3; ++i) a.in_stride[w][i] = h->in_stride[i], a.out_stride[w][i] = h->out_stride[i];
        }
        a.q_heads = (int)q->heads;
        a.heads = (int)(q->heads + (k ? k->heads : 0));
        a.tokens = (uint32_t)(B * T);
        a.T = (uint32_t)T;
        a.D = (int)D;
        a.R = (int)R;
        a.table = reinterpret_cast<const float2 *>(table);
        a.n_pos = (int)n_pos;
        a.positions = positions;
        a.pos_batch = (uint32_t)pos_batch;
        a.n_axes = n_axes;
        int first = 0;
        for (int i = 0; i < kMaxAxes - 1; ++i) {
            first = i < n_axes - 1 ? first + sections[i] / 2 : (int)(R / 2);
            a.bound[i] = first;
        }
        a.inverse = inverse;
        const int per_unit = interleaved ? E::kVec : 2 * E::kVec;
        a.rot_units = (int)((R + per_unit - 1) / per_unit);
        // (in place, the part that is not rotated stays where it is)
        const int units = a.rot_units + (in_place ? 0 : (int)((D - R + E::kVec - 1) / E::kVec));
        // (both parts rounded up: 257 pieces of fp32 where a part of a head of 1023 or 1024 is rotated; the last one is a second workgroup's)
        a.units = std::min(units, kThreads);
        // heads of a thread: as many as are in flight at a time, fewer where that leaves the chip with less than 512 threads per compute unit
        // (and, where a head is no whole lines, so that those that a token's threads write at once are 384 bytes at least: 46400 x 6 heads
        // of 72 16.5 us with three at once, 24 with one)
        const int head_bytes = (int)(D * sizeof(typename E::Raw)), at_once = head_bytes % 128 == 0 ? 1 : (383 + head_bytes) / head_bytes;
        int per_thread = std::clamp(a.heads / at_once, 1, kHeadsPerThread);
        while (per_thread > 1 && (int64_t)a.tokens * a.units * ((a.heads + per_thread - 1) / per_thread) < 256 * 512) --per_thread;
        a.heads_at_once = std::min((a.heads + per_thread - 1) / per_thread, kThreads / a.units);
        a.tokens_per_block = kThreads / (a.units * a.heads_at_once);
        a.heads_per_block = a.heads_at_once * per_thread;
        const dim3 grid((a.tokens + a.tokens_per_block - 1) / a.tokens_per_block, (a.heads + a.heads_per_block - 1) / a.heads_per_block,
                        (units + kThreads - 1) / kThreads);
        // Streaming stores from 4 MB on, which is what an XCD's L2 holds: 2000 x 40 heads of 128 9.4 us, cached 13.6; below that the
        // outputs stay in the L2 for what reads them next (1022 x 16 heads of 80, 2.6 MB: 7.1 us, streaming 7.2).
        const bool stream_out = (int64_t)a.tokens * a.heads * D * (int64_t)sizeof(typename E::Raw) >= (4 << 20);
        const auto kernel = interleaved ? (stream_out ? rope_kernel<E, true, true> : rope_kernel<E, true, false>)
                                        : (stream_out ? rope_kernel<E, false, true> : rope_kernel<E, false, false>);
        kernel<<<grid, kThreads, 0, stream>>>(a);
        return check_launch();
    });
}

}  // namespace dvdq
