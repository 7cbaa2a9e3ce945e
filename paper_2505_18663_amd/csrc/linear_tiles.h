// Tiled matrix products with their epilogue, of 16-bit elements (linear16.hip) and of 8-bit codes (linear8.hip):
//
//   y[m, n] = residual[m, n] + gate[m / (M / G), n] * act(sum_k x[m, k] w[n, k] (times scales) + bias[n])
//
// Ways: linear_few (few tokens), linear_tiles (five shapes of tile, K in parts where there are few tiles: linear_join), rows that are no whole
// 16-byte pieces copied first (linear_pad) or through registers (linear_any).  Times in comments are of 16-bit products unless said.
#pragma once
#include <algorithm>

#include "elem.h"
#include "gemm_common.h"

namespace dvdq {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// Operands of a product: 16 bytes of a row of each are a lane's share of a matrix instruction, whatever the type, so that tiles, slices and
// their places in LDS are those of bytes.  Out: the type of the output, and of what goes into the epilogue.
template <typename E>
struct Op16 {                          // 16-bit elements, sums in fp32
    using Out = E;
    using Acc = v4f;
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ v4f mfma(uint4 a, uint4 b, v4f c) {
        if constexpr (std::is_same<E, Bf16>::value)
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    }
    static constexpr int kBytes = 2;
};
template <typename E>
struct Op8 {                           // 8-bit codes, exact sums, a scale per token and per channel
    using Out = E;
    using Acc = v4i;
    static constexpr bool kScaled = true;
    static constexpr int kBytes = 1;
    static __device__ __forceinline__ v4i mfma(uint4 a, uint4 b, v4i c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, a), __builtin_bit_cast(v4i, b), c, 0, 0, 0);
    }
};
// 16 bytes at any element's address, of which `left` belong to the row, whose length is K
template <typename P>
static __device__ __forceinline__ uint4 load_operand(const uint8_t *p, int left, int K) {
    struct __attribute__((packed, aligned(P::kBytes))) Sixteen {
        uint32_t w[4];
    };
    if (left >= 16) return __builtin_bit_cast(uint4, *reinterpret_cast<const Sixteen *>(p));
    return load_end<P::kBytes>(p, left, K >= 16);
}

struct LinearArgs {
    const uint8_t *x, *w;
    const float *x_scale, *w_scale;    // of 8-bit operands
    const void *bias, *gate, *residual;
    void *y;
    int64_t ldx, ldw;                  // bytes between rows
    int64_t ldr, ldy, ldg;             // elements between rows
    int M, N, K;                       // K: bytes of a row
    int gate_rows;                     // tokens of one row of the gate
    float4 *parts;                     // sums of parts of K, in the order of the accumulators (kPart)
    int splits, slices;                // parts of K; slices of 128 bytes of a part
    // Outputs past the caches, where they are larger than an XCD's L2 and the 64 bytes that the lanes of a token write are sectors of their own
    // (rows and address multiples of 64 bytes): 32760 x 1536 x 8960 with tanh GELU 823 -> 775 us, 32760 x 1536 x 4608 395 -> 364, 118800 x 1536 x 1536 513 -> 510.  (fp32
    // outputs: see launch_linear8.)
    bool streaming;
};
constexpr int kPart = 4;               // in the place of an activation: leave the sums of a part of K for linear_join

// Eight elements as words, which stay so many registers where a branch or a row's end puts them together (as an array of elements each would have
// a register of its own).
template <typename E>
struct Eight {
    static constexpr int kWords = sizeof(typename E::Raw);   // twice that many words
    uint32_t w[2 * kWords];
    __device__ __forceinline__ float at(int i) const {
        if constexpr (kWords == 2) return E::to_f32((uint16_t)(w[i / 2] >> 16 * (i % 2)));
        else return __builtin_bit_cast(float, w[i]);
    }
    // n of them, at least one; what comes past those is not to be used
    static __device__ __forceinline__ Eight load(const typename E::Raw *p, int n) {
        if (n >= 8) return __builtin_bit_cast(Eight, *reinterpret_cast<const Piece<E, 8> *>(p));
        uint32_t e[8];                                       // (the last one in the place of those past it: no load hangs on a condition)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kWords == 2) e[i] = p[min(i, n - 1)];
            else e[i] = __builtin_bit_cast(uint32_t, p[min(i, n - 1)]);
        }
        Eight r;
#pragma unroll
        for (int i = 0; i < 2 * kWords; ++i) r.w[i] = kWords == 2 ? e[2 * i % 8] | e[(2 * i + 1) % 8] << 16 : e[i];
        return r;
    }
    static __device__ __forceinline__ Eight rounded(const float (&v)[8]) {
        Eight r;
#pragma unroll
        for (int i = 0; i < 2 * kWords; ++i) {
            if constexpr (kWords == 2) r.w[i] = E::from_f32(v[2 * i]) | (uint32_t)E::from_f32(v[2 * i + 1]) << 16;
            else r.w[i] = __builtin_bit_cast(uint32_t, v[i]);
        }
        return r;
    }
    __device__ __forceinline__ Piece<E, 8> piece() const { return __builtin_bit_cast(Piece<E, 8>, *this); }
};

// n elements on from a kernel's argument p, n the same for all lanes.  (A pointer that is put together from scalar registers itself, as by
// uniform_ptr, is of no address space to the compiler: flat accesses, which count as LDS ones too, at 64-bit addresses in vector registers.)
template <typename T>
static __device__ __forceinline__ T *uniform_on(T *p, int64_t n) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)n), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)n >> 32));
    return p + (int64_t)((uint64_t)hi << 32 | lo);
}
// p is the same for all lanes, the offset 32 bits of each lane's own: one register an address
template <typename T>
static __device__ __forceinline__ T *bytes_on(T *p, uint32_t offset) {
    using Byte = std::conditional_t<std::is_const<T>::value, const uint8_t, uint8_t>;
    return reinterpret_cast<T *>(reinterpret_cast<Byte *>(p) + offset);
}

// What follows the sums of a wave's 64 channels x 16 FM tokens, from channel n0 of token m0 on: the lane's token of fragment j is
// m0 + 16 j + lane % 16, its channels 8 (lane / 16) .. + 7 and the same 32 further on (channel_of_row).
template <typename P, int ACT, int FM>
static __device__ __forceinline__ void epilogue(const LinearArgs &a, const typename P::Acc (&acc)[4][FM], int m0, int n0) {
    using E = typename P::Out;
    using Raw = typename E::Raw;
    using Row8 = Eight<E>;
    const Raw *bias_row = static_cast<const Raw *>(a.bias), *gate_rows = static_cast<const Raw *>(a.gate);
    const int lane = threadIdx.x & 63, row = lane & 15, col = 8 * (lane >> 4);
    if (m0 >= a.M || n0 >= a.N) return;
    const bool shared_gate = a.gate && m0 / a.gate_rows == (min(m0 + 16 * FM, a.M) - 1) / a.gate_rows;   // one row for all tokens
    const uint32_t off_y = (row * (uint32_t)a.ldy + col) * (uint32_t)sizeof(Raw), off_r = (row * (uint32_t)a.ldr + col) * (uint32_t)sizeof(Raw);   // bytes
    Raw *y = uniform_on(static_cast<Raw *>(a.y), m0 * a.ldy + n0);
    const Raw *res = a.residual ? uniform_on(static_cast<const Raw *>(a.residual), m0 * a.ldr + n0) : nullptr;
    // scales of 8 channels (from n on, `count` of them) and of the tokens
    struct Scales {
        float e[P::kScaled ? 8 : 1];
    };
    float token_scale[P::kScaled ? FM : 1];
    if constexpr (P::kScaled) {
#pragma unroll
        for (int j = 0; j < FM; ++j) token_scale[j] = a.x_scale[min(m0 + 16 * j + row, a.M - 1)];
    }
    auto scales = [&](int n, int count) {
        Scales s = {};
        if constexpr (P::kScaled) {
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                #pragma unroll
                for (int e = 0; e < 4; ++e) s.e[i + e] = a.w_scale[count == 8 ? n + i + e : min(n + i + e, a.N - 1)];
            }
        }
        return s;
    };
    auto values = [&](float (&v)[8], int h, int j, const Row8 &bias, const Scales &s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const auto sum = acc[2 * h + i / 4][j][i & 3];
            if constexpr (P::kScaled) v[i] = activate<ACT>(fmaf((float)sum * s.e[i], token_scale[j], bias.at(i)));
            else v[i] = activate<ACT>(sum + bias.at(i));
        }
    };
    auto times = [](float (&v)[8], const Row8 &p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= p.at(i);
    };
    auto plus = [](float (&v)[8], const Row8 &p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += p.at(i);
    };
    // The lane's row of the gate, token by token (16 apart): a division once, for the first
    struct GateRow {
        int q, left, first_q, first_left, by, by_left, tokens;
        __device__ __forceinline__ GateRow(const LinearArgs &a, int m) : tokens(a.gate_rows) {
            first_q = m / tokens, first_left = m - first_q * tokens;
            by = 16 / tokens, by_left = 16 - by * tokens;
            q = first_q, left = first_left;
        }
        __device__ __forceinline__ void begin() {
            q = first_q, left = first_left;
            asm volatile("" : "+v"(q));   // (or the second half's addresses are the first's, kept in registers)
        }
        __device__ __forceinline__ int next() {
            const int here = q;
            left += by_left;
            q += by + (left >= tokens ? 1 : 0);
            left -= left >= tokens ? tokens : 0;
            return here;
        }
    };
    if (m0 + 16 * FM <= a.M && n0 + 64 <= a.N) {
        // Loads come back behind the stores in front of them, and behind a branch around a load the compiler waits for all of both.  So each
        // combination of gate and residual has its own way without branches, and what the next chunk of B tokens is made of is requested before the
        // stores of the present one, the residual (which y may be: the compiler could not move its loads above a store) two chunks ahead, and
        // with it the gate where tokens have rows of their own (as edge tiles have it, token by token behind the stores, 32760 x 1536 x 1536 with a
        // residual took 201 us in place of 174, 8011 x 293 x 9621 208 in place of 161, 6240 x 1536 x 1536 51.5 in place of 43.2).
        const auto whole = [&](auto gated, auto added) {
            constexpr int GATE = decltype(gated)::value;     // 1: one row for all tokens, 2: rows of their own
            constexpr bool RES = decltype(added)::value, AHEAD = RES || GATE == 2;
            // As many tokens as registers hold: with four of 256 x 256 tiles' 8-bit ones, 29 to 105 words spilt, 118800 x 1536 x 1536 with gate and residual 407 us in
            // place of 367, 32760 x 5120 x 13824 2150 and 2065, fp32 outputs 32760 x 1536 x 5120 592 and 498.
            constexpr int B = std::min(FM, GATE < 2 ? (FM == 8 && P::kScaled ? 2 : 4) : FM == 8 ? 1 : sizeof(Raw) == 4 ? 2 : 4), C = FM / B;   // tokens of a chunk, chunks of 32 channels
            Scales s;
            Row8 bias, gate, r[2][RES ? B : 1], g[2][GATE == 2 ? B : 1], out[B];
            auto vectors = [&](int h) {
                const int n = n0 + 32 * h + col;
                s = scales(n, 8);
                bias = Row8();
                if (a.bias) bias = Row8::load(bias_row + n, 8);
                if constexpr (GATE == 1) gate = Row8::load(gate_rows + (m0 / a.gate_rows) * a.ldg + n, 8);
            };
            GateRow gate_row(a, m0 + row);
            auto fetch = [&](int c) {
                if constexpr (RES) {
#pragma unroll
                    for (int j = 0; j < B; ++j) r[c & 1][j] = Row8::load(bytes_on(res + 16 * (c % C * B + j) * a.ldr + 32 * (c / C), off_r), 8);
                }
                if constexpr (GATE == 2) {
                    if (c % C == 0) gate_row.begin();
#pragma unroll
                    for (int j = 0; j < B; ++j) g[c & 1][j] = Row8::load(gate_rows + gate_row.next() * a.ldg + (n0 + 32 * (c / C) + col), 8);
                }
            };
            vectors(0);
            if constexpr (AHEAD) {
                fetch(0);
                fetch(1);
            }
#pragma unroll
            for (int c = 0; c < 2 * C; ++c) {
                const int h = c / C, j0 = c % C * B;
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    float v[8];
                    values(v, h, j0 + j, bias, s);
                    if constexpr (GATE == 1) times(v, gate);
                    if constexpr (GATE == 2) times(v, g[c & 1][j]);
                    if constexpr (RES) plus(v, r[c & 1][j]);
                    out[j] = Row8::rounded(v);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (c == C - 1) vectors(1);
                if constexpr (AHEAD)
                    if (c + 2 < 2 * C) fetch(c + 2);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    Raw *to = bytes_on(y + 16 * (j0 + j) * a.ldy + 32 * h, off_y);
                    if (a.streaming) store_piece<E, 8, true>(to, out[j].piece(), 8);
                    else store_piece<E, 8>(to, out[j].piece(), 8);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        const auto gated = [&](auto which) {
            if (res) whole(which, std::true_type());
            else whole(which, std::false_type());
        };
        if (!a.gate) gated(std::integral_constant<int, 0>());
        else if (shared_gate) gated(std::integral_constant<int, 1>());
        else gated(std::integral_constant<int, 2>());
    } else {
        constexpr int B = FM == 8 ? 2 : FM;
        // WHOLE: the lanes have 8 channels or none.  (Code that is run once takes longer to fetch than to run: without that for parts of 8 channels
        // 500 x 131 x 512 8.6 -> 7.7 us, 2559 x 87 x 160 6.7 -> 5.8.)
        const auto edge = [&](auto whole_pieces) {
            constexpr bool WHOLE = decltype(whole_pieces)::value;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = n0 + 32 * h + col, count = WHOLE ? 8 : min(8, a.N - n);
                if (n >= a.N) continue;
                const Scales s = scales(n, count);
                Row8 bias = {};
                if (a.bias) bias = Row8::load(bias_row + n, count);
#pragma unroll
                for (int j0 = 0; j0 < FM; j0 += B) {
                    Row8 r[B] = {}, g[B] = {};
                    if (a.gate) {
                        GateRow gate_row(a, m0 + 16 * j0 + row);
#pragma unroll
                        for (int j = 0; j < B; ++j) g[j] = Row8::load(gate_rows + min(gate_row.next(), (a.M - 1) / a.gate_rows) * a.ldg + n, count);
                    }
                    if (res)
#pragma unroll
                        for (int j = 0; j < B; ++j) {
                            const int from = min(16 * (j0 + j) + row, a.M - 1 - m0);   // tokens past the last read the last one's.  In 64 bits: one token's pitch may be anything
                            r[j] = Row8::load(res + from * a.ldr + 32 * h + col, count);
                        }
#pragma unroll
                    for (int j = 0; j < B; ++j) {
                        const int m = m0 + 16 * (j0 + j) + row;
                        if (m < a.M) {
                            float v[8];
                            values(v, h, j0 + j, bias, s);
                            if (a.gate) times(v, g[j]);
                            if (res) plus(v, r[j]);
                            store_piece<E, 8>(bytes_on(y + 16 * (j0 + j) * a.ldy + 32 * h, off_y), Row8::rounded(v).piece(), count);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        };
        if (FM < 8 && (a.N % 8 == 0 || n0 + 64 <= a.N)) edge(std::true_type());
        else edge(std::false_type());
    }
}

// The weights are the matrix instruction's rows, the tokens its columns, so that a lane's four results are four channels of one
// token.  Row r of fragment f of 64 channels is channel 32 (f / 2) + 8 (r / 4) + 4 (f % 2) + r % 4: two fragments are then 8
// consecutive channels of a lane, 16 bytes, and the four lanes of a token store 64 bytes in a row, without a detour.
static __device__ __forceinline__ int channel_of_row(int row) {
    return (row & ~63) + 32 * ((row >> 5) & 1) + 8 * ((row & 15) >> 2) + 4 * ((row >> 4) & 1) + (row & 3);
}

// The sums of a wave, for linear_join: `at` numbers its fragments
template <typename Acc, int FM>
static __device__ __forceinline__ void store_part(const LinearArgs &a, const Acc (&acc)[4][FM], int64_t at) {
#pragma unroll
    for (int j = 0; j < FM; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) a.parts[((at + j) * 4 + i) * 64 + (threadIdx.x & 63)] = __builtin_bit_cast(float4, acc[i][j]);
}

// Any sizes, pitches and addresses: tiles as in linear_tiles, a workgroup each, operands through registers into LDS rows of 128 bytes of K, a
// slice ahead.  LDS as there.
template <typename P, int ACT, int FM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM, 2) void linear_any(LinearArgs a, int group_n) {
    constexpr int W = WN * WM, BN = 64 * WN, BM = 16 * FM * WM, R = 8 * W;   // R: rows that the threads have a piece each of
    constexpr int LW = BN / R, LX = BM / R;
    extern __shared__ uint4 lds[];                           // two slices of BN rows of weights, BM of tokens
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_tiles = (a.N + BN - 1) / BN, m_tiles = (a.M + BM - 1) / BM, tiles = n_tiles * m_tiles, grid = gridDim.x;
    // A run of tiles for each XCD, as there.  (Divisions that a launch can do without are left out: 512 x 131 x 512 8.1 -> 7.9 us.)
    const int xcd = blockIdx.x & 7, t = (grid >> 3) * xcd + min(xcd, grid & 7) + (blockIdx.x >> 3), split = a.splits == 1 ? 0 : t / tiles;
    int m0, n0;
    if (group_n >= n_tiles) {
        const int tile = t - split * tiles, tile_m = tile / n_tiles;
        m0 = tile_m * BM, n0 = (tile - tile_m * n_tiles) * BN;
    } else {
        tile_origin(t - split * tiles, m_tiles, n_tiles, group_n, BM, BN, m0, n0);
    }
    const int wn = wave % WN * 64, wm = wave / WN * 16 * FM;
    const int q0 = split * a.slices, q1 = min(q0 + a.slices, (a.K + 127) >> 7);
    typename P::Acc acc[4][FM] = {};
    const int piece = tid & 7, row0 = tid >> 3;
    uint4 pw[LW], px[LX];
    // Of a slice across the rows' end a thread loads the 16 bytes that end with the row, in the place of its piece or of one past the end, and shifts
    // them on their way to LDS: as pieces that hang on conditions, each load was waited for (40 x 100 x 1536 7.2 -> 6.8 us).
    auto load = [&](int q) __attribute__((always_inline)) {
        const auto rows = [&](int from, int count) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < LW; ++i) pw[i] = load_operand<P>(a.w + min(n0 + channel_of_row(row0 + R * i), a.N - 1) * a.ldw + from, count, a.K);
#pragma unroll
            for (int i = 0; i < LX; ++i) px[i] = load_operand<P>(a.x + min(m0 + row0 + R * i, a.M - 1) * a.ldx + from, count, a.K);
        };
        const int k = q * 128 + piece * 16;
        if ((q + 1) * 128 <= a.K) rows(k, 16);
        else if (a.K >= 16) rows(min(k, a.K - 16), 16);
        else rows(k, a.K - k);
    };
    if (q0 < q1) load(q0);
    for (int q = q0; q < q1; ++q) {
        uint4 *lds_w = lds + (q & 1) * (8 * (BN + BM)), *lds_x = lds_w + 8 * BN;
        const int at = row0 * 8 + (piece ^ ((row0 >> 1) & 7));   // (R is a multiple of 16: the same exchange of pieces in all of a thread's rows)
        const auto put = [&](auto of) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < LW; ++i) lds_w[at + 8 * R * i] = of(pw[i]);
#pragma unroll
            for (int i = 0; i < LX; ++i) lds_x[at + 8 * R * i] = of(px[i]);
        };
        const int past = q * 128 + piece * 16 - (a.K - 16);  // bytes of the thread's piece that are past the end
        if ((q + 1) * 128 <= a.K || a.K < 16) put([](const uint4 &v) { return v; });
        else put([&](const uint4 &v) { return past >= 16 ? uint4() : shifted_down(v, max(past, 0)); });
        __syncthreads();                                     // (and every wave has read the slice before the last)
        if (q + 1 < q1) load(q + 1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uint4 fw[4], fx[FM];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int rw = wn + 16 * f + (lane & 15), p = 4 * ks + (lane >> 4);
                fw[f] = lds_w[rw * 8 + (p ^ ((rw >> 1) & 7))];
            }
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                const int rx = wm + 16 * f + (lane & 15), p = 4 * ks + (lane >> 4);
                fx[f] = lds_x[rx * 8 + (p ^ ((rx >> 1) & 7))];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < FM; ++j) acc[i][j] = P::mfma(fw[i], fx[j], acc[i][j]);
        }
    }
    if constexpr (ACT == kPart) store_part(a, acc, ((int64_t)t * W + wave) * FM);
    else epilogue<P, ACT>(a, acc, __builtin_amdgcn_readfirstlane(m0 + wm), __builtin_amdgcn_readfirstlane(n0 + wn));
}

// ---- few tokens (at most 16): bound by the weights, which are read once, straight into registers
// A workgroup has 16 channels, its waves parts of K: a lane reads 32 bytes of a channel (the four lanes of a channel a whole line) and the same part of its
// token, two matrix instructions' worth, twice over before the first product; the waves' sums meet in LDS in their order.
// (The instruction's order of K does not matter as long as it is the same on both sides.)
// 2 x 1536 x 9216, 28 MB of weights: 9.1 us with 8 waves (8.3 where the caches hold the weights), 9.5 with 16, 9.6 with 4; as tiles 14.1.
// 1 x 1536 x 4608 6.5 and 11.9, 16 x 1536 x 13824 15.0 and 18.2, 2 x 5120 x 30720 57 and 67.  Few channels leave compute units idle and long rows their
// waves with too little in flight: 8 x 13824 x 128 22 and 15, 16 x 5120 x 5120 23 and 19, 2 x 13824 x 5120 36 and 36; these are tiles.
constexpr int kFewWaves = 8;
// 8-bit codes, us, this and tiles: 1 x 13824 x 5120 19.0 and 24.8, 8 x 13824 x 5120 23.9 and 24.9, 16 x 13824 x 5120 28.8 and 24.3 (a step loads as many bytes of
// tokens as of weights by then), 16 x 5120 x 5120 11.5 and 13.3, 16 x 5120 x 30720 47 and 41, 8 x 5120 x 30720 37 and 41, 16 x 8960 x 1536 10.2 and 12.3,
// 8 x 13824 x 512 12.5 and 12.2, 16 x 13824 x 512 14.2 and 12.0.  32 tokens as two groups: 5120 x 5120 16 and 14.
inline bool few_tokens(int64_t M, int64_t N, int64_t K, bool codes) {   // K: bytes of a row
    return codes ? M <= 8 || (M <= 16 && K <= 12288 && N * K <= (int64_t)1 << 26) : M <= 16 && (K <= 8192 || N >= 16384);
}
template <typename P, int ACT>
__global__ __launch_bounds__(512) void linear_few(LinearArgs a) {
    using E = typename P::Out;
    using Raw = typename E::Raw;
    using Acc = typename P::Acc;
    extern __shared__ uint4 lds[];
    Acc *sums = reinterpret_cast<Acc *>(lds);                // [wave][token][channels / 4]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, n0 = blockIdx.x * 16;
    const uint8_t *w = a.w + min(n0 + (lane & 15), a.N - 1) * a.ldw, *x = a.x + min(lane & 15, a.M - 1) * a.ldx;
    const int steps = (a.K + 127) >> 7, q0 = (int)((int64_t)steps * wave / waves), q1 = (int)((int64_t)steps * (wave + 1) / waves);
    constexpr int AHEAD = 2;
    Acc acc[2] = {};
    const int whole = min(q1, a.K >> 7);                     // steps of 128 bytes that there are
    w += (lane >> 4) * 32, x += (lane >> 4) * 32;
    int q = q0;
    for (; q + AHEAD <= whole; q += AHEAD) {
        uint4 pw[AHEAD][2], px[AHEAD][2];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pw[i][h] = load_operand<P>(w + (q + i) * 128 + 16 * h, 16, a.K);
                px[i][h] = load_operand<P>(x + (q + i) * 128 + 16 * h, 16, a.K);
            }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[h] = P::mfma(pw[i][h], px[i][h], acc[h]);
    }
    if (q < whole) {                                         // fewer than AHEAD: the rest once more, as nothing
        uint4 pw[AHEAD - 1][2], px[AHEAD - 1][2];
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pw[i][h] = load_operand<P>(w + min(q + i, whole - 1) * 128 + 16 * h, 16, a.K);
                px[i][h] = load_operand<P>(x + min(q + i, whole - 1) * 128 + 16 * h, 16, a.K);
            }
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i)
            if (q + i < whole) {
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[h] = P::mfma(pw[i][h], px[i][h], acc[h]);
            }
    }
    if (whole < q1) {                                        // the last step, of fewer than 128 bytes
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = whole * 128 + 16 * h, left = a.K - k - (lane >> 4) * 32;
            uint4 pw = {}, px = {};
            if (left > 0) {
                pw = load_operand<P>(w + k, left, a.K);
                px = load_operand<P>(x + k, left, a.K);
            }
            acc[h] = P::mfma(pw, px, acc[h]);
        }
    }
    sums[(wave * 16 + (lane & 15)) * 4 + (lane >> 4)] = acc[0] + acc[1];
    __syncthreads();
    const int m = threadIdx.x >> 4, n = n0 + (threadIdx.x & 15);
    if (threadIdx.x >= 256 || m >= a.M || n >= a.N) return;
    using Sum = std::remove_reference_t<decltype(acc[0][0])>;
    Sum sum = 0;
    for (int i = 0; i < waves; ++i) sum += reinterpret_cast<const Sum *>(sums)[i * 256 + threadIdx.x];
    float v = (float)sum;
    if constexpr (P::kScaled) v = v * a.w_scale[n] * a.x_scale[m];
    if (a.bias) v += E::to_f32(static_cast<const Raw *>(a.bias)[n]);
    v = activate<ACT>(v);
    if (a.gate) v *= E::to_f32(static_cast<const Raw *>(a.gate)[(m / a.gate_rows) * a.ldg + n]);
    if (a.residual) v += E::to_f32(static_cast<const Raw *>(a.residual)[m * a.ldr + n]);
    static_cast<Raw *>(a.y)[m * a.ldy + n] = E::from_f32(v);
}

// Rows of K bytes at any address -> rows of `pitch` bytes, a multiple of 128, zero past K: activations (rows_x of them), then weights.  A
// workgroup has `rows` rows, whose pieces are numbered through: piece i is in row i * mul >> 32, mul = 2^32 / pieces rounded up, which is exact for
// the 512 pieces that rows share a workgroup up to; longer rows have one each (mul = 0).
template <typename P>
__global__ __launch_bounds__(256) void linear_pad(const uint8_t *x, int64_t ldx, int rows_x, const uint8_t *w, int64_t ldw, int rows_w, int K,
                                                  int pitch, int rows, uint32_t mul, uint8_t *out) {
    const uint32_t pieces = (uint32_t)pitch / 16;
    const int64_t row0 = (int64_t)blockIdx.x * rows;
    const uint32_t here = pieces * (uint32_t)min((int64_t)rows, rows_x + (int64_t)rows_w - row0);
    uint4 *to = reinterpret_cast<uint4 *>(out) + row0 * pieces;
    constexpr int AHEAD = 2;
    for (uint32_t i = threadIdx.x; i < here; i += 256 * AHEAD) {
        uint4 p[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const uint32_t at = i + 256 * e, r = __umulhi(at, mul);
            const int k = (int)(at - r * pieces) * 16;
            const int64_t row = row0 + r;
            p[e] = uint4();
            if (at < here && k < K) p[e] = load_operand<P>((row < rows_x ? x + row * ldx : w + (row - rows_x) * ldw) + k, min(16, K - k), K);
        }
#pragma unroll
        for (int e = 0; e < AHEAD; ++e)
            if (i + 256 * e < here) to[i + 256 * e] = p[e];
    }
}

// Joins the parts of K, in their order, and finishes: a wave per 64 channels x 16 tokens of tiles of WN x WM waves of 64 channels x 16 FM tokens.
template <typename P, int ACT>
__global__ __launch_bounds__(256) void linear_join(LinearArgs a, int FM, int WN, int WM, int group_n) {
    const int lane = threadIdx.x & 63, per_tile = FM * WN * WM;
    const int n_tiles = (a.N + 64 * WN - 1) / (64 * WN), m_tiles = (a.M + 16 * FM * WM - 1) / (16 * FM * WM);
    const int64_t g = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), stride = (int64_t)n_tiles * m_tiles * per_tile * 256;
    const int tile = (int)(g / per_tile), in = (int)(g - (int64_t)tile * per_tile), wave = in / FM, j = in - wave * FM;
    if (tile >= n_tiles * m_tiles) return;
    int m0, n0;
    tile_origin(tile, m_tiles, n_tiles, group_n, 16 * FM * WM, 64 * WN, m0, n0);
    m0 += wave / WN * 16 * FM + 16 * j;
    n0 += wave % WN * 64;
    if (m0 >= a.M || n0 >= a.N) return;
    typename P::Acc acc[4][1] = {};
    const float4 *p = a.parts + g * 256 + lane;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s, p += stride)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][0] += __builtin_bit_cast(typename P::Acc, p[i * 64]);
    epilogue<P, ACT>(a, acc, m0, n0);
}

// ---- rows of whole 16-byte pieces: operands straight into LDS

// 16 bytes per lane from each lane's own address to LDS address lds_base + 16 * lane (completion awaited by hand, as with
// lds_direct_load16)
static __device__ __forceinline__ void lds_direct_load16_at(const void *p, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds_base) : "memory");
}

__device__ uint4 zero_piece;   // what the pieces past K of the last slice are read from

// Tiles of 64 WN channels x 16 FM WM tokens, WN x WM waves of 64 channels x 16 FM tokens each; slices of 128 bytes of K.
// Tokens have three slices in LDS, weights two, or the other way round (slices_of_weights): while a slice is multiplied, the next is there, the tokens of
// the one after it come in, and its weights follow as soon as those of the present slice have been read.  (The tokens are what comes from further away: with three
// slices of weights and two of tokens, 256 x 256 tiles, 8-bit 32760 x 13824 x 5120 took 1734 to 1810 us in place of 1693 to 1757, 32760 x 8960 x 1536 360 in place of 351.
// What bounds the loop on a full chip is the way from the L2s into LDS, 54 to 69 GB/s per compute unit where 32 of them share panels; it must not run dry.
// Five slices of tokens and four of weights for 128 x 128 and smaller tiles: 8-bit 600 x 4608 x 1536 20.1 -> 16.0 us, 17 x 13824 x 5120 23.7 -> 20.3, 1000 x 8960 x 1536
// 28.1 -> 25.6, but 1560 x 1536 x 1536 11.3 -> 11.9, 512 x 4096 x 5120 level, and one workgroup a compute unit; not kept.)
// A slice is worked off in phases of 16 matrix instructions (or fewer), and a phase begins by requesting the fragments of the next one.
// Before the last phase of a slice, whose fragments are then in registers, stands the slice's one barrier: behind it the next slice is
// in LDS for every wave, and this one's place is free.
// A workgroup takes tile after tile, without a seam: the last slices of a tile load the first ones of the next, which is multiplied
// while the outputs are still being written.
// Tiles of 256 x 128 and 128 x 64, two thirds of whose loads are weights: 886 x 9984 x 6016 106 to 114 -> 102 us, 1000 x 5120 x 5120 58.8 to 62 -> 56.7, 8-bit 57.4 -> 55.0 and
// 34.3 -> 32.9; where rows are no whole lines 2 x 7592 x 3080 18.0 -> 16.2, 33 x 5000 x 5000 19.2 -> 17.5, 8-bit 40 x 7600 x 3080 14.2 -> 13.5; but 7212 x 64 x 1093
// 12.5 -> 13.5, 8-bit 17 x 5120 x 13824 19.2 -> 20.1.
constexpr int slices_of_weights(int BN, int BM) { return BN > BM ? 3 : 2; }
template <typename P, int ACT, int FM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM, 2) void linear_tiles(LinearArgs a, int group_n) {
    constexpr int W = WN * WM, BN = 64 * WN, BM = 16 * FM * WM, FH = FM < 4 ? FM : 4, NH = FM / FH, PH = 2 * NH;
    constexpr int LW = BN / 8 / W, LX = BM / 8 / W;          // loads of a wave per slice, 8 rows each
    constexpr int kAhead = slices_of_weights(BN, BM) == 3 ? LW : LX;   // of the operand that is loaded two slices ahead
    constexpr int kStores = ACT == kPart || sizeof(typename P::Out::Raw) == 4 ? 4 * FM : 2 * FM;   // of a wave per whole tile, at least
    constexpr uint32_t kUnitW = BN * 128, kUnitX = BM * 128;
    constexpr int SW = slices_of_weights(BN, BM), SX = 5 - SW;
    extern __shared__ uint4 lds[];                           // weights: SW units, tokens: SX
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_tiles = (a.N + BN - 1) / BN, m_tiles = (a.M + BM - 1) / BM, tiles = n_tiles * m_tiles, items = tiles * a.splits, grid = gridDim.x;
    const int wn = wave % WN * 64, wm = wave / WN * 16 * FM;
    const int slices = a.slices;                             // at least 2; what lies past K is zero

    // Consecutive workgroups go to different XCDs.  Each XCD has one run of tiles, which its workgroups take in order: those that run
    // at the same time share panels, and so do those of the next round (as interleaved rounds of the whole chip, 32760 x 13824 x 5120
    // took 3340 us in place of 3190).
    const int xcds = min(8, grid), xcd = blockIdx.x % xcds, step = (grid - xcd + xcds - 1) / xcds;
    const int share = items / xcds, more = items % xcds;     // (the first XCDs have one more, of workgroups as well as of tiles)
    const int end = share * (xcd + 1) + min(xcd + 1, more);
    const uint32_t lds_w = lds_address(lds) + wave * (1024 * LW), lds_x = lds_address(lds) + SW * kUnitW + wave * (1024 * LX);
    const uint8_t *src_w, *src_x;
    uint32_t off_w[LW], off_x[LX];
    const bool spread_w = a.N * a.ldw < (int64_t)1 << 32, spread_x = a.M * a.ldx < (int64_t)1 << 32;   // offsets of 32 bits
    int m0, n0, k_left;
    auto aim = [&](int t) {                                  // the loads' source: part t / tiles of K of tile t % tiles
        const int part = ACT == kPart ? t / tiles : 0, k0 = part * slices * 128;
        tile_origin(t - part * tiles, m_tiles, n_tiles, group_n, BM, BN, m0, n0);
        k_left = a.K - k0;
        // Rows past the matrix are read from other rows of it (their products are dropped), spread over it: the last row for all of them
        // is one line that every workgroup of a column of tiles asks for at once (24017 x 3608 x 176, 256-channel tiles, 118 us).
        const int base_n = spread_w && n0 + BN > a.N ? 0 : n0, base_m = spread_x && m0 + BM > a.M ? 0 : m0;
        src_w = uniform_ptr(a.w + (base_n * a.ldw + k0));
        src_x = uniform_ptr(a.x + (base_m * a.ldx + k0));
        // Rows are worked out for each tile anew (the compiler does not see that `own` is the same): kept from tile to tile they were spilt, and read back behind
        // every load and store under way: 8-bit 32760 x 1536 x 8960 468 -> 431 us, with tanh GELU 484 -> 464, 32760 x 13824 x 5120 with gate and residual 1717 -> 1707.
        int own = lane;
        asm volatile("" : "+v"(own));
        auto inside = [](int row, int first, int rows, int base) {
            row += first;
            return (row < rows ? row : base + (row - base) % (rows - base)) - base;
        };
#pragma unroll
        for (int j = 0; j < LW; ++j) {
            const int row = wave * (8 * LW) + 8 * j + (own >> 3);
            off_w[j] = (uint32_t)(inside(channel_of_row(row), n0, a.N, base_n) * a.ldw) + 16 * ((own & 7) ^ ((row >> 1) & 7));
        }
#pragma unroll
        for (int j = 0; j < LX; ++j) {
            const int row = wave * (8 * LX) + 8 * j + (own >> 3);
            off_x[j] = (uint32_t)(inside(row, m0, a.M, base_m) * a.ldx) + 16 * ((own & 7) ^ ((row >> 1) & 7));
        }
    };
    // slice q of the aimed tile; `whole`: known to lie within K
    auto load_w = [&](int q, int slot, bool whole) {
        const uint8_t *src = src_w + (uint32_t)q * 128u;
        if (whole || (q + 1) * 128 <= k_left) {
#pragma unroll
            for (int j = 0; j < LW; ++j) lds_direct_load16(src, off_w[j], lds_w + slot * kUnitW + 1024 * j);
        } else {
#pragma unroll
            for (int j = 0; j < LW; ++j) {
                const int piece = 16 * ((lane & 7) ^ (((wave * (8 * LW) + 8 * j + (lane >> 3)) >> 1) & 7));
                lds_direct_load16_at(piece < k_left - q * 128 ? static_cast<const void *>(src + off_w[j]) : &zero_piece, lds_w + slot * kUnitW + 1024 * j);
            }
        }
    };
    auto load_x = [&](int q, int slot, bool whole) {
        const uint8_t *src = src_x + (uint32_t)q * 128u;
        if (whole || (q + 1) * 128 <= k_left) {
#pragma unroll
            for (int j = 0; j < LX; ++j) lds_direct_load16(src, off_x[j], lds_x + slot * kUnitX + 1024 * j);
        } else {
#pragma unroll
            for (int j = 0; j < LX; ++j) {
                const int piece = 16 * ((lane & 7) ^ (((wave * (8 * LX) + 8 * j + (lane >> 3)) >> 1) & 7));
                lds_direct_load16_at(piece < k_left - q * 128 ? static_cast<const void *>(src + off_x[j]) : &zero_piece, lds_x + slot * kUnitX + 1024 * j);
            }
        }
    };

    // fragment reads: LDS row r of 128 bytes holds its 16-byte piece c at c ^ ((r >> 1) & 7), so that the 16 rows that a read takes at
    // once lie in different banks
    const int at = (lane & 15) * 8 + ((lane >> 4) ^ ((lane & 15) >> 1));   // of k-step 0; k-step 1 is piece ^ 4
    const int at_w = wn * 8 + at, at_x = SW * (kUnitW / 16) + wm * 8 + at;
    typename P::Acc acc[4][FM] = {};
    uint4 fw[2][4], fx[2][FH];
    auto read = [&](int sw, int sx, int p) {                 // the fragments of phase p of the slice in these places
        const int ks = p / NH, h = p % NH;
        if (h == 0)
#pragma unroll
            for (int f = 0; f < 4; ++f) fw[ks][f] = lds[sw * (kUnitW / 16) + (at_w ^ (4 * ks)) + 128 * f];
#pragma unroll
        for (int f = 0; f < FH; ++f) fx[p & 1][f] = lds[sx * (kUnitX / 16) + (at_x ^ (4 * ks)) + 128 * (h * FH + f)];
    };

    int t = share * xcd + min(xcd, more) + blockIdx.x / xcds, sw = 0, sx = 0;   // places of the present slice
    if (t >= end) return;
    aim(t);
    load_w(0, 0, false);
    load_x(0, 0, false);
    load_w(1, 1, false);
    load_x(1, 1, false);
    wait_vmcnt<LW + LX>();
    asm volatile("s_barrier" ::: "memory");
    read(0, 0, 0);
    bool stored = false;                                     // the outputs of a whole tile are on their way
    while (true) {
        const int cur_m = m0, cur_n = n0, next = t + step, whole = min(slices - 3, (k_left >> 7) - 2);
        // STEADY: slices of this tile follow, all within K
        auto slice = [&](int q, auto steady) {
            constexpr bool STEADY = decltype(steady)::value;
            const int nw = sw == SW - 1 ? 0 : sw + 1, nx = sx == SX - 1 ? 0 : sx + 1;   // of the next slice
            bool loads = true;                               // what is loaded two slices ahead
            int lq = q + 2;
            if (!STEADY && lq >= slices) {
                lq -= slices;
                loads = next < end;
                if (lq == 0 && loads) aim(next);
            }
#pragma unroll
            for (int p = 0; p < PH; ++p) {
                if (p < PH - 1) {
                    read(sw, sx, p + 1);
                    if (p == 0 && loads) {
                        if constexpr (SW == 3) load_w(lq, nw == 2 ? 0 : nw + 1, STEADY);
                        else load_x(lq, nx == 2 ? 0 : nx + 1, STEADY);
                    }
                } else if (STEADY || q + 1 < slices || next < end) {
                    if (!STEADY && !loads) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    else if (STEADY || !(stored && q == 0)) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kAhead) : "memory");
                    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kAhead + kStores) : "memory");
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                    if (loads) {
                        if constexpr (SW == 3) load_x(lq, sx, STEADY);
                        else load_w(lq, sw, STEADY);
                    }
                    if (STEADY || q + 1 < slices) read(nw, nx, 0);   // (of the next tile: behind the outputs)
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < FH; ++j) acc[i][(p % NH) * FH + j] = P::mfma(fw[p / NH][i], fx[p & 1][j], acc[i][(p % NH) * FH + j]);
                __builtin_amdgcn_sched_barrier(0);
            }
            sw = nw;
            sx = nx;
        };
        const int steady = stored ? 1 : 0;
#pragma unroll 1
        for (int q = 0; q < slices; ++q) {
            if (q == steady)
                for (; q < whole; ++q) slice(q, std::true_type());
            slice(q, std::false_type());
        }
        if constexpr (ACT == kPart) store_part(a, acc, ((int64_t)t * W + wave) * FM);
        else epilogue<P, ACT>(a, acc, cur_m + wm, cur_n + wn);
        if (next >= end) return;
        read(sw, sx, 0);
        t = next;
        stored = ACT == kPart || (cur_m + BM <= a.M && cur_n + BN <= a.N);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = typename P::Acc{};
    }
}

template <typename P, int ACT, int FM, int WN, int WM>
int launch_tiles(const LinearArgs &a, int per_cu, int group_n, hipStream_t stream) {
    constexpr int BN = 64 * WN, BM = 16 * FM * WM;
    constexpr int SW = slices_of_weights(BN, BM);
    constexpr size_t kLds = (SW * BN + (5 - SW) * BM) * 128;
    static std::atomic<uint64_t> done{0};
    const auto kernel = linear_tiles<P, ACT, FM, WN, WM>;
    allow_dynamic_lds(reinterpret_cast<const void *>(kernel), kLds, done);
    const int items = ((a.N + BN - 1) / BN) * ((a.M + BM - 1) / BM) * a.splits;
    kernel<<<dim3(min(items, 256 * per_cu)), 64 * WN * WM, kLds, stream>>>(a, group_n);
    return check_launch();
}

// The shapes of tiles: channels, tokens, workgroups per compute unit (LDS)
struct Shape { int fm, wn, wm, per_cu; };
constexpr Shape kShapes[] = {{8, 4, 2, 1}, {4, 4, 2, 1}, {4, 2, 2, 2}, {2, 2, 2, 2}, {2, 1, 2, 4}};
constexpr int kShapeAny = 2;   // linear_any's; for codes it has the smallest too

struct LinearPlan { int shape, splits, slices, group_n; size_t parts_bytes, pad_bytes; float time; };

// Estimated time of a shape of tile and a number of parts of K, in us.  A slice takes a workgroup 0.34 us and 0.23 us per 64 KB of it (1.85
// times that where rows do not begin at a multiple of 128 bytes) or, where its compute unit is busy, its share of the loads (275 GB/s for one
// compute unit alone, 74 where all of them load, 13 % less with such rows) and of the matrix cores (1.19 us for 256 x 256 x 64), and 0.1 us
// per 256 x 256 of outputs.  A round of tiles has 1.6 us and 0.4 us per 256 x 256 of outputs beside its slices, 6.2 where one workgroup has the
// compute unit for itself and nothing hides its outputs.  Parts of K are written and read back at 9.2 TB/s (they stay in the caches), by a
// launch of 3.2 us.  The constants are fitted to 818 timings of 67 outputs (32 to 118800 tokens, 64 to 11384 channels, K 64 to 13824) with every shape
// and 1 to 12 parts: the choice takes 2 % longer than the best of them in the mean, 13 % at most; always 128 x 128 without parts
// 35 % in the mean, 6.2 times at most.  8-bit codes, whose slices have as many bytes and matrix instructions: at 15 sizes 4 % longer than the best in the mean,
// 15 % at most (17 x 13824 x 5120, 600 x 4608 x 1536).
// Through registers: 16-bit products, 1.7 times that.  8-bit ones, a slice alone 0.3 us and 1.2 per 64 KB, or 1.4 times the share of the loads: of 18 sizes
// with rows that are no whole pieces (40 to 50000 tokens, 100 to 12000 channels, K 88 to 9001) the choice, copies among it, takes 1.3 % longer than
// the best in the mean, 6 % at most (256 x 128 and 128 x 64 tiles are faster by that where they are at all).  us, 128 x 128 tiles, 64 x 64, copied:
// 6242 x 1160 x 1156 20.5, 30.2, 26.4; 188 x 1720 x 1376 17.9, 13.8 (11.3 in parts), 14.1; 3000 x 1000 x 1500 16.9, 22.3, 19.0; 40 x 9001 x 1000 93, 62 (15.8 in parts), 20.1; 50000 x 777 x 100 20.9, 30.9, 30.9; 22268 x 4824 x 752 161, 215, 125;
// 10000 x 5000 x 5120 362, 544, 279.
// K: bytes of a row; codes: 8-bit ones
inline LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, bool any, bool codes) {
    const int total = (int)((K + 127) / 128);
    const bool lines = K % 128 == 0;
    LinearPlan best = {};
    best.time = 1e30f;
    for (int i = 0; i < (int)(sizeof(kShapes) / sizeof(kShapes[0])); ++i) {
        if (any && i != kShapeAny && !(codes && i == 4)) continue;
        const Shape &sh = kShapes[i];
        const int bn = 64 * sh.wn, bm = 16 * sh.fm * sh.wm, n_tiles = (int)((N + bn - 1) / bn), slots = 256 * sh.per_cu;
        const int64_t tiles = n_tiles * ((M + bm - 1) / bm);
        const float area = (float)(bn * bm) / 65536, bytes = (float)((bn + bm) * 128);
        for (const int want : {1, 2, 3, 4, 6, 8, 12}) {
            const int per = std::max(2, (total + want - 1) / want), splits = (total + per - 1) / per;
            if (want > 1 && (per < 4 || splits == 1 || tiles * splits > slots)) break;
            const int64_t items = tiles * splits, full = items / slots;
            const int rest = (int)(items - full * slots);
            const bool held = any && codes;                  // (on the way to LDS in registers)
            const float load = bytes * (lines ? 1.0f : 1.15f) * (held ? 1.4f : 1.0f) * (1 / 275e3f + (items < 256 ? (float)items / 256 : 1.0f) / 100e3f);
            const float lone = held ? 0.3f + 1.2f / 65536 * bytes : 0.34f + (lines ? 0.23f : 0.43f) / 65536 * bytes;
            auto round = [&](int resident) {
                return 1.6f + (0.4f * (float)resident + (sh.per_cu == 1 ? 5.7f : 0.0f)) * area +
                       (float)per * (std::max(lone, (float)resident * std::max(load, 1.19f * area)) + 0.1f * (float)resident * area);
            };
            float time = (float)full * round(sh.per_cu) + (rest ? round((rest + 255) / 256) : 0.0f);
            if (splits > 1) time += 3.2f + (float)items * area * (8 * 65536 / 9.2e6f);
            if (any && !codes) time *= 1.7f;
            if (time < best.time) {
                const int groups = (n_tiles + 5) / 6;   // columns of tiles that are run through before the next row
                best = {i, splits, per, any && !codes ? n_tiles : (n_tiles + groups - 1) / groups, splits > 1 ? (size_t)(items * bn * bm) * sizeof(float) : 0, 0, time};
            }
        }
    }
    // Rows that are no whole pieces: copied into ones that are, where that takes less than what linear_any loses (its registers on the way to
    // LDS cost it 1.4 to 1.9 times the time of 128 x 128 tiles: 32760 x 1533 x 8960 1388 us, copied 780).
    if (any && K % 16 != 0) {
        const int64_t pitch = (K + 127) / 128 * 128;
        LinearPlan p = linear_plan(M, N, pitch, false, codes);
        p.pad_bytes = (size_t)((M + N) * pitch);
        p.time += 3.0f + (float)p.pad_bytes * (2 / 5e6f);
        if (p.time < best.time) return p;
    }
    return best;
}
inline size_t plan_bytes(const LinearPlan &p) { return (p.pad_bytes + 255) / 256 * 256 + p.parts_bytes; }

template <typename P, int ACT, int FM, int WN, int WM>
int launch_any(const LinearArgs &a, int group_n, hipStream_t stream) {
    constexpr int BN = 64 * WN, BM = 16 * FM * WM;
    constexpr size_t kLds = 2 * (BN + BM) * 128;
    static std::atomic<uint64_t> done{0};
    const auto kernel = linear_any<P, ACT, FM, WN, WM>;
    allow_dynamic_lds(reinterpret_cast<const void *>(kernel), kLds, done);
    kernel<<<dim3((unsigned)(((a.N + BN - 1) / BN) * ((a.M + BM - 1) / BM) * a.splits)), 64 * WN * WM, kLds, stream>>>(a, group_n);
    return check_launch();
}

template <typename P, int ACT>
int launch_product(const LinearArgs &a, const LinearPlan &p, bool any, hipStream_t stream) {
    if (any) {
        if constexpr (P::kScaled) {
            if (p.shape == 4) return launch_any<P, ACT, 2, 1, 2>(a, p.group_n, stream);
        }
        return launch_any<P, ACT, 4, 2, 2>(a, p.group_n, stream);
    }
    switch (p.shape) {
        case 0: return launch_tiles<P, ACT, 8, 4, 2>(a, 1, p.group_n, stream);
        case 1: return launch_tiles<P, ACT, 4, 4, 2>(a, 1, p.group_n, stream);
        case 2: return launch_tiles<P, ACT, 4, 2, 2>(a, 2, p.group_n, stream);
        case 3: return launch_tiles<P, ACT, 2, 2, 2>(a, 2, p.group_n, stream);
        default: return launch_tiles<P, ACT, 2, 1, 2>(a, 4, p.group_n, stream);
    }
}

// addresses and pitches of an operand that tiles read straight into LDS
inline bool whole_pieces(const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld & 15) == 0 && ld < (int64_t)1 << 23; }

// see dvdq_bench_linear_choice
inline int choice_for(int64_t M, int64_t N, int64_t K, bool any, bool codes) {
    if (few_tokens(M, N, K, codes)) return -1;
    const LinearPlan p = linear_plan(M, N, K, any, codes);
    return p.shape + 16 * p.splits + (p.pad_bytes ? 4096 : any ? 8192 : 0);
}

inline size_t workspace_for(int64_t M, int64_t N, int64_t K, bool codes) {
    if (few_tokens(M, N, K, codes)) return 0;
    const size_t any = plan_bytes(linear_plan(M, N, K, true, codes));   // (addresses and pitches are not known here)
    return K % 16 == 0 ? std::max(any, plan_bytes(linear_plan(M, N, K, false, codes))) : any;
}

// The product of operands P; those of the output's type come into play in the last of the launches only.
template <typename P, typename Parts, int ACT>
int launch_few_or_tiles(LinearArgs a, void *workspace, hipStream_t stream) {
    if (few_tokens(a.M, a.N, a.K, P::kScaled)) {
        linear_few<P, ACT><<<dim3((unsigned)((a.N + 15) / 16)), 64 * kFewWaves, kFewWaves * 1024, stream>>>(a);
        return check_launch();
    }
    bool any = a.K % 16 != 0 || !whole_pieces(a.x, a.M > 1 ? a.ldx : 0) || !whole_pieces(a.w, a.N > 1 ? a.ldw : 0);
    const LinearPlan p = linear_plan(a.M, a.N, a.K, any, P::kScaled);
    a.parts = reinterpret_cast<float4 *>(static_cast<uint8_t *>(workspace) + (p.pad_bytes + 255) / 256 * 256);
    if (p.pad_bytes) {
        const int pitch = (a.K + 127) / 128 * 128;
        uint8_t *rows = static_cast<uint8_t *>(workspace);
        const int pieces = pitch / 16, at_once = std::max(1, std::min(16, 512 / pieces));
        const uint32_t mul = at_once == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + pieces - 1) / pieces);
        const int64_t groups = ((int64_t)a.M + a.N + at_once - 1) / at_once;
        linear_pad<Parts><<<dim3((unsigned)groups), 256, 0, stream>>>(a.x, a.ldx, a.M, a.w, a.ldw, a.N, a.K, pitch, at_once, mul, rows);
        const int rc = check_launch();
        if (rc != DVDQ_OK) return rc;
        a.x = rows, a.w = rows + (int64_t)a.M * pitch;
        a.ldx = a.ldw = a.K = pitch;
        any = false;
    }
    a.splits = p.splits;
    a.slices = p.slices;
    if (p.splits == 1) return launch_product<P, ACT>(a, p, any, stream);
    const int rc = launch_product<Parts, kPart>(a, p, any, stream);
    if (rc != DVDQ_OK) return rc;
    const Shape &sh = kShapes[p.shape];
    const int64_t waves = (((int64_t)a.N + 64 * sh.wn - 1) / (64 * sh.wn)) * (((int64_t)a.M + 16 * sh.fm * sh.wm - 1) / (16 * sh.fm * sh.wm)) * sh.fm * sh.wn * sh.wm;
    linear_join<P, ACT><<<dim3((unsigned)((waves + 3) / 4)), 256, 0, stream>>>(a, sh.fm, sh.wn, sh.wm, p.group_n);
    return check_launch();
}

}  // namespace

}  // namespace dvdq
