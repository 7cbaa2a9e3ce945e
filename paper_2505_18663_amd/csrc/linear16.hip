// Matrix product of 16-bit activations and weights with its epilogue:
//
//   y[m, n] = residual[m, n] + gate[m / (M / G), n] * act(sum_k x[m, k] w[n, k] + bias[n])
//
// Products on the matrix cores, sums and epilogue in fp32, one rounding to the tensors' type.
//
// Ways: linear_few (few tokens), linear_tiles (five shapes of tile, K in parts where there are few tiles: linear_join), rows that are no whole
// 16-byte pieces copied first (linear_pad) or through registers (linear_any).  Against the library's product of the card's torch, which has no
// epilogue, weights out of the caches (a fast card and a slow one): 32760 x 13824 x 5120 with a residual 3260 to 3520 us and 2920 to 3120, 32760 x 1536 x 8960
// with tanh GELU 755 to 820 and 660 to 750, 512 x 4096 x 5120 35 to 37 and 36 to 38, 64 x 5120 x 5120 20 and 22, 1560 x 1536 x 1536 17 and 20, 2 x 1536 x 9216
// 9.1 and 20, 32760 x 1533 x 8960 740 to 780 and 890 to 910.
#include <algorithm>

#include "elem.h"
#include "gemm_common.h"

namespace dvdq {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

template <typename E>
static __device__ __forceinline__ v4f mfma(uint4 a, uint4 b, v4f c) {
    if constexpr (std::is_same<E, Bf16>::value)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

struct LinearArgs {
    const uint16_t *x, *w, *bias, *gate, *residual;
    uint16_t *y;
    int64_t ldx, ldw, ldr, ldy, ldg;   // elements between rows
    int M, N, K;
    int gate_rows;                     // tokens of one row of the gate
    float4 *parts;                     // sums of parts of K, in the order of the accumulators (kPart)
    int splits, slices;                // parts of K; slices of 64 of a part
    // Outputs past the caches, where they are larger than an XCD's L2 and the 64 bytes that the lanes of a token write are sectors of their own
    // (rows and address multiples of 64 bytes): 32760 x 1536 x 8960 with tanh GELU 823 -> 775 us, 32760 x 1536 x 4608 395 -> 364, 118800 x 1536 x 1536 513 -> 510.
    bool streaming;
};
constexpr int kPart = 4;               // in the place of an activation: leave the sums of a part of K for linear_join

// What follows the sums of a wave's 64 channels x 16 FM tokens, from channel n0 of token m0 on: the lane's token of fragment j is
// m0 + 16 j + lane % 16, its channels 8 (lane / 16) .. + 7 and the same 32 further on (channel_of_row).
template <typename E, int ACT, int FM>
static __device__ __forceinline__ void epilogue(const LinearArgs &a, const v4f (&acc)[4][FM], int m0, int n0) {
    constexpr int B = FM < 4 ? FM : 4;
    const int lane = threadIdx.x & 63, row = lane & 15, col = 8 * (lane >> 4);
    if (m0 >= a.M || n0 >= a.N) return;
    const bool shared_gate = a.gate && m0 / a.gate_rows == (min(m0 + 16 * FM, a.M) - 1) / a.gate_rows;   // one row for all tokens
    const uint32_t off_y = row * (uint32_t)a.ldy + col, off_r = row * (uint32_t)a.ldr + col;             // elements
    uint16_t *y = const_cast<uint16_t *>(uniform_ptr(a.y + (m0 * a.ldy + n0)));
    const uint16_t *res = a.residual ? uniform_ptr(a.residual + (m0 * a.ldr + n0)) : nullptr;
    auto values = [&](float (&v)[8], int h, int j, const Piece<E> &bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = activate<ACT>(acc[2 * h + i / 4][j][i & 3] + E::to_f32(bias.e[i]));
    };
    auto times = [](float (&v)[8], const Piece<E> &p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= E::to_f32(p.e[i]);
    };
    auto plus = [](float (&v)[8], const Piece<E> &p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += E::to_f32(p.e[i]);
    };
    auto rounded = [](const float (&v)[8]) {
        Piece<E> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.e[i] = E::from_f32(v[i]);
        return o;
    };
    if (m0 + 16 * FM <= a.M && n0 + 64 <= a.N) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = n0 + 32 * h + col;
            Piece<E> bias = {}, gate;
            if (a.bias) bias = load_piece<E>(a.bias + n, 8);
            if (shared_gate) gate = load_piece<E>(a.gate + (m0 / a.gate_rows) * a.ldg + n, 8);
            // the residual of B tokens is on its way while the B before are worked off (y may be the residual: the compiler could not
            // move a load above a store)
            Piece<E> r[2][B];
            auto fetch = [&](int j0) {
#pragma unroll
                for (int j = 0; j < B; ++j) r[(j0 / B) & 1][j] = load_piece<E>(res + 16 * (j0 + j) * a.ldr + 32 * h + off_r, 8);
            };
            if (res) fetch(0);
#pragma unroll
            for (int j0 = 0; j0 < FM; j0 += B) {
                if (j0 + B < FM && res) fetch(j0 + B);
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    float v[8];
                    values(v, h, j0 + j, bias);
                    if (a.gate) {
                        if (!shared_gate) gate = load_piece<E>(a.gate + ((m0 + 16 * (j0 + j) + row) / a.gate_rows) * a.ldg + n, 8);
                        times(v, gate);
                    }
                    if (res) plus(v, r[(j0 / B) & 1][j]);
                    uint16_t *to = y + 16 * (j0 + j) * a.ldy + 32 * h + off_y;
                    if (a.streaming) store_piece<E, 8, true>(to, rounded(v), 8);
                    else store_piece<E>(to, rounded(v), 8);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = n0 + 32 * h + col, count = min(8, a.N - n);
            Piece<E> bias = {};
            if (a.bias && count > 0) bias = load_piece<E>(a.bias + n, count);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const int m = m0 + 16 * j + row;
                if (m < a.M && count > 0) {
                    float v[8];
                    values(v, h, j, bias);
                    if (a.gate) times(v, load_piece<E>(a.gate + (m / a.gate_rows) * a.ldg + n, count));
                    if (res) plus(v, load_piece<E>(res + 16 * j * a.ldr + 32 * h + off_r, count));
                    store_piece<E>(y + 16 * j * a.ldy + 32 * h + off_y, rounded(v), count);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
}

// The weights are the matrix instruction's rows, the tokens its columns, so that a lane's four results are four channels of one
// token.  Row r of fragment f of 64 channels is channel 32 (f / 2) + 8 (r / 4) + 4 (f % 2) + r % 4: two fragments are then 8
// consecutive channels of a lane, 16 bytes, and the four lanes of a token store 64 bytes in a row, without a detour.
static __device__ __forceinline__ int channel_of_row(int row) {
    return (row & ~63) + 32 * ((row >> 5) & 1) + 8 * ((row & 15) >> 2) + 4 * ((row >> 4) & 1) + (row & 3);
}

// The sums of a wave, for linear_join: `at` numbers its fragments
template <int FM>
static __device__ __forceinline__ void store_part(const LinearArgs &a, const v4f (&acc)[4][FM], int64_t at) {
#pragma unroll
    for (int j = 0; j < FM; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) a.parts[((at + j) * 4 + i) * 64 + (threadIdx.x & 63)] = __builtin_bit_cast(float4, acc[i][j]);
}

// Any sizes, pitches and addresses: 128 x 128 outputs of four waves, 64 x 64 each, operands through registers into LDS rows of 64
// elements of K, a slice ahead.  LDS as in linear_tiles.
template <typename E, int ACT>
__global__ __launch_bounds__(256, 2) void linear_any(LinearArgs a) {
    extern __shared__ uint4 lds[];                           // two slices of 128 rows of weights, 128 of tokens
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_tiles = (a.N + 127) / 128, m_tiles = (a.M + 127) / 128, tiles = n_tiles * m_tiles;
    const int split = blockIdx.x / tiles, tile = blockIdx.x - split * tiles;
    const int tile_m = tile / n_tiles;
    const int n0 = (tile - tile_m * n_tiles) * 128, m0 = tile_m * 128;
    const int wn = (wave & 1) * 64, wm = (wave >> 1) * 64;
    const int q0 = split * a.slices, q1 = min(q0 + a.slices, (a.K + 63) >> 6);
    v4f acc[4][4] = {};
    const int piece = tid & 7, row0 = tid >> 3;
    Piece<E> pw[4], px[4];
    auto load = [&](int q) {
        const int k = q * 64 + piece * 8, count = min(8, a.K - k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i;
            pw[i] = load_piece<E>(a.w + min(n0 + channel_of_row(row), a.N - 1) * a.ldw + k, count);
            px[i] = load_piece<E>(a.x + min(m0 + row, a.M - 1) * a.ldx + k, count);
        }
    };
    if (q0 < q1) load(q0);
    for (int q = q0; q < q1; ++q) {
        uint4 *lds_w = lds + (q & 1) * 2048, *lds_x = lds_w + 1024;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i, at = row * 8 + (piece ^ ((row >> 1) & 7));
            lds_w[at] = __builtin_bit_cast(uint4, pw[i]);
            lds_x[at] = __builtin_bit_cast(uint4, px[i]);
        }
        __syncthreads();                                     // (and every wave has read the slice before the last)
        if (q + 1 < q1) load(q + 1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uint4 fw[4], fx[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int rw = wn + 16 * f + (lane & 15), rx = wm + 16 * f + (lane & 15), p = 4 * ks + (lane >> 4);
                fw[f] = lds_w[rw * 8 + (p ^ ((rw >> 1) & 7))];
                fx[f] = lds_x[rx * 8 + (p ^ ((rx >> 1) & 7))];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma<E>(fw[i], fx[j], acc[i][j]);
        }
    }
    if constexpr (ACT == kPart) store_part(a, acc, ((int64_t)blockIdx.x * 4 + wave) * 4);
    else epilogue<E, ACT>(a, acc, __builtin_amdgcn_readfirstlane(m0 + wm), __builtin_amdgcn_readfirstlane(n0 + wn));
}

// ---- few tokens (at most 16): bound by the weights, which are read once, straight into registers
// A workgroup has 16 channels, its waves parts of K: a lane reads 32 bytes of a channel (the four lanes of a channel a whole line) and the same part of its
// token, two matrix instructions' worth, twice over before the first product; the waves' sums meet in LDS in their order.
// (The instruction's order of K does not matter as long as it is the same on both sides.)
// 2 x 1536 x 9216, 28 MB of weights: 9.1 us with 8 waves (8.3 where the caches hold the weights), 9.5 with 16, 9.6 with 4; as tiles 14.1.
// 1 x 1536 x 4608 6.5 and 11.9, 16 x 1536 x 13824 15.0 and 18.2, 2 x 5120 x 30720 57 and 67.  Few channels leave compute units idle and long rows their
// waves with too little in flight: 8 x 13824 x 128 22 and 15, 16 x 5120 x 5120 23 and 19, 2 x 13824 x 5120 36 and 36; these are tiles.
constexpr int kFewWaves = 8;
inline bool few_tokens(int64_t M, int64_t N, int64_t K) { return M <= 16 && (K <= 4096 || N >= 16384); }
template <typename E, int ACT>
__global__ __launch_bounds__(512) void linear_few(LinearArgs a) {
    extern __shared__ uint4 lds[];
    float *sums = reinterpret_cast<float *>(lds);            // [wave][token][channel]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, n0 = blockIdx.x * 16;
    const uint16_t *w = a.w + min(n0 + (lane & 15), a.N - 1) * a.ldw, *x = a.x + min(lane & 15, a.M - 1) * a.ldx;
    const int steps = (a.K + 63) >> 6, q0 = (int)((int64_t)steps * wave / waves), q1 = (int)((int64_t)steps * (wave + 1) / waves);
    constexpr int AHEAD = 2;
    v4f acc[2] = {};
    const auto multiply = [&](const Piece<E> &pw, const Piece<E> &px, int h) {
        acc[h] = mfma<E>(__builtin_bit_cast(uint4, pw), __builtin_bit_cast(uint4, px), acc[h]);
    };
    const int whole = min(q1, a.K >> 6);                     // steps of 64 elements that there are
    w += (lane >> 4) * 16, x += (lane >> 4) * 16;
    int q = q0;
    for (; q + AHEAD <= whole; q += AHEAD) {
        Piece<E> pw[AHEAD][2], px[AHEAD][2];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pw[i][h] = load_piece<E>(w + (q + i) * 64 + 8 * h, 8);
                px[i][h] = load_piece<E>(x + (q + i) * 64 + 8 * h, 8);
            }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) multiply(pw[i][h], px[i][h], h);
    }
    if (q < whole) {                                         // fewer than AHEAD: the rest once more, as nothing
        Piece<E> pw[AHEAD - 1][2], px[AHEAD - 1][2];
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pw[i][h] = load_piece<E>(w + min(q + i, whole - 1) * 64 + 8 * h, 8);
                px[i][h] = load_piece<E>(x + min(q + i, whole - 1) * 64 + 8 * h, 8);
            }
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i)
            if (q + i < whole) {
#pragma unroll
                for (int h = 0; h < 2; ++h) multiply(pw[i][h], px[i][h], h);
            }
    }
    if (whole < q1) {                                        // the last step, of fewer than 64 elements
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = whole * 64 + 8 * h, left = a.K - k - (lane >> 4) * 16;
            Piece<E> pw = {}, px = {};
            if (left > 0) {
                pw = load_piece<E>(w + k, left);
                px = load_piece<E>(x + k, left);
            }
            multiply(pw, px, h);
        }
    }
    const v4f sum = acc[0] + acc[1];
    reinterpret_cast<v4f *>(sums)[(wave * 16 + (lane & 15)) * 4 + (lane >> 4)] = sum;
    __syncthreads();
    const int m = threadIdx.x >> 4, n = n0 + (threadIdx.x & 15);
    if (threadIdx.x >= 256 || m >= a.M || n >= a.N) return;
    float v = 0.0f;
    for (int i = 0; i < waves; ++i) v += sums[i * 256 + threadIdx.x];
    if (a.bias) v += E::to_f32(a.bias[n]);
    v = activate<ACT>(v);
    if (a.gate) v *= E::to_f32(a.gate[(m / a.gate_rows) * a.ldg + n]);
    if (a.residual) v += E::to_f32(a.residual[m * a.ldr + n]);
    a.y[m * a.ldy + n] = E::from_f32(v);
}

// Rows of K elements at any address -> rows of `pitch` elements, a multiple of 64, zero past K: activations (rows_x of them), then weights.
template <typename E>
__global__ __launch_bounds__(256) void linear_pad(const uint16_t *x, int64_t ldx, int rows_x, const uint16_t *w, int64_t ldw, int rows_w, int K,
                                                  int pitch, uint16_t *out) {
    const uint32_t pieces = (uint32_t)pitch / 8;
    const int64_t total = (int64_t)(rows_x + rows_w) * pieces;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < total; i += gridDim.x * (int64_t)256) {
        const int64_t row = i / pieces;
        const int k = (int)(i - row * pieces) * 8;
        const uint16_t *src = row < rows_x ? x + row * ldx : w + (row - rows_x) * ldw;
        Piece<E> p = {};
        if (k < K) p = load_piece<E>(src + k, min(8, K - k));
        reinterpret_cast<uint4 *>(out)[i] = __builtin_bit_cast(uint4, p);
    }
}

// Joins the parts of K, in their order, and finishes: a wave per 64 channels x 16 tokens of tiles of WN x WM waves of 64 channels x 16 FM tokens.
template <typename E, int ACT>
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
    v4f acc[4][1] = {};
    const float4 *p = a.parts + g * 256 + lane;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s, p += stride)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][0] += __builtin_bit_cast(v4f, p[i * 64]);
    epilogue<E, ACT>(a, acc, m0, n0);
}

// ---- rows of whole 16-byte pieces: operands straight into LDS

// 16 bytes per lane from each lane's own address to LDS address lds_base + 16 * lane (completion awaited by hand, as with
// lds_direct_load16)
static __device__ __forceinline__ void lds_direct_load16_at(const void *p, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds_base) : "memory");
}

__device__ uint4 zero_piece;   // what the pieces past K of the last slice are read from

// Tiles of 64 WN channels x 16 FM WM tokens, WN x WM waves of 64 channels x 16 FM tokens each; slices of 64 elements of K.
// Weights have three slices in LDS, tokens two: while a slice is multiplied, the next is there, the weights of the one after it
// come in, and its tokens follow as soon as those of the present slice have been read.  (What bounds the loop on a full chip is the way from
// the L2s into LDS, 54 to 69 GB/s per compute unit where 32 of them share panels; it must not run dry.)
// A slice is worked off in phases of 16 matrix instructions (or fewer), and a phase begins by requesting the fragments of the next one.
// Before the last phase of a slice, whose fragments are then in registers, stands the slice's one barrier: behind it the next slice is
// in LDS for every wave, and this one's place is free.
// A workgroup takes tile after tile, without a seam: the last slices of a tile load the first ones of the next, which is multiplied
// while the outputs are still being written.
template <typename E, int ACT, int FM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM, 2) void linear_tiles(LinearArgs a, int group_n) {
    constexpr int W = WN * WM, BN = 64 * WN, BM = 16 * FM * WM, FH = FM < 4 ? FM : 4, NH = FM / FH, P = 2 * NH;
    constexpr int LW = BN / 8 / W, LX = BM / 8 / W;          // loads of a wave per slice, 8 rows each
    constexpr int kStores = ACT == kPart ? 4 * FM : 2 * FM;  // of a wave per whole tile
    constexpr uint32_t kUnitW = BN * 128, kUnitX = BM * 128;
    extern __shared__ uint4 lds[];                           // weights: 3 units, tokens: 2
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
    const uint32_t lds_w = lds_address(lds) + wave * (1024 * LW), lds_x = lds_address(lds) + 3 * kUnitW + wave * (1024 * LX);
    const uint8_t *src_w, *src_x;
    uint32_t off_w[LW], off_x[LX];
    const bool spread_w = a.N * a.ldw < (int64_t)1 << 31, spread_x = a.M * a.ldx < (int64_t)1 << 31;   // offsets of 32 bits
    int m0, n0, k_left;
    auto aim = [&](int t) {                                  // the loads' source: part t / tiles of K of tile t % tiles
        const int part = ACT == kPart ? t / tiles : 0, k0 = part * slices * 64;
        tile_origin(t - part * tiles, m_tiles, n_tiles, group_n, BM, BN, m0, n0);
        k_left = a.K - k0;
        // Rows past the matrix are read from other rows of it (their products are dropped), spread over it: the last row for all of them
        // is one line that every workgroup of a column of tiles asks for at once (24017 x 3608 x 176, 256-channel tiles, 118 us).
        const int base_n = spread_w && n0 + BN > a.N ? 0 : n0, base_m = spread_x && m0 + BM > a.M ? 0 : m0;
        src_w = reinterpret_cast<const uint8_t *>(uniform_ptr(a.w + (base_n * a.ldw + k0)));
        src_x = reinterpret_cast<const uint8_t *>(uniform_ptr(a.x + (base_m * a.ldx + k0)));
        auto inside = [](int row, int first, int rows, int base) {
            row += first;
            return (row < rows ? row : base + (row - base) % (rows - base)) - base;
        };
#pragma unroll
        for (int j = 0; j < LW; ++j) {
            const int row = wave * (8 * LW) + 8 * j + (lane >> 3);
            off_w[j] = (uint32_t)(inside(channel_of_row(row), n0, a.N, base_n) * a.ldw * 2) + 16 * ((lane & 7) ^ ((row >> 1) & 7));
        }
#pragma unroll
        for (int j = 0; j < LX; ++j) {
            const int row = wave * (8 * LX) + 8 * j + (lane >> 3);
            off_x[j] = (uint32_t)(inside(row, m0, a.M, base_m) * a.ldx * 2) + 16 * ((lane & 7) ^ ((row >> 1) & 7));
        }
    };
    // slice q of the aimed tile; `whole`: known to lie within K
    auto load_w = [&](int q, int slot, bool whole) {
        const uint8_t *src = src_w + (uint32_t)q * 128u;
        if (whole || (q + 1) * 64 <= k_left) {
#pragma unroll
            for (int j = 0; j < LW; ++j) lds_direct_load16(src, off_w[j], lds_w + slot * kUnitW + 1024 * j);
        } else {
#pragma unroll
            for (int j = 0; j < LW; ++j) {
                const int piece = 16 * ((lane & 7) ^ (((wave * (8 * LW) + 8 * j + (lane >> 3)) >> 1) & 7));
                lds_direct_load16_at(piece < (k_left - q * 64) * 2 ? static_cast<const void *>(src + off_w[j]) : &zero_piece, lds_w + slot * kUnitW + 1024 * j);
            }
        }
    };
    auto load_x = [&](int q, int slot, bool whole) {
        const uint8_t *src = src_x + (uint32_t)q * 128u;
        if (whole || (q + 1) * 64 <= k_left) {
#pragma unroll
            for (int j = 0; j < LX; ++j) lds_direct_load16(src, off_x[j], lds_x + slot * kUnitX + 1024 * j);
        } else {
#pragma unroll
            for (int j = 0; j < LX; ++j) {
                const int piece = 16 * ((lane & 7) ^ (((wave * (8 * LX) + 8 * j + (lane >> 3)) >> 1) & 7));
                lds_direct_load16_at(piece < (k_left - q * 64) * 2 ? static_cast<const void *>(src + off_x[j]) : &zero_piece, lds_x + slot * kUnitX + 1024 * j);
            }
        }
    };

    // fragment reads: LDS row r of 128 bytes holds its 16-byte piece c at c ^ ((r >> 1) & 7), so that the 16 rows that a read takes at
    // once lie in different banks
    const int at = (lane & 15) * 8 + ((lane >> 4) ^ ((lane & 15) >> 1));   // of k-step 0; k-step 1 is piece ^ 4
    const int at_w = wn * 8 + at, at_x = 3 * (kUnitW / 16) + wm * 8 + at;
    v4f acc[4][FM] = {};
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
        const int cur_m = m0, cur_n = n0, next = t + step, whole = min(slices - 3, (k_left >> 6) - 2);
        // STEADY: slices of this tile follow, all within K
        auto slice = [&](int q, auto steady) {
            constexpr bool STEADY = decltype(steady)::value;
            const int nw = sw == 2 ? 0 : sw + 1, aw = nw == 2 ? 0 : nw + 1;
            bool loads = true;                               // what is loaded two slices ahead
            int lq = q + 2;
            if (!STEADY && lq >= slices) {
                lq -= slices;
                loads = next < end;
                if (lq == 0 && loads) aim(next);
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (p < P - 1) {
                    read(sw, sx, p + 1);
                    if (p == 0 && loads) load_w(lq, aw, STEADY);
                } else if (STEADY || q + 1 < slices || next < end) {
                    if (!STEADY && !loads) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    else if (STEADY || !(stored && q == 0)) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LW) : "memory");
                    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LW + kStores) : "memory");
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                    if (loads) load_x(lq, sx, STEADY);
                    if (STEADY || q + 1 < slices) read(nw, sx ^ 1, 0);   // (of the next tile: behind the outputs)
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < FH; ++j) acc[i][(p % NH) * FH + j] = mfma<E>(fw[p / NH][i], fx[p & 1][j], acc[i][(p % NH) * FH + j]);
                __builtin_amdgcn_sched_barrier(0);
            }
            sw = nw;
            sx ^= 1;
        };
        const int steady = stored ? 1 : 0;
#pragma unroll 1
        for (int q = 0; q < slices; ++q) {
            if (q == steady)
                for (; q < whole; ++q) slice(q, std::true_type());
            slice(q, std::false_type());
        }
        if constexpr (ACT == kPart) store_part(a, acc, ((int64_t)t * W + wave) * FM);
        else epilogue<E, ACT>(a, acc, cur_m + wm, cur_n + wn);
        if (next >= end) return;
        read(sw, sx, 0);
        t = next;
        stored = ACT == kPart || (cur_m + BM <= a.M && cur_n + BN <= a.N);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = v4f{};
    }
}

template <typename E, int ACT, int FM, int WN, int WM>
int launch_tiles(const LinearArgs &a, int per_cu, int group_n, hipStream_t stream) {
    constexpr int BN = 64 * WN, BM = 16 * FM * WM;
    constexpr size_t kLds = (3 * BN + 2 * BM) * 128;
    static std::atomic<uint64_t> done{0};
    const auto kernel = linear_tiles<E, ACT, FM, WN, WM>;
    allow_dynamic_lds(reinterpret_cast<const void *>(kernel), kLds, done);
    const int items = ((a.N + BN - 1) / BN) * ((a.M + BM - 1) / BM) * a.splits;
    kernel<<<dim3(min(items, 256 * per_cu)), 64 * WN * WM, kLds, stream>>>(a, group_n);
    return check_launch();
}

// The shapes of tiles: channels, tokens, workgroups per compute unit (LDS)
struct Shape { int fm, wn, wm, per_cu; };
constexpr Shape kShapes[] = {{8, 4, 2, 1}, {4, 4, 2, 1}, {4, 2, 2, 2}, {2, 2, 2, 2}, {2, 1, 2, 4}};
constexpr int kShapeAny = 2;   // linear_any's

struct LinearPlan { int shape, splits, slices, group_n; size_t parts_bytes, pad_bytes; float time; };

// Estimated time of a shape of tile and a number of parts of K, in us.  A slice takes a workgroup 0.34 us and 0.23 us per 64 KB of it (1.85
// times that where rows do not begin at a multiple of 128 bytes) or, where its compute unit is busy, its share of the loads (275 GB/s for one
// compute unit alone, 74 where all of them load, 13 % less with such rows) and of the matrix cores (1.19 us for 256 x 256 x 64), and 0.1 us
// per 256 x 256 of outputs.  A round of tiles has 1.6 us and 0.4 us per 256 x 256 of outputs beside its slices, 6.2 where one workgroup has the
// compute unit for itself and nothing hides its outputs.  Parts of K are written and read back at 9.2 TB/s (they stay in the caches), by a
// launch of 3.2 us.  The constants are fitted to 818 timings of 67 outputs (32 to 118800 tokens, 64 to 11384 channels, K 64 to 13824) with every shape
// and 1 to 12 parts: the choice takes 2 % longer than the best of them in the mean, 13 % at most; always 128 x 128 without parts
// 35 % in the mean, 6.2 times at most.
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, bool any) {
    const int total = (int)((K + 63) / 64);
    const bool lines = K % 64 == 0;
    LinearPlan best = {};
    best.time = 1e30f;
    for (int i = 0; i < (int)(sizeof(kShapes) / sizeof(kShapes[0])); ++i) {
        if (any && i != kShapeAny) continue;
        const Shape &sh = kShapes[i];
        const int bn = 64 * sh.wn, bm = 16 * sh.fm * sh.wm, n_tiles = (int)((N + bn - 1) / bn), slots = 256 * sh.per_cu;
        const int64_t tiles = n_tiles * ((M + bm - 1) / bm);
        const float area = (float)(bn * bm) / 65536, bytes = (float)((bn + bm) * 128);
        for (const int want : {1, 2, 3, 4, 6, 8, 12}) {
            const int per = std::max(2, (total + want - 1) / want), splits = (total + per - 1) / per;
            if (want > 1 && (per < 4 || splits == 1 || tiles * splits > slots)) break;
            const int64_t items = tiles * splits, full = items / slots;
            const int rest = (int)(items - full * slots);
            const float load = bytes * (lines ? 1.0f : 1.15f) * (1 / 275e3f + (items < 256 ? (float)items / 256 : 1.0f) / 100e3f);
            const float lone = 0.34f + (lines ? 0.23f : 0.43f) / 65536 * bytes;
            auto round = [&](int resident) {
                return 1.6f + (0.4f * (float)resident + (sh.per_cu == 1 ? 5.7f : 0.0f)) * area +
                       (float)per * (std::max(lone, (float)resident * std::max(load, 1.19f * area)) + 0.1f * (float)resident * area);
            };
            float time = (float)full * round(sh.per_cu) + (rest ? round((rest + 255) / 256) : 0.0f);
            if (splits > 1) time += 3.2f + (float)items * area * (8 * 65536 / 9.2e6f);
            if (any) time *= 1.7f;
            if (time < best.time) {
                const int groups = (n_tiles + 5) / 6;   // columns of tiles that are run through before the next row
                best = {i, splits, per, any ? n_tiles : (n_tiles + groups - 1) / groups, splits > 1 ? (size_t)(items * bn * bm) * sizeof(float) : 0, 0, time};
            }
        }
    }
    // Rows that are no whole pieces: copied into ones that are, where that takes less than what linear_any loses (its registers on the way to
    // LDS cost it 1.4 to 1.9 times the time of 128 x 128 tiles: 32760 x 1533 x 8960 1388 us, copied 780).
    if (any && K % 8 != 0) {
        const int64_t pitch = (K + 63) / 64 * 64;
        LinearPlan p = linear_plan(M, N, pitch, false);
        p.pad_bytes = (size_t)((M + N) * pitch) * 2;
        p.time += 3.0f + (float)p.pad_bytes * (2 / 5e6f);
        if (p.time < best.time) return p;
    }
    return best;
}
inline size_t plan_bytes(const LinearPlan &p) { return (p.pad_bytes + 255) / 256 * 256 + p.parts_bytes; }

template <typename E, int ACT>
int launch_product(const LinearArgs &a, const LinearPlan &p, bool any, hipStream_t stream) {
    if (any) {
        static std::atomic<uint64_t> done{0};
        constexpr size_t kLds = 2 * 256 * 128;
        allow_dynamic_lds(reinterpret_cast<const void *>(linear_any<E, ACT>), kLds, done);
        linear_any<E, ACT><<<dim3((unsigned)(((a.N + 127) / 128) * ((a.M + 127) / 128) * a.splits)), 256, kLds, stream>>>(a);
        return check_launch();
    }
    switch (p.shape) {
        case 0: return launch_tiles<E, ACT, 8, 4, 2>(a, 1, p.group_n, stream);
        case 1: return launch_tiles<E, ACT, 4, 4, 2>(a, 1, p.group_n, stream);
        case 2: return launch_tiles<E, ACT, 4, 2, 2>(a, 2, p.group_n, stream);
        case 3: return launch_tiles<E, ACT, 2, 2, 2>(a, 2, p.group_n, stream);
        default: return launch_tiles<E, ACT, 2, 1, 2>(a, 4, p.group_n, stream);
    }
}

}  // namespace

size_t linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (few_tokens(M, N, K)) return 0;
    const size_t any = plan_bytes(linear_plan(M, N, K, true));   // (addresses and pitches are not known here)
    return K % 8 == 0 ? std::max(any, plan_bytes(linear_plan(M, N, K, false))) : any;
}

int linear_choice(int64_t M, int64_t N, int64_t K, bool any) {
    if (few_tokens(M, N, K)) return -1;
    const LinearPlan p = linear_plan(M, N, K, any);
    return p.shape + 16 * p.splits + (p.pad_bytes ? 4096 : any ? 8192 : 0);
}

int launch_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *bias, int act, const void *gate, int64_t gate_rows,
                  int64_t ldg, const void *residual, int64_t ldr, int64_t M, int64_t N, int64_t K, int dtype, void *y, int64_t ldy,
                  void *workspace, hipStream_t stream) {
    LinearArgs a = {};
    a.x = static_cast<const uint16_t *>(x), a.w = static_cast<const uint16_t *>(w), a.bias = static_cast<const uint16_t *>(bias);
    a.gate = static_cast<const uint16_t *>(gate), a.residual = static_cast<const uint16_t *>(residual), a.y = static_cast<uint16_t *>(y);
    a.ldx = ldx, a.ldw = ldw, a.ldr = ldr, a.ldy = ldy, a.ldg = ldg;
    a.M = (int)M, a.N = (int)N, a.K = (int)K;
    a.gate_rows = gate ? (int)(M / gate_rows) : 1;
    a.streaming = M * N >= (2 << 20) && ldy % 32 == 0 && (reinterpret_cast<uintptr_t>(y) & 63) == 0;
    const auto whole = [](const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld & 7) == 0 && ld < (int64_t)1 << 22; };
    if (few_tokens(M, N, K))
        return with_type(dtype, [&](auto type) {
            using E = decltype(type);
            if constexpr (sizeof(typename E::Raw) == 2) {
                return with_act(act, [&](auto which) {
                    constexpr int ACT = decltype(which)::value;
                    linear_few<E, ACT><<<dim3((unsigned)((N + 15) / 16)), 64 * kFewWaves, kFewWaves * 1024, stream>>>(a);
                    return check_launch();
                });
            } else {
                return (int)DVDQ_ERR_UNSUPPORTED;
            }
        });
    bool any = K % 8 != 0 || !whole(x, M > 1 ? ldx : 0) || !whole(w, N > 1 ? ldw : 0);
    const LinearPlan p = linear_plan(M, N, K, any);
    a.parts = reinterpret_cast<float4 *>(static_cast<uint8_t *>(workspace) + (p.pad_bytes + 255) / 256 * 256);
    if (p.pad_bytes) {
        const int pitch = (int)((K + 63) / 64 * 64);
        uint16_t *rows = static_cast<uint16_t *>(workspace);
        const int64_t blocks = std::min((int64_t)256 * 32, ((M + N) * (pitch / 8) + 255) / 256);
        linear_pad<Bf16><<<dim3((unsigned)blocks), 256, 0, stream>>>(a.x, ldx, a.M, a.w, ldw, a.N, a.K, pitch, rows);   // (bits: any 16-bit type)
        const int rc = check_launch();
        if (rc != DVDQ_OK) return rc;
        a.x = rows, a.w = rows + M * pitch;
        a.ldx = a.ldw = a.K = pitch;
        any = false;
    }
    a.splits = p.splits;
    a.slices = p.slices;
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        if constexpr (sizeof(typename E::Raw) == 2) {
            return with_act(act, [&](auto which) {
                constexpr int ACT = decltype(which)::value;
                if (p.splits == 1) return launch_product<E, ACT>(a, p, any, stream);
                const int rc = launch_product<E, kPart>(a, p, any, stream);
                if (rc != DVDQ_OK) return rc;
                const Shape &sh = kShapes[p.shape];
                const int64_t waves = ((N + 64 * sh.wn - 1) / (64 * sh.wn)) * ((M + 16 * sh.fm * sh.wm - 1) / (16 * sh.fm * sh.wm)) * sh.fm * sh.wn * sh.wm;
                linear_join<E, ACT><<<dim3((unsigned)((waves + 3) / 4)), 256, 0, stream>>>(a, sh.fm, sh.wn, sh.wm, p.group_n);
                return check_launch();
            });
        } else {
            return (int)DVDQ_ERR_UNSUPPORTED;
        }
    });
}

}  // namespace dvdq
