// Matrix product of 16-bit activations and weights with its epilogue:
//
//   y[m, n] = residual[m, n] + gate[m / (M / G), n] * act(sum_k x[m, k] w[n, k] + bias[n])
//
// Products on the matrix cores, sums and epilogue in fp32, one rounding to the tensors' type.
#include "elem.h"

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
    int act;
};

template <typename E, int ACT, int V>
static __device__ __forceinline__ void finish(const LinearArgs &a, float (&v)[V], int m, int n, int count) {
    if (a.bias) {
        const Piece<E> p = load_piece<E>(a.bias + n, count);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += E::to_f32(p.e[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = activate<ACT>(v[i]);
    if (a.gate) {
        const Piece<E> p = load_piece<E>(a.gate + (m / a.gate_rows) * a.ldg + n, count);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] *= E::to_f32(p.e[i]);
    }
    if (a.residual) {
        const Piece<E> p = load_piece<E>(a.residual + m * a.ldr + n, count);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += E::to_f32(p.e[i]);
    }
    Piece<E> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.e[i] = E::from_f32(v[i]);
    store_piece<E>(a.y + m * a.ldy + n, o, count);
}

// Bias, activation, gate, residual and store of 8 consecutive channels of a token.
template <typename E>
static __device__ __forceinline__ void epilogue(const LinearArgs &a, float (&v)[8], int m, int n) {
    const int count = min(8, a.N - n);
    if (m >= a.M || count <= 0) return;
    switch (a.act) {
        case DVDQ_ACT_SILU: finish<E, DVDQ_ACT_SILU>(a, v, m, n, count); break;
        case DVDQ_ACT_GELU_TANH: finish<E, DVDQ_ACT_GELU_TANH>(a, v, m, n, count); break;
        case DVDQ_ACT_GELU: finish<E, DVDQ_ACT_GELU>(a, v, m, n, count); break;
        default: finish<E, DVDQ_ACT_NONE>(a, v, m, n, count);
    }
}

// The weights are the matrix instruction's rows, the tokens its columns, so that a lane's four results are four channels of one
// token.  Row r of fragment f of 64 channels is channel 16 (r / 4) + 4 f + r % 4: over the four fragments a lane then holds 16
// consecutive channels of a token, and the four lanes of a token 64, which are stored without a detour.
static __device__ __forceinline__ int channel_of_row(int row) { return (row & ~63) + 16 * ((row & 15) >> 2) + 4 * ((row & 63) >> 4) + (row & 3); }

// Any sizes, pitches and addresses: 128 x 128 outputs of four waves, 64 x 64 each, operands through registers into LDS rows of 64
// elements of K.  The 16-byte pieces of an LDS row are permuted by its row number, so that the 16 rows that a read takes at once
// lie in different banks.
template <typename E>
__global__ __launch_bounds__(256) void linear_any(LinearArgs a) {
    constexpr int BK = 64;
    __shared__ uint4 lds_w[128 * 8], lds_x[128 * 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_tiles = (a.N + 127) / 128, tile_m = blockIdx.x / n_tiles;
    const int n0 = (blockIdx.x - tile_m * n_tiles) * 128, m0 = tile_m * 128;
    const int wn = (wave & 1) * 64, wm = (wave >> 1) * 64;
    v4f acc[4][4] = {};
    const int piece = tid & 7, row0 = tid >> 3;
    for (int k0 = 0; k0 < a.K; k0 += BK) {
        const int k = k0 + piece * 8, count = min(8, a.K - k);
        Piece<E> pw[4], px[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i;
            const int n = min(n0 + channel_of_row(row), a.N - 1), m = min(m0 + row, a.M - 1);
            pw[i] = load_piece<E>(a.w + n * a.ldw + k, count);
            px[i] = load_piece<E>(a.x + m * a.ldx + k, count);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i, at = row * 8 + (piece ^ ((row >> 1) & 7));
            lds_w[at] = __builtin_bit_cast(uint4, pw[i]);
            lds_x[at] = __builtin_bit_cast(uint4, px[i]);
        }
        __syncthreads();
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
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = acc[2 * h + i / 4][j][i & 3];
            epilogue<E>(a, v, m0 + wm + 16 * j + (lane & 15), n0 + wn + 16 * (lane >> 4) + 8 * h);
        }
}

}  // namespace

size_t linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    (void)M, (void)N, (void)K;
    return 0;
}

int launch_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *bias, int act, const void *gate, int64_t gate_rows,
                  int64_t ldg, const void *residual, int64_t ldr, int64_t M, int64_t N, int64_t K, int dtype, void *y, int64_t ldy,
                  void *workspace, hipStream_t stream) {
    (void)workspace;
    LinearArgs a = {};
    a.x = static_cast<const uint16_t *>(x), a.w = static_cast<const uint16_t *>(w), a.bias = static_cast<const uint16_t *>(bias);
    a.gate = static_cast<const uint16_t *>(gate), a.residual = static_cast<const uint16_t *>(residual), a.y = static_cast<uint16_t *>(y);
    a.ldx = ldx, a.ldw = ldw, a.ldr = ldr, a.ldy = ldy, a.ldg = ldg;
    a.M = (int)M, a.N = (int)N, a.K = (int)K;
    a.gate_rows = gate ? (int)(M / gate_rows) : 1;
    a.act = act;
    const dim3 grid((unsigned)(((N + 127) / 128) * ((M + 127) / 128)));
    if (dtype == DVDQ_BF16) linear_any<Bf16><<<grid, 256, 0, stream>>>(a);
    else linear_any<Fp16><<<grid, 256, 0, stream>>>(a);
    return check_launch();
}

}  // namespace dvdq
