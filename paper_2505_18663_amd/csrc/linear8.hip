// Matrix product of 8-bit codes and 8-bit weights with its epilogue:
//
//   y[m, n] = residual[m, n] + gate[m / (M / G), n] * act(x_scale[m] w_scale[n] sum_k codes[m, k] w[n, k] + bias[n])
//
// Products on the INT8 matrix cores, summed exactly in int32; scales and epilogue in fp32, one rounding to the tensors' type.
#include <algorithm>

#include "elem.h"
#include "gemm_common.h"

namespace dvdq {

namespace {

struct Linear8Args {
    const int8_t *x, *w;
    const float *x_scale, *w_scale;
    const void *bias, *gate, *residual;
    void *y;
    int64_t ldx, ldw, ldr, ldy, ldg;   // elements between rows
    int M, N, K;
    int gate_rows;                     // tokens of one row of the gate
};

struct I8 {
    using Raw = int8_t;
};

// 16 channels x 16 tokens a workgroup, its waves parts of K: a lane reads 16 bytes of a channel and of a token, the waves' sums meet in LDS.
template <typename E, int ACT>
__global__ __launch_bounds__(256) void linear8_few(Linear8Args a) {
    using Raw = typename E::Raw;
    __shared__ v4i sums[4 * 64];                             // [wave][token][channels / 4]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, columns = (a.N + 15) / 16;
    const int64_t tiles = (int64_t)columns * ((a.M + 15) / 16);
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int n0 = (int)(tile % columns) * 16, m0 = (int)(tile / columns) * 16;
        const int8_t *w = a.w + min(n0 + (lane & 15), a.N - 1) * a.ldw, *x = a.x + min(m0 + (lane & 15), a.M - 1) * a.ldx;
        const int steps = (a.K + 63) >> 6, q0 = steps * wave / 4, q1 = steps * (wave + 1) / 4;
        v4i acc = {};
        for (int q = q0; q < q1; ++q) {
            const int k = q * 64 + (lane >> 4) * 16, left = a.K - k;
            Piece<I8, 16> pw = {}, px = {};
            if (left > 0) pw = load_piece<I8, 16>(w + k, left), px = load_piece<I8, 16>(x + k, left);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, pw), __builtin_bit_cast(v4i, px), acc, 0, 0, 0);
        }
        __syncthreads();                                     // (the sums of the tile before have been read)
        sums[(wave * 16 + (lane & 15)) * 4 + (lane >> 4)] = acc;
        __syncthreads();
        const int m = m0 + (threadIdx.x >> 4), n = n0 + (threadIdx.x & 15);
        if (m >= a.M || n >= a.N) continue;
        int sum = 0;
        for (int i = 0; i < 4; ++i) sum += reinterpret_cast<const int *>(sums)[i * 256 + threadIdx.x];
        float v = (float)sum * a.x_scale[m] * a.w_scale[n];
        if (a.bias) v += E::to_f32(static_cast<const Raw *>(a.bias)[n]);
        v = activate<ACT>(v);
        if (a.gate) v *= E::to_f32(static_cast<const Raw *>(a.gate)[(m / a.gate_rows) * a.ldg + n]);
        if (a.residual) v += E::to_f32(static_cast<const Raw *>(a.residual)[m * a.ldr + n]);
        static_cast<Raw *>(a.y)[m * a.ldy + n] = E::from_f32(v);
    }
}

}  // namespace

size_t linear8_workspace_bytes(int64_t M, int64_t N, int64_t K) { return 0; }

int launch_linear8(const int8_t *codes, int64_t ldc, const float *x_scale, const int8_t *w, int64_t ldw, const float *w_scale, const void *bias, int act,
                   const void *gate, int64_t gate_rows, int64_t ldg, const void *residual, int64_t ldr, int64_t M, int64_t N, int64_t K, int dtype,
                   void *y, int64_t ldy, void *workspace, hipStream_t stream) {
    Linear8Args a = {};
    a.x = codes, a.w = w, a.x_scale = x_scale, a.w_scale = w_scale, a.bias = bias, a.gate = gate, a.residual = residual, a.y = y;
    a.ldx = ldc, a.ldw = ldw, a.ldr = ldr, a.ldy = ldy, a.ldg = ldg;
    a.M = (int)M, a.N = (int)N, a.K = (int)K;
    a.gate_rows = gate ? (int)(M / gate_rows) : 1;
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        return with_act(act, [&](auto which) {
            constexpr int ACT = decltype(which)::value;
            linear8_few<E, ACT><<<dim3((unsigned)std::min<int64_t>(((N + 15) / 16) * ((M + 15) / 16), 1 << 20)), 256, 0, stream>>>(a);
            return check_launch();
        });
    });
}

}  // namespace dvdq
