// Matrix product of 8-bit codes and 8-bit weights with its epilogue:
//
//   y[m, n] = residual[m, n] + gate[m / (M / G), n] * act(x_scale[m] w_scale[n] sum_k codes[m, k] w[n, k] + bias[n])
//
// Products on the INT8 matrix cores, summed exactly in int32; scales and epilogue in fp32, one rounding to the tensors' type.  The kernels
// are those of linear_tiles.h: 128 bytes of a row are a slice, whatever the type, and a matrix instruction takes as long for them.
//
// us, with what the library's int8 product takes (int32 outputs, no scales, no epilogue): 32760 x 13824 x 5120 with gate and residual 1670 to 1735 and 1750 to 1870,
// 32760 x 1536 x 8960 with tanh GELU 464 to 470 and 512 to 520, 8192^3 409 and 441, 512 x 4096 x 5120 with tanh GELU 21 and 20 to 23, 1560 x 1536 x 1536 11 and 19,
// 6242 x 1168 x 1160 19 and 35, 64 x 5120 x 5120 14 and 18, 2 x 1536 x 9216 5.6.  2.67 to 2.77 POP/s where K is large: the way from the L2s into LDS and the power
// limit (1.93 GHz); outputs of short K wait for the acknowledgement of the stores in front of the next tile's loads (8 us a tile beside 1.6 us a slice).
#include "linear_tiles.h"

namespace dvdq {

size_t linear8_workspace_bytes(int64_t M, int64_t N, int64_t K) { return workspace_for(M, N, K, true); }

int linear8_choice(int64_t M, int64_t N, int64_t K, bool any) { return choice_for(M, N, K, any, true); }

int launch_linear8(const int8_t *codes, int64_t ldc, const float *x_scale, const int8_t *w, int64_t ldw, const float *w_scale, const void *bias, int act,
                   const void *gate, int64_t gate_rows, int64_t ldg, const void *residual, int64_t ldr, int64_t M, int64_t N, int64_t K, int dtype,
                   void *y, int64_t ldy, void *workspace, hipStream_t stream) {
    LinearArgs a = {};
    a.x = reinterpret_cast<const uint8_t *>(codes), a.w = reinterpret_cast<const uint8_t *>(w), a.x_scale = x_scale, a.w_scale = w_scale;
    a.bias = bias, a.gate = gate, a.residual = residual, a.y = y;
    a.ldx = ldc, a.ldw = ldw, a.ldr = ldr, a.ldy = ldy, a.ldg = ldg;
    a.M = (int)M, a.N = (int)N, a.K = (int)K;
    a.gate_rows = gate ? (int)(M / gate_rows) : 1;
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        // A lane's 8 fp32 outputs are two stores of 16 bytes with a gap between those of the token's lanes, which caches fill and stores past them do
        // not: 8192 x 1024 x 8192 137 us past them, 98 through them, 32760 x 1536 x 1536 114 and 94, 32760 x 8960 x 1536 365 and 360.  Where outputs and residual are more than
        // the last cache, 256 MB, it is the other way round: 32760 x 1536 x 1536 with a residual 148 and 157, 32760 x 5120 x 13824 2386 and 2438, 118800 x 1536 x 1536
        // without one 343 and 352.
        constexpr bool WIDE = sizeof(typename E::Raw) == 4;
        a.streaming = (WIDE ? M * N * (residual ? 2 : 1) > (64 << 20) : M * N >= (2 << 20)) && ldy * sizeof(typename E::Raw) % 64 == 0 && (reinterpret_cast<uintptr_t>(y) & 63) == 0;
        return with_act(act, [&](auto which) { return launch_few_or_tiles<Op8<E>, Op8<Bf16>, decltype(which)::value>(a, workspace, stream); });
    });
}

}  // namespace dvdq
