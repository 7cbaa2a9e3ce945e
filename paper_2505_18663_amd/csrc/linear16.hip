// Matrix product of 16-bit activations and weights with its epilogue:
//
//   y[m, n] = residual[m, n] + gate[m / (M / G), n] * act(sum_k x[m, k] w[n, k] + bias[n])
//
// Products on the matrix cores, sums and epilogue in fp32, one rounding to the tensors' type.
//
// The kernels are those of linear_tiles.h.  Against the library's product of the card's torch, which has no
// epilogue, weights out of the caches: 32760 x 13824 x 5120 with a residual 3170 to 3367 us and 2920 to 3120, 32760 x 1536 x 8960
// with tanh GELU 740 to 807 and 660 to 750, 512 x 4096 x 5120 33 to 37 and 36 to 38, 64 x 5120 x 5120 20 and 22, 1560 x 1536 x 1536 17 and 20, 2 x 1536 x 9216
// 8.4 to 9.1 and 20, 32760 x 1533 x 8960 740 to 780 and 890 to 910.
#include "linear_tiles.h"

namespace dvdq {

size_t linear_workspace_bytes(int64_t M, int64_t N, int64_t K) { return workspace_for(M, N, 2 * K, false); }

int linear_choice(int64_t M, int64_t N, int64_t K, bool any) { return choice_for(M, N, 2 * K, any, false); }

int launch_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *bias, int act, const void *gate, int64_t gate_rows,
                  int64_t ldg, const void *residual, int64_t ldr, int64_t M, int64_t N, int64_t K, int dtype, void *y, int64_t ldy,
                  void *workspace, hipStream_t stream) {
    LinearArgs a = {};
    a.x = static_cast<const uint8_t *>(x), a.w = static_cast<const uint8_t *>(w), a.bias = bias;
    a.gate = gate, a.residual = residual, a.y = y;
    a.ldx = 2 * ldx, a.ldw = 2 * ldw, a.ldr = ldr, a.ldy = ldy, a.ldg = ldg;
    a.M = (int)M, a.N = (int)N, a.K = (int)(2 * K);
    a.gate_rows = gate ? (int)(M / gate_rows) : 1;
    a.streaming = M * N >= (2 << 20) && ldy % 32 == 0 && (reinterpret_cast<uintptr_t>(y) & 63) == 0;
    return with_type(dtype, [&](auto type) {
        using E = decltype(type);
        if constexpr (sizeof(typename E::Raw) == 2)
            return with_act(act, [&](auto which) { return launch_few_or_tiles<Op16<E>, Op16<E>, decltype(which)::value>(a, workspace, stream); });
        else
            return (int)DVDQ_ERR_UNSUPPORTED;
    });
}

}  // namespace dvdq
