// The linear operator's products of an operand whose summed index is not the contiguous one: a [K,N] weight in the forward, an
// [N,K] one in dA, and A in dW, read as the caller has them. The copies that this spares, with their cost against the slower
// reads (us): forward with a [K,N] weight, copied / in place, K 8192, N 3584: M 512 63 / 43, M 2048 124 / 104, M 16384 727 / 724;
// the backward of M 8192 of it, A copied / in place 780 / 725.
#include "ficco_linear.h"

namespace ficco {

int launch_tiles_strided(int tile, bool a_strided, const LinearLaunch &a, hipStream_t s)
{
    switch (tile) {
#define X(id, T)                                                                                                    \
    case id:                                                                                                        \
        if constexpr (!T::BURST) {                                                                                  \
            if (!a_strided) return launch_tiles_t<T, false, true>(a, s);                                            \
            if constexpr (T::BM % 64 == 0) return launch_tiles_t<T, true, false>(a, s);                              \
        }                                                                                                           \
        return FICCO_ERR_ARG;
    FICCO_FOR_EACH_TILE(X)
#undef X
    default: return FICCO_ERR_ARG;
    }
}

}  // namespace ficco
