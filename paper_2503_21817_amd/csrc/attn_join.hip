// attn_join.hpp as a kernel
#include "attn_join.hpp"

namespace skipffn {

template <int DP>
__global__ __launch_bounds__(ATT_THREADS) void attn_join_kernel(const AttnJoinArgs P) { attn_join<DP>(P, (int)blockIdx.x); }

hipError_t launch_attn_join(const AttnJoinArgs& a, hipStream_t s) {
    const uint32_t wgs = (uint32_t)(((int64_t)a.T * a.Hq + ATT_WAVES - 1) / ATT_WAVES);
    if (a.D <= 64) attn_join_kernel<64><<<wgs, ATT_THREADS, 0, s>>>(a);
    else attn_join_kernel<128><<<wgs, ATT_THREADS, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace skipffn
