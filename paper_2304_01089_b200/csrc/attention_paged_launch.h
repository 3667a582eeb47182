// Choice and launch of a paged attention kernel instance. Included by the files that have the instances.
#pragma once
#include "attention_paged.cuh"

namespace rptq {
namespace attn_paged {

struct Launch {
    int bits_v, un, nq, smem, grid, dev;
    cudaStream_t stream;
};

int launch_keys3(const Params& p, const Launch& l);
int launch_keys4(const Params& p, const Launch& l);
int launch_keys8(const Params& p, const Launch& l);

constexpr int SMEM_MAX = 227 * 1024;

template <int BK, int BV, int UN, int NQ>
int launch_one(const Params& p, const Launch& l)
{
    static SmemAllowed done;
    if (allow_smem(reinterpret_cast<const void*>(paged_kernel<BK, BV, UN, NQ>), l.dev, SMEM_MAX, done) != RPTQ_OK) return RPTQ_ERR_CUDA;
    return launch_kernel(paged_kernel<BK, BV, UN, NQ>, dim3((unsigned)l.grid), THREADS, (size_t)l.smem, 0, l.stream, p);
}
template <int BK, int BV>
int launch_size(const Params& p, const Launch& l)
{
    if (l.un == 4) {
        if (l.nq == 2) return launch_one<BK, BV, 4, 2>(p, l);
        return l.nq == 4 ? launch_one<BK, BV, 4, 4>(p, l) : launch_one<BK, BV, 4, 8>(p, l);
    }
    return l.nq == 2 ? launch_one<BK, BV, 8, 2>(p, l) : launch_one<BK, BV, 8, 4>(p, l);
}
template <int BK>
int launch_values(const Params& p, const Launch& l)
{
    return l.bits_v == 3 ? launch_size<BK, 3>(p, l) : l.bits_v == 4 ? launch_size<BK, 4>(p, l) : launch_size<BK, 8>(p, l);
}

}  // namespace attn_paged
}  // namespace rptq
