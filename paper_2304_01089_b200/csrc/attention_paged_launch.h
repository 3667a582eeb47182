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

template <int BK, int BV, int UN, int NQ, bool EXACT>
int launch_one(const Params& p, const Launch& l)
{
    static SmemAllowed done;
    if (allow_smem(reinterpret_cast<const void*>(paged_kernel<BK, BV, UN, NQ, EXACT>), l.dev, SMEM_MAX, done) != RPTQ_OK) return RPTQ_ERR_CUDA;
    return launch_kernel(paged_kernel<BK, BV, UN, NQ, EXACT>, dim3((unsigned)l.grid), THREADS, (size_t)l.smem, 0, l.stream, p);
}
template <int BK, int BV, int UN, bool EXACT>
int launch_heads(const Params& p, const Launch& l)
{
    if (l.nq == 2) return launch_one<BK, BV, UN, 2, EXACT>(p, l);
    if constexpr (UN <= 4) {
        if (l.nq == 8) return launch_one<BK, BV, UN, 8, EXACT>(p, l);
    }
    return launch_one<BK, BV, UN, 4, EXACT>(p, l);
}
// The common sizes of heads in a cache whose tensors have the same bits know their sizes when they are compiled.
template <int BK, int BV>
int launch_size(const Params& p, const Launch& l)
{
    if constexpr (BK == BV) {
        if (p.nu == 2) return launch_heads<BK, BV, 2, true>(p, l);
        if (p.nu == 3) return launch_heads<BK, BV, 3, true>(p, l);
        if (p.nu == 4) return launch_heads<BK, BV, 4, true>(p, l);
        if (p.nu == 8) return launch_heads<BK, BV, 8, true>(p, l);
    }
    return l.un == 4 ? launch_heads<BK, BV, 4, false>(p, l) : launch_heads<BK, BV, 8, false>(p, l);
}
template <int BK>
int launch_values(const Params& p, const Launch& l)
{
    return l.bits_v == 3 ? launch_size<BK, 3>(p, l) : l.bits_v == 4 ? launch_size<BK, 4>(p, l) : launch_size<BK, 8>(p, l);
}

}  // namespace attn_paged
}  // namespace rptq
