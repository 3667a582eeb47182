// Choice and launch of a paged attention kernel instance. Included by the files that have the instances.
#pragma once
#include "attention_paged.cuh"

namespace rptq {
namespace attn_paged {

struct Launch {
    int bits_v, un, smem, grid, dev;
    cudaStream_t stream;
};

int launch_keys3(const Params& p, const Launch& l);
int launch_keys4(const Params& p, const Launch& l);
int launch_keys8(const Params& p, const Launch& l);

template <int BK, int BV, int UN, bool EXACT, int R>
int launch_one(const Params& p, const Launch& l)
{
    static SmemAllowed done;
    if (allow_smem(reinterpret_cast<const void*>(paged_kernel<BK, BV, UN, EXACT, R>), l.dev, SMEM_MAX, done) != RPTQ_OK) return RPTQ_ERR_CUDA;
    return launch_kernel(paged_kernel<BK, BV, UN, EXACT, R>, dim3((unsigned)l.grid), THREADS, (size_t)l.smem, 0, l.stream, p);
}
template <int BK, int BV, int UN>
int launch_exact(const Params& p, const Launch& l)
{
    return p.warps == 1 ? launch_one<BK, BV, UN, true, 1>(p, l) : p.warps == 2 ? launch_one<BK, BV, UN, true, 2>(p, l) : launch_one<BK, BV, UN, true, 4>(p, l);
}
// The common sizes of heads are known when the instance is compiled, which saves 10 to 20 % (16 sequences of up to 3000 keys, keys of 8 and values
// of 4 bits, 32 heads of 128 channels: 33.0 -> 29.4 us; 8 cached heads for 32: 21.2 -> 18.5).
template <int BK, int BV>
int launch_size(const Params& p, const Launch& l)
{
    if (p.nu == 2) return launch_exact<BK, BV, 2>(p, l);
    if (p.nu == 3) return launch_exact<BK, BV, 3>(p, l);
    if (p.nu == 4) return launch_exact<BK, BV, 4>(p, l);
    if (p.nu == 8) return launch_exact<BK, BV, 8>(p, l);
    return l.un == 4 ? launch_one<BK, BV, 4, false, 0>(p, l) : launch_one<BK, BV, 8, false, 0>(p, l);
}
template <int BK>
int launch_values(const Params& p, const Launch& l)
{
    return l.bits_v == 3 ? launch_size<BK, 3>(p, l) : l.bits_v == 4 ? launch_size<BK, 4>(p, l) : launch_size<BK, 8>(p, l);
}

}  // namespace attn_paged
}  // namespace rptq
