// rptq_attention_paged: one new token per sequence attends over the sequence's pages of the quantised cache.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>

#include "kv_pages.cuh"
#include "unpack.cuh"

namespace rptq {
namespace attn_paged {

using namespace kv;

constexpr int THREADS = 128, TILE = 128;

struct Params {
    const uint8_t *k, *v;
    int bits_k, bits_v;
    int64_t k_slab, v_slab, k_page, v_page, n_pages;
    const float2 *val_k, *val_v;
    const void* q; int64_t ldq; void* out; int64_t ldo; int bf16;
    const int32_t* table; int64_t ld_table; int width;
    const int32_t* lens;
    int H, G, d, nu, P;
    float scale_log2e;
    int* status;
};

template <int BITS>
__device__ __forceinline__ float dot_key(const uint8_t* slab, int nu, int r, const float* q)
{
    float s = 0.f;
    for (int u = 0; u < nu; ++u) {
        uint32_t w[BITS], o[8];
#pragma unroll
        for (int i = 0; i < BITS; ++i) w[i] = *reinterpret_cast<const uint32_t*>(slab + k_word<BITS>(nu, u, i, r));
        unpack_act32<BITS>(w, o);
#pragma unroll
        for (int c = 0; c < 32; ++c) s = __fmaf_rn(q[32 * u + c], (float)((o[c >> 2] >> (8 * (c & 3))) & 255u), s);
    }
    return s;
}
template <int BITS>
__device__ __forceinline__ float v_code(const uint8_t* slab, int ch, int r)
{
    const int u = ch >> 5, at = ch & 31, e = at & 3, sh = at & 4;
    auto byte = [&](int w) -> uint32_t { return slab[v_byte<BITS>(u, w, e, r)]; };
    if constexpr (BITS == 8) return (float)byte(at >> 2);
    else if constexpr (BITS == 4) return (float)((byte(at >> 3) >> sh) & 15u);
    else return at < 24 ? (float)((byte(at >> 3) >> sh) & 7u)
                        : (float)(((byte(0) >> (sh + 3)) & 1u) | (((byte(1) >> (sh + 3)) & 1u) << 1) | (((byte(2) >> (sh + 3)) & 1u) << 2));
}

// One block per (query head, sequence): tiles of 128 keys with a running maximum and sum; a thread scores a key, then owns one or two
// channels of the output.
__global__ void __launch_bounds__(THREADS) paged_kernel(const Params p)
{
    __shared__ float s_q[32 * MAX_UNITS], s_p[TILE], s_red[THREADS / 32];
    const int tid = threadIdx.x, hq = blockIdx.x, h = hq / p.G, seq = blockIdx.y;
    pdl_trigger();
    pdl_wait();
    const int len = min(max(p.lens[seq], 0), (int)min((int64_t)p.width * p.P, (int64_t)INT_MAX));
    for (int c = tid; c < 32 * p.nu; c += THREADS) {
        float x = 0.f;
        if (c < p.d) {
            const int64_t at = (int64_t)seq * p.ldq + (int64_t)hq * p.d + c;
            x = p.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.q)[at]) : __half2float(static_cast<const __half*>(p.q)[at]);
        }
        s_q[c] = isfinite(x) ? x * p.val_k[(int64_t)h * p.nu * 32 + c].x : __int_as_float(0x7FC00000);
    }
    float m = -1.0e30f, l = 0.f, acc[2] = {0.f, 0.f};
    for (int j0 = 0; j0 < len; j0 += TILE) {
        __syncthreads();
        const int j = j0 + tid;
        auto slab_of = [&](int key, const uint8_t* pool, int64_t page_bytes, int64_t slab_bytes) -> const uint8_t* {
            const int page_i = key / p.P;
            const int64_t page = p.table[(int64_t)seq * p.ld_table + page_i];
            if (page < 0 || page >= p.n_pages) return nullptr;
            return pool + slab_offset(page, page_bytes, h, p.P / SLAB, (key - page_i * p.P) / SLAB, slab_bytes);
        };
        float s = -INFINITY;
        if (j < len) {
            const uint8_t* slab = slab_of(j, p.k, p.k_page, p.k_slab);
            if (!slab) { if (p.status) *p.status = RPTQ_ERR_BAD_SLOT; }
            else s = p.scale_log2e * (p.bits_k == 3 ? dot_key<3>(slab, p.nu, j % SLAB, s_q) : p.bits_k == 4 ? dot_key<4>(slab, p.nu, j % SLAB, s_q) : dot_key<8>(slab, p.nu, j % SLAB, s_q));
        }
        float top = s;
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if ((tid & 31) == 0) s_red[tid >> 5] = top;
        __syncthreads();
        const float m_new = fmaxf(fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])), m), f = exp2f(m - m_new);
        s_p[tid] = exp2f(s - m_new);
        m = m_new;
        __syncthreads();
        l *= f; acc[0] *= f; acc[1] *= f;
        const int n = min(TILE, len - j0);
        for (int i = 0; i < n; ++i) {
            const float pi = s_p[i];
            if (pi == 0.f) continue;
            l += pi;
            const uint8_t* slab = slab_of(j0 + i, p.v, p.v_page, p.v_slab);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int ch = tid + t * THREADS;
                if (ch >= p.d) continue;
                const int r = (j0 + i) % SLAB;
                acc[t] = __fmaf_rn(pi, p.bits_v == 3 ? v_code<3>(slab, ch, r) : p.bits_v == 4 ? v_code<4>(slab, ch, r) : v_code<8>(slab, ch, r), acc[t]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int ch = tid + t * THREADS;
        if (ch >= p.d) continue;
        const float2 sz = p.val_v[(int64_t)h * p.nu * 32 + ch];
        const float o = l == 0.f ? 0.f : sz.x * (acc[t] / l - sz.y);
        const int64_t at = (int64_t)seq * p.ldo + (int64_t)hq * p.d + ch;
        if (p.bf16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(o);
        else static_cast<__half*>(p.out)[at] = __float2half_rn(o);
    }
}

}  // namespace attn_paged
}  // namespace rptq

extern "C" {

int64_t rptq_attention_paged_workspace_bytes(const rptq_kv_cache_t* cache, int n_q_heads)
{
    if (!cache || n_q_heads < 1 || n_q_heads % cache->H) return RPTQ_ERR_INVALID_ARG;
    return 16;
}

int rptq_attention_paged(const rptq_kv_cache_t* cache, const void* q, int64_t ldq, int q_type, int n_q_heads, int n_seq,
                         const void* k_pages, const void* v_pages, int64_t n_pages, const int32_t* page_table, int64_t ld_table, int table_width,
                         const int32_t* seq_lens, float qk_scale, void* out, int64_t ldo, void* workspace, void* stream)
{
    using namespace rptq;
    using namespace rptq::attn_paged;
    if (!cache || n_seq < 0 || n_pages < 0 || table_width < 0 || !(qk_scale >= 0.f)) return RPTQ_ERR_INVALID_ARG;
    if (n_q_heads < 1 || n_q_heads % cache->H || ld_table < table_width) return RPTQ_ERR_INVALID_ARG;
    if (q_type != RPTQ_ROWS_F16 && q_type != RPTQ_ROWS_BF16) return RPTQ_ERR_INVALID_ARG;
    const int64_t Cq = (int64_t)n_q_heads * cache->d;
    if (ldq < Cq || ldo < Cq) return RPTQ_ERR_INVALID_ARG;
    if (!aligned16(k_pages) || !aligned16(v_pages)) return RPTQ_ERR_INVALID_ARG;
    if ((int64_t)table_width * cache->P > INT_MAX || n_seq > 65535 || n_q_heads > 65535) return RPTQ_ERR_UNSUPPORTED;
    if (n_seq == 0) return RPTQ_OK;
    if (!k_pages || !v_pages || !q || !out || !seq_lens || !workspace || (table_width > 0 && !page_table)) return RPTQ_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 1u) || !aligned16(workspace)) return RPTQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(page_table) | reinterpret_cast<uintptr_t>(seq_lens)) & 3u) return RPTQ_ERR_INVALID_ARG;
    int dev = -1;
    if (cache->device < 0 || cudaGetDevice(&dev) != cudaSuccess) return RPTQ_ERR_CUDA;
    if (dev != cache->device) return RPTQ_ERR_INVALID_ARG;

    Params p{};
    p.k = static_cast<const uint8_t*>(k_pages); p.v = static_cast<const uint8_t*>(v_pages);
    p.bits_k = cache->k.bits; p.bits_v = cache->v.bits;
    p.k_slab = cache->k.slab_bytes; p.v_slab = cache->v.slab_bytes; p.k_page = cache->k.page_bytes; p.v_page = cache->v.page_bytes; p.n_pages = n_pages;
    p.val_k = cache->k.value; p.val_v = cache->v.value;
    p.q = q; p.ldq = ldq; p.out = out; p.ldo = ldo; p.bf16 = q_type == RPTQ_ROWS_BF16;
    p.table = page_table; p.ld_table = ld_table; p.width = table_width; p.lens = seq_lens;
    p.H = cache->H; p.G = n_q_heads / cache->H; p.d = cache->d; p.nu = cache->nu; p.P = cache->P;
    p.scale_log2e = qk_scale * 1.4426950408889634f;
    p.status = device_status_word();
    return launch_kernel(paged_kernel, dim3((unsigned)n_q_heads, (unsigned)n_seq), THREADS, 0, 0, static_cast<cudaStream_t>(stream), p);
}

}  // extern "C"
