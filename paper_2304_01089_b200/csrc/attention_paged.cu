// rptq_attention_paged: argument checks, the choice of the kernel's instance, and the launches. The kernel: attention_paged.cuh.
#include <chrono>
#include <climits>
#include <cmath>

#include "attention_paged.cuh"
#include "attention_paged_launch.h"

namespace rptq {
namespace attn_paged {

constexpr int MAX_KEYS = 1 << 30;              // per sequence
constexpr int MIN_SHARE = PAIR_COST + 2;       // least share of a group

// How a cache is worked on with G query heads per cached head: the instance knows its sizes (`exact`), warps of a group, blocks per SM.
struct Plan { bool exact; int un, warps, chunks, smem, blocks; };
static Plan plan_of(const rptq_kv_cache_t* c, int G)
{
    Plan x{};
    x.exact = c->nu == 8 || (c->nu >= 2 && c->nu <= 4);
    x.un = x.exact ? c->nu : c->nu <= 4 ? 4 : 8;
    x.warps = G <= WARP_Q ? 1 : G <= 2 * WARP_Q ? 2 : 4;
    x.chunks = (G + x.warps * WARP_Q - 1) / (x.warps * WARP_Q);
    x.smem = WARPS / x.warps * STAGES * stage_bytes(c->k.bits, c->v.bits, c->nu) + WARPS * scratch_bytes(c->k.bits, x.un);
    const int by_smem = (SMEM_MAX + 1024) / (x.smem + 1024);
    x.blocks = by_smem < blocks_per_sm(x.un) ? by_smem : blocks_per_sm(x.un);
    return x;
}

// In the upper 48 bits; drawn from the clock, so that what an earlier process left in the memory is not taken for this one's counts.
static unsigned long long process_mark()
{
    static const unsigned long long mark = ((unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull) & ~0xFFFFull;
    return mark;
}

}  // namespace attn_paged
}  // namespace rptq

extern "C" {

int64_t rptq_attention_paged_workspace_bytes(const rptq_kv_cache_t* cache, int n_q_heads)
{
    using namespace rptq;
    using namespace rptq::attn_paged;
    if (!cache || n_q_heads < 1 || n_q_heads % cache->H) return RPTQ_ERR_INVALID_ARG;
    const int n_sm = cache->device < 0 ? 0 : sm_count(cache->device);
    if (n_sm == 0) return RPTQ_ERR_CUDA;
    const Plan x = plan_of(cache, n_q_heads / cache->H);
    return (int64_t)n_sm * x.blocks * WARPS * (3 * 8 + 2 * WARP_Q * 4 * part_pitch(cache->nu));
}

int rptq_attention_paged(const rptq_kv_cache_t* cache, const void* q, int64_t ldq, int q_type, int n_q_heads, int n_seq,
                         const void* k_pages, const void* v_pages, int64_t n_pages, const int32_t* page_table, int64_t ld_table, int table_width,
                         const int32_t* seq_lens, float qk_scale, void* out, int64_t ldo, void* workspace, void* stream)
{
    using namespace rptq;
    using namespace rptq::attn_paged;
    if (!cache || n_seq < 0 || n_pages < 0 || table_width < 0 || !(qk_scale >= 0.f) || !std::isfinite(qk_scale)) return RPTQ_ERR_INVALID_ARG;
    if (n_q_heads < 1 || n_q_heads % cache->H || ld_table < table_width) return RPTQ_ERR_INVALID_ARG;
    if (q_type != RPTQ_ROWS_F16 && q_type != RPTQ_ROWS_BF16) return RPTQ_ERR_INVALID_ARG;
    const int64_t Cq = (int64_t)n_q_heads * cache->d;
    if (ldq < Cq || ldo < Cq) return RPTQ_ERR_INVALID_ARG;
    if (!aligned16(k_pages) || !aligned16(v_pages)) return RPTQ_ERR_INVALID_ARG;
    if ((int64_t)table_width * cache->P > MAX_KEYS || n_seq > 65535 || n_q_heads > 65535) return RPTQ_ERR_UNSUPPORTED;
    const Plan x = plan_of(cache, n_q_heads / cache->H);
    // what the longest sequences could need, in tiles: places in the list are 32 bits, groups' shares of it included
    const int64_t max_tiles = ((int64_t)table_width * cache->P + TILE - 1) / TILE, all_pairs = (int64_t)n_seq * cache->H * x.chunks;
    if (all_pairs * (max_tiles + PAIR_COST) > INT_MAX / 2) return RPTQ_ERR_UNSUPPORTED;
    if (n_seq == 0) return RPTQ_OK;
    if (!k_pages || !v_pages || !q || !out || !seq_lens || !workspace || (table_width > 0 && !page_table)) return RPTQ_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 1u) || !aligned16(workspace)) return RPTQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(page_table) | reinterpret_cast<uintptr_t>(seq_lens)) & 3u) return RPTQ_ERR_INVALID_ARG;
    int dev = -1;
    if (cache->device < 0 || cudaGetDevice(&dev) != cudaSuccess) return RPTQ_ERR_CUDA;
    if (dev != cache->device) return RPTQ_ERR_INVALID_ARG;
    const int n_sm = sm_count(dev);
    if (n_sm == 0) return RPTQ_ERR_CUDA;

    Params p{};
    p.k = static_cast<const uint8_t*>(k_pages); p.v = static_cast<const uint8_t*>(v_pages);
    p.k_page = (uint32_t)cache->k.page_bytes; p.v_page = (uint32_t)cache->v.page_bytes;
    p.n_pages = (uint32_t)(n_pages < INT_MAX ? n_pages : INT_MAX);          // (a page number is an int32)
    p.val_k = cache->k.value; p.val_v = cache->v.rest; p.centre_v = cache->v.centre;
    p.q = q; p.ldq = ldq; p.out = out; p.ldo = ldo; p.bf16 = q_type == RPTQ_ROWS_BF16;
    p.vector_out = aligned16(out) && ldo % 8 == 0 && cache->d % 8 == 0;
    p.table = page_table; p.ld_table = ld_table; p.lens = seq_lens;
    p.n_seq = n_seq; p.H = cache->H; p.G = n_q_heads / cache->H; p.d = cache->d; p.nu = cache->nu; p.P = cache->P;
    p.max_len = table_width * cache->P;
    p.chunks = x.chunks;
    p.scale_log2e = qk_scale * 1.4426950408889634f;
    p.arrived = static_cast<unsigned long long*>(workspace);
    p.mark = process_mark();
    p.status = device_status_word();
    p.warps = x.warps;
    const int64_t most = (int64_t)n_sm * x.blocks;
    p.parts = reinterpret_cast<float*>(p.arrived + 3 * most * WARPS);

    // a grid that fills the GPU is the most
    p.whole = max_tiles <= FEW_TILES;
    p.min_share = MIN_SHARE;
    const int64_t groups = p.whole ? all_pairs : (all_pairs * (max_tiles + PAIR_COST) + MIN_SHARE - 1) / MIN_SHARE;
    Launch l{};
    l.bits_v = cache->v.bits; l.un = x.un; l.smem = x.smem; l.dev = dev; l.stream = static_cast<cudaStream_t>(stream);
    l.grid = (int)(groups < most ? (groups < 1 ? 1 : groups) : most);       // (every block's first group has a share before any has a second)
    return cache->k.bits == 3 ? launch_keys3(p, l) : cache->k.bits == 4 ? launch_keys4(p, l) : launch_keys8(p, l);
}

}  // extern "C"
