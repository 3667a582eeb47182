// The kernel of rptq_attention_paged: one new token per sequence over the paged cache. attention_paged.cu has the checks and the choice
// of the instance; attention_paged_k3.cu, _k4.cu and _k8.cu have the instances, by the bits of the keys.
//
// With one token per sequence every code of the cache is used once (once per query head that shares it), so the call is bound by
// reading the cache: 2 d bits / 8 bytes per key and cached head. What follows from that:
//   - the keys of all (sequence, cached head) pairs, cut into tiles of 32, are one long list, and every WARP of a grid that fills the
//     GPU takes an equal share of it, whatever the sequences' lengths are (the host does not know them). A warp has its own ring
//     of tiles in shared memory (cp.async, up to the end of its share: the next pair's tiles travel while this one's are finished) and
//     never waits for another warp;
//   - of a pair whose keys are shared by several warps each leaves a partial output in the workspace, and the one that comes last
//     joins them, in their order: a result does not depend on the order in which warps finish;
//   - softmax with a running reference: P = 2^(S - ref) with a whole number ref. It moves only when a score passes it, and then to
//     HEAD above the tile's maximum, so that nearly all tiles need no maximum and no scaling; moving by whole
//     numbers scales by exact powers of two;
//   - K's scale of a channel multiplies the query, V's the result, so neither product has clusters in it (the zero points of K shift all
//     scores of a row alike). The query becomes integers of 31 bits with one exponent per head, four signed bytes in four
//     columns of mma.sync m16n8k32 (u8 codes x s8 bytes, exact). Of 4-bit codes the packed word itself is an operand: its bytes are 16 hi + lo, so with the
//     integer y of hi's channel counted in units 16 times larger and x - y in place of lo's x, x lo + 16 y hi = (x - y) lo + y (16 hi + lo)
//     takes one AND for eight codes. A channel's query is off by at most 2^-27 of the head's largest: less than 32-bit sums lose;
//   - one or two query heads a cached head: probabilities as unsigned 32-bit integers, four bytes in four columns, V^T as operand A. The
//     sums are exact, and keys behind the last one or on a page that does not exist have P = 0 whatever bytes lie there;
//   - more query heads: P 2^15 as a sum of two fp16 numbers in two columns, codes as fp16 (1024 + n - 1024), sums in fp32. Four query
//     heads to a set of eight columns. (As bytes, eight heads would take four times the accumulators of fp32 sums.)
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "attn_common.cuh"
#include "kv_pages.cuh"

namespace rptq {
namespace attn_paged {

using namespace kv;
using attn::ex2;
using attn::mma_f16;
using attn::mma_u8;
using attn::mma_u8s8;
using tc::cp_async16;
using tc::cp_async_commit;
using tc::cp_async_wait;
using tc::smem_u32;

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int TILE = 2 * SLAB;                 // keys
constexpr int STAGES = 3;
constexpr float HEAD = 4.0f;                   // how far above the largest score a moved reference lies, in powers of two
constexpr float NO_REF = -1.0e30f;
constexpr int FLUSH_TILES = 1000;              // 32 keys x 255 x 255 a tile stay below 2^31 in 32-bit sums for 1032 tiles
constexpr int UNIT_PITCH = 36;                 // words between the units of the staged query: the four pieces of a row group in different banks

struct Params {
    const uint8_t *k, *v;
    const float2 *val_k, *val_v;
    const void* q; int64_t ldq; void* out; int64_t ldo; int bf16, vector_out;
    const int32_t* table; int64_t ld_table;
    const int32_t* lens;
    uint32_t k_page, v_page, n_pages;          // bytes of a page; pages
    int n_seq, H, G, d, nu, P, max_len;
    int chunks;                                // groups of NQ query heads per cached head
    int whole;                                 // a warp takes whole pairs, every n_workers-th; nothing is split
    int min_tiles;                             // least share of a warp
    float scale_log2e;
    unsigned long long* arrived;               // [n_workers] parts that are there of the pair that began in the warp's share and goes on
    unsigned long long call;                   // this call's mark in them, its lowest 16 bits zero
    float* parts;                              // [n_workers][2][NQ][2 + 32 nu]: reference, sum, outputs of a pair's part
    int* status;
};

__device__ __forceinline__ int len_of(const Params& p, int s) { return min(max(p.lens[s], 0), p.max_len); }
__device__ __forceinline__ int tiles_of(int len) { return (len + TILE - 1) / TILE; }

// Where a warp is in its share: sequence, pair of the sequence (cached head and group of query heads), tiles of the pair.
struct Cursor {
    int s, pair, t, n, nt, len;                // t: the next tile, n: how many of the pair are mine from here on, nt: all of the pair
    int64_t left;                              // tiles of my share behind these (whole: the pair's number in the batch)
    bool ok;
};

// All lanes: the number of tiles of one pair of every sequence together.
__device__ __forceinline__ int64_t tiles_per_pair(const Params& p)
{
    int64_t n = 0;
    for (int s = threadIdx.x & 31; s < p.n_seq; s += 32) n += tiles_of(len_of(p, s));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    return n;
}
// All lanes: the share of `share` tiles from tile `at` of the list on.
__device__ __forceinline__ void find_tile(const Params& p, int pairs, int64_t at, int64_t share, Cursor& c)
{
    const int lane = threadIdx.x & 31;
    const int64_t x = at / pairs;
    int64_t before = 0;
    c.ok = false;
    for (int s0 = 0; s0 < p.n_seq; s0 += 32) {
        const int len = s0 + lane < p.n_seq ? len_of(p, s0 + lane) : 0;
        int64_t run = tiles_of(len);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += y;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + run > x);
        if (past) {
            const int l = __ffs(past) - 1;
            c.ok = true;
            c.s = s0 + l;
            c.len = __shfl_sync(0xffffffffu, len, l);
            c.nt = tiles_of(c.len);
            const int64_t rest = at - (before + __shfl_sync(0xffffffffu, run, l) - c.nt) * pairs;
            c.pair = (int)(rest / c.nt);
            c.t = (int)(rest - (int64_t)c.pair * c.nt);
            c.n = (int)min((int64_t)(c.nt - c.t), share);
            c.left = share - c.n;
            return;
        }
        before += __shfl_sync(0xffffffffu, run, 31);
    }
}
// whole: the pair c.left or the next of my pairs that has keys.
__device__ __forceinline__ void find_pair(const Params& p, int pairs, int64_t step, Cursor& c)
{
    c.t = 0;
    const int64_t n = (int64_t)p.n_seq * pairs;
    for (; c.left < n; c.left += step) {
        c.s = (int)(c.left / pairs);
        c.pair = (int)(c.left - (int64_t)c.s * pairs);
        c.len = len_of(p, c.s);
        c.n = c.nt = tiles_of(c.len);
        if (c.nt > 0) return;
    }
    c.ok = false;
}
// From the end of my part of a pair to the next pair.
__device__ __forceinline__ void next_pair(const Params& p, int pairs, int64_t step, Cursor& c)
{
    if (p.whole) { c.left += step; find_pair(p, pairs, step, c); return; }
    if (c.left == 0) { c.ok = false; return; }
    c.t = 0;
    if (++c.pair == pairs) {
        c.pair = 0;
        do {
            if (++c.s >= p.n_seq) { c.ok = false; return; }
            c.len = len_of(p, c.s);
            c.nt = tiles_of(c.len);
        } while (c.nt == 0);
    }
    c.n = (int)min((int64_t)c.nt, c.left);
    c.left -= c.n;
}

__device__ __forceinline__ float query_value(const Params& p, int s, int head, int ch)
{
    const int64_t at = (int64_t)s * p.ldq + (int64_t)head * p.d + ch;
    return p.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.q)[at]) : __half2float(static_cast<const __half*>(p.q)[at]);
}
// N results of consecutive channels from `ch` on (1, 4 or 8).
template <int N>
__device__ __forceinline__ void store_out(const Params& p, int s, int head, int ch, const float (&o)[N])
{
    uint16_t h[N];
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = p.bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(o[i])) : __half_as_ushort(__float2half_rn(o[i]));
    uint16_t* to = static_cast<uint16_t*>(p.out) + (int64_t)s * p.ldo + (int64_t)head * p.d + ch;
    if constexpr (N > 1) {
        if (p.vector_out && ch + N <= p.d) {
            uint32_t w[N / 2];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) w[i] = h[2 * i] | ((uint32_t)h[2 * i + 1] << 16);
            if constexpr (N == 8) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
            else *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (ch + i < p.d) to[i] = h[i];
}

// 8-bit numbers at bits 0-7 (or nibbles at bits 0-3, 4-7) of the halves of w as fp16: the number itself, or 16 times the nibble.
template <uint32_t MASK>
__device__ __forceinline__ uint32_t to_half2(uint32_t w)
{
    const uint32_t t = (w & MASK) | 0x64006400u;                                   // 1024 + n
    const __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&t), __float2half2_rn(-1024.0f));
    return *reinterpret_cast<const uint32_t*>(&r);
}

// bytes of a stage of a warp's ring: two slabs of each tensor
__host__ __device__ constexpr int stage_bytes(int bits_k, int bits_v, int nu) { return 2 * SLAB * 4 * nu * (bits_k + bits_v); }
__host__ __device__ inline int scratch_bytes(int un, int nq) { return nq * TILE * 4 > 2 * un * UNIT_PITCH * 4 ? nq * TILE * 4 : 2 * un * UNIT_PITCH * 4; }
__host__ __device__ inline int part_floats(int nq, int nu) { return nq * (2 + 32 * nu); }

// BK, BV: bits of the keys' and the values' codes; UN: units of 32 channels a head may have (EXACT: has); NQ: query heads at a time.
template <int BK, int BV, int UN, int NQ, bool EXACT>
__global__ void __launch_bounds__(THREADS, (UN <= 4 && NQ <= 4) ? 4 : 3)
paged_kernel(const Params p)
{
    constexpr bool LIMB = NQ == 2;
    constexpr int NPAIR = NQ / 2;                          // score fragments: two query heads each
    constexpr int NSET = LIMB ? 1 : NQ / 4;                // output fragments
    constexpr int KQ = BK == 8 ? (UN + 1) / 2 : (UN + 3) / 4, KI = BK == 8 ? 2 : 4;      // groups of four 16-byte pieces, products per group
    constexpr int NB = BV != 3 ? (UN + 1) / 2 : UN <= 4 ? 2 : 4;                         // blocks of four products of 16 channels
    constexpr float HI = BV == 8 ? 1.0f : 0.0625f;         // channels of the upper nibbles count 16 n
    constexpr bool RAW = LIMB && BV == 4;                  // their rows hold 16 hi + lo
    using Acc = typename std::conditional<LIMB, int, float>::type;
    extern __shared__ __align__(16) uint8_t smem[];

    const int nu = EXACT ? UN : p.nu;
    const int k_slab = SLAB * 4 * BK * nu, v_slab = SLAB * 4 * BV * nu, stage = 2 * (k_slab + v_slab);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    const int64_t n_workers = (int64_t)gridDim.x * WARPS, worker = (int64_t)warp * gridDim.x + blockIdx.x;
    uint8_t* ring = smem + warp * (STAGES * stage + scratch_bytes(UN, NQ));
    uint32_t* scratch = reinterpret_cast<uint32_t*>(ring + STAGES * stage);
    const int pairs = p.H * p.chunks, slabs_per_page = p.P / SLAB;

    pdl_trigger();
    pdl_wait();

    // rows of sequences without keys
    for (int64_t s = worker; s < p.n_seq; s += n_workers)
        if (len_of(p, (int)s) == 0)
            for (int i = lane; i < p.H * p.G * p.d; i += 32) static_cast<uint16_t*>(p.out)[s * p.ldo + i] = 0;

    Cursor in{};                                           // what is loaded next
    int64_t share = 0, list0 = 0;                          // list0: place of the pair's first tile in the list
    if (p.whole) {
        in.ok = true;
        in.left = worker;
        find_pair(p, pairs, n_workers, in);
    } else {
        const int64_t total = tiles_per_pair(p) * pairs;
        share = max((total + n_workers - 1) / n_workers, (int64_t)p.min_tiles);
        const int64_t first = worker * share;
        if (first >= total) return;
        find_tile(p, pairs, first, min(share, total - first), in);
        list0 = first - in.t;
    }
    if (!in.ok) return;
    Cursor c = in;                                         // what is worked on
    int first_t = c.t;                                     // my first tile of c's pair

    // ---- loads: a window of 32 page numbers, one per lane, and the window behind it
    int win_s = -1, win0 = 0, page_now = -1, page_next = -1, page_i = 0, slab_i = 0;
    uint32_t head_k = 0, head_v = 0;                       // where the pair's head begins in a page
    uint32_t missing = 0;                                  // two bits per tile under way: its slabs on pages that do not exist
    auto load_window = [&](int first) {
        const int i = first + lane;
        return i < (in.len + p.P - 1) / p.P ? p.table[(int64_t)in.s * p.ld_table + i] : -1;
    };
    auto seek = [&]() {                                    // to the next tile of another pair
        page_i = 2 * in.t / slabs_per_page;
        slab_i = 2 * in.t - page_i * slabs_per_page;
        const int h = in.pair / p.chunks;
        head_k = (uint32_t)(h * slabs_per_page) * (uint32_t)k_slab;
        head_v = (uint32_t)(h * slabs_per_page) * (uint32_t)v_slab;
        if (in.s != win_s || page_i < win0 || page_i >= win0 + 32) {
            win_s = in.s; win0 = page_i & ~31;
            page_now = load_window(win0);
            page_next = load_window(win0 + 32);
        }
    };
    seek();
    int in_stage = 0;
    auto issue = [&]() {
        missing <<= 2;
        if (in.ok) {
            const uint32_t to = smem_u32(ring) + in_stage * stage + 16 * lane;
            const int keys = in.len - in.t * TILE;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const bool want = half * SLAB < keys;
                if (page_i == win0 + 32) {
                    win0 += 32;
                    page_now = page_next;
                    page_next = load_window(win0 + 32);
                }
                uint32_t page = (uint32_t)__shfl_sync(0xffffffffu, page_now, page_i);
                const bool there = want && page < p.n_pages;
                if (!there) {
                    if (want) {
                        missing |= 1u << half;
                        if (p.status) *p.status = RPTQ_ERR_BAD_SLOT;
                    }
                    page = 0;
                }
                const uint8_t* k = p.k + ((uint64_t)page * p.k_page + (head_k + (uint32_t)(slab_i * k_slab) + 16 * lane));
                const uint8_t* v = p.v + ((uint64_t)page * p.v_page + (head_v + (uint32_t)(slab_i * v_slab) + 16 * lane));
#pragma unroll
                for (int i = 0; i < (UN * 4 * BK + 31) / 32; ++i)
                    if (512 * (i + 1) <= SLAB * 4 * BK * (EXACT ? UN : 0) || 512 * i + 16 * lane < k_slab)
                        cp_async16(to + half * k_slab + 512 * i, k + 512 * i, there);
#pragma unroll
                for (int i = 0; i < (UN * 4 * BV + 31) / 32; ++i)
                    if (512 * (i + 1) <= SLAB * 4 * BV * (EXACT ? UN : 0) || 512 * i + 16 * lane < v_slab)
                        cp_async16(to + 2 * k_slab + half * v_slab + 512 * i, v + 512 * i, there);
                if (++slab_i == slabs_per_page) { slab_i = 0; ++page_i; }
            }
            ++in.t;
            if (--in.n == 0) {
                next_pair(p, pairs, n_workers, in);
                if (in.ok) seek();
            }
        }
        cp_async_commit();
        in_stage = in_stage + 1 == STAGES ? 0 : in_stage + 1;
    };
#pragma unroll 1
    for (int i = 0; i < STAGES - 1; ++i) issue();

    // ---- per pair
    uint32_t qb[NPAIR][KQ * KI][2];
    float coef[NPAIR], ref[NPAIR];                         // of query head 2 i + (t4 >> 1)
    Acc O[NSET][NB][4][4], L[NSET][4];
    float F[LIMB ? NB : 1][4][2], Fl = 0.f;                // LIMB: sums that were taken out of the integers; my two of the four digits
    int since = 0;
    const float weight = (t4 & 1) ? 65536.0f : 1.0f;       // of my two digits d0 + 2^8 d1
    const uint32_t limb_sel = (uint32_t)(g8 & 3) * 0x11u + 0x40u;      // byte g8 & 3 of two words

    auto start_pair = [&]() {
        const int h = c.pair / p.chunks, head0 = h * p.G + (c.pair - h * p.chunks) * NQ;
        const int n_heads = min(NQ, p.G - (c.pair - h * p.chunks) * NQ);
        const float2* val = p.val_k + (int64_t)h * nu * 32;
        float s[UN];
#pragma unroll
        for (int i = 0; i < UN; ++i) s[i] = i < nu ? val[32 * i + lane].x : 0.f;
#pragma unroll
        for (int ps = 0; ps < NPAIR; ++ps) {
            float x[2][UN];
            uint32_t top[2] = {0u, 0u};
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    const int ch = 32 * i + lane;
                    x[q][i] = ch < p.d && 2 * ps + q < n_heads ? query_value(p, c.s, head0 + 2 * ps + q, ch) * s[i] : 0.f;
                    top[q] = max(top[q], __float_as_uint(x[q][i]) & 0x7FFFFFFFu);
                }
            __syncwarp();
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t m = __reduce_max_sync(0xffffffffu, top[q]);
                const bool finite = m < 0x7F800000u;
                const int e = max((int)(m >> 23), 30);                     // |x| < 2^(e - 126): |x| 2^(156 - e) < 2^30
                const float f = finite ? __int_as_float((283 - e) << 23) : 0.f;
                if ((t4 >> 1) == q) coef[ps] = finite ? __int_as_float((e - 29) << 23) * p.scale_log2e : __int_as_float(0x7FC00000);
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    int X = __float2int_rn(x[q][i] * f);
                    if constexpr (BK != 8) {
                        // channels whose codes are upper nibbles are multiplied by 16 n (3 bits) or, of 4 bits, by the whole byte
                        if (lane & 4) X = __float2int_rn(x[q][i] * (f * 0.0625f));
                        if constexpr (BK == 4) {
                            const int y = __shfl_xor_sync(0xffffffffu, X, 4);
                            if (!(lane & 4)) X -= y;
                        }
                    }
                    // signed bytes d with X = d0 + 2^8 d1 + 2^16 d2 + 2^24 d3
                    if (i < nu) scratch[(q * UN + i) * UNIT_PITCH + lane] = ((uint32_t)X + 0x00808080u) ^ 0x00808080u;
                }
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < KQ; ++j)
#pragma unroll
                for (int i = 0; i < KI; ++i) {
                    const int unit = BK == 8 ? 2 * j + (t4 >> 1) : 4 * j + t4, at = BK == 8 ? 16 * (t4 & 1) + 8 * i : 8 * i;
                    uint32_t b0 = 0u, b1 = 0u;
                    if (unit < nu) {
                        const uint4* z = reinterpret_cast<const uint4*>(scratch + ((g8 >> 2) * UN + unit) * UNIT_PITCH + at);
                        const uint4 a = z[0], b = z[1];
                        b0 = __byte_perm(__byte_perm(a.x, a.y, limb_sel), __byte_perm(a.z, a.w, limb_sel), 0x5410);
                        b1 = __byte_perm(__byte_perm(b.x, b.y, limb_sel), __byte_perm(b.z, b.w, limb_sel), 0x5410);
                    }
                    qb[ps][j * KI + i][0] = b0; qb[ps][j * KI + i][1] = b1;
                }
            __syncwarp();
            ref[ps] = NO_REF;
        }
#pragma unroll
        for (int a = 0; a < NSET; ++a) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) O[a][b][e][i] = (Acc)0;
#pragma unroll
            for (int i = 0; i < 4; ++i) L[a][i] = (Acc)0;
        }
        if constexpr (LIMB) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) F[b][e][0] = F[b][e][1] = 0.f;
            Fl = 0.f;
        }
        since = 0;
    };
    // LIMB: the integers move into the 32-bit floating sums, times f. The two digits are joined in floating point: a sum may have 31 bits
    auto flush = [&](float f) {
        if constexpr (LIMB) {
            const float w0 = weight, w1 = 256.0f * weight;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    int (&o)[4] = O[0][b][e];
                    if constexpr (RAW) { o[2] -= o[0]; o[3] -= o[1]; }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        F[b][e][r] = f * (F[b][e][r] + __fmaf_rn(w1, (float)o[2 * r + 1], w0 * (float)o[2 * r]));
                        o[2 * r] = o[2 * r + 1] = 0;
                    }
                }
            Fl = f * (Fl + __fmaf_rn(w1, (float)L[0][1], w0 * (float)L[0][0]));
#pragma unroll
            for (int i = 0; i < 4; ++i) L[0][i] = 0;
            since = 0;
        }
    };
    // What the join and the direct end of a pair have in common: o / l with V's parameters.
    auto result = [&](float o, float l, float inv, float2 sz) { return l == 0.f ? 0.f : sz.x * (o * inv - sz.y); };

    bool begins = true;
    int out_stage = 0;
#pragma unroll 1
    while (c.ok) {
        if (begins) start_pair();
        issue();
        cp_async_wait<STAGES - 1>();
        __syncwarp();
        const uint8_t* ks = ring + out_stage * stage;
        const uint8_t* vs = ks + 2 * k_slab;
        out_stage = out_stage + 1 == STAGES ? 0 : out_stage + 1;

        // ---------------------------------------------------------------- scores: key g8 + 8 (t4 & 1) of each slab
        float S[2][NPAIR];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            int acc[NPAIR][4] = {};
            const uint8_t* base = ks + half * k_slab;
#pragma unroll
            for (int j = 0; j < KQ; ++j) {
                const int pieces = (BK == 8 ? 2 * nu : nu) - 4 * j;
                if (!EXACT && pieces <= 0) break;
                const int n = min(pieces, 4), piece = min(t4, n - 1);
                if constexpr (BK == 3) {
                    const uint8_t* a = base + SLAB * 48 * j + (n * g8 + piece) * 4;
                    uint32_t x[4], y[4];
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        x[i] = *reinterpret_cast<const uint32_t*>(a + SLAB * 4 * n * i);
                        y[i] = *reinterpret_cast<const uint32_t*>(a + SLAB * 4 * n * i + 32 * n);
                    }
                    x[3] = ((x[0] >> 3) & 0x11111111u) | ((x[1] >> 2) & 0x22222222u) | ((x[2] >> 1) & 0x44444444u);
                    y[3] = ((y[0] >> 3) & 0x11111111u) | ((y[1] >> 2) & 0x22222222u) | ((y[2] >> 1) & 0x44444444u);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int ps = 0; ps < NPAIR; ++ps)
                            mma_u8s8(acc[ps], x[i] & 0x07070707u, y[i] & 0x07070707u, x[i] & 0x70707070u, y[i] & 0x70707070u, qb[ps][4 * j + i][0], qb[ps][4 * j + i][1]);
                } else {
                    const uint8_t* a = base + SLAB * 64 * j + (n * g8 + piece) * 16;
                    const uint4 xa = *reinterpret_cast<const uint4*>(a), ya = *reinterpret_cast<const uint4*>(a + 128 * n);
                    const uint32_t x[4] = {xa.x, xa.y, xa.z, xa.w}, y[4] = {ya.x, ya.y, ya.z, ya.w};
                    if constexpr (BK == 4) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int ps = 0; ps < NPAIR; ++ps)
                                mma_u8s8(acc[ps], x[i] & 0x0F0F0F0Fu, y[i] & 0x0F0F0F0Fu, x[i], y[i], qb[ps][4 * j + i][0], qb[ps][4 * j + i][1]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int ps = 0; ps < NPAIR; ++ps)
                                mma_u8s8(acc[ps], x[2 * i], y[2 * i], x[2 * i + 1], y[2 * i + 1], qb[ps][2 * j + i][0], qb[ps][2 * j + i][1]);
                    }
                }
            }
#pragma unroll
            for (int ps = 0; ps < NPAIR; ++ps) {
                // My two digits of keys g8 and g8 + 8 (d0 + 2^8 d1: at most 257 x 128 x 255 x 256 < 2^31); the lane beside me has the other
                // two. It takes key g8 + 8 if I take g8
                const float a = weight * (float)(acc[ps][1] * 256 + acc[ps][0]), b = weight * (float)(acc[ps][3] * 256 + acc[ps][2]);
                const float other = __shfl_xor_sync(0xffffffffu, (t4 & 1) ? a : b, 1);
                S[half][ps] = coef[ps] * (((t4 & 1) ? b : a) + other);
            }
        }
        const int t_left = c.len - c.t * TILE;                 // keys from this tile on
        const uint32_t gone = (missing >> (2 * (STAGES - 1))) & 3u;
        if (t_left < TILE || gone) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const bool seen = half * SLAB + g8 + 8 * (t4 & 1) < t_left && !((gone >> half) & 1u);
#pragma unroll
                for (int ps = 0; ps < NPAIR; ++ps) S[half][ps] = seen ? S[half][ps] : -INFINITY;
            }
        }
        // ---------------------------------------------------------------- probabilities relative to the reference
        bool above = false;
#pragma unroll
        for (int ps = 0; ps < NPAIR; ++ps) above |= fmaxf(S[0][ps], S[1][ps]) > ref[ps];
        if (__any_sync(0xffffffffu, above || (LIMB && ++since == FLUSH_TILES))) {
            float f[NPAIR];
#pragma unroll
            for (int ps = 0; ps < NPAIR; ++ps) {
                float m = fmaxf(S[0][ps], S[1][ps]);
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                const float to = m > ref[ps] ? ceilf(m) + HEAD : ref[ps];
                f[ps] = ex2(fmaxf(ref[ps] - to, -1000.0f));
                ref[ps] = to;
            }
            if constexpr (LIMB) {
                flush(f[0]);
            } else {
                // the outputs' columns: query head 4 a + t4, whose scores are those of fragment 2 a + (t4 >> 1), lanes t4 & 1
#pragma unroll
                for (int a = 0; a < NSET; ++a) {
                    const float lo = __shfl_sync(0xffffffffu, f[2 * a], (t4 & 1) * 2), hi = __shfl_sync(0xffffffffu, f[2 * a + 1], (t4 & 1) * 2);
                    const float g = (t4 >> 1) ? hi : lo;
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int i = 0; i < 4; ++i) O[a][b][e][i] *= g;
#pragma unroll
                    for (int i = 0; i < 4; ++i) L[a][i] *= g;
                }
            }
        }
        uint32_t pb[2][NSET][2];                           // operand B of the second product
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int ps = 0; ps < NPAIR; ++ps) {
                uint32_t w;
                // (S - ref first: a whole number added to the exponent before would be rounded with the score)
                if constexpr (LIMB) {
                    w = __float2uint_rn(ex2(S[half][ps] - ref[ps]) * 2147483648.0f);
                } else {
                    const float x = ex2(S[half][ps] - ref[ps]) * 32768.0f;
                    const __half hi = __float2half_rn(x), lo = __float2half_rn(x - __half2float(hi));
                    w = __half_as_ushort(hi) | ((uint32_t)__half_as_ushort(lo) << 16);
                }
                scratch[(half * NQ + 2 * ps + (t4 >> 1)) * SLAB + g8 + 8 * (t4 & 1)] = w;
            }
        __syncwarp();
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int a = 0; a < NSET; ++a) {
                const int q = LIMB ? g8 >> 2 : 4 * a + (g8 >> 1);
                const uint4 x = *reinterpret_cast<const uint4*>(scratch + (half * NQ + q) * SLAB + 4 * t4);
                if constexpr (LIMB) {
                    pb[half][0][0] = __byte_perm(__byte_perm(x.x, x.y, limb_sel), __byte_perm(x.z, x.w, limb_sel), 0x5410);
                } else {
                    const uint32_t sel = (g8 & 1) ? 0x7632u : 0x5410u;
                    pb[half][a][0] = __byte_perm(x.x, x.z, sel); pb[half][a][1] = __byte_perm(x.y, x.w, sel);
                }
            }
        // ---------------------------------------------------------------- outputs: V^T times the probabilities
        if constexpr (LIMB) {
            mma_u8(L[0], 0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u, pb[0][0][0], pb[1][0][0]);
        } else {
#pragma unroll
            for (int a = 0; a < NSET; ++a)
#pragma unroll
                for (int half = 0; half < 2; ++half) mma_f16(L[a], 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, pb[half][a][0], pb[half][a][1]);
        }
        // Four words (keys 4 t4 .. 4 t4 + 3 as bytes) of block b of a slab.
        uint32_t three[2][3][4];                           // BV == 3: the words of my unit
        if constexpr (BV == 3) {
            const int unit = min(UN <= 4 ? g8 >> 1 : g8, nu - 1);
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int w = 0; w < 3; ++w) {
                    const uint4 x = *reinterpret_cast<const uint4*>(vs + half * v_slab + 64 * (3 * unit + w) + 16 * t4);
                    three[half][w][0] = x.x; three[half][w][1] = x.y; three[half][w][2] = x.z; three[half][w][3] = x.w;
                }
        }
        auto block = [&](int half, int b, uint32_t (&w)[4]) {                  // 3 and 4 bits: eight channels in four words
            if constexpr (BV == 3) {
                const auto& c3 = three[half];
                auto tail = [&](int e) { return ((c3[0][e] >> 3) & 0x11111111u) | ((c3[1][e] >> 2) & 0x22222222u) | ((c3[2][e] >> 1) & 0x44444444u); };
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (UN <= 4) w[e] = b == 0 ? ((g8 & 1) ? c3[2][e] : c3[0][e]) : ((g8 & 1) ? tail(e) : c3[1][e]);
                    else w[e] = b < 3 ? c3[b < 3 ? b : 0][e] : tail(e);
                }
            } else {
                const int group = 8 * (b + 1) <= 4 * (EXACT ? UN : 0) ? 8 * b + g8 : min(8 * b + g8, 4 * nu - 1);
                const uint4 x = *reinterpret_cast<const uint4*>(vs + half * v_slab + 64 * group + 16 * t4);
                w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
            }
        };
        constexpr uint32_t LO = BV == 3 ? 0x07070707u : 0x0F0F0F0Fu, UP = BV == 3 ? 0x70707070u : RAW ? 0xFFFFFFFFu : 0xF0F0F0F0u;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (!EXACT && BV != 3 && 2 * b >= nu) break;
            if constexpr (BV == 8) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (EXACT && 2 * b + x >= UN) break;
                    const uint8_t* at = vs + 64 * min(8 * (2 * b + x) + g8, 8 * nu - 1) + 16 * t4;
                    const uint4 m = *reinterpret_cast<const uint4*>(at), n = *reinterpret_cast<const uint4*>(at + v_slab);
                    const uint32_t u[2][4] = {{m.x, m.y, m.z, m.w}, {n.x, n.y, n.z, n.w}};
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int e = 2 * x + y;
                        if constexpr (LIMB) {
                            mma_u8(O[0][b][e], u[0][2 * y], u[0][2 * y + 1], u[1][2 * y], u[1][2 * y + 1], pb[0][0][0], pb[1][0][0]);
                        } else {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const uint32_t r0 = u[half][2 * y], r1 = u[half][2 * y + 1];
                                const uint32_t a0 = to_half2<0x00FF00FFu>(r0), a1 = to_half2<0x00FF00FFu>(r1), a2 = to_half2<0x00FF00FFu>(r0 >> 8), a3 = to_half2<0x00FF00FFu>(r1 >> 8);
#pragma unroll
                                for (int a = 0; a < NSET; ++a) mma_f16(O[a][b][e], a0, a1, a2, a3, pb[half][a][0], pb[half][a][1]);
                            }
                        }
                    }
                }
            } else {
                uint32_t u[2][4];
                block(0, b, u[0]);
                block(1, b, u[1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (LIMB) {
                        mma_u8(O[0][b][e], u[0][e] & LO, u[0][e] & UP, u[1][e] & LO, u[1][e] & UP, pb[0][0][0], pb[1][0][0]);
                    } else {
                        constexpr uint32_t HLO = LO & 0x00FF00FFu, HUP = UP & 0x00FF00FFu;
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t r = u[half][e], s = r >> 8;
                            const uint32_t a0 = to_half2<HLO>(r), a1 = to_half2<HUP>(r), a2 = to_half2<HLO>(s), a3 = to_half2<HUP>(s);
#pragma unroll
                            for (int a = 0; a < NSET; ++a) mma_f16(O[a][b][e], a0, a1, a2, a3, pb[half][a][0], pb[half][a][1]);
                        }
                    }
                }
            }
        }
        __syncwarp();                                      // the stage may be overwritten, and the scratch
        ++c.t;
        begins = --c.n == 0;
        if (!begins) continue;

        // ---------------------------------------------------------------- the end of my part of the pair
        const bool complete = c.t == c.nt && first_t == 0;
        const int h = c.pair / p.chunks, chunk = c.pair - h * p.chunks, head0 = h * p.G + chunk * NQ, n_heads = min(NQ, p.G - chunk * NQ);
        const float2* val = p.val_v + (int64_t)h * nu * 32;
        const int part_pitch = 2 + 32 * nu;
        if constexpr (LIMB) flush(1.0f);
#pragma unroll
        for (int a = 0; a < NSET; ++a) {
            const int q = LIMB ? t4 >> 1 : 4 * a + t4;                         // the query head of my columns
            float l, my_ref, my_coef;
            if constexpr (LIMB) {
                l = Fl + __shfl_xor_sync(0xffffffffu, Fl, 1);
                my_ref = ref[0]; my_coef = coef[0];
            } else {
                l = L[a][0] + L[a][1];
                const int from = (t4 & 1) * 2;
                const float r0 = __shfl_sync(0xffffffffu, ref[2 * a], from), r1 = __shfl_sync(0xffffffffu, ref[2 * a + 1], from);
                const float c0 = __shfl_sync(0xffffffffu, coef[2 * a], from), c1 = __shfl_sync(0xffffffffu, coef[2 * a + 1], from);
                my_ref = (t4 >> 1) ? r1 : r0; my_coef = (t4 >> 1) ? c1 : c0;
            }
            // a query that is not finite has no sum; nor has a pair none of whose pages exist, which gives zeros
            if (isnan(my_coef)) l = my_coef;
            const float inv = 1.0f / l;
            float* part = p.parts + ((worker * 2 + (first_t == 0)) * NQ + q) * part_pitch;
            const bool mine = q < n_heads && (!LIMB || (t4 & 1) == 0);
            if (!complete && mine && g8 == 0) { part[0] = my_ref; part[1] = l; }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (!EXACT && BV != 3 && 2 * b >= nu) break;
                float o[8];                                                    // channels ch .. ch + 7 (8 bits: two runs of four)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float x;
                        if constexpr (LIMB) x = F[b][e][r] + __shfl_xor_sync(0xffffffffu, F[b][e][r], 1);
                        else x = O[a][b][e][2 * r] + O[a][b][e][2 * r + 1];
                        if (r == 1) x *= HI;
                        o[BV == 8 ? 2 * e + r : e + 4 * r] = x;
                    }
                constexpr int N = BV == 8 ? 4 : 8;
#pragma unroll
                for (int x = 0; x < 8 / N; ++x) {
                    const int ch = BV == 8 ? 4 * (8 * (2 * b + x) + g8) : BV == 4 ? 8 * (8 * b + g8) : UN <= 4 ? 32 * (g8 >> 1) + 16 * (g8 & 1) + 8 * b : 32 * g8 + 8 * b;
                    if (!mine || ch >= 32 * nu) continue;
                    float y[N];
#pragma unroll
                    for (int i = 0; i < N; ++i) y[i] = complete ? result(o[N * x + i], l, inv, val[ch + i]) : o[N * x + i];
                    if (complete) {
                        store_out<N>(p, c.s, head0 + q, ch, y);
                    } else {
#pragma unroll
                        for (int i = 0; i < N; i += 2) *reinterpret_cast<float2*>(part + 2 + ch + i) = make_float2(y[i], y[i + 1]);
                    }
                }
            }
        }
        if (!complete) {
            // The pair began in the share of warp w_first; the last of its parts to arrive joins them all, in the order of the shares.
            const int64_t w_first = list0 / share, w_last = (list0 + c.nt - 1) / share;
            __threadfence();
            __syncwarp();
            int last = 0;
            if (lane == 0) {
                // (a count that an earlier call or anything else left there does not carry this call's mark and counts as none)
                unsigned long long* at = p.arrived + w_first;
                unsigned long long seen = *reinterpret_cast<volatile unsigned long long*>(at), old;
                do {
                    old = seen;
                    const unsigned n = (old & ~0xFFFFull) == p.call ? (unsigned)(old & 0xFFFF) : 0u;
                    last = n == (unsigned)(w_last - w_first);
                    seen = atomicCAS(at, old, last ? p.call : p.call + n + 1);
                } while (seen != old);
            }
            if (__shfl_sync(0xffffffffu, last, 0)) {
                __threadfence();
                for (int q = 0; q < n_heads; ++q) {
                    auto part = [&](int64_t w) { return p.parts + ((w * 2 + (w == w_first)) * NQ + q) * part_pitch; };
                    float top = NO_REF;
                    for (int64_t w = w_first + lane; w <= w_last; w += 32) top = fmaxf(top, __ldcg(part(w)));
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    float l = 0.f, o[UN] = {};
#pragma unroll 4
                    for (int64_t w = w_first; w <= w_last; ++w) {
                        const float* x = part(w);
                        const float f = ex2(fmaxf(__ldcg(x) - top, -1000.0f));
                        l = __fmaf_rn(f, __ldcg(x + 1), l);
#pragma unroll
                        for (int i = 0; i < UN; ++i)
                            if (i < nu) o[i] = __fmaf_rn(f, __ldcg(x + 2 + 32 * i + lane), o[i]);
                    }
                    const float inv = 1.0f / l;
#pragma unroll
                    for (int i = 0; i < UN; ++i) {
                        const int ch = 32 * i + lane;
                        if (ch >= p.d) continue;
                        const float y[1] = {result(o[i], l, inv, val[ch])};
                        store_out<1>(p, c.s, head0 + q, ch, y);
                    }
                }
            }
        }
        list0 += c.nt;
        next_pair(p, pairs, n_workers, c);
        first_t = 0;
    }
    cp_async_wait<0>();
}

}  // namespace attn_paged
}  // namespace rptq
