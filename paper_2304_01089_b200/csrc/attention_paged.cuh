// The kernel of rptq_attention_paged: one new token per sequence over the paged cache. attention_paged.cu has the checks and the choice
// of the instance; attention_paged_k3.cu, _k4.cu and _k8.cu have the instances, by the bits of the keys.
//
// With one token per sequence every code of the cache is used once (once per query head that shares it), so the call is bound by
// reading the cache: 2 d bits / 8 bytes per key and cached head. What follows from that:
//   - the keys of all (sequence, cached head) pairs, cut into tiles of 32, are one long list, and every WARP of a grid that fills the
//     GPU takes an equal share of it, whatever the sequences' lengths are (the host does not know them). A warp has its own ring
//     of tiles in shared memory (cp.async, up to the end of its share: the next pair's tiles travel while this one's are finished) and
//     never waits for another warp;
//   - a pair whose keys are shared by several warps leaves partial outputs in the workspace, and a second kernel joins them in their
//     order, so that a result does not depend on the order in which warps finish;
//   - softmax with a running reference: P = 2^(S - ref) with a whole number ref. It moves only when a score passes it, and then to
//     HEAD above the tile's maximum, so that nearly all tiles need no maximum and no scaling; moving by whole
//     numbers scales by exact powers of two;
//   - K's scale of a channel multiplies the query, V's the result, so neither product has clusters in it (the zero points of K shift all
//     scores of a row alike). The query becomes integers of 31 bits with one exponent per head, four signed bytes in four
//     columns of mma.sync m16n8k32 (u8 codes x s8 bytes, exact): of 4-bit codes the upper nibbles are used where they are, as 16 n,
//     with the query's integers of those channels shifted down by four, so a packed word needs two AND instructions for eight codes. A channel's
//     query is off by at most 2^-27 of the head's largest: less than 32-bit sums lose;
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
    int64_t k_page, v_page, n_pages;
    int k_slab, v_slab;
    const float2 *val_k, *val_v;
    const void* q; int64_t ldq; void* out; int64_t ldo; int bf16, vector_out;
    const int32_t* table; int64_t ld_table; int width;
    const int32_t* lens;
    int n_seq, H, G, d, nu, P, max_len;
    int chunks;                                // groups of NQ query heads per cached head
    int whole;                                 // a warp takes whole pairs, every n_workers-th; nothing is split
    int min_tiles;                             // least share of a warp
    float scale_log2e;
    float* parts;                              // [n_workers][2][NQ][2 + 32 nu]: reference, sum, outputs of a pair's part
    int* status;
};

__device__ __forceinline__ int len_of(const Params& p, int s) { return min(max(p.lens[s], 0), p.max_len); }
__device__ __forceinline__ int tiles_of(int len) { return (len + TILE - 1) / TILE; }

// The share of a warp: sequence, pair of the sequence (cached head and group of query heads), tile of the pair.
struct Cursor {
    int s, pair, t, nt, len;
    int64_t left;                              // tiles (whole == 0); the pair's number in the batch (whole != 0)
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
// All lanes: where tile `at` of the list lies.
__device__ __forceinline__ void find_tile(const Params& p, int pairs, int64_t at, Cursor& c)
{
    const int lane = threadIdx.x & 31;
    const int64_t x = at / pairs;
    int64_t before = 0;
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
            c.s = s0 + l;
            c.len = __shfl_sync(0xffffffffu, len, l);
            c.nt = tiles_of(c.len);
            const int64_t rest = at - (before + __shfl_sync(0xffffffffu, run, l) - c.nt) * pairs;
            c.pair = (int)(rest / c.nt);
            c.t = (int)(rest - (int64_t)c.pair * c.nt);
            return;
        }
        before += __shfl_sync(0xffffffffu, run, 31);
    }
    c.ok = false;
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
        c.nt = tiles_of(c.len);
        if (c.nt > 0) return;
    }
    c.ok = false;
}
__device__ __forceinline__ void advance(const Params& p, int pairs, int64_t step, Cursor& c)
{
    ++c.t;
    if (!p.whole && --c.left == 0) { c.ok = false; return; }
    if (c.t < c.nt) return;
    if (p.whole) { c.left += step; find_pair(p, pairs, step, c); return; }
    c.t = 0;
    if (++c.pair < pairs) return;
    c.pair = 0;
    do {
        if (++c.s >= p.n_seq) { c.ok = false; return; }
        c.len = len_of(p, c.s);
        c.nt = tiles_of(c.len);
    } while (c.nt == 0);
}

__device__ __forceinline__ float query_value(const Params& p, int s, int head, int ch)
{
    const int64_t at = (int64_t)s * p.ldq + (int64_t)head * p.d + ch;
    return p.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.q)[at]) : __half2float(static_cast<const __half*>(p.q)[at]);
}
// n results of consecutive channels from `ch` on (n = 4 or 8).
template <int N>
__device__ __forceinline__ void store_out(const Params& p, int s, int head, int ch, const float (&o)[N])
{
    uint16_t h[N];
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = p.bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(o[i])) : __half_as_ushort(__float2half_rn(o[i]));
    uint16_t* to = static_cast<uint16_t*>(p.out) + (int64_t)s * p.ldo + (int64_t)head * p.d + ch;
    if (p.vector_out && ch + N <= p.d) {
        uint32_t w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = h[2 * i] | ((uint32_t)h[2 * i + 1] << 16);
        if constexpr (N == 8) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (ch + i < p.d) to[i] = h[i];
    }
}

// 8-bit numbers at bits 0-7 (or nibbles at bits 0-3, 4-7) of the halves of w as fp16: the number itself, or 16 times the nibble.
template <uint32_t MASK>
__device__ __forceinline__ uint32_t to_half2(uint32_t w)
{
    const uint32_t t = (w & MASK) | 0x64006400u;                                   // 1024 + n
    const __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&t), __float2half2_rn(-1024.0f));
    return *reinterpret_cast<const uint32_t*>(&r);
}

__host__ __device__ inline int stage_bytes(int k_slab, int v_slab) { return 2 * (k_slab + v_slab); }
__host__ __device__ inline int scratch_bytes(int un, int nq) { return nq * TILE * 4 > 2 * un * UNIT_PITCH * 4 ? nq * TILE * 4 : 2 * un * UNIT_PITCH * 4; }
__host__ __device__ inline int part_floats(int nq, int nu) { return nq * (2 + 32 * nu); }

// BK, BV: bits of the keys' and the values' codes; UN: units of 32 channels a head may have; NQ: query heads at a time.
template <int BK, int BV, int UN, int NQ>
__global__ void __launch_bounds__(THREADS, (UN == 4 && NQ <= 4) ? 4 : 3)
paged_kernel(const Params p)
{
    constexpr bool LIMB = NQ == 2;
    constexpr int NPAIR = NQ / 2;                          // score fragments: two query heads each
    constexpr int NSET = LIMB ? 1 : NQ / 4;                // output fragments
    constexpr int KQ = BK == 8 ? UN / 2 : UN / 4, KI = BK == 8 ? 2 : 4;      // groups of four 16-byte pieces, products per group
    constexpr int NB = UN / 2;                             // blocks of four products of 16 channels
    constexpr float HI = BV == 8 ? 1.0f : 0.0625f;         // channels of the upper nibbles count 16 n
    using Acc = typename std::conditional<LIMB, int, float>::type;
    extern __shared__ __align__(16) uint8_t smem[];

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    const int64_t n_workers = (int64_t)gridDim.x * WARPS, worker = (int64_t)warp * gridDim.x + blockIdx.x;
    const int stage = stage_bytes(p.k_slab, p.v_slab);
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
    in.ok = true;
    if (p.whole) {
        in.left = worker;
        find_pair(p, pairs, n_workers, in);
    } else {
        const int64_t total = tiles_per_pair(p) * pairs;
        const int64_t share = max((total + n_workers - 1) / n_workers, (int64_t)p.min_tiles), first = worker * share;
        in.left = min(share, total - first);
        if (in.left <= 0) return;
        find_tile(p, pairs, first, in);
    }
    if (!in.ok) return;
    Cursor c = in;                                         // what is worked on
    int first_t = c.t;                                     // my first tile of c's pair

    // ---- loads: a window of 32 page numbers, one per lane, and the window behind it
    int win_s = -1, win0 = 0, page_now = -1, page_next = -1, page_i = 0, slab_i = 0;
    bool seek = true;
    uint32_t missing = 0;                                  // two bits per tile under way: its slabs on pages that do not exist
    auto load_window = [&](int s, int first, int len) {
        const int i = first + lane;
        return i < (len + p.P - 1) / p.P ? p.table[(int64_t)s * p.ld_table + i] : -1;
    };
    int in_stage = 0;
    auto issue = [&]() {
        missing <<= 2;
        if (in.ok) {
            if (seek) {
                page_i = 2 * in.t / slabs_per_page;
                slab_i = 2 * in.t - page_i * slabs_per_page;
                if (in.s != win_s || page_i < win0 || page_i >= win0 + 32) {
                    win_s = in.s; win0 = page_i & ~31;
                    page_now = load_window(in.s, win0, in.len);
                    page_next = win0 + 32 < (in.len + p.P - 1) / p.P ? load_window(in.s, win0 + 32, in.len) : -1;
                }
                seek = false;
            }
            const int h = in.pair / p.chunks;
            const uint32_t to = smem_u32(ring) + in_stage * stage;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const bool want = (2 * in.t + half) * SLAB < in.len;
                if (page_i >= win0 + 32) {
                    win0 += 32;
                    page_now = page_next;
                    page_next = win0 + 32 < (in.len + p.P - 1) / p.P ? load_window(in.s, win0 + 32, in.len) : -1;
                }
                const int page = __shfl_sync(0xffffffffu, page_now, page_i - win0);
                const bool there = want && page >= 0 && page < p.n_pages;
                if (want && !there) {
                    missing |= 1u << half;
                    if (p.status) *p.status = RPTQ_ERR_BAD_SLOT;
                }
                const int64_t in_page = (int64_t)h * slabs_per_page + slab_i, pg = there ? page : 0;
                const uint8_t* k = p.k + (there ? pg * p.k_page + in_page * p.k_slab : 0);
                const uint8_t* v = p.v + (there ? pg * p.v_page + in_page * p.v_slab : 0);
                const uint32_t to_k = to + half * p.k_slab, to_v = to + 2 * p.k_slab + half * p.v_slab;
#pragma unroll
                for (int i = 0; i < (UN * 4 * BK + 31) / 32; ++i) {
                    const int at = 16 * (lane + 32 * i);
                    if (at < p.k_slab) cp_async16(to_k + at, k + (there ? at : 0), there);
                }
#pragma unroll
                for (int i = 0; i < (UN * 4 * BV + 31) / 32; ++i) {
                    const int at = 16 * (lane + 32 * i);
                    if (at < p.v_slab) cp_async16(to_v + at, v + (there ? at : 0), there);
                }
                if (++slab_i == slabs_per_page) { slab_i = 0; ++page_i; }
            }
            const int pair = in.pair, s = in.s;
            advance(p, pairs, n_workers, in);
            if (in.pair != pair || in.s != s) seek = true;
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
    const float w0 = (t4 & 1) ? 65536.0f : 1.0f, w1 = (t4 & 1) ? 16777216.0f : 256.0f;

    auto start_pair = [&]() {
        const int h = c.pair / p.chunks, head0 = h * p.G + (c.pair - h * p.chunks) * NQ;
        const int n_heads = min(NQ, p.G - (c.pair - h * p.chunks) * NQ);
        const float2* val = p.val_k + (int64_t)h * p.nu * 32;
#pragma unroll
        for (int ps = 0; ps < NPAIR; ++ps) {
            float x[2][UN];
            uint32_t top[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                const int ch = 32 * i + lane;
                const float s = i < p.nu ? val[ch].x : 0.f;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    x[q][i] = ch < p.d && 2 * ps + q < n_heads ? query_value(p, c.s, head0 + 2 * ps + q, ch) * s : 0.f;
                    top[q] = max(top[q], __float_as_uint(x[q][i]) & 0x7FFFFFFFu);
                }
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
                    // channels whose codes are upper nibbles are multiplied by 16 n
                    const float g = BK != 8 && (lane & 4) ? f * 0.0625f : f;
                    const uint32_t X = (uint32_t)__float2int_rn(x[q][i] * g);
                    // signed bytes d with X = d0 + 2^8 d1 + 2^16 d2 + 2^24 d3
                    if (i < p.nu) scratch[(q * UN + i) * UNIT_PITCH + lane] = (X + 0x00808080u) ^ 0x00808080u;
                }
            }
            __syncwarp();
            const uint32_t byte = (uint32_t)(g8 & 3), sel = byte | ((byte + 4) << 4);
#pragma unroll
            for (int j = 0; j < KQ; ++j)
#pragma unroll
                for (int i = 0; i < KI; ++i) {
                    const int unit = BK == 8 ? 2 * j + (t4 >> 1) : 4 * j + t4, at = BK == 8 ? 16 * (t4 & 1) + 8 * i : 8 * i;
                    uint32_t b0 = 0u, b1 = 0u;
                    if (unit < p.nu) {
                        const uint4* z = reinterpret_cast<const uint4*>(scratch + ((g8 >> 2) * UN + unit) * UNIT_PITCH + at);
                        const uint4 a = z[0], b = z[1];
                        b0 = __byte_perm(__byte_perm(a.x, a.y, sel), __byte_perm(a.z, a.w, sel), 0x5410);
                        b1 = __byte_perm(__byte_perm(b.x, b.y, sel), __byte_perm(b.z, b.w, sel), 0x5410);
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
    // LIMB: the integers move into the 32-bit floating sums, times f
    auto flush = [&](float f) {
        if constexpr (LIMB) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        F[b][e][r] = f * (F[b][e][r] + __fmaf_rn(w1, (float)O[0][b][e][2 * r + 1], w0 * (float)O[0][b][e][2 * r]));
                        O[0][b][e][2 * r] = O[0][b][e][2 * r + 1] = 0;
                    }
            Fl = f * (Fl + __fmaf_rn(w1, (float)L[0][1], w0 * (float)L[0][0]));
#pragma unroll
            for (int i = 0; i < 4; ++i) L[0][i] = 0;
            since = 0;
        }
    };

    int out_stage = 0;
#pragma unroll 1
    while (c.ok) {
        issue();
        cp_async_wait<STAGES - 1>();
        __syncwarp();
        if (c.t == first_t) start_pair();
        const uint8_t* ks = ring + out_stage * stage;
        const uint8_t* vs = ks + 2 * p.k_slab;
        out_stage = out_stage + 1 == STAGES ? 0 : out_stage + 1;

        // ---------------------------------------------------------------- scores: key g8 + 8 (t4 & 1) of each slab
        float S[2][NPAIR];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            int acc[NPAIR][4] = {};
            const uint8_t* base = ks + half * p.k_slab;
#pragma unroll
            for (int j = 0; j < KQ; ++j) {
                const int pieces = (BK == 8 ? 2 * p.nu : p.nu) - 4 * j;
                if (pieces <= 0) break;
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
                                mma_u8s8(acc[ps], x[i] & 0x0F0F0F0Fu, y[i] & 0x0F0F0F0Fu, x[i] & 0xF0F0F0F0u, y[i] & 0xF0F0F0F0u, qb[ps][4 * j + i][0], qb[ps][4 * j + i][1]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int ps = 0; ps < NPAIR; ++ps)
                                mma_u8s8(acc[ps], x[2 * i], y[2 * i], x[2 * i + 1], y[2 * i + 1], qb[ps][2 * j + i][0], qb[ps][2 * j + i][1]);
                    }
                }
            }
            const int j = c.t * TILE + half * SLAB + g8 + 8 * (t4 & 1);
            const bool seen = j < c.len && !((missing >> (2 * (STAGES - 1) + half)) & 1u);
#pragma unroll
            for (int ps = 0; ps < NPAIR; ++ps) {
                // my two digits of keys g8 and g8 + 8; the lane beside me has the other two. It takes key g8 + 8 if I take g8
                const float a = __fmaf_rn(w1, (float)acc[ps][1], w0 * (float)acc[ps][0]), b = __fmaf_rn(w1, (float)acc[ps][3], w0 * (float)acc[ps][2]);
                const float other = __shfl_xor_sync(0xffffffffu, (t4 & 1) ? a : b, 1);
                S[half][ps] = seen ? ((t4 & 1) ? b : a) + other : -INFINITY;
                S[half][ps] *= seen ? coef[ps] : 1.0f;
            }
        }
        // ---------------------------------------------------------------- probabilities relative to the reference
        bool above = false;
#pragma unroll
        for (int ps = 0; ps < NPAIR; ++ps) above |= fmaxf(S[0][ps], S[1][ps]) > ref[ps];
        if (__any_sync(0xffffffffu, above) || (LIMB && ++since == FLUSH_TILES)) {
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
                // the outputs' columns: query head 4 a + t4, whose score lanes are those of fragment 2 a + (t4 >> 1), lane pair t4 & 1
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
                    const uint32_t byte = (uint32_t)(g8 & 3), sel = byte | ((byte + 4) << 4);
                    pb[half][0][0] = __byte_perm(__byte_perm(x.x, x.y, sel), __byte_perm(x.z, x.w, sel), 0x5410);
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
            const int unit = min(UN == 4 ? g8 >> 1 : g8, p.nu - 1);
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int w = 0; w < 3; ++w) {
                    const uint4 x = *reinterpret_cast<const uint4*>(vs + half * p.v_slab + 64 * (3 * unit + w) + 16 * t4);
                    three[half][w][0] = x.x; three[half][w][1] = x.y; three[half][w][2] = x.z; three[half][w][3] = x.w;
                }
        }
        auto block = [&](int half, int b, uint32_t (&w)[4]) {                  // 3 and 4 bits: eight channels in four words
            if constexpr (BV == 3) {
                const auto& c3 = three[half];
                auto tail = [&](int e) { return ((c3[0][e] >> 3) & 0x11111111u) | ((c3[1][e] >> 2) & 0x22222222u) | ((c3[2][e] >> 1) & 0x44444444u); };
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (UN == 4) w[e] = b == 0 ? ((g8 & 1) ? c3[2][e] : c3[0][e]) : ((g8 & 1) ? tail(e) : c3[1][e]);
                    else w[e] = b < 3 ? c3[b < 3 ? b : 0][e] : tail(e);
                }
            } else {
                const uint4 x = *reinterpret_cast<const uint4*>(vs + half * p.v_slab + 64 * min(8 * b + g8, 4 * p.nu - 1) + 16 * t4);
                w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
            }
        };
        constexpr uint32_t LO = BV == 3 ? 0x07070707u : 0x0F0F0F0Fu, UP = BV == 3 ? 0x70707070u : 0xF0F0F0F0u;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (BV != 3 && 2 * b >= p.nu) break;
            if constexpr (BV == 8) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint8_t* at = vs + 64 * min(8 * (2 * b + x) + g8, 8 * p.nu - 1) + 16 * t4;
                    const uint4 m = *reinterpret_cast<const uint4*>(at), n = *reinterpret_cast<const uint4*>(at + p.v_slab);
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

        // ---------------------------------------------------------------- the end of my part of the pair
        const Cursor done = c;
        advance(p, pairs, n_workers, c);
        const bool last = done.t == done.nt - 1;
        if (last || !c.ok) {
            const bool complete = last && first_t == 0;
            const int h = done.pair / p.chunks, chunk = done.pair - h * p.chunks, head0 = h * p.G + chunk * NQ, n_heads = min(NQ, p.G - chunk * NQ);
            const float2* val = p.val_v + (int64_t)h * p.nu * 32;
            if constexpr (LIMB) flush(1.0f);
#pragma unroll
            for (int a = 0; a < NSET; ++a) {
                const int q = LIMB ? t4 >> 1 : 4 * a + t4;                     // the query head of my columns
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
                float* part = p.parts + ((worker * 2 + (first_t == 0)) * NQ + q) * (2 + 32 * p.nu);
                const bool mine = q < n_heads && (!LIMB || (t4 & 1) == 0);
                if (!complete && mine && g8 == 0) { part[0] = my_ref; part[1] = l; }
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if (BV != 3 && 2 * b >= p.nu) break;
                    float o[8];                                                // channels ch0 .. ch0 + 7 (8 bits: two runs of four)
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
                        const int ch = BV == 8 ? 4 * (8 * (2 * b + x) + g8) : BV == 4 ? 8 * (8 * b + g8) : UN == 4 ? 32 * (g8 >> 1) + 16 * (g8 & 1) + 8 * b : 32 * g8 + 8 * b;
                        if (!mine || ch >= 32 * p.nu) continue;
                        float y[N];
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            y[i] = o[N * x + i];
                            if (complete) {
                                const float2 sz = val[ch + i];
                                y[i] = l == 0.f ? 0.f : sz.x * (y[i] * inv - sz.y);
                            }
                        }
                        if (complete) {
                            store_out<N>(p, done.s, head0 + q, ch, y);
                        } else {
#pragma unroll
                            for (int i = 0; i < N; i += 2) *reinterpret_cast<float2*>(part + 2 + ch + i) = make_float2(y[i], y[i + 1]);
                        }
                    }
                }
            }
            first_t = c.t;
        }
        __syncwarp();                                      // the stage may be overwritten, and the scratch
    }
    cp_async_wait<0>();
}

// The parts of split pairs. Block i looks at the end of warp i's share: if a pair lies across it that began in that share, the block joins
// the pair's parts, in the order of the shares (a thread per channel or two).
template <int NQ>
__global__ void __launch_bounds__(THREADS) join_kernel(const Params p, int64_t n_workers)
{
    __shared__ Cursor s_c;
    __shared__ int64_t s_total;
    pdl_trigger();
    pdl_wait();
    const int pairs = p.H * p.chunks;
    if (threadIdx.x < 32) {
        const int64_t total = tiles_per_pair(p) * pairs;
        const int64_t share = max((total + n_workers - 1) / n_workers, (int64_t)p.min_tiles), at = (blockIdx.x + 1) * share;
        Cursor c{};
        c.ok = at < total;
        if (c.ok) find_tile(p, pairs, at, c);
        c.left = share;
        if (c.ok && (c.t == 0 || c.t > share)) c.ok = false;               // no pair lies across, or it began in an earlier share
        if (threadIdx.x == 0) { s_c = c; s_total = total; }
    }
    __syncthreads();
    const Cursor c = s_c;
    if (!c.ok) return;
    const int64_t share = c.left, end = (blockIdx.x + 1) * share - c.t + c.nt;     // the tile behind the pair's last
    const int64_t w_first = blockIdx.x, w_last = (end - 1) / share;
    const int h = c.pair / p.chunks, chunk = c.pair - h * p.chunks, n_heads = min(NQ, p.G - chunk * NQ);
    const int64_t pitch = 2 + 32 * p.nu;
    for (int i = threadIdx.x; i < n_heads * p.d; i += THREADS) {
        const int q = i / p.d, ch = i - q * p.d;
        // my part of worker w: its last pair's is the second, its first one's the first
        auto part = [&](int64_t w) { return p.parts + ((w * 2 + (w == w_first)) * NQ + q) * pitch; };
        float top = NO_REF;
        for (int64_t w = w_first; w <= w_last; ++w) top = fmaxf(top, part(w)[0]);
        float l = 0.f, o = 0.f;
#pragma unroll 4
        for (int64_t w = w_first; w <= w_last; ++w) {
            const float* x = part(w);
            const float f = ex2(fmaxf(x[0] - top, -1000.0f));
            l = __fmaf_rn(f, x[1], l);
            o = __fmaf_rn(f, x[2 + ch], o);
        }
        const float2 sz = p.val_v[(int64_t)h * p.nu * 32 + ch];
        const float y = l == 0.f ? 0.f : sz.x * (o / l - sz.y);
        uint16_t* to = static_cast<uint16_t*>(p.out) + (int64_t)c.s * p.ldo + (int64_t)(h * p.G + chunk * NQ + q) * p.d + ch;
        *to = p.bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
    }
}

}  // namespace attn_paged
}  // namespace rptq
