// The kernel of rptq_attention_paged: one new token per sequence over the paged cache. attention_paged.cu has the checks and the choice
// of the instance; attention_paged_k3.cu, _k4.cu and _k8.cu have the instances, by the bits of the keys.
//
// With one token per sequence every code of the cache is used once (once per query head that shares it), so the call is bound by
// reading the cache: 2 d bits / 8 bytes per key and cached head. What follows from that:
//   - the keys of all (sequence, cached head) pairs, cut into tiles of 32, are one long list, and every GROUP of warps of a grid that
//     fills the GPU takes an equal share of it, whatever the sequences' lengths are (the host does not know them). Beginning and ending
//     a pair counts as PAIR_COST tiles. A group is one warp, or two or four that work on the same tiles for two query heads
//     each; it has a ring of tiles in shared memory (cp.async, to the end of its share: the next pair's tiles travel while this one's
//     are finished) and never waits for another group;
//   - of a pair whose keys are shared by several groups each leaves a partial output in the workspace, and the one that comes last
//     joins them, in their order (of more than MANY_PARTS in two levels: the last of a run of parts joins the run, the last of the runs their
//     sums): a result does not depend on the order in which groups finish;
//   - softmax with a running reference: P = 2^(S - ref) with a whole number ref. It moves when a score passes it, and then to
//     HEAD above the tile's maximum, so that nearly all tiles need no maximum and no scaling; moving by whole
//     numbers scales by exact powers of two. After RUN_TILES tiles it begins anew, higher or lower: probabilities are integers, and lose
//     what lies 2^-30 below the largest of those that have a reference in common;
//   - K's scale of a channel multiplies the query, V's the result, so neither product has clusters in it (the zero points of K shift all
//     scores of a row alike). The query becomes integers of 31 bits with one exponent per head, four signed bytes in four
//     columns of mma.sync m16n8k32 (u8 codes x s8 bytes, exact): two query heads fill the eight columns. Of 4-bit codes the packed word itself
//     is an operand: its bytes are 16 hi + lo, so with the integer y of hi's channel counted in units 16 times larger and x - y in place
//     of lo's x, x lo + 16 y hi = (x - y) lo + y (16 hi + lo) takes one AND for eight codes; 3-bit pages are made for the same (kv_pages.cuh). A
//     channel's query, whose largest lies in [2^29, 2^30), is off by at most 2^-26 of the head's largest (a step of 16; 8 bits: 2^-30; 3
//     bits, a step of 64: 2^-24);
//   - probabilities as unsigned 32-bit integers, four bytes in four columns, V^T as operand A. The sums are exact, and keys behind the last
//     one or on a page that does not exist have P = 0 whatever bytes lie there. (Codes as fp16 with eight query heads in a warp's eight
//     columns took three instructions per four codes to convert, twice the registers, and 50 us where this takes 24 us: 64 sequences of
//     up to 1337 keys, 32 query heads on 8 cached ones, 8 bits.)
// Measured: 72 heads of 128 channels, eight sequences of up to 2011 keys (10859 in all), 4 bits: 24.9 us, of which finding the share, the
// first tiles, parts and join take 8 and the rest runs at 5.8 TB/s; one sequence of 65553 keys, 32 heads: 53.3 us, 5.0 TB/s over all; 3 bits, 96
// heads, sixteen sequences of up to 1700 keys: 35.6 us, 3.2 TB/s: there a warp's tile is 474 instructions one behind the other, and with 2.8 warps a
// scheduler neither memory nor the issue slots (48 %) are full.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_common.cuh"
#include "kv_pages.cuh"

namespace rptq {
namespace attn_paged {

using namespace kv;
using attn::ex2;
using attn::mma_u8;
using attn::mma_u8s8;
using tc::cp_async16;
using tc::cp_async_commit;
using tc::cp_async_wait;
using tc::smem_u32;

constexpr int TILE = 2 * SLAB;                 // keys
constexpr int WARPS = 4, THREADS = 32 * WARPS;  // of a block: 4, 2 or 1 groups
constexpr int PAIR_COST = 4;                   // tiles that beginning and ending a pair counts as
constexpr int WARP_Q = 2;                      // query heads of a warp
constexpr int FEW_TILES = 4;                   // pairs of at most so many tiles are not split, nor
constexpr int WHOLE_TILES = 10;                // those of at most so many where every pair can have a group of its own: splitting and joining costs about
                                               // as much as six tiles. (4 sequences of 130 keys, 8 cached heads of 128 for 32, 4 bits: 12.4 us split, 7.2
                                               // whole; of 330 keys 11.6 and 11.2. 64 sequences of 330 keys, 32 heads, more pairs than groups: 18.5 and 23.2.
                                               // The groups decide, because only they know the lengths: long calls pay 0.3 to 0.6 us for it)
constexpr int MANY_PARTS = 32;                 // more parts of a pair than these are joined in two levels
constexpr int MAX_TRIES = 1 << 14;             // (every failed one is another group's success, of which there are a few per part)
constexpr float HEAD = 2.0f;                   // how far above the largest score a moved reference lies, in powers of two: room for the next, taken from the
                                               // resolution of the probabilities. (8 x 2011 keys 4: 24.77 us, 2: 24.77, 1: 24.91; 3 bits 34.8, 35.4, 35.9)
constexpr float NO_REF = -0x1p127f;
constexpr float MAX_UNIT = 0x1p80f;            // of the integers that scores are: a score is less than 2^46 of them, and stays above NO_REF
constexpr int RUN_TILES = 32;                  // tiles that have a reference in common at most: what the largest key's distance costs the others is then
                                               // bounded by 1024 keys, however many a group has. (Emptying the integers that often costs a long share
                                               // less than 1 %: 64 sequences of up to 8000 keys, 16 heads, 82.3 and 82.5 us. 32 keys x 255 x 255
                                               // a tile would pass 31 bits after 1032)
constexpr float ONE = 4294967040.0f;           // a probability of 1 relative to its reference: the largest float that is a 32-bit integer

constexpr int SMEM_MAX = 227 * 1024;           // of a block
constexpr int STAGES = 2;                      // of a group's ring. (Three, more of the cache under way: 2 to 4 % slower; four: 5 %)
// 168 registers a thread. (Four, 128: 4 to 17 % slower; two: up to 12 %.) Heads of more than 128 channels need up to 255: with 168 they spill, 32
// sequences of up to 3000 keys, 16 heads of 256 channels, 4 bits, took 60.5 us with three blocks, 45.0 with two; 8 bits, 8 heads for 32, 65.9 and 45.4.
__host__ __device__ constexpr int blocks_per_sm(int un) { return un <= 4 ? 3 : 2; }
// bytes of a stage of a ring: two slabs of each tensor
__host__ __device__ constexpr int stage_bytes(int bits_k, int bits_v, int nu) { return 2 * SLAB * 4 * nu * (bits_k + bits_v); }
// a warp's own: the staged query of one head, or the tile's probabilities; behind them V's zero points of the pair's head, a byte each
__host__ __device__ constexpr int unit_pitch(int bits_k) { return bits_k == 3 ? 44 : 36; }       // words between the units of the staged query: the
                                                                 // four pieces of a row group in different banks
__host__ __device__ constexpr int zeros_at(int bits_k, int un) { return un * unit_pitch(bits_k) * 4 > WARP_Q * TILE * 4 ? un * unit_pitch(bits_k) * 4 : WARP_Q * TILE * 4; }
__host__ __device__ constexpr int scratch_bytes(int bits_k, int un) { return zeros_at(bits_k, un) + (un + 3) / 4 * 128; }
__host__ __device__ constexpr int part_pitch(int nu) { return 4 + 32 * nu; }
struct Params {
    const uint8_t *k, *v;
    const float2 *val_k, *val_v;               // [H * 32 nu] K's {s, z}; V's {s, z - centre}
    const uint8_t* centre_v;                   // [H * 32 nu] V's zero points, or the codes nearest to them
    const void* q; int64_t ldq; void* out; int64_t ldo; int bf16, vector_out;
    const int32_t* table; int64_t ld_table;
    const int32_t* lens;
    uint32_t k_page, v_page, n_pages;          // bytes of a page; pages
    int n_seq, H, G, d, nu, P, max_len;
    int chunks;                                // sets of WARP_Q * warps query heads per cached head
    int warps;                                 // of a group
    int whole;                                 // the table has room for FEW_TILES a pair at most
    int min_share;                             // least share of a group
    float scale_log2e;
    // [groups][3][warps] parts that are there, under the process's mark: of the run of parts that begins with the group's part of the pair which
    // comes into its share from before; of the run that begins with its part of the pair which begins there; and of the latter pair's runs
    unsigned long long* arrived;
    unsigned long long mark;                   // its lowest 16 bits are zero
    float* parts;                              // [groups][2][warps][WARP_Q][4 + 32 nu]: reference, sum, -, -, outputs of a pair's part
    int* status;
};

__device__ __forceinline__ int len_of(const Params& p, int s) { return min(max(p.lens[s], 0), p.max_len); }
__device__ __forceinline__ int tiles_of(int len) { return (len + TILE - 1) / TILE; }

// Where a group is in its share: sequence, pair of the sequence (cached head and set of query heads), tiles of the pair.
struct Cursor {
    int s, pair, t, n, nt, len;                // t: the next tile, n: how many of the pair are mine from here on, nt: all of the pair
    int begin;                                 // the pair's place in the list (whole: the pair's number in the batch)
    bool ok;
};

// All lanes: a group's share of the list (0: groups take whole pairs), and the list's length. (The host sees to it that the list and its
// places stay below 2^31.)
__device__ __forceinline__ int find_shares(const Params& p, int pairs, int n_groups, int& share)
{
    const int whole = p.n_seq * pairs <= n_groups ? WHOLE_TILES : FEW_TILES;
    int n = 0;
    bool split = false;
    for (int s = threadIdx.x & 31; s < p.n_seq; s += 32) {
        const int nt = tiles_of(len_of(p, s));
        n += nt > 0 ? nt + PAIR_COST : 0;
        split |= nt > whole;
    }
    const int total = __reduce_add_sync(0xffffffffu, n) * pairs;
    share = __any_sync(0xffffffffu, split) ? max((total + n_groups - 1) / n_groups, p.min_share) : 0;
    return total;
}
// My tiles of the pair c.s, c.pair, which begins at c.begin: those at places first .. end - 1 of the list.
__device__ __forceinline__ void cut(Cursor& c, int first, int end)
{
    const int t0 = c.begin + PAIR_COST;
    c.t = max(first - t0, 0);
    c.n = min(end - t0, c.nt) - c.t;
    if (c.n <= 0) c.ok = false;                // the share ends at this pair's beginning
}
// All lanes: the first tiles of places first .. end - 1 of the list.
__device__ __forceinline__ void find_tile(const Params& p, int pairs, int first, int end, Cursor& c)
{
    const int lane = threadIdx.x & 31;
    const int x = first / pairs;
    int before = 0;
    for (int s0 = 0; s0 < p.n_seq; s0 += 32) {
        const int len = s0 + lane < p.n_seq ? len_of(p, s0 + lane) : 0;
        int run = len > 0 ? tiles_of(len) + PAIR_COST : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += y;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + run > x);
        if (past) {
            const int l = __ffs(past) - 1;
            c.ok = true;
            c.s = s0 + l;
            c.len = __shfl_sync(0xffffffffu, len, l);
            c.nt = tiles_of(c.len);
            const int seq0 = (before + __shfl_sync(0xffffffffu, run, l) - (c.nt + PAIR_COST)) * pairs;
            c.pair = (first - seq0) / (c.nt + PAIR_COST);
            c.begin = seq0 + c.pair * (c.nt + PAIR_COST);
            cut(c, first, end);
            return;
        }
        before += __shfl_sync(0xffffffffu, run, 31);
    }
}
// whole: the pair number c.begin or the next of my pairs that has keys.
__device__ __forceinline__ void find_pair(const Params& p, int pairs, int step, Cursor& c)
{
    c.t = 0;
    const int n = p.n_seq * pairs;
    for (; c.begin < n; c.begin += step) {
        c.s = c.begin / pairs;
        c.pair = c.begin - c.s * pairs;
        c.len = len_of(p, c.s);
        c.n = c.nt = tiles_of(c.len);
        if (c.nt > 0) return;
    }
    c.ok = false;
}
// From the end of my part of a pair to the next pair; `end`: of my share.
__device__ __forceinline__ void next_pair(const Params& p, int pairs, bool whole, int step, int end, Cursor& c)
{
    if (whole) { c.begin += step; find_pair(p, pairs, step, c); return; }
    c.begin += c.nt + PAIR_COST;
    if (c.begin >= end) { c.ok = false; return; }
    if (++c.pair == pairs) {
        c.pair = 0;
        do {
            if (++c.s >= p.n_seq) { c.ok = false; return; }
            c.len = len_of(p, c.s);
            c.nt = tiles_of(c.len);
        } while (c.nt == 0);
    }
    cut(c, 0, end);
}

__device__ __forceinline__ uint16_t query_bits(const Params& p, int s, int head, int ch)
{
    return static_cast<const uint16_t*>(p.q)[(int64_t)s * p.ldq + (int64_t)head * p.d + ch];
}
__device__ __forceinline__ float query_value(const Params& p, uint16_t bits)
{
    return p.bf16 ? __bfloat162float(__ushort_as_bfloat16(bits)) : __half2float(__ushort_as_half(bits));
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

// BK, BV: bits of the keys' and the values' codes; UN: units of 32 channels a head may have (EXACT: has); R: warps of a group (0: p.warps).
template <int BK, int BV, int UN, bool EXACT, int R>
__global__ void __launch_bounds__(THREADS, blocks_per_sm(UN))
paged_kernel(const Params p)
{
    constexpr int KQ = BK == 8 ? (UN + 1) / 2 : (UN + 3) / 4, KI = BK == 8 ? 2 : BK == 4 ? 4 : 5;      // groups of four 16-byte pieces, products per group
    // A lane's channels of the outputs: NB runs of eight (8 bits: of twice four; 3 bits: a half of a unit is two runs), and the products they take
    constexpr int NB = BV != 3 ? (UN + 1) / 2 : UN <= 4 ? 2 : 4, NM = BV == 3 ? 5 * NB : 4 * NB;
    constexpr float HI = BV == 4 ? 0.0625f : 1.0f;         // 4 bits: channels of the upper nibbles count 16 n
    constexpr bool RAW = BV == 4;                          // their rows hold 16 hi + lo
    extern __shared__ __align__(16) uint8_t smem[];

    const int nu = EXACT ? UN : p.nu;
    const int k_slab = SLAB * 4 * BK * nu, v_slab = SLAB * 4 * BV * nu, stage = 2 * (k_slab + v_slab);
    const int warps = R ? R : p.warps;
    const int warp_in_block = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    const int group = warp_in_block / warps, warp = warp_in_block - group * warps;
    const int n_groups = gridDim.x * (WARPS / warps), me = group * gridDim.x + blockIdx.x;
    uint8_t* ring = smem + group * STAGES * stage;
    uint32_t* scratch = reinterpret_cast<uint32_t*>(smem + (WARPS / warps) * STAGES * stage + warp_in_block * scratch_bytes(BK, UN));
    const int pairs = p.H * p.chunks, slabs_per_page = p.P / SLAB;
    auto sync_group = [&]() {
        if (R == 4) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * warps) : "memory");
    };

    pdl_trigger();
    pdl_wait();

    // rows of sequences without keys
    for (int s = me; s < p.n_seq; s += n_groups)
        if (len_of(p, s) == 0)
            for (int i = 32 * warp + lane; i < p.H * p.G * p.d; i += 32 * warps) static_cast<uint16_t*>(p.out)[(int64_t)s * p.ldo + i] = 0;

    Cursor in{};                                           // what is loaded next
    int share = 0, end = 0;
    const int total = p.whole ? 0 : find_shares(p, pairs, n_groups, share);
    if (share > 0) {
        if (me <= (total - 1) / share) {
            end = min(me * share + share, total);
            find_tile(p, pairs, me * share, end, in);
        }
    } else {
        in.ok = true;
        in.begin = me;
        find_pair(p, pairs, n_groups, in);
    }
    if (!in.ok) return;
    Cursor c = in;                                         // what is worked on
    int first_t = c.t;                                     // my first tile of c's pair

    // ---- loads: a window of 32 page numbers, one per lane, and the window behind it. Of two warps each copies a slab of both tensors,
    // of four a slab of one
    int win_s = -1, win0 = 0, page_now = -1, page_next = -1, page_i = 0, slab_i = 0;
    const uint8_t *head_k = nullptr, *head_v = nullptr;    // my 16 bytes of the head's first slab in page 0
    uint32_t missing = 0;                                  // two bits per tile under way: its slabs on pages that do not exist
    auto load_window = [&](int first) {
        const int i = first + lane;
        return i < (in.len + p.P - 1) / p.P ? p.table[(int64_t)in.s * p.ld_table + i] : -1;
    };
    auto seek = [&]() {                                    // to the next tile of another pair
        page_i = 2 * in.t / slabs_per_page;
        slab_i = 2 * in.t - page_i * slabs_per_page;
        const uint32_t slab0 = (uint32_t)(in.pair / p.chunks * slabs_per_page);
        head_k = p.k + slab0 * (uint32_t)k_slab + 16 * lane;
        head_v = p.v + slab0 * (uint32_t)v_slab + 16 * lane;
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
                if (page_i == win0 + 32) {
                    win0 += 32;
                    page_now = page_next;
                    page_next = load_window(win0 + 32);
                }
                const uint32_t page = (uint32_t)__shfl_sync(0xffffffffu, page_now, page_i);
                const bool want = half * SLAB < keys, there = want && page < p.n_pages;
                missing |= want && !there ? 1u << half : 0u;
                const uint64_t from = there ? page : 0u;
                if (R == 1 || (half * warps >> 1) == (warps == 4 ? warp & 2 : warp)) {
                    if (warps < 4 || !(warp & 1)) {
                        const uint8_t* k = head_k + from * p.k_page + (uint32_t)(slab_i * k_slab);
#pragma unroll
                        for (int i = 0; i < (UN * 4 * BK + 31) / 32; ++i)
                            if (512 * (i + 1) <= SLAB * 4 * BK * (EXACT ? UN : 0) || 512 * i + 16 * lane < k_slab)
                                cp_async16(to + half * k_slab + 512 * i, k + 512 * i, there);
                    }
                    if (warps < 4 || (warp & 1)) {
                        const uint8_t* v = head_v + from * p.v_page + (uint32_t)(slab_i * v_slab);
#pragma unroll
                        for (int i = 0; i < (UN * 4 * BV + 31) / 32; ++i)
                            if (512 * (i + 1) <= SLAB * 4 * BV * (EXACT ? UN : 0) || 512 * i + 16 * lane < v_slab)
                                cp_async16(to + 2 * k_slab + half * v_slab + 512 * i, v + 512 * i, there);
                    }
                }
                if (++slab_i == slabs_per_page) { slab_i = 0; ++page_i; }
            }
            if ((missing & 3u) && lane == 0) record_bad_slot(p.status);
            ++in.t;
            if (--in.n == 0) {
                next_pair(p, pairs, share == 0, n_groups, end, in);
                if (in.ok) seek();
            }
        }
        cp_async_commit();
        in_stage = in_stage + 1 == STAGES ? 0 : in_stage + 1;
    };
#pragma unroll 1
    for (int i = 0; i < STAGES - 1; ++i) issue();

    // ---- per pair
    uint32_t qb[KQ * KI][2];
    float coef = 0.f, ref = NO_REF, sum_ref = NO_REF;      // of query head t4 >> 1; ref: of the integers, sum_ref: of the floating sums
    int O[NM][4], L[4];
    float F[NB][4][2], Fl = 0.f;                           // sums that were taken out of the integers; my two of the four digits
    int since = 0, n_heads = 0;
    const float weight = (t4 & 1) ? 65536.0f : 1.0f;       // of my two digits d0 + 2^8 d1
    const uint32_t limb_sel = (uint32_t)(g8 & 3) * 0x11u + 0x40u;      // byte g8 & 3 of two words

    // my channels 32 i + lane of the query heads and of K's scales, loaded a tile before they are used
    uint32_t q_bits[UN];
    float k_scale[UN];
    uint32_t zero_words[(UN + 3) / 4];                     // of channels 128 i + 4 lane ..
    auto load_query = [&](const Cursor& of) {
        const int h = of.pair / p.chunks, q0 = (of.pair - h * p.chunks) * (WARP_Q * warps) + WARP_Q * warp, n = p.G - q0;
        const float2* val = p.val_k + (int64_t)h * nu * 32;
#pragma unroll
        for (int i = 0; i < UN; i += 4) zero_words[i / 4] = 32 * i + 4 * lane < 32 * nu ? *reinterpret_cast<const uint32_t*>(p.centre_v + h * nu * 32 + 32 * i + 4 * lane) : 0u;
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int ch = 32 * i + lane;
            k_scale[i] = i < nu && n > 0 ? val[ch].x : 0.f;
            q_bits[i] = ch < p.d && n > 0 ? query_bits(p, of.s, h * p.G + q0, ch) : 0u;
            if (ch < p.d && n > 1) q_bits[i] |= (uint32_t)query_bits(p, of.s, h * p.G + q0 + 1, ch) << 16;
        }
    };
    uint8_t* const zeros = reinterpret_cast<uint8_t*>(scratch) + zeros_at(BK, UN);
    auto start_pair = [&]() {
        n_heads = min(WARP_Q, p.G - (c.pair % p.chunks) * (WARP_Q * warps) - WARP_Q * warp);
        if (n_heads <= 0) return;
        float x[WARP_Q][UN];
#pragma unroll
        for (int j = 0; j < KQ * KI; ++j) qb[j][0] = qb[j][1] = 0u;
#pragma unroll
        for (int q = 0; q < WARP_Q; ++q) {
            if (q >= n_heads) break;
            uint32_t top = 0u;
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                x[q][i] = query_value(p, (uint16_t)(q_bits[i] >> (16 * q))) * k_scale[i];
                top = max(top, __float_as_uint(x[q][i]) & 0x7FFFFFFFu);
            }
            top = __reduce_max_sync(0xffffffffu, top);
            const int e = max((int)(top >> 23), 30);                       // |x| < 2^(e - 126): |x| 2^(156 - e) < 2^30
            const float unit = __int_as_float((e - 29) << 23) * p.scale_log2e;
            const bool finite = top < 0x7F800000u && unit < MAX_UNIT;
            const float f = finite ? __int_as_float((283 - e) << 23) : 0.f;
            if ((t4 >> 1) == q) coef = finite ? unit : __int_as_float(0x7FC00000);
            // signed bytes d with X = d0 + 2^8 d1 + 2^16 d2 + 2^24 d3
            auto digits = [](int X) { return ((uint32_t)X + 0x00808080u) ^ 0x00808080u; };
            constexpr int PITCH = unit_pitch(BK);
            __syncwarp();
            if constexpr (BK == 3) {
                // A product has c0, c0 + 8 c1, c0 + 8 c1 + 64 b, .. as factors: the query's integers of c0, c1 / 8, b / 64 (of the single bits on top,
                // worth 4: / 16 and / 32), each less the next. First the integers, channel by channel and those of the single bits behind them
                const int in_half = lane & 15;
                const float g = f * (in_half >= 12 ? 0.015625f : (in_half >= 4 && in_half < 8) || in_half >= 10 ? 0.125f : 1.0f);
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    if (i >= nu) break;
                    scratch[i * PITCH + lane] = (uint32_t)__float2int_rn(x[q][i] * g);
                    if (in_half >= 12) scratch[i * PITCH + 32 + 4 * (lane >> 4) + (lane & 3)] = (uint32_t)__float2int_rn(x[q][i] * (f * (lane & 1 ? 0.03125f : 0.0625f)));
                }
                __syncwarp();
                // then the 10 operands' four bytes each
                uint32_t z[UN][2];
                auto entry = [&](const uint32_t* y, int e) {
                    const int op = e >> 2, i = e & 3;
                    int a, b;                                                  // b < 0: nothing is taken off
                    if (op < 6) {
                        const int h = op >= 3 ? 16 : 0, of = op >= 3 ? op - 3 : op;
                        a = h + (of == 2 ? 12 : 4 * of) + i;
                        b = of == 2 ? -1 : h + (of == 1 ? 12 : 4) + i;
                    } else {
                        const int h = 16 * (i >> 1), bit = 32 + 4 * (i >> 1) + 2 * (i & 1);
                        a = op == 6 ? h + 8 + (i & 1) : op == 7 ? h + 10 + (i & 1) : op == 8 ? bit : bit + 1;
                        b = op == 6 ? h + 10 + (i & 1) : op == 7 ? bit : op == 8 ? bit + 1 : -1;
                    }
                    return digits((int)y[a] - (b < 0 ? 0 : (int)y[b]));
                };
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    const uint32_t* y = scratch + min(i, nu - 1) * PITCH;
                    z[i][0] = entry(y, lane);
                    z[i][1] = entry(y, 32 + (lane & 7));
                }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    if (i >= nu) break;
                    scratch[i * PITCH + lane] = z[i][0];
                    if (lane < 8) scratch[i * PITCH + 32 + lane] = z[i][1];
                }
            } else {
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    int X = __float2int_rn(x[q][i] * (BK == 4 && (lane & 4) ? f * 0.0625f : f));
                    if constexpr (BK == 4) {                                   // channels whose codes are upper nibbles are multiplied by the whole byte
                        const int y = __shfl_xor_sync(0xffffffffu, X, 4);
                        if (!(lane & 4)) X -= y;
                    }
                    if (i < nu) scratch[i * PITCH + lane] = digits(X);
                }
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < KQ; ++j)
#pragma unroll
                for (int i = 0; i < KI; ++i) {
                    const int unit = BK == 8 ? 2 * j + (t4 >> 1) : 4 * j + t4, at = BK == 8 ? 16 * (t4 & 1) + 8 * i : 8 * i;
                    if (unit < nu && (g8 >> 2) == q) {
                        const uint4* z = reinterpret_cast<const uint4*>(scratch + unit * PITCH + at);
                        const uint4 a = z[0], b = z[1];
                        qb[j * KI + i][0] = __byte_perm(__byte_perm(a.x, a.y, limb_sel), __byte_perm(a.z, a.w, limb_sel), 0x5410);
                        qb[j * KI + i][1] = __byte_perm(__byte_perm(b.x, b.y, limb_sel), __byte_perm(b.z, b.w, limb_sel), 0x5410);
                    }
                }
        }
#pragma unroll
        for (int i = 0; i < UN; i += 4) *reinterpret_cast<uint32_t*>(zeros + 32 * i + 4 * lane) = zero_words[i / 4];
        __syncwarp();
        ref = sum_ref = NO_REF;
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) O[m][i] = 0;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) F[b][e][0] = F[b][e][1] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) L[i] = 0;
        Fl = 0.f;
        since = 0;
    };
    // The integers move into the 32-bit floating sums, both relative to the larger of their references from there on. The two digits are joined in
    // floating point: one's sum has up to 26 bits, the other counts 2^8 times as much.
    // The floating sums are of code - zero point (of one outside the codes: less the nearest code), the subtraction still exact: in sums of the
    // codes the outputs, which are means of values around zero, would be differences of far larger numbers.
    auto flush = [&]() {
        const float top = fmaxf(ref, sum_ref), f = ex2(fmaxf(sum_ref - top, -1000.0f)), w0 = weight * ex2(fmaxf(ref - top, -1000.0f)), w1 = 256.0f * w0;
        sum_ref = top;
        if constexpr (BV == 3) {
            // operand k of a half of a unit is row k & 1 of product k >> 1: of A byte e c0, c0 + 8 c1, all of it; of C byte i c0, c0 + 8 c1, and the
            // single bits on top
#pragma unroll
            for (int j = 0; j < NB / 2; ++j) {
                const uint4 zs = *reinterpret_cast<const uint4*>(zeros + 128 * j + 16 * g8);
                const uint32_t z[4] = {zs.x, zs.y, zs.z, zs.w};
                int v[2][16];
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    auto sum = [&](int k) { return O[10 * j + (k >> 1)][2 * (k & 1) + d]; };
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[d][e] = sum(3 * e);
                        v[d][4 + e] = (sum(3 * e + 1) - sum(3 * e)) >> 3;
                        v[d][12 + e] = (sum(3 * e + 2) - sum(3 * e + 1)) >> 6;
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        v[d][8 + i] = sum(12 + 4 * i);
                        v[d][10 + i] = (sum(13 + 4 * i) - sum(12 + 4 * i)) >> 3;
                        v[d][12 + 2 * i] += ((sum(14 + 4 * i) - sum(13 + 4 * i)) >> 6) * 4;
                        v[d][13 + 2 * i] += ((sum(15 + 4 * i) - sum(14 + 4 * i)) >> 7) * 4;
                    }
                }
#pragma unroll
                for (int n = 0; n < 16; ++n)
#pragma unroll
                    for (int d = 0; d < 2; ++d) v[d][n] -= (int)((z[n >> 2] >> (8 * (n & 3))) & 255u) * L[d];
#pragma unroll
                for (int n = 0; n < 16; ++n) {
                    float& x = F[2 * j + (n >> 3)][n & 3][(n >> 2) & 1];
                    x = __fmaf_rn(f, x, __fmaf_rn(w1, (float)v[1][n], w0 * (float)v[0][n]));
                }
            }
        } else {
            uint2 z = make_uint2(0u, 0u);
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                if (!EXACT && 2 * (m >> 2) >= nu) break;
                if (BV == 8 && m % 2 == 0) z.x = *reinterpret_cast<const uint32_t*>(zeros + 32 * (m >> 1) + 4 * g8);
                if (BV == 4 && m % 4 == 0) z = *reinterpret_cast<const uint2*>(zeros + 64 * (m >> 2) + 8 * g8);
                int (&o)[4] = O[m];
                if constexpr (RAW) { o[2] -= o[0]; o[3] -= o[1]; }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t word = BV == 4 && i >= 2 ? z.y : z.x, byte = BV == 8 ? 2 * (m & 1) + (i >> 1) : m & 3;
                    o[i] -= (int)((word >> (8 * byte)) & 255u) * (BV == 4 && i >= 2 ? 16 * L[i & 1] : L[i & 1]);
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) F[m >> 2][m & 3][r] = __fmaf_rn(f, F[m >> 2][m & 3][r], __fmaf_rn(w1, (float)o[2 * r + 1], w0 * (float)o[2 * r]));
            }
        }
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) O[m][i] = 0;
        Fl = __fmaf_rn(f, Fl, __fmaf_rn(w1, (float)L[1], w0 * (float)L[0]));
#pragma unroll
        for (int i = 0; i < 4; ++i) L[i] = 0;
        since = 0;
    };
    // What the join and the direct end of a pair have in common: o / l with V's parameters, the zero point but for what the sums have lost of it.
    auto result = [&](float o, float l, float inv, float2 sz) { return l == 0.f ? 0.f : sz.x * (o * inv - sz.y); };

    // One tile.
    auto work = [&](const uint8_t* ks, const uint8_t* vs) {
        // ---------------------------------------------------------------- scores: key g8 + 8 (t4 & 1) of each slab
        float S[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            int acc[4] = {};
            const uint8_t* base = ks + half * k_slab;
#pragma unroll
            for (int j = 0; j < KQ; ++j) {
                const int pieces = (BK == 8 ? 2 * nu : nu) - 4 * j;
                if (!EXACT && pieces <= 0) break;
                const int n = min(pieces, 4), piece = min(t4, n - 1);
                if constexpr (BK == 3) {
                    const uint8_t* a = base + SLAB * 48 * j + (n * g8 + piece) * 4;
                    uint32_t x[3], y[3];
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        x[i] = *reinterpret_cast<const uint32_t*>(a + SLAB * 4 * n * i);
                        y[i] = *reinterpret_cast<const uint32_t*>(a + SLAB * 4 * n * i + 32 * n);
                    }
                    constexpr uint32_t M7 = 0x07070707u, M3F = 0x3F3F3F3Fu, M7F = 0x7F7F7F7Fu;
                    const uint32_t (*b)[2] = qb + 5 * j;
                    mma_u8s8(acc, x[0] & M7, y[0] & M7, x[0] & M3F, y[0] & M3F, b[0][0], b[0][1]);
                    mma_u8s8(acc, x[0], y[0], x[1] & M7, y[1] & M7, b[1][0], b[1][1]);
                    mma_u8s8(acc, x[1] & M3F, y[1] & M3F, x[1], y[1], b[2][0], b[2][1]);
                    mma_u8s8(acc, x[2] & M7, y[2] & M7, x[2] & M3F, y[2] & M3F, b[3][0], b[3][1]);
                    mma_u8s8(acc, x[2] & M7F, y[2] & M7F, x[2], y[2], b[4][0], b[4][1]);
                } else {
                    const uint8_t* a = base + SLAB * 64 * j + (n * g8 + piece) * 16;
                    const uint4 xa = *reinterpret_cast<const uint4*>(a), ya = *reinterpret_cast<const uint4*>(a + 128 * n);
                    const uint32_t x[4] = {xa.x, xa.y, xa.z, xa.w}, y[4] = {ya.x, ya.y, ya.z, ya.w};
                    if constexpr (BK == 4) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) mma_u8s8(acc, x[i] & 0x0F0F0F0Fu, y[i] & 0x0F0F0F0Fu, x[i], y[i], qb[4 * j + i][0], qb[4 * j + i][1]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) mma_u8s8(acc, x[2 * i], y[2 * i], x[2 * i + 1], y[2 * i + 1], qb[2 * j + i][0], qb[2 * j + i][1]);
                    }
                }
            }
            // My two digits of keys g8 and g8 + 8 (d0 + 2^8 d1: at most 257 x 128 x 255 x 256 < 2^31); the lane beside me has the other two. It
            // takes key g8 + 8 if I take g8
            const float a = weight * (float)(acc[1] * 256 + acc[0]), b = weight * (float)(acc[3] * 256 + acc[2]);
            const float other = __shfl_xor_sync(0xffffffffu, (t4 & 1) ? a : b, 1);
            S[half] = coef * (((t4 & 1) ? b : a) + other);
        }
        const int keys = c.len - c.t * TILE;                   // from this tile on
        const uint32_t gone = (missing >> (2 * (STAGES - 1))) & 3u;
        if (keys < TILE || gone) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
                if (half * SLAB + g8 + 8 * (t4 & 1) >= keys || ((gone >> half) & 1u)) S[half] = -INFINITY;
        }
        // ---------------------------------------------------------------- probabilities relative to the reference
        if (__any_sync(0xffffffffu, fmaxf(S[0], S[1]) > ref) || since == RUN_TILES) {
            float m = fmaxf(S[0], S[1]);
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float to = fmaxf(ceilf(m) + HEAD, NO_REF);
            const bool anew = m > ref || since == RUN_TILES;                   // (the other query head's reference may stay)
            if (since > 0) flush();                                            // (nothing is there at a pair's first tile)
            if (anew) ref = to;
        }
        ++since;
        // (S - ref first: a whole number added to the exponent before would be rounded with the score)
#pragma unroll
        for (int half = 0; half < 2; ++half)
            scratch[(half * WARP_Q + (t4 >> 1)) * SLAB + g8 + 8 * (t4 & 1)] = __float2uint_rn(ex2(S[half] - ref) * ONE);
        __syncwarp();
        uint32_t pb[2];                                        // operand B of the second product: byte g8 & 3 of four keys
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint4 x = *reinterpret_cast<const uint4*>(scratch + (half * WARP_Q + (g8 >> 2)) * SLAB + 4 * t4);
            pb[half] = __byte_perm(__byte_perm(x.x, x.y, limb_sel), __byte_perm(x.z, x.w, limb_sel), 0x5410);
        }
        // ---------------------------------------------------------------- outputs: V^T times the probabilities
        mma_u8(L, 0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u, pb[0], pb[1]);
        if constexpr (BV == 8) {
#pragma unroll
            for (int x = 0; x < UN; ++x) {
                if (!EXACT && x >= nu) break;
                const uint8_t* at = vs + 64 * (8 * x + g8) + 16 * t4;
                const uint4 m = *reinterpret_cast<const uint4*>(at), n = *reinterpret_cast<const uint4*>(at + v_slab);
                mma_u8(O[2 * x], m.x, m.y, n.x, n.y, pb[0], pb[1]);
                mma_u8(O[2 * x + 1], m.z, m.w, n.z, n.w, pb[0], pb[1]);
            }
        } else if constexpr (BV == 4) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (!EXACT && 2 * b >= nu) break;
                const int group = 8 * (b + 1) <= 4 * (EXACT ? UN : 0) ? 8 * b + g8 : min(8 * b + g8, 4 * nu - 1);
                const uint4 x = *reinterpret_cast<const uint4*>(vs + 64 * group + 16 * t4), y = *reinterpret_cast<const uint4*>(vs + v_slab + 64 * group + 16 * t4);
                mma_u8(O[4 * b + 0], x.x & 0x0F0F0F0Fu, x.x, y.x & 0x0F0F0F0Fu, y.x, pb[0], pb[1]);
                mma_u8(O[4 * b + 1], x.y & 0x0F0F0F0Fu, x.y, y.y & 0x0F0F0F0Fu, y.y, pb[0], pb[1]);
                mma_u8(O[4 * b + 2], x.z & 0x0F0F0F0Fu, x.z, y.z & 0x0F0F0F0Fu, y.z, pb[0], pb[1]);
                mma_u8(O[4 * b + 3], x.w & 0x0F0F0F0Fu, x.w, y.w & 0x0F0F0F0Fu, y.w, pb[0], pb[1]);
            }
        } else {
            // a row group has a half of a unit: four words of A and two of C
            constexpr uint32_t M7 = 0x07070707u, M3F = 0x3F3F3F3Fu, M7F = 0x7F7F7F7Fu;
#pragma unroll
            for (int j = 0; j < NB / 2; ++j) {
                const int unit = min(4 * j + (g8 >> 1), nu - 1);
                const uint8_t* at = vs + 64 * (3 * unit) + 16 * t4;
                uint32_t w[2][6];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint4 a = *reinterpret_cast<const uint4*>(at + half * v_slab + 64 * (g8 & 1));
                    const uint2 c = *reinterpret_cast<const uint2*>(at + half * v_slab + 128 + 8 * (g8 & 1));
                    w[half][0] = a.x; w[half][1] = a.y; w[half][2] = a.z; w[half][3] = a.w; w[half][4] = c.x; w[half][5] = c.y;
                }
                auto op = [&](int half, int k) -> uint32_t {                   // operand k of 20
                    if (k < 12) return k % 3 == 0 ? w[half][k / 3] & M7 : k % 3 == 1 ? w[half][k / 3] & M3F : w[half][k / 3];
                    const uint32_t c = w[half][4 + (k - 12) / 4];
                    return k % 4 == 0 ? c & M7 : k % 4 == 1 ? c & M3F : k % 4 == 2 ? c & M7F : c;
                };
#pragma unroll
                for (int m = 0; m < 10; ++m) mma_u8(O[10 * j + m], op(0, 2 * m), op(0, 2 * m + 1), op(1, 2 * m), op(1, 2 * m + 1), pb[0], pb[1]);
            }
        }
        __syncwarp();                                          // the scratch may be written again (one warp: and the stage)
    };

    // My part of the pair is done: to the output if it is all of the pair, else to the workspace.
    auto finish = [&]() {
        const bool complete = c.t == c.nt && first_t == 0;
        const int h = c.pair / p.chunks, head0 = h * p.G + (c.pair - h * p.chunks) * (WARP_Q * warps) + WARP_Q * warp;
        const float2* val = p.val_v + (int64_t)h * nu * 32;
        const int pitch = part_pitch(nu);
        auto part_of = [&](int of, bool begins, int q) { return p.parts + (int64_t)(((of * 2 + begins) * warps + warp) * WARP_Q + q) * pitch; };
        flush();
        float l = Fl + __shfl_xor_sync(0xffffffffu, Fl, 1);
        // a query that is not finite has no sum; nor has a pair none of whose pages exist, which gives zeros
        if (isnan(coef)) l = coef;
        const float inv = 1.0f / l;
        const int q = t4 >> 1;
        const bool mine = q < n_heads && (t4 & 1) == 0;
        float* part = part_of(me, first_t == 0, q);
        if (!complete && mine && g8 == 0) *reinterpret_cast<float2*>(part) = make_float2(sum_ref, l);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (!EXACT && BV != 3 && 2 * b >= nu) break;
            float o[8];                                                        // channels ch .. ch + 7 (8 bits: two runs of four)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float x = F[b][e][r] + __shfl_xor_sync(0xffffffffu, F[b][e][r], 1);
                    o[BV == 8 ? 2 * e + r : e + 4 * r] = r == 1 ? x * HI : x;
                }
            constexpr int N = BV == 8 ? 4 : 8;
#pragma unroll
            for (int x = 0; x < 8 / N; ++x) {
                const int ch = BV == 8 ? 4 * (8 * (2 * b + x) + g8) : BV == 4 ? 8 * (8 * b + g8) : 32 * (4 * (b >> 1) + (g8 >> 1)) + 16 * (g8 & 1) + 8 * (b & 1);
                if (!mine || ch >= 32 * nu) continue;
                float y[N];
#pragma unroll
                for (int i = 0; i < N; ++i) y[i] = complete ? result(o[N * x + i], l, inv, val[ch + i]) : o[N * x + i];
                if (complete) {
                    store_out<N>(p, c.s, head0 + q, ch, y);
                } else {
#pragma unroll
                    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(part + 4 + ch + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
                }
            }
        }
        if (complete) return;
        // The pair's first tile is in the share of group g_first. The last of its parts to arrive joins them, in the order of the shares. Many
        // parts are joined in runs first, by the last of each run, and the run's sum takes the place of its first part.
        const int g_first = (c.begin + PAIR_COST) / share, n_parts = (c.begin + PAIR_COST + c.nt - 1) / share - g_first + 1;
        const int run = n_parts <= MANY_PARTS ? 1 : ((int)sqrtf((float)n_parts) + 8) & ~7;
#pragma unroll 1
        for (int level = run == 1 ? 1 : 0; level < 2; ++level) {
            // what I may have to join: `count` parts, `step` apart, or the runs' sums
            const int from = level == 0 ? (me - g_first) / run * run : 0;
            const int step = level == 0 ? 1 : run, count = level == 0 ? min(run, n_parts - from) : (n_parts + run - 1) / run;
            __threadfence();
            __syncwarp();
            int last = 0;
            if (lane == 0) {
                // A count is 0 again after every call. What is no count of this process lacks its mark: one of those that come first puts a
                // count in its place.
                unsigned long long* at = p.arrived + ((g_first + from) * 3 + (level == 1 ? 2 : from == 0)) * warps + warp;
                unsigned long long before = atomicAdd(at, 1ull);
                for (int tries = 0; (before & ~0xFFFFull) != p.mark && tries < MAX_TRIES; ++tries) {
                    const unsigned long long seen = *reinterpret_cast<volatile unsigned long long*>(at);
                    if ((seen & ~0xFFFFull) == p.mark) before = atomicAdd(at, 1ull);
                    else if (atomicCAS(at, seen, p.mark + 1) == seen) before = p.mark;
                }
                last = before == p.mark + (unsigned)(count - 1);
                if ((before & ~0xFFFFull) != p.mark && p.status) atomicExch(p.status, RPTQ_ERR_DEVICE_TIMEOUT);
                if (last) *reinterpret_cast<volatile unsigned long long*>(at) = p.mark;
            }
            if (!__shfl_sync(0xffffffffu, last, 0)) return;
            __threadfence();
            // the parts of both heads in a row, AHEAD of them under way; a running reference as for the tiles
            constexpr int AHEAD = UN <= 4 ? 8 : 4, V = UN <= 4 ? 1 : 2;        // four channels a lane, twice
            const int all = count * n_heads;
            float4 o[V];
            float2 sz[V][4];
            float top = NO_REF;
            int head = 0, i = 0;                                               // head and part of the next sum
#pragma unroll
            for (int x = 0; x < V; ++x)
#pragma unroll
                for (int k = 0; k < 4; ++k) sz[x][k] = val[min(4 * lane + 128 * x, 32 * nu - 4) + k];
            l = 0.f;
#pragma unroll
            for (int x = 0; x < V; ++x) o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
            for (int n0 = 0; n0 < all; n0 += AHEAD) {
                float4 v[AHEAD][V];
                float2 sums[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const int n = min(n0 + k, all - 1), second = n >= count, b = from + (n - (second ? count : 0)) * step;
                    const float* at = part_of(g_first + b, b == 0, second);
                    sums[k] = __ldcg(reinterpret_cast<const float2*>(at));
#pragma unroll
                    for (int x = 0; x < V; ++x) v[k][x] = __ldcg(reinterpret_cast<const float4*>(at + 4 + min(4 * lane + 128 * x, 32 * nu - 4)));
                }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    if (n0 + k >= all) break;
                    const float to = fmaxf(top, sums[k].x), f = ex2(fmaxf(top - to, -1000.0f)), g = ex2(fmaxf(sums[k].x - to, -1000.0f));
                    top = to;
                    l = __fmaf_rn(g, sums[k].y, f * l);
#pragma unroll
                    for (int x = 0; x < V; ++x) {
                        o[x].x = __fmaf_rn(g, v[k][x].x, f * o[x].x); o[x].y = __fmaf_rn(g, v[k][x].y, f * o[x].y);
                        o[x].z = __fmaf_rn(g, v[k][x].z, f * o[x].z); o[x].w = __fmaf_rn(g, v[k][x].w, f * o[x].w);
                    }
                    if (++i < count) continue;
                    float* sum = part_of(g_first + from, from == 0, head);
                    __syncwarp();                                              // every lane has read the first part's reference and sum, which lane 0 replaces
                    if (level == 0 && lane == 0) *reinterpret_cast<float2*>(sum) = make_float2(top, l);
                    const float to_one = 1.0f / l;
#pragma unroll
                    for (int x = 0; x < V; ++x) {
                        const int ch = 4 * lane + 128 * x;
                        if (ch < 32 * nu) {
                            if (level == 0) {
                                *reinterpret_cast<float4*>(sum + 4 + ch) = o[x];
                            } else {
                                const float y[4] = {result(o[x].x, l, to_one, sz[x][0]), result(o[x].y, l, to_one, sz[x][1]), result(o[x].z, l, to_one, sz[x][2]),
                                                    result(o[x].w, l, to_one, sz[x][3])};
                                store_out<4>(p, c.s, head0 + head, ch, y);
                            }
                        }
                        o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                    top = NO_REF; l = 0.f; i = 0;
                    ++head;
                }
            }
        }
    };

    bool begins = true;
    int out_stage = 0;
    load_query(c);
#pragma unroll 1
    while (c.ok) {
        if (begins) start_pair();
        if constexpr (R == 1) {
            issue();
            cp_async_wait<STAGES - 1>();
            __syncwarp();
        } else {
            cp_async_wait<STAGES - 2>();
            sync_group();                                      // everybody's copies of this tile are here, and the tile before is done with
            issue();
        }
        begins = --c.n == 0;                                   // of the next pair
        if (begins) {
            Cursor next = c;
            next_pair(p, pairs, share == 0, n_groups, end, next);
            if (next.ok) load_query(next);
        }
        if (R == 1 || n_heads > 0) work(ring + out_stage * stage, ring + out_stage * stage + 2 * k_slab);
        out_stage = out_stage + 1 == STAGES ? 0 : out_stage + 1;
        ++c.t;
        if (begins) {
            if (R == 1 || n_heads > 0) finish();
            next_pair(p, pairs, share == 0, n_groups, end, c);
            first_t = 0;
        }
    }
    cp_async_wait<0>();
}

}  // namespace attn_paged
}  // namespace rptq
