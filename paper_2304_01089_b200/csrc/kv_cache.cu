// The paged key / value cache: handle, quantise-on-write and read-back.
//
// Writing reads 2 to 4 bytes and writes 3 to 8 bits an element, reading back the reverse: both are bound by memory. A warp takes 256 channels
// (8 a lane: one 16-byte access of 16-bit rows, one word of 4-bit codes) of the tokens of a window, and keeps their parameters in
// registers. Tokens whose slots follow one another inside a group of four keys (a prompt's, whatever key it starts at) are taken together: the
// bytes of V that one token owns lie four apart, but four tokens' bytes of a word are 16 in a row (a 4 x 4 transposition in registers). One
// token alone writes its bytes one by one.
// The next group's loads are under way while a group is worked on. Rows of values are read and written past the caches (they are
// used once; with the default policy writing and reading 4096 tokens took 77 us instead of 72).
// Measured (4096 tokens, 72 heads of 128 channels, 4 bits, fp16, caches cold): writing 41 us, 4.6 TB/s; reading back 34 us, 5.6 TB/s.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <climits>
#include <cstring>
#include <new>
#include <type_traits>

#include "kv_pages.cuh"
#include "pack.cuh"
#include "tc.cuh"
#include "unpack.cuh"

namespace rptq {
namespace kv {

constexpr int THREADS = 128;

// One tensor (K or V) of a call.
struct Side {
    int bits;
    int64_t slab_bytes, page_bytes;
    const float2 *quant, *value;
    const uint16_t* pos;
    const int32_t* chan;
    int n_units_row;               // units of a code row
    uint8_t* pages;
    void* rows;
    int64_t ld;                    // elements (bytes for code rows) between rows
    int vector;                    // rows may be read and written 16 bytes at a time
};
struct Params {
    Side side[2];                  // K, V
    const int64_t* slots;
    int n_tokens, H, d, nu, P;
    int window;                    // tokens of a warp, 1 .. MAX_WINDOW
    int64_t n_slots;
    int* status;
};

__device__ __forceinline__ int64_t page_of(int64_t slot, int P) { return slot >> 31 ? slot / P : (int64_t)((uint32_t)slot / (uint32_t)P); }

// A token's key in its page; false: the token is left alone.
__device__ __forceinline__ bool find_slot(const Params& p, int token, int64_t& page, int& key)
{
    const int64_t slot = p.slots[token];
    if (slot < 0) return false;
    if (slot >= p.n_slots) {
        record_bad_slot(p.status);
        return false;
    }
    page = page_of(slot, p.P);
    key = (int)(slot - page * p.P);
    return true;
}

template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Code at position `pos` of a packed code row (rows are 4-byte aligned).
template <int BITS>
__device__ __forceinline__ uint32_t row_code(const uint8_t* row, int pos)
{
    if constexpr (BITS == 8) return row[pos];
    if constexpr (BITS == 4) return (row[(pos >> 3) * 4 + (pos & 3)] >> (pos & 4)) & 15u;
    const uint8_t* u = row + (pos >> 5) * 12;
    const int r = pos & 31, t = r & 7, at = t & 3, sh = t & 4;
    if (r < 24) return (u[4 * (r >> 3) + at] >> sh) & 7u;
    return ((u[at] >> (sh + 3)) & 1u) | (((u[4 + at] >> (sh + 3)) & 1u) << 1) | (((u[8 + at] >> (sh + 3)) & 1u) << 2);
}

// ---------------------------------------------------------------- rows of values
// The tokens that go together among first .. end - 1, at most MAX_WINDOW: lane l stands for token first + l. A token leads when it is the
// first of its call in a group of four keys whose slots follow one another; `n` tokens from it on are its group.
constexpr int MAX_WINDOW = 16;
struct Window {
    int64_t at;                    // byte of the token's slab of head 0 in the pool
    int key_n;                     // 8 (key in the slab) + n
    uint32_t leaders;
};
__device__ __forceinline__ Window find_groups(const Params& p, const Side& s, int first, int end)
{
    const int lane = threadIdx.x & 31, i = first + lane;
    const int64_t before = i > 0 && i <= p.n_tokens ? p.slots[i - 1] : -2;     // the one load: a lane's slot is the next lane's `before`
    const int64_t slot = __shfl_down_sync(0xffffffffu, before, 1);
    const int in_four = (int)(slot & 3);
    int n = 1;
#pragma unroll
    for (int k = 1; k < 4; ++k) {
        const int64_t next = __shfl_down_sync(0xffffffffu, before, 1 + k);
        if (n == k && in_four + k < 4 && next == slot + k && next < p.n_slots) ++n;
    }
    Window w{0, 0, 0u};
    bool leads = false;
    if (i < end && slot >= 0) {
        if (slot >= p.n_slots) {
            record_bad_slot(p.status);
        } else {
            leads = in_four == 0 || before != slot - 1;
            const int64_t page = page_of(slot, p.P);
            const int key = (int)(slot - page * p.P);
            w.at = page * s.page_bytes + (int64_t)(key / SLAB) * s.slab_bytes;
            w.key_n = 8 * (key % SLAB) + n;
        }
    }
    w.leaders = __ballot_sync(0xffffffffu, leads);
    return w;
}
// Eight channels of a head: the lane's place among all heads' groups of eight.
struct Place {
    int h, u, w, ch, real;         // head, unit, group of the unit, first channel in the head, channels that exist
    bool valid;
};
__device__ __forceinline__ Place find_place(const Params& p, int group)
{
    Place x;
    x.valid = group < p.H * p.nu * 4;
    const int unit = x.valid ? group >> 2 : 0;
    x.h = unit / p.nu;
    x.u = unit - x.h * p.nu;
    x.w = group & 3;
    x.ch = 32 * x.u + 8 * x.w;
    x.real = x.valid ? min(max(p.d - x.ch, 0), 8) : 0;
    return x;
}
// byte e of word k -> byte k of word e
__device__ __forceinline__ void transpose4(uint32_t (&w)[4])
{
    const uint32_t a = __byte_perm(w[0], w[1], 0x5140), b = __byte_perm(w[0], w[1], 0x7362);
    const uint32_t c = __byte_perm(w[2], w[3], 0x5140), d = __byte_perm(w[2], w[3], 0x7362);
    w[0] = __byte_perm(a, c, 0x5410); w[1] = __byte_perm(a, c, 0x7632);
    w[2] = __byte_perm(b, d, 0x5410); w[3] = __byte_perm(b, d, 0x7632);
}

// Eight elements of a row as raw 16-byte vectors.
template <class T> struct Raw { static constexpr int N = sizeof(T) / 2; uint4 v[N]; };
template <class T> struct Rows { Raw<T> of[4]; };                   // of four tokens
template <int N> struct Words { uint32_t w[N][4]; };                // N words of four tokens
template <class T, bool VECTOR>
__device__ __forceinline__ Raw<T> load8(const T* from, int real)
{
    Raw<T> r;
    if constexpr (VECTOR) {
#pragma unroll
        for (int i = 0; i < Raw<T>::N; ++i) r.v[i] = real > 0 ? __ldcs(reinterpret_cast<const uint4*>(from) + i) : make_uint4(0, 0, 0, 0);
    } else {
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < real ? from[i] : from_float<T>(0.f);
        memcpy(&r, e, sizeof r);
    }
    return r;
}
// Elements 2 i, 2 i + 1.
template <class T> __device__ __forceinline__ float2 pair_of(const Raw<T>& r, int i);
template <> __device__ __forceinline__ float2 pair_of(const Raw<float>& r, int i)
{
    const uint4 v = r.v[i >> 1];
    return i & 1 ? make_float2(__uint_as_float(v.z), __uint_as_float(v.w)) : make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
}
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
template <> __device__ __forceinline__ float2 pair_of(const Raw<__half>& r, int i)
{
    const uint32_t w = word_of(r.v[0], i);
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <> __device__ __forceinline__ float2 pair_of(const Raw<__nv_bfloat16>& r, int i)
{
    const uint32_t w = word_of(r.v[0], i);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
// Two numbers into elements 2 i, 2 i + 1.
__device__ __forceinline__ uint32_t join2(float2 x, __half) { const __half2 h = __float22half2_rn(x); return *reinterpret_cast<const uint32_t*>(&h); }
__device__ __forceinline__ uint32_t join2(float2 x, __nv_bfloat16) { const __nv_bfloat162 h = __float22bfloat162_rn(x); return *reinterpret_cast<const uint32_t*>(&h); }

template <int BITS, bool V, class T>
__device__ __forceinline__ void write_rows(const Params& p, const Side& s, int first, int end, int chunk)
{
    const int lane = threadIdx.x & 31;
    const Place at = find_place(p, 32 * chunk + lane);
    float2 inv[4];
    int zc[8];
    const float4* par = reinterpret_cast<const float4*>(s.quant + ((int64_t)at.h * p.nu * 32 + at.ch));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 x = par[i];
        inv[i] = make_float2(x.x, x.z); zc[2 * i] = __float_as_int(x.y); zc[2 * i + 1] = __float_as_int(x.w);
    }
    constexpr int WORDS = BITS == 8 ? 2 : 1;               // a lane's (3 bits: the unit's first and third lane have A, the second has C)
    const bool writes = at.valid && (BITS == 3 ? at.w < 3 : at.real > 0);
    const int word = BITS == 8 ? 2 * at.w : BITS == 4 ? at.w : (3 - at.w) % 3;
    // my first word of key 0 of the head's first slab, and the bytes between keys
    uint8_t* const mine = s.pages + slab_offset(0, 0, at.h, p.P / SLAB, 0, s.slab_bytes) + (V ? v_byte<BITS>(at.u, writes ? word : 0, 0, 0) : k_word<BITS>(p.nu, at.u, writes ? word : 0, 0));
    const int key_step = V ? 0 : k_word<BITS>(p.nu, at.u, 0, 1) - k_word<BITS>(p.nu, at.u, 0, 0);
    const T* const row0 = static_cast<const T*>(s.rows) + (int64_t)first * s.ld + at.h * p.d + at.ch;
    const Window groups = find_groups(p, s, first, end);

    // n tokens; FOUR: n == 4
    auto group = [&](const Rows<T>& rows, uint8_t* slab, int r, int n, auto four) {
        constexpr bool FOUR = decltype(four)::value;
        uint32_t w[WORDS][4] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!FOUR && k >= n) break;
            int v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 t = tc::fma2(pair_of(rows.of[k], i), inv[i], make_float2(12582912.0f, 12582912.0f));
                v[2 * i] = quant_int(t.x, zc[2 * i]);
                v[2 * i + 1] = quant_int(t.y, zc[2 * i + 1]);
            }
            if constexpr (BITS == 8) {
                w[0][k] = sat_pack_u8(v[1], v[0], sat_pack_u8(v[3], v[2], 0u));
                w[1][k] = sat_pack_u8(v[5], v[4], sat_pack_u8(v[7], v[6], 0u));
            } else if constexpr (BITS == 4) {
                w[0][k] = sat_nibble_word(v);
            } else {
                // code i in the low nibble of byte i, code 4 + i in the high one; odd lanes have codes 8 .. 15 of the half
                const uint32_t x = sat_nibble_word_max7(v), beside = __shfl_xor_sync(0xffffffffu, x, 1);
                const uint32_t c = (x & 0x0747u) | ((x >> 13) & 0x3838u) | ((x >> 7) & 0x80u) | ((x >> 8) & 0x4000u) | ((x >> 15) & 0x8000u);
                const uint32_t other = __shfl_xor_sync(0xffffffffu, c, 2);
                w[0][k] = at.w & 1 ? c | (other << 16) : (x & 0x07070707u) | ((x >> 1) & 0x38383838u) | ((beside << 2) & 0xC0C0C0C0u);
            }
        }
        if (!writes) return;
        if constexpr (!V) {
            uint8_t* to = slab + r * key_step;
#pragma unroll
            for (int k = 0; k < 4; ++k, to += key_step) {
                if (!FOUR && k >= n) break;
                if constexpr (BITS == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0][k], w[1][k]);
                else *reinterpret_cast<uint32_t*>(to) = w[0][k];
            }
        } else {
            uint8_t* to = slab + 16 * (r >> 2) + (r & 3);
#pragma unroll
            for (int x = 0; x < WORDS; ++x) {
                if constexpr (FOUR) {
                    transpose4(w[x]);
                    *reinterpret_cast<uint4*>(to + 64 * x) = make_uint4(w[x][0], w[x][1], w[x][2], w[x][3]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k >= n) break;
#pragma unroll
                        for (int e = 0; e < 4; ++e) to[64 * x + 4 * e + k] = (uint8_t)(w[x][k] >> (8 * e));
                    }
                }
            }
        }
    };
    // a group's rows are on their way while the one before is quantised
    Rows<T> rows, ahead;
    uint32_t left = groups.leaders;
    auto load = [&](Rows<T>& to) {
        const int l = __ffs(left) - 1, n = __shfl_sync(0xffffffffu, groups.key_n, l) & 7;
        const T* row = row0 + (int64_t)l * s.ld;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n) to.of[k] = s.vector ? load8<T, true>(row + k * s.ld, at.real) : load8<T, false>(row + k * s.ld, at.real);
    };
    if (left) load(rows);
    while (left) {
        const int l = __ffs(left) - 1, key_n = __shfl_sync(0xffffffffu, groups.key_n, l), r = key_n >> 3, n = key_n & 7;
        uint8_t* slab = mine + __shfl_sync(0xffffffffu, groups.at, l);
        left &= left - 1;
        if (left) load(ahead);
        if (n == 4) group(rows, slab, r, n, std::true_type());
        else group(rows, slab, r, n, std::false_type());
        rows = ahead;
    }
}

template <int BITS, bool V, class T>
__device__ __forceinline__ void read_rows(const Params& p, const Side& s, int first, int end, int chunk)
{
    const int lane = threadIdx.x & 31;
    const Place at = find_place(p, 32 * chunk + lane);
    float2 scale[4], zero[4];                              // zero: -(2^23 + z)
    const float4* par = reinterpret_cast<const float4*>(s.value + ((int64_t)at.h * p.nu * 32 + at.ch));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 x = par[i];
        scale[i] = make_float2(x.x, x.z); zero[i] = make_float2(-8388608.0f - x.y, -8388608.0f - x.w);
    }
    pdl_wait();                                            // (the handle's tables were there before any launch)
    constexpr int WORDS = BITS == 8 ? 2 : 1;
    const bool reads = at.valid && (BITS == 3 ? at.w < 3 : at.real > 0);
    const int word = BITS == 8 ? 2 * at.w : BITS == 4 ? at.w : (3 - at.w) % 3;
    const uint8_t* const mine = s.pages + slab_offset(0, 0, at.h, p.P / SLAB, 0, s.slab_bytes) + (V ? v_byte<BITS>(at.u, reads ? word : 0, 0, 0) : k_word<BITS>(p.nu, at.u, reads ? word : 0, 0));
    const int key_step = V ? 0 : k_word<BITS>(p.nu, at.u, 0, 1) - k_word<BITS>(p.nu, at.u, 0, 0);
    T* const row0 = static_cast<T*>(s.rows) + (int64_t)first * s.ld + at.h * p.d + at.ch;
    const Window groups = find_groups(p, s, first, end);

    auto load = [&](Words<WORDS>& to, int l) {
        const int key_n = __shfl_sync(0xffffffffu, groups.key_n, l), r = key_n >> 3, n = key_n & 7;
        const uint8_t* slab = mine + __shfl_sync(0xffffffffu, groups.at, l);
        if (reads) {
            if constexpr (!V) {
                const uint8_t* from = slab + r * key_step;
#pragma unroll
                for (int k = 0; k < 4; ++k, from += key_step) {
                    if (k >= n) break;
                    if constexpr (BITS == 8) {
                        const uint2 x = *reinterpret_cast<const uint2*>(from);
                        to.w[0][k] = x.x; to.w[1][k] = x.y;
                    } else {
                        to.w[0][k] = *reinterpret_cast<const uint32_t*>(from);
                    }
                }
            } else {
#pragma unroll
                for (int x = 0; x < WORDS; ++x) {
                    // all four keys' bytes, whichever of them are wanted
                    const uint4 y = *reinterpret_cast<const uint4*>(slab + 64 * x + 16 * (r >> 2));
                    to.w[x][0] = y.x; to.w[x][1] = y.y; to.w[x][2] = y.z; to.w[x][3] = y.w;
                }
            }
        }
    };
    auto group = [&](Words<WORDS> words, T* row, int r, int n, auto four, auto vector) {
        constexpr bool FOUR = decltype(four)::value, VECTOR = decltype(vector)::value;
        if constexpr (V) {
#pragma unroll
            for (int x = 0; x < WORDS; ++x) {
                uint32_t (&t)[4] = words.w[x];
                transpose4(t);
                if constexpr (!FOUR) {
                    const int skip = r & 3;
                    if (skip & 1) { t[0] = t[1]; t[1] = t[2]; t[2] = t[3]; }
                    if (skip & 2) { t[0] = t[2]; t[1] = t[3]; }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k, row += s.ld) {
            if (!FOUR && k >= n) break;
            uint32_t q[2];                                 // codes as bytes
            if constexpr (BITS == 8) {
                q[0] = words.w[0][k]; q[1] = words.w[1][k];
            } else if constexpr (BITS == 4) {
                const uint32_t x = words.w[0][k];
                q[0] = x & 0x0F0F0F0Fu; q[1] = (x >> 4) & 0x0F0F0F0Fu;
            } else {
                const uint32_t x = words.w[0][k], a = __shfl_sync(0xffffffffu, x, lane & ~1);
                const uint32_t c = __shfl_sync(0xffffffffu, x, (lane & ~3) + 1) >> (at.w == 3 ? 16 : 0);      // (its low half)
                if (at.w & 1) {
                    q[0] = (c & 0x0707u) | (((c >> 3) & 0x0707u) << 16);
                    q[1] = ((a >> 6) & 0x03030303u) | ((c >> 4) & 0x4u) | ((c << 3) & 0x400u) | ((c << 4) & 0x40000u) | ((c << 11) & 0x4000000u);
                } else {
                    q[0] = a & 0x07070707u; q[1] = (a >> 3) & 0x07070707u;
                }
            }
            float2 y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {                  // 2^23 + code, exactly; minus 2^23 + z, exactly; one rounding with s
                const uint32_t b = q[i >> 1];
                const float2 c = make_float2(__uint_as_float(__byte_perm(b, 0x4B000000u, i & 1 ? 0x7542u : 0x7540u)),
                                             __uint_as_float(__byte_perm(b, 0x4B000000u, i & 1 ? 0x7543u : 0x7541u)));
                y[i] = tc::mul2(tc::add2(c, zero[i]), scale[i]);
            }
            if (at.real == 0) continue;
            if constexpr (VECTOR) {
                if constexpr (std::is_same<T, float>::value) {
                    __stcs(reinterpret_cast<float4*>(row), make_float4(y[0].x, y[0].y, y[1].x, y[1].y));
                    __stcs(reinterpret_cast<float4*>(row) + 1, make_float4(y[2].x, y[2].y, y[3].x, y[3].y));
                } else {
                    __stcs(reinterpret_cast<uint4*>(row), make_uint4(join2(y[0], T()), join2(y[1], T()), join2(y[2], T()), join2(y[3], T())));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < at.real) row[i] = from_float<T>(i & 1 ? y[i >> 1].y : y[i >> 1].x);
            }
        }
    };
    Words<WORDS> words{}, ahead{};
    uint32_t left = groups.leaders;
    if (left) load(words, __ffs(left) - 1);
    while (left) {
        const int l = __ffs(left) - 1, key_n = __shfl_sync(0xffffffffu, groups.key_n, l), r = key_n >> 3, n = key_n & 7;
        T* row = row0 + (int64_t)l * s.ld;
        left &= left - 1;
        if (left) load(ahead, __ffs(left) - 1);
        using Yes = std::true_type; using No = std::false_type;
        if (!s.vector) group(words, row, r, n, No(), No());
        else if (n == 4) group(words, row, r, n, Yes(), Yes());
        else group(words, row, r, n, No(), Yes());
        words = ahead;
    }
}

// A warp takes a chunk of 256 channels of K or V (blockIdx.y) and a window of the tokens; the four warps of a block take neighbouring
// chunks. Six blocks per SM write (80 registers; rows of fp32 four, 128), eight read (64). (Parts as long as make all warps resident at once, K's and V's at the same
// time, were 15 % slower when that was tried, before the rows passed the caches by: 90 us against 77 for writing and reading 4096 tokens.)
template <class T> constexpr int rows_blocks_per_sm(bool write) { return !write ? 8 : sizeof(T) == 4 ? 4 : 6; }
template <class T, bool WRITE>
__global__ void __launch_bounds__(THREADS, rows_blocks_per_sm<T>(WRITE)) rows_kernel(const Params p)
{
    pdl_trigger();
    if constexpr (WRITE) pdl_wait();                       // (inside, behind the loads of the parameters, it costs the write's instances registers)
    const int n_chunks = (p.H * p.nu * 4 + 31) / 32;
    const int64_t id = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5), window = id / n_chunks;
    const bool is_v = blockIdx.y != 0;
    const int chunk = (int)(id - window * n_chunks);
    if (window * p.window >= p.n_tokens) { if constexpr (!WRITE) pdl_wait(); return; }
    const int first = (int)window * p.window, end = (int)min((int64_t)first + p.window, (int64_t)p.n_tokens);
    const Side& s = p.side[is_v];
    auto run = [&](auto bits) {
        constexpr int BITS = decltype(bits)::value;
        if (!is_v) {
            if constexpr (WRITE) write_rows<BITS, false, T>(p, s, first, end, chunk);
            else read_rows<BITS, false, T>(p, s, first, end, chunk);
        } else {
            if constexpr (WRITE) write_rows<BITS, true, T>(p, s, first, end, chunk);
            else read_rows<BITS, true, T>(p, s, first, end, chunk);
        }
    };
    if (s.bits == 3) run(std::integral_constant<int, 3>());
    else if (s.bits == 4) run(std::integral_constant<int, 4>());
    else run(std::integral_constant<int, 8>());
}

// ---------------------------------------------------------------- code rows
template <int BITS>
__device__ __forceinline__ void store_unit(uint8_t* slab, bool is_v, int nu, int u, int r, const uint32_t (&w)[BITS])
{
#pragma unroll
    for (int i = 0; i < BITS; ++i) {
        if (is_v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) slab[v_byte<BITS>(u, i, e, r)] = (uint8_t)(w[i] >> (8 * e));
        } else {
            *reinterpret_cast<uint32_t*>(slab + k_word<BITS>(nu, u, i, r)) = w[i];
        }
    }
}
// One thread per unit of a token's head.
template <int BITS>
__device__ void write_code_rows(const Params& p, const Side& s, bool is_v)
{
    const int64_t n = (int64_t)p.n_tokens * p.H * p.nu;
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * THREADS) {
        const int token = (int)(i / (p.H * p.nu)), hu = (int)(i - (int64_t)token * (p.H * p.nu)), h = hu / p.nu, u = hu - h * p.nu;
        int64_t page; int key;
        if (!find_slot(p, token, page, key)) continue;
        uint32_t q[32], w[BITS];
        const int ch0 = h * p.d + 32 * u, real = min(32, p.d - 32 * u);
        const uint8_t* row = static_cast<const uint8_t*>(s.rows) + (int64_t)token * s.ld;
#pragma unroll
        for (int c = 0; c < 32; ++c) q[c] = c < real ? row_code<BITS>(row, s.pos[ch0 + c]) : 0u;
        if constexpr (BITS == 3) pack_three(q, w);
        else pack32<BITS>(q, w);
        store_unit<BITS>(s.pages + slab_offset(page, s.page_bytes, h, p.P / SLAB, key / SLAB, s.slab_bytes), is_v, p.nu, u, key % SLAB, w);
    }
}
// One thread per unit of the padded row.
template <int BITS>
__device__ void read_code_rows(const Params& p, const Side& s, bool is_v)
{
    const int64_t n = (int64_t)p.n_tokens * s.n_units_row;
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * THREADS) {
        const int token = (int)(i / s.n_units_row), unit = (int)(i - (int64_t)token * s.n_units_row);
        int64_t page; int key;
        if (!find_slot(p, token, page, key)) continue;
        uint32_t q[32], w[BITS];
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            const int ch = s.chan[32 * unit + c];
            q[c] = 0;
            if (ch < 0) continue;
            const int h = ch / p.d, in_head = ch - h * p.d, u = in_head >> 5, at = in_head & 31;
            const uint8_t* slab = s.pages + slab_offset(page, s.page_bytes, h, p.P / SLAB, key / SLAB, s.slab_bytes);
            const int r = key % SLAB, b = at & 3, sh = at & 4;
            auto byte = [&](int word) -> uint32_t { return is_v ? slab[v_byte<BITS>(u, word, b, r)] : slab[k_word<BITS>(p.nu, u, word, r) + b]; };
            if constexpr (BITS == 8) q[c] = byte(at >> 2);
            else if constexpr (BITS == 4) q[c] = (byte(at >> 3) >> sh) & 15u;
            else q[c] = code_of_three([&](int w, int e) -> uint32_t { return is_v ? slab[v_byte<BITS>(u, w, e, r)] : slab[k_word<BITS>(p.nu, u, w, r) + e]; }, at);
        }
        pack32<BITS>(q, w);
        uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(s.rows) + (int64_t)token * s.ld) + (int64_t)unit * BITS;
#pragma unroll
        for (int k = 0; k < BITS; ++k) out[k] = w[k];
    }
}
template <bool WRITE>
__global__ void __launch_bounds__(THREADS) code_rows_kernel(const Params p)
{
    pdl_trigger();
    pdl_wait();
    const bool is_v = blockIdx.y != 0;
    const Side& s = p.side[blockIdx.y];
    if constexpr (WRITE) {
        if (s.bits == 3) write_code_rows<3>(p, s, is_v);
        else if (s.bits == 4) write_code_rows<4>(p, s, is_v);
        else write_code_rows<8>(p, s, is_v);
    } else {
        if (s.bits == 3) read_code_rows<3>(p, s, is_v);
        else if (s.bits == 4) read_code_rows<4>(p, s, is_v);
        else read_code_rows<8>(p, s, is_v);
    }
}

// Tokens per warp: as many as leave WARPS_PER_SM warps for every SM. (Measured with 8, 16, 32, 64: one token and 16 rows back for eight sequences 6.9,
// 7.1, 8.7, 8.7 us; chunks of 333 tokens for three 15.6, 11.5, 12.8, 16.3; 2011 rows of 3 bits 18.2, 18.2, 18.2, 20.7; 4096 tokens 68 with each.)
constexpr int WARPS_PER_SM = 16;
template <class T, bool WRITE>
static int launch_values(Params& p, int n_sm, cudaStream_t st)
{
    const int64_t n_chunks = (p.H * p.nu * 4 + 31) / 32;
    auto windows = [&]() { return ((int64_t)p.n_tokens + p.window - 1) / p.window; };
    p.window = MAX_WINDOW;
    while (p.window > 1 && windows() * n_chunks * 2 < (int64_t)n_sm * WARPS_PER_SM) p.window /= 2;
    const int64_t blocks = (windows() * n_chunks + THREADS / 32 - 1) / (THREADS / 32);
    if (blocks > INT_MAX) return RPTQ_ERR_UNSUPPORTED;
    return launch_kernel(rows_kernel<T, WRITE>, dim3((unsigned)blocks, 2), THREADS, 0, 0, st, p);
}
template <bool WRITE>
static int launch_rows(Params& p, int rows_type, int n_sm, cudaStream_t st)
{
    if (rows_type == RPTQ_ROWS_CODES) {
        const int units = WRITE ? p.H * p.nu : p.side[0].n_units_row > p.side[1].n_units_row ? p.side[0].n_units_row : p.side[1].n_units_row;
        const int64_t want = ((int64_t)p.n_tokens * units + THREADS - 1) / THREADS, most = (int64_t)n_sm * 16;
        return launch_kernel(code_rows_kernel<WRITE>, dim3((unsigned)(want < most ? want : most), 2), THREADS, 0, 0, st, p);
    }
    if (rows_type == RPTQ_ROWS_F32) return launch_values<float, WRITE>(p, n_sm, st);
    if (rows_type == RPTQ_ROWS_F16) return launch_values<__half, WRITE>(p, n_sm, st);
    return launch_values<__nv_bfloat16, WRITE>(p, n_sm, st);
}

static int element_bytes(int rows_type) { return rows_type == RPTQ_ROWS_F32 ? 4 : rows_type == RPTQ_ROWS_CODES ? 1 : 2; }

// Checks of a write or read call and its launch parameters.
static int make_params(const rptq_kv_cache_t* c, const void* k, int64_t ldk, const void* v, int64_t ldv, int rows_type, const int64_t* slots,
                       int n_tokens, const void* k_pages, const void* v_pages, int64_t n_pages, Params* p, bool* nothing, int* n_sm)
{
    *nothing = false;
    if (!c || n_tokens < 0 || n_pages < 0) return RPTQ_ERR_INVALID_ARG;
    if (rows_type < RPTQ_ROWS_F32 || rows_type > RPTQ_ROWS_BF16) return RPTQ_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!k_pages || !v_pages)) return RPTQ_ERR_INVALID_ARG;
    if (!aligned16(k_pages) || !aligned16(v_pages)) return RPTQ_ERR_INVALID_ARG;
    if (n_pages > INT64_MAX / c->P) return RPTQ_ERR_UNSUPPORTED;
    if (n_tokens == 0) { *nothing = true; return RPTQ_OK; }
    if (!k || !v || !slots || (reinterpret_cast<uintptr_t>(slots) & 7u)) return RPTQ_ERR_INVALID_ARG;
    const int e = element_bytes(rows_type);
    const bool codes = rows_type == RPTQ_ROWS_CODES;
    const int64_t need_k = codes ? c->k.row_bytes : c->C, need_v = codes ? c->v.row_bytes : c->C;
    const uintptr_t mask = codes ? 3u : (uintptr_t)e - 1u;
    if (ldk < need_k || ldv < need_v || (codes && ((ldk | ldv) & 3))) return RPTQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(k) & mask) || (reinterpret_cast<uintptr_t>(v) & mask)) return RPTQ_ERR_INVALID_ARG;
    int dev = -1;
    if (c->device < 0 || cudaGetDevice(&dev) != cudaSuccess) return RPTQ_ERR_CUDA;
    if (dev != c->device) return RPTQ_ERR_INVALID_ARG;
    *n_sm = sm_count(dev);
    if (*n_sm == 0) return RPTQ_ERR_CUDA;
    for (int t = 0; t < 2; ++t) {
        const rptq_kv_cache::Tensor& x = t ? c->v : c->k;
        Side& s = p->side[t];
        s.bits = x.bits; s.slab_bytes = x.slab_bytes; s.page_bytes = x.page_bytes;
        s.quant = x.quant; s.value = x.value; s.pos = x.pos; s.chan = x.chan; s.n_units_row = x.K_pad / 32;
        s.pages = static_cast<uint8_t*>(const_cast<void*>(t ? v_pages : k_pages));
        s.rows = const_cast<void*>(t ? v : k);
        s.ld = t ? ldv : ldk;
        s.vector = aligned16(s.rows) && (s.ld * e) % 16 == 0 && c->d % 8 == 0;
    }
    p->slots = slots; p->n_tokens = n_tokens; p->H = c->H; p->d = c->d; p->nu = c->nu; p->P = c->P;
    p->n_slots = n_pages * c->P;
    p->status = device_status_word();
    return RPTQ_OK;
}

// The device tables of a handle, gathered on the host: one allocation and one copy.
struct Tables {
    std::vector<uint8_t> bytes;
    template <class T>
    size_t add(const std::vector<T>& x)
    {
        const size_t at = (bytes.size() + 15) / 16 * 16;
        bytes.resize(at + x.size() * sizeof(T));
        std::memcpy(bytes.data() + at, x.data(), x.size() * sizeof(T));
        return at;
    }
};
struct TensorTables { size_t quant, value, centre, rest, pos, chan; };

static TensorTables make_tensor(const rptq_layout_t* L, const rptq_kv_cache& c, rptq_kv_cache::Tensor& t, Tables& tables)
{
    t.bits = L->bits; t.K_pad = L->K_pad; t.row_bytes = L->row_bytes;
    t.slab_bytes = (int64_t)SLAB * c.nu * 4 * L->bits;
    t.page_bytes = t.slab_bytes * (c.P / SLAB) * c.H;
    const size_t n = (size_t)c.H * c.nu * 32;
    std::vector<float2> quant(n), value(n, make_float2(0.f, 0.f)), rest(value);
    std::vector<uint8_t> centre(n, 0);
    std::vector<uint16_t> pos((size_t)c.C);
    std::vector<int32_t> chan((size_t)L->K_pad, -1);
    const int32_t magic = -0x4B400000;                       // pads: 0 * 0 rounds to 0, code 0
    for (auto& q : quant) { q.x = 0.f; std::memcpy(&q.y, &magic, 4); }
    size_t j = 0;
    for (int cl = 0; cl < L->g; ++cl)
        for (int i = 0; i < L->size[(size_t)cl]; ++i, ++j) {
            const int ch = L->perm[j], h = ch / c.d;
            const size_t at = (size_t)h * c.nu * 32 + (size_t)(ch - h * c.d);
            const int32_t zc = L->zero[(size_t)cl] - 0x4B400000;
            quant[at].x = (float)(1.0 / (double)L->scale[(size_t)cl]);
            std::memcpy(&quant[at].y, &zc, 4);
            value[at] = make_float2(L->scale[(size_t)cl], (float)L->zero[(size_t)cl]);
            centre[at] = (uint8_t)std::min(std::max(L->zero[(size_t)cl], 0), (1 << L->bits) - 1);
            rest[at] = make_float2(L->scale[(size_t)cl], (float)(L->zero[(size_t)cl] - centre[at]));
            pos[(size_t)ch] = (uint16_t)L->pos[j];
            chan[(size_t)L->pos[j]] = ch;
        }
    return {tables.add(quant), tables.add(value), tables.add(centre), tables.add(rest), tables.add(pos), tables.add(chan)};
}
static void set_tables(rptq_kv_cache::Tensor& t, const TensorTables& at, const uint8_t* base)
{
    t.quant = reinterpret_cast<const float2*>(base + at.quant);
    t.value = reinterpret_cast<const float2*>(base + at.value);
    t.centre = base + at.centre;
    t.rest = reinterpret_cast<const float2*>(base + at.rest);
    t.pos = reinterpret_cast<const uint16_t*>(base + at.pos);
    t.chan = reinterpret_cast<const int32_t*>(base + at.chan);
}

}  // namespace kv
}  // namespace rptq

extern "C" {

int rptq_kv_cache_create(rptq_kv_cache_t** out, const rptq_layout_t* LK, const rptq_layout_t* LV, int n_heads, int page_size)
{
    using namespace rptq::kv;
    if (!out) return RPTQ_ERR_INVALID_ARG;
    *out = nullptr;
    if (!LK || !LV || n_heads < 1 || page_size < 1) return RPTQ_ERR_INVALID_ARG;
    if (LK->C != LV->C || LK->C % n_heads || LK->device != LV->device) return RPTQ_ERR_INVALID_ARG;
    if (LK->C / n_heads > 32 * MAX_UNITS || page_size % SLAB || page_size > 65536) return RPTQ_ERR_UNSUPPORTED;
    const int bits = LK->bits > LV->bits ? LK->bits : LV->bits;             // offsets inside a page are 32 bits
    if ((int64_t)page_size * n_heads * ((LK->C / n_heads + 31) / 32) * 4 * bits > INT_MAX) return RPTQ_ERR_UNSUPPORTED;
    int dev = -1;
    if (LK->device >= 0 && (cudaGetDevice(&dev) != cudaSuccess || dev != LK->device)) return RPTQ_ERR_INVALID_ARG;
    rptq_kv_cache_t* c = new (std::nothrow) rptq_kv_cache();
    if (!c) return RPTQ_ERR_ALLOC;
    c->C = LK->C; c->H = n_heads; c->d = LK->C / n_heads; c->nu = (c->d + 31) / 32; c->P = page_size; c->device = LK->device;
    int rc = RPTQ_OK;
    try {
        Tables tables;
        const TensorTables k = make_tensor(LK, *c, c->k, tables), v = make_tensor(LV, *c, c->v, tables);
        if (c->device >= 0) {                                               // (without a device the handle knows sizes only, as a layout does)
            if (cudaMalloc(&c->tables, tables.bytes.size()) != cudaSuccess) { c->tables = nullptr; rc = RPTQ_ERR_ALLOC; }
            else if (cudaMemcpy(c->tables, tables.bytes.data(), tables.bytes.size(), cudaMemcpyHostToDevice) != cudaSuccess ||
                     cudaStreamSynchronize(nullptr) != cudaSuccess) rc = RPTQ_ERR_CUDA;         // (other streams may use them at once)
            set_tables(c->k, k, static_cast<const uint8_t*>(c->tables));
            set_tables(c->v, v, static_cast<const uint8_t*>(c->tables));
        }
    } catch (const std::bad_alloc&) {
        rc = RPTQ_ERR_ALLOC;
    }
    if (rc != RPTQ_OK) { rptq_kv_cache_destroy(c); return rc; }
    *out = c;
    return RPTQ_OK;
}

int rptq_kv_cache_query(const rptq_kv_cache_t* cache, int64_t* k_page_bytes, int64_t* v_page_bytes)
{
    if (!cache) return RPTQ_ERR_INVALID_ARG;
    if (k_page_bytes) *k_page_bytes = cache->k.page_bytes;
    if (v_page_bytes) *v_page_bytes = cache->v.page_bytes;
    return RPTQ_OK;
}

int rptq_kv_cache_destroy(rptq_kv_cache_t* cache)
{
    if (!cache) return RPTQ_OK;
    cudaFree(cache->tables);
    delete cache;
    return RPTQ_OK;
}

int rptq_kv_cache_write(const rptq_kv_cache_t* cache, const void* k, int64_t ldk, const void* v, int64_t ldv, int rows_type,
                        const int64_t* slots, int n_tokens, void* k_pages, void* v_pages, int64_t n_pages, void* stream)
{
    using namespace rptq;
    using namespace rptq::kv;
    Params p{};
    bool nothing;
    int n_sm = 0;
    const int rc = make_params(cache, k, ldk, v, ldv, rows_type, slots, n_tokens, k_pages, v_pages, n_pages, &p, &nothing, &n_sm);
    if (rc != RPTQ_OK || nothing) return rc;
    return launch_rows<true>(p, rows_type, n_sm, static_cast<cudaStream_t>(stream));
}

int rptq_kv_cache_read(const rptq_kv_cache_t* cache, const void* k_pages, const void* v_pages, int64_t n_pages, const int64_t* slots,
                       int n_tokens, void* k, int64_t ldk, void* v, int64_t ldv, int rows_type, void* stream)
{
    using namespace rptq;
    using namespace rptq::kv;
    Params p{};
    bool nothing;
    int n_sm = 0;
    const int rc = make_params(cache, k, ldk, v, ldv, rows_type, slots, n_tokens, k_pages, v_pages, n_pages, &p, &nothing, &n_sm);
    if (rc != RPTQ_OK || nothing) return rc;
    return launch_rows<false>(p, rows_type, n_sm, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
