// The paged key / value cache: its handle, and where a code lies in a page. Shared by kv_cache.cu (which writes and reads pages) and
// attention_paged.cu (which attends over them).
//
// A page holds page_size keys of every head: [head][slab of 16 keys]. A head's channels are kept in their own order, rounded up to
// units of 32 (what pads hold does not matter: their integers of the query are 0, their outputs are not stored). The reorder's
// clusters do not appear: attention multiplies the query by the channels' scales first, so that one sum over all channels takes the place of a sum per cluster, and a cluster need not start at a unit of its own. (Four clusters
// of 128 channels take 4 units here and about 5.5 in a row of the padded layout.)
// 32 codes of a unit are BITS words in both tensors: with 4 and 8 bits those of the library's packed format. With 3 bits a byte holds two codes
// and two single bits, so that AND and the byte itself bring them apart as far as a product needs (c0, c0 + 8 c1, c0 + 8 c1 + 64 b; the
// differences are taken of the factors or of the sums): of each half of 16 codes
//   A byte i = 0..3   c[i] | c[4 + i] << 3 | (c[12 + i] & 3) << 6                                   words 0 and 1: the halves' A
//   C byte i = 0, 1   c[8 + i] | c[10 + i] << 3 | (c[12 + 2 i] >> 2) << 6 | (c[13 + 2 i] >> 2) << 7     word 2: C of the first half, of the second
// What differs between the tensors is the order of a slab's bytes:
//   K   the tensor-core operand is keys x channels: a lane reads one key's 16 bytes. Units are taken four at a time (8 bits: two), so
//       that the four lanes of a row group read 64 contiguous bytes of a key and neighbouring keys follow: 128 bytes, all banks, per
//       eight lanes. 4 bits: [quad of units][key][unit][word]; 8 bits: the same with a unit as two pieces of four words;
//       3 bits: [quad][word 0..2][key][unit], a word at a time.
//   V   the operand is channels x keys with four keys in a register: byte e of word W of the four keys 4 t .. 4 t + 3 are one word,
//       [W][t][e][key in four]. No bytes have to be brought together when the cache is read, and a token that is
//       written owns its bytes.
#pragma once
#include "rptq_internal.h"

struct rptq_kv_cache {
    int C = 0, H = 0, d = 0, nu = 0, P = 0, device = -1;   // channels, cached heads, channels and units per head, keys per page
    struct Tensor {
        int bits = 0, K_pad = 0;
        int64_t row_bytes = 0, slab_bytes = 0, page_bytes = 0;
        const float2* quant = nullptr;     // [H * 32 nu] {inv_s, bits of z - 0x4B400000}; pads give code 0
        const float2* value = nullptr;     // [H * 32 nu] {s, (float) z}
        const uint8_t* centre = nullptr;   // [H * 32 nu] z, or the code nearest to it: what sums of codes are counted from
        const float2* rest = nullptr;      // [H * 32 nu] {s, (float) (z - centre)}
        const uint16_t* pos = nullptr;     // [C] position of the channel in a code row of the layout
        const int32_t* chan = nullptr;     // [K_pad] channel at the position, -1 at pads
    } k, v;
    void* tables = nullptr;          // all of the device tables
};

namespace rptq {
namespace kv {

constexpr int SLAB = 16;             // keys
constexpr int MAX_UNITS = 8;         // of a head: at most 256 channels

// Byte of word w (of the unit's BITS) of unit u, key r of a K slab; nu units in the head.
template <int BITS>
__host__ __device__ __forceinline__ int k_word(int nu, int u, int w, int r)
{
    if constexpr (BITS == 3) {
        const int j = u >> 2, n = nu - 4 * j < 4 ? nu - 4 * j : 4;
        return SLAB * (48 * j + 4 * n * w) + (n * r + (u & 3)) * 4;
    } else {
        const int piece = BITS == 4 ? u : 2 * u + (w >> 2), pieces = BITS == 4 ? nu : 2 * nu;
        const int j = piece >> 2, n = pieces - 4 * j < 4 ? pieces - 4 * j : 4;
        return SLAB * 64 * j + (n * r + (piece & 3)) * 16 + 4 * (w & 3);
    }
}

// Byte of byte e of word w of unit u, key r of a V slab.
template <int BITS>
__host__ __device__ __forceinline__ int v_byte(int u, int w, int e, int r) { return 64 * (BITS * u + w) + 16 * (r >> 2) + 4 * e + (r & 3); }

// 3 bits: the page's words of a unit's 32 codes.
__device__ __forceinline__ void pack_three(const uint32_t (&q)[32], uint32_t (&w)[3])
{
    w[0] = w[1] = w[2] = 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t* c = q + 16 * h;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[h] |= (c[i] | (c[4 + i] << 3) | ((c[12 + i] & 3u) << 6)) << (8 * i);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w[2] |= (c[8 + i] | (c[10 + i] << 3) | ((c[12 + 2 * i] >> 2) << 6) | ((c[13 + 2 * i] >> 2) << 7)) << (8 * (2 * h + i));
    }
}
// Code `at` of the unit; byte(word, e): byte e of a word.
template <class Byte>
__device__ __forceinline__ uint32_t code_of_three(Byte byte, int at)
{
    const int h = at >> 4, c = at & 15, i = c & 3;
    if (c < 4) return byte(h, i) & 7u;
    if (c < 8) return (byte(h, i) >> 3) & 7u;
    if (c < 10) return byte(2, 2 * h + (c & 1)) & 7u;
    if (c < 12) return (byte(2, 2 * h + (c & 1)) >> 3) & 7u;
    return (byte(h, i) >> 6) | (((byte(2, 2 * h + (i >> 1)) >> (6 + (i & 1))) & 1u) << 2);
}

// A slot or page outside its pool. A time-out that is recorded already stays: it says that an output is undefined, this only that something was
// left out.
__device__ __forceinline__ void record_bad_slot(int* status)
{
    if (status) atomicCAS(status, RPTQ_OK, RPTQ_ERR_BAD_SLOT);
}

// Where a slot's slab begins in the pool: page, head, slab of the page.
__host__ __device__ __forceinline__ int64_t slab_offset(int64_t page, int64_t page_bytes, int head, int slabs_per_page, int slab, int64_t slab_bytes)
{
    return page * page_bytes + ((int64_t)head * slabs_per_page + slab) * slab_bytes;
}

}  // namespace kv
}  // namespace rptq
