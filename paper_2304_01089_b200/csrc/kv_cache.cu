// The paged key / value cache: handle, quantise-on-write and read-back.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>
#include <cstring>
#include <new>

#include "kv_pages.cuh"
#include "pack.cuh"
#include "unpack.cuh"

namespace rptq {
namespace kv {

constexpr int THREADS = 128;

// One tensor (K or V) of a call.
struct Side {
    int bits;
    int64_t row_bytes, slab_bytes, page_bytes;
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
    int n_tokens, H, d, nu, P, C;
    int64_t n_slots;
    int* status;
};

// A token's key in its page; false: the token is left alone.
__device__ __forceinline__ bool find_slot(const Params& p, int token, int64_t& page, int& key)
{
    const int64_t slot = p.slots[token];
    if (slot < 0) return false;
    if (slot >= p.n_slots) {
        if (p.status) *p.status = RPTQ_ERR_BAD_SLOT;
        return false;
    }
    page = slot / p.P;
    key = (int)(slot - page * p.P);
    return true;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
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
template <int BITS>
__device__ __forceinline__ void load_unit(const uint8_t* slab, bool is_v, int nu, int u, int r, uint32_t (&w)[BITS])
{
#pragma unroll
    for (int i = 0; i < BITS; ++i) {
        if (is_v) {
            w[i] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[i] |= (uint32_t)slab[v_byte<BITS>(u, i, e, r)] << (8 * e);
        } else {
            w[i] = *reinterpret_cast<const uint32_t*>(slab + k_word<BITS>(nu, u, i, r));
        }
    }
}

// One thread per unit of a token's head.
template <int BITS, class T, bool CODES>
__device__ void write_units(const Params& p, const Side& s, bool is_v)
{
    const int64_t n = (int64_t)p.n_tokens * p.H * p.nu;
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * THREADS) {
        const int token = (int)(i / (p.H * p.nu)), hu = (int)(i - (int64_t)token * (p.H * p.nu)), h = hu / p.nu, u = hu - h * p.nu;
        int64_t page; int key;
        if (!find_slot(p, token, page, key)) continue;
        uint32_t q[32], w[BITS];
        const int ch0 = h * p.d + 32 * u, real = min(32, p.d - 32 * u);
        if constexpr (CODES) {
            const uint8_t* row = static_cast<const uint8_t*>(s.rows) + (int64_t)token * s.ld;
#pragma unroll
            for (int c = 0; c < 32; ++c) q[c] = c < real ? row_code<BITS>(row, s.pos[ch0 + c]) : 0u;
            pack32<BITS>(q, w);
        } else {
            const T* row = static_cast<const T*>(s.rows) + (int64_t)token * s.ld + ch0;
            const float2* par = s.quant + (int64_t)hu * 32;
            int v[32];
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                const float2 a = par[c];
                v[c] = quant_int(__fmaf_rn(c < real ? to_float(row[c]) : 0.f, a.x, 12582912.0f), __float_as_int(a.y));
            }
            pack32_sat<BITS>(v, w);
        }
        store_unit<BITS>(s.pages + slab_offset(page, s.page_bytes, h, p.P / SLAB, key / SLAB, s.slab_bytes), is_v, p.nu, u, key % SLAB, w);
    }
}
template <class T, bool CODES>
__global__ void __launch_bounds__(THREADS) write_kernel(const Params p)
{
    pdl_trigger();
    pdl_wait();
    const bool is_v = blockIdx.y != 0;
    const Side& s = p.side[blockIdx.y];
    if (s.bits == 3) write_units<3, T, CODES>(p, s, is_v);
    else if (s.bits == 4) write_units<4, T, CODES>(p, s, is_v);
    else write_units<8, T, CODES>(p, s, is_v);
}

template <int BITS, class T>
__device__ void read_units(const Params& p, const Side& s, bool is_v)
{
    const int64_t n = (int64_t)p.n_tokens * p.H * p.nu;
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * THREADS) {
        const int token = (int)(i / (p.H * p.nu)), hu = (int)(i - (int64_t)token * (p.H * p.nu)), h = hu / p.nu, u = hu - h * p.nu;
        int64_t page; int key;
        if (!find_slot(p, token, page, key)) continue;
        uint32_t w[BITS], o[8];
        load_unit<BITS>(s.pages + slab_offset(page, s.page_bytes, h, p.P / SLAB, key / SLAB, s.slab_bytes), is_v, p.nu, u, key % SLAB, w);
        unpack_act32<BITS>(w, o);
        const int ch0 = h * p.d + 32 * u, real = min(32, p.d - 32 * u);
        const float2* par = s.value + (int64_t)hu * 32;
        T* row = static_cast<T*>(s.rows) + (int64_t)token * s.ld + ch0;
#pragma unroll
        for (int c = 0; c < 32; ++c)
            if (c < real) row[c] = from_float<T>(((float)((o[c >> 2] >> (8 * (c & 3))) & 255u) - par[c].y) * par[c].x);
    }
}
// Code rows: one thread per unit of the padded row.
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
            else if (at < 24) q[c] = (byte(at >> 3) >> sh) & 7u;
            else q[c] = ((byte(0) >> (sh + 3)) & 1u) | (((byte(1) >> (sh + 3)) & 1u) << 1) | (((byte(2) >> (sh + 3)) & 1u) << 2);
        }
        pack32<BITS>(q, w);
        uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(s.rows) + (int64_t)token * s.ld) + (int64_t)unit * BITS;
#pragma unroll
        for (int k = 0; k < BITS; ++k) out[k] = w[k];
    }
}
template <class T, bool CODES>
__global__ void __launch_bounds__(THREADS) read_kernel(const Params p)
{
    pdl_trigger();
    pdl_wait();
    const bool is_v = blockIdx.y != 0;
    const Side& s = p.side[blockIdx.y];
    if constexpr (CODES) {
        if (s.bits == 3) read_code_rows<3>(p, s, is_v);
        else if (s.bits == 4) read_code_rows<4>(p, s, is_v);
        else read_code_rows<8>(p, s, is_v);
    } else {
        if (s.bits == 3) read_units<3, T>(p, s, is_v);
        else if (s.bits == 4) read_units<4, T>(p, s, is_v);
        else read_units<8, T>(p, s, is_v);
    }
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
        s.bits = x.bits; s.row_bytes = x.row_bytes; s.slab_bytes = x.slab_bytes; s.page_bytes = x.page_bytes;
        s.quant = x.quant; s.value = x.value; s.pos = x.pos; s.chan = x.chan; s.n_units_row = x.K_pad / 32;
        s.pages = static_cast<uint8_t*>(const_cast<void*>(t ? v_pages : k_pages));
        s.rows = const_cast<void*>(t ? v : k);
        s.ld = t ? ldv : ldk;
        s.vector = aligned16(s.rows) && (s.ld * e) % 16 == 0 && (c->d * e) % 16 == 0;
    }
    p->slots = slots; p->n_tokens = n_tokens; p->H = c->H; p->d = c->d; p->nu = c->nu; p->P = c->P; p->C = c->C;
    p->n_slots = n_pages * c->P;
    p->status = device_status_word();
    return RPTQ_OK;
}

template <class T>
static int upload(T** dst, const std::vector<T>& src)
{
    if (cudaMalloc(reinterpret_cast<void**>(dst), src.size() * sizeof(T)) != cudaSuccess) { *dst = nullptr; return RPTQ_ERR_ALLOC; }
    return cudaMemcpy(*dst, src.data(), src.size() * sizeof(T), cudaMemcpyHostToDevice) == cudaSuccess ? RPTQ_OK : RPTQ_ERR_CUDA;
}

static int make_tensor(const rptq_layout_t* L, const rptq_kv_cache& c, rptq_kv_cache::Tensor& t)
{
    t.bits = L->bits; t.K_pad = L->K_pad; t.row_bytes = L->row_bytes;
    t.slab_bytes = (int64_t)SLAB * c.nu * 4 * L->bits;
    t.page_bytes = t.slab_bytes * (c.P / SLAB) * c.H;
    if (c.device < 0) return RPTQ_OK;
    const size_t n = (size_t)c.H * c.nu * 32;
    std::vector<float2> quant(n), value(n, make_float2(0.f, 0.f));
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
            pos[(size_t)ch] = (uint16_t)L->pos[j];
            chan[(size_t)L->pos[j]] = ch;
        }
    int rc = upload(&t.quant, quant);
    if (rc == RPTQ_OK) rc = upload(&t.value, value);
    if (rc == RPTQ_OK) rc = upload(&t.pos, pos);
    if (rc == RPTQ_OK) rc = upload(&t.chan, chan);
    return rc;
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
    int rc;
    try {
        rc = make_tensor(LK, *c, c->k);
        if (rc == RPTQ_OK) rc = make_tensor(LV, *c, c->v);
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
    for (auto* t : {&cache->k, &cache->v}) {
        cudaFree(t->quant);
        cudaFree(t->value);
        cudaFree(t->pos);
        cudaFree(t->chan);
    }
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
    auto st = static_cast<cudaStream_t>(stream);
    const int64_t want = ((int64_t)n_tokens * p.H * p.nu + THREADS - 1) / THREADS, most = (int64_t)n_sm * 16;
    const dim3 grid((unsigned)(want < most ? want : most), 2);
    if (rows_type == RPTQ_ROWS_F32) return launch_kernel(write_kernel<float, false>, grid, THREADS, 0, 0, st, p);
    if (rows_type == RPTQ_ROWS_F16) return launch_kernel(write_kernel<__half, false>, grid, THREADS, 0, 0, st, p);
    if (rows_type == RPTQ_ROWS_BF16) return launch_kernel(write_kernel<__nv_bfloat16, false>, grid, THREADS, 0, 0, st, p);
    return launch_kernel(write_kernel<uint8_t, true>, grid, THREADS, 0, 0, st, p);
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
    auto st = static_cast<cudaStream_t>(stream);
    const int units = rows_type == RPTQ_ROWS_CODES ? (p.side[0].n_units_row > p.side[1].n_units_row ? p.side[0].n_units_row : p.side[1].n_units_row) : p.H * p.nu;
    const int64_t want = ((int64_t)n_tokens * units + THREADS - 1) / THREADS, most = (int64_t)n_sm * 16;
    const dim3 grid((unsigned)(want < most ? want : most), 2);
    if (rows_type == RPTQ_ROWS_F32) return launch_kernel(read_kernel<float, false>, grid, THREADS, 0, 0, st, p);
    if (rows_type == RPTQ_ROWS_F16) return launch_kernel(read_kernel<__half, false>, grid, THREADS, 0, 0, st, p);
    if (rows_type == RPTQ_ROWS_BF16) return launch_kernel(read_kernel<__nv_bfloat16, false>, grid, THREADS, 0, 0, st, p);
    return launch_kernel(read_kernel<uint8_t, true>, grid, THREADS, 0, 0, st, p);
}

}  // extern "C"
