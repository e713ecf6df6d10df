// Retained rows in 8 bits: quantised as they are written, read back, and the entry points of the calls over them.
#include "vs_cache8.h"

#include <algorithm>

namespace vs {
namespace {

constexpr int kThreads = 256;

struct RowsParams {
    char* slab;
    char* k;  // [n_caches][rows_per_cache][Hkv][128] bf16
    char* v;
    int64_t cache_bytes;
    int64_t rows_stride;  // bytes between caches in k and v
    int first;            // first row taken of k and v
    int n_rows;
    int Hkv, items;       // items: (block, KV head) pairs of a cache, at most
    LenTable at;          // the cache's row that the first of them is
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// What the code in the low byte stands for (15 + 8 bits: exact before the rounding).
__device__ __forceinline__ __bf16 row_value(unsigned code, float scale) { return (__bf16)((float)((int)(code & 255u) - 128) * scale); }

// A wavefront per (block, KV head), four a workgroup: the quantiser's lanes keep a row's maximum in 16 lanes and end up with whole words of the block
// (vs_cache8.h), so that nothing passes through LDS.  Bound by memory (4 caches x 11016 rows of 4 heads, 136 MB: 26.8 us = 5.1 TB/s).
__global__ __launch_bounds__(kThreads) void cache8_append_kernel(RowsParams p) {
    const int lane = threadIdx.x & 63, item = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int at = p.at.v[blockIdx.y], block = at / kBlockRows + item / p.Hkv, g = item % p.Hkv;
    if (item >= p.items || block * kBlockRows >= at + p.n_rows) return;
    const int64_t row_bytes = (int64_t)p.Hkv * 256, src = blockIdx.y * p.rows_stride + p.first * row_bytes + (int64_t)g * 256 + 16 * (lane & 15);
    write_block(p.slab + blockIdx.y * p.cache_bytes + ((int64_t)block * p.Hkv + g) * kBlockBytes, p.k + src, p.v + src, row_bytes, block * kBlockRows, at,
                at + p.n_rows, lane);
}

// 16 lanes per (row, KV head): a row's codes of V go out byte by byte, so that nothing of the block is read.  Bound by the launch and the
// chain load, maximum, divide, store.
__global__ __launch_bounds__(kThreads) void cache8_append_rows_kernel(RowsParams p) {
    const int c = threadIdx.x & 15, item = blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    if (item >= p.n_rows * p.Hkv) return;
    const int n = item / p.Hkv, g = item - n * p.Hkv, at = p.at.v[blockIdx.y] + n, key = at % kBlockRows;
    const int64_t src = blockIdx.y * p.rows_stride + ((int64_t)(p.first + n) * p.Hkv + g) * 256 + 16 * c;
    char* const blk = p.slab + blockIdx.y * p.cache_bytes + ((int64_t)(at / kBlockRows) * p.Hkv + g) * kBlockBytes;
    uint2 k_codes;
    unsigned v_codes[8];
    const unsigned pair = quantise(*reinterpret_cast<const raw16*>(p.k + src), *reinterpret_cast<const raw16*>(p.v + src), k_codes, v_codes);
    *reinterpret_cast<uint2*>(blk + k_code_offset(key, c)) = k_codes;
#pragma unroll
    for (int j = 0; j < 8; ++j) blk[v_code_offset(key, c, j)] = (char)v_codes[j];
    if (c == 0) *reinterpret_cast<unsigned*>(blk + kBlockScales + 4 * key) = pair;
}

// The lanes of write_block the other way round.  136 MB as above: 22.4 us = 6.1 TB/s.
__global__ __launch_bounds__(kThreads) void cache8_read_kernel(RowsParams p) {
    const int lane = threadIdx.x & 63, item = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, h = lane >> 4;
    const int first = p.at.v[blockIdx.y], block = first / kBlockRows + item / p.Hkv, g = item % p.Hkv;
    const int row0 = block * kBlockRows, end = first + p.n_rows;
    if (item >= p.items || row0 >= end) return;
    const char* const blk = p.slab + blockIdx.y * p.cache_bytes + ((int64_t)block * p.Hkv + g) * kBlockBytes;
    const int64_t dst = blockIdx.y * p.rows_stride + ((int64_t)g * 128 + 8 * c) * 2;
    uint2 k[8];
    raw16 v[4], s[2];
#pragma unroll
    for (int u = 0; u < 8; ++u) k[u] = *reinterpret_cast<const uint2*>(blk + k_code_offset(16 * (u >> 2) + 4 * h + (u & 3), c));
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const raw16*>(blk + kBlockV + j * 1024 + lane * 16);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) s[kt] = *reinterpret_cast<const raw16*>(blk + kBlockScales + 64 * kt + 16 * h);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int row = row0 + 16 * (u >> 2) + 4 * h + (u & 3);
        if (row < first || row >= end) continue;
        const unsigned pair = s[u >> 2][u & 3];
        const float ks = __uint_as_float(pair << 16), vs = __uint_as_float(pair & 0xffff0000u);
        bf16x8 kx, vx;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned kw = j < 4 ? k[u].x : k[u].y;
            kx[j] = row_value(kw >> (8 * (j & 3)), ks);
            const unsigned vw = v[j >> 1][2 * (j & 1) + (u >> 2)];
            vx[j] = row_value(vw >> (8 * (u & 3)), vs);
        }
        const int64_t at = dst + (int64_t)(row - first + p.first) * p.Hkv * 256;
        *reinterpret_cast<bf16x8*>(p.k + at) = kx;
        *reinterpret_cast<bf16x8*>(p.v + at) = vx;
    }
}

// 16 lanes per (row, KV head), as for few rows written.
__global__ __launch_bounds__(kThreads) void cache8_read_rows_kernel(RowsParams p) {
    const int c = threadIdx.x & 15, item = blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    if (item >= p.n_rows * p.Hkv) return;
    const int n = item / p.Hkv, g = item - n * p.Hkv, at = p.at.v[blockIdx.y] + n, key = at % kBlockRows;
    const char* const blk = p.slab + blockIdx.y * p.cache_bytes + ((int64_t)(at / kBlockRows) * p.Hkv + g) * kBlockBytes;
    const uint2 k = *reinterpret_cast<const uint2*>(blk + k_code_offset(key, c));
    const unsigned pair = *reinterpret_cast<const unsigned*>(blk + kBlockScales + 4 * key);
    unsigned char v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const unsigned char*>(blk + v_code_offset(key, c, j));
    const float ks = __uint_as_float(pair << 16), vs = __uint_as_float(pair & 0xffff0000u);
    bf16x8 kx, vx;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        kx[j] = row_value((j < 4 ? k.x : k.y) >> (8 * (j & 3)), ks);
        vx[j] = row_value(v[j], vs);
    }
    const int64_t dst = blockIdx.y * p.rows_stride + ((int64_t)(p.first + n) * p.Hkv + g) * 256 + 16 * c;
    *reinterpret_cast<bf16x8*>(p.k + dst) = kx;
    *reinterpret_cast<bf16x8*>(p.v + dst) = vx;
}

// Few rows go one by one, many in blocks.  us written and read, caches x KV heads x rows, one by one / in blocks: 28 x 4 x 1 2.9, 2.6 / 4.4, 3.8;
// 28 x 4 x 37 4.3, 3.9 / 6.6, 5.4; 28 x 8 x 64 6.7, 6.1 / 7.0, 6.3; 4 x 4 x 1000 6.9, 6.1 / 6.9, 6.3; 28 x 4 x 170 7.8, 7.0 / 7.1, 6.5;
// 4 x 4 x 2000 11.3, 8.9 / 7.8, 7.5.
bool by_rows(const vs_shape& s, int32_t n_caches, int32_t n_rows) { return (int64_t)n_caches * n_rows * s.n_kv_heads <= 16384; }

// (block, KV head) pairs that n_rows rows of any of the caches can touch
int items_of(const vs_shape& s, int32_t n_caches, const LenTable& at, int32_t n_rows) {
    int most = 0;
    for (int i = 0; i < n_caches; ++i)
        most = std::max(most, (int)(((int64_t)at.v[i] + n_rows - 1) / kBlockRows - at.v[i] / kBlockRows + 1));
    return most * s.n_kv_heads;
}

RowsParams rows_params(const vs_shape& s, int32_t n_caches, const void* slab, int32_t capacity, const LenTable& at, const void* k,
                       const void* v, int32_t rows_per_cache, int32_t first, int32_t n_rows) {
    RowsParams p;
    p.slab = (char*)slab;
    p.k = (char*)k;
    p.v = (char*)v;
    p.cache_bytes = cache8_bytes(s, capacity);
    p.rows_stride = (int64_t)rows_per_cache * s.n_kv_heads * 256;
    p.first = first;
    p.n_rows = n_rows;
    p.Hkv = s.n_kv_heads;
    p.items = items_of(s, n_caches, at, n_rows);
    p.at = at;
    return p;
}

}  // namespace

hipError_t launch_cache8_append(const vs_shape& s, int32_t n_caches, void* slab, int32_t capacity, const LenTable& lens, const void* k_rows,
                                const void* v_rows, int32_t n_tokens, int32_t first_kept, hipStream_t st) {
    const RowsParams p = rows_params(s, n_caches, slab, capacity, lens, k_rows, v_rows, n_tokens, first_kept, n_tokens - first_kept);
    if (by_rows(s, n_caches, p.n_rows)) {
        cache8_append_rows_kernel<<<dim3((p.n_rows * p.Hkv + 15) / 16, n_caches), kThreads, 0, st>>>(p);
        return hipGetLastError();
    }
    cache8_append_kernel<<<dim3((p.items + 3) / 4, n_caches), kThreads, 0, st>>>(p);
    return hipGetLastError();
}

hipError_t launch_cache8_read(const vs_shape& s, int32_t n_caches, const void* slab, int32_t capacity, const LenTable& first, int32_t n_rows,
                              void* k_out, void* v_out, hipStream_t st) {
    const RowsParams p = rows_params(s, n_caches, slab, capacity, first, k_out, v_out, n_rows, 0, n_rows);
    if (by_rows(s, n_caches, p.n_rows)) {
        cache8_read_rows_kernel<<<dim3((p.n_rows * p.Hkv + 15) / 16, n_caches), kThreads, 0, st>>>(p);
        return hipGetLastError();
    }
    cache8_read_kernel<<<dim3((p.items + 3) / 4, n_caches), kThreads, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace vs

using namespace vs;

namespace {

constexpr int32_t kMaxTokens = 4096, kMaxStreams = 1024, kMaxCaches = 1 << 20;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t x) { return (x + 255) & ~size_t(255); }

vs_status check_shape8(const vs_shape* s) {
    const vs_status st = check_shape(s);
    return st == VS_OK && s->dtype != VS_BF16 ? VS_ERR_UNSUPPORTED : st;
}
// (a slab beyond any memory; within it, numbers of blocks fit 32 bits)
inline bool capacity_in_range(const vs_shape& s, int32_t capacity) { return capacity >= 1 && cache8_bytes(s, capacity) <= int64_t(1) << 40; }

inline int64_t row_bytes(const vs_shape& s) { return (int64_t)s.n_kv_heads * s.head_dim * 2; }

}  // namespace

extern "C" {

size_t vs_cache8_bytes(const vs_shape* shape, int32_t capacity) {
    return check_shape8(shape) == VS_OK && capacity_in_range(*shape, capacity) ? (size_t)cache8_bytes(*shape, capacity) : 0;
}

size_t vs_cache8_workspace_bytes(const vs_shape* shape, int32_t max_q_tokens, int32_t max_cache_rows, int32_t n_streams) {
    if (check_shape8(shape) != VS_OK) return 0;
    if (max_q_tokens < 0 || max_q_tokens > kMaxTokens || max_cache_rows < 0 || n_streams < 0 || n_streams > kMaxStreams) return 0;
    size_t need = control_block_bytes(*shape) + 256;
    if (max_q_tokens > 0) need = std::max(need, control_block_bytes(*shape) + round256(prefill8_workspace_bytes(*shape, max_q_tokens, max_cache_rows)));
    if (n_streams > 0)
        need = std::max(need, control_block_bytes(*shape) + decode8_workspace_bytes(*shape, std::min(n_streams, kMaxStreamsPerLaunch)));
    return need;
}

vs_status vs_cache8_append(const vs_shape* shape, int32_t n_caches, void* slab, int32_t capacity, int32_t* lens, const void* k_rows,
                           const void* v_rows, int32_t n_tokens, int32_t first_kept, void* hip_stream) {
    (void)hipGetLastError();
    const vs_status st = check_shape8(shape);
    if (st != VS_OK) return st;
    if (!slab || !lens || !k_rows || !v_rows) return VS_ERR_NULL;
    if (n_caches < 1 || n_caches > kMaxCaches || !capacity_in_range(*shape, capacity) || n_tokens < 1 || first_kept < 0 || first_kept >= n_tokens) return VS_ERR_SHAPE;
    if (!aligned16(slab) || !aligned16(k_rows) || !aligned16(v_rows)) return VS_ERR_ALIGN;
    const int32_t n_kept = n_tokens - first_kept;
    for (int32_t i = 0; i < n_caches; ++i) {
        if (lens[i] < 0) return VS_ERR_SHAPE;
        if ((int64_t)lens[i] + n_kept > capacity) return VS_ERR_CAPACITY;
    }
    const int64_t per_cache = (int64_t)n_tokens * row_bytes(*shape), bytes = cache8_bytes(*shape, capacity);
    for (int32_t i0 = 0; i0 < n_caches; i0 += kMaxStreamsPerLaunch) {
        const int32_t n = std::min(n_caches - i0, kMaxStreamsPerLaunch);
        LenTable t{};
        for (int32_t i = 0; i < n; ++i) t.v[i] = lens[i0 + i];
        if (launch_cache8_append(*shape, n, static_cast<char*>(slab) + i0 * bytes, capacity, t, static_cast<const char*>(k_rows) + i0 * per_cache,
                                 static_cast<const char*>(v_rows) + i0 * per_cache, n_tokens, first_kept,
                                 static_cast<hipStream_t>(hip_stream)) != hipSuccess)
            return VS_ERR_HIP;
        for (int32_t i = 0; i < n; ++i) lens[i0 + i] += n_kept;
    }
    return VS_OK;
}

vs_status vs_cache8_read(const vs_shape* shape, int32_t n_caches, const void* slab, int32_t capacity, const int32_t* lens,
                         const int32_t* first_rows, int32_t n_rows, void* k_out, void* v_out, void* hip_stream) {
    (void)hipGetLastError();
    const vs_status st = check_shape8(shape);
    if (st != VS_OK) return st;
    if (!slab || !lens || !k_out || !v_out) return VS_ERR_NULL;
    if (n_caches < 1 || n_caches > kMaxCaches || !capacity_in_range(*shape, capacity) || n_rows < 1) return VS_ERR_SHAPE;
    if (!aligned16(slab) || !aligned16(k_out) || !aligned16(v_out)) return VS_ERR_ALIGN;
    for (int32_t i = 0; i < n_caches; ++i) {
        if (lens[i] < 0 || (first_rows && first_rows[i] < 0)) return VS_ERR_SHAPE;
        if (lens[i] > capacity) return VS_ERR_CAPACITY;
        if ((first_rows ? (int64_t)first_rows[i] : 0) + n_rows > lens[i]) return VS_ERR_SHAPE;
    }
    const int64_t per_cache = (int64_t)n_rows * row_bytes(*shape), bytes = cache8_bytes(*shape, capacity);
    for (int32_t i0 = 0; i0 < n_caches; i0 += kMaxStreamsPerLaunch) {
        const int32_t n = std::min(n_caches - i0, kMaxStreamsPerLaunch);
        LenTable t{};
        for (int32_t i = 0; i < n; ++i) t.v[i] = first_rows ? first_rows[i0 + i] : 0;
        if (launch_cache8_read(*shape, n, static_cast<const char*>(slab) + i0 * bytes, capacity, t, n_rows, static_cast<char*>(k_out) + i0 * per_cache,
                               static_cast<char*>(v_out) + i0 * per_cache, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
            return VS_ERR_HIP;
    }
    return VS_OK;
}

vs_status vs_cache8_decode_attn(const vs_shape* shape, int32_t n_streams, void* slab, int32_t capacity, int32_t* lens, const void* q,
                                const void* k_new, const void* v_new, void* out, void* workspace, size_t workspace_bytes,
                                void* hip_stream) {
    (void)hipGetLastError();
    const vs_status st = check_shape8(shape);
    if (st != VS_OK) return st;
    if (!slab || !lens || !q || !out || (k_new == nullptr) != (v_new == nullptr)) return VS_ERR_NULL;
    if (n_streams < 1 || n_streams > kMaxStreams || !capacity_in_range(*shape, capacity)) return VS_ERR_SHAPE;
    if (!aligned16(slab) || !aligned16(q) || !aligned16(out) || !aligned16(k_new) || !aligned16(v_new)) return VS_ERR_ALIGN;
    const int32_t add = k_new ? 1 : 0;
    for (int32_t i = 0; i < n_streams; ++i) {
        if (lens[i] < 0) return VS_ERR_SHAPE;
        if (lens[i] > capacity - add) return VS_ERR_CAPACITY;
        if (lens[i] + add < 1) return VS_ERR_SHAPE;
    }
    const size_t ctrl = control_block_bytes(*shape);
    if (!workspace || workspace_bytes < ctrl + decode8_workspace_bytes(*shape, std::min(n_streams, kMaxStreamsPerLaunch))) return VS_ERR_WORKSPACE;
    if (!aligned16(workspace)) return VS_ERR_ALIGN;
    const int64_t rb = row_bytes(*shape), qb = (int64_t)shape->n_q_heads * 256, bytes = cache8_bytes(*shape, capacity);
    for (int32_t i0 = 0; i0 < n_streams; i0 += kMaxStreamsPerLaunch) {
        const int32_t n = std::min(n_streams - i0, kMaxStreamsPerLaunch);
        LenTable t{};
        for (int32_t i = 0; i < n; ++i) t.v[i] = lens[i0 + i] + add;
        if (launch_decode8(*shape, n, static_cast<char*>(slab) + i0 * bytes, capacity, t, static_cast<const char*>(q) + i0 * qb,
                           add ? static_cast<const char*>(k_new) + i0 * rb : nullptr, add ? static_cast<const char*>(v_new) + i0 * rb : nullptr,
                           static_cast<char*>(out) + i0 * qb, workspace, static_cast<char*>(workspace) + ctrl, static_cast<hipStream_t>(hip_stream)) !=
            hipSuccess)
            return VS_ERR_HIP;
        for (int32_t i = 0; i < n; ++i) lens[i0 + i] += add;
    }
    return VS_OK;
}

vs_status vs_cache8_prefill_attn(const vs_shape* shape, vs_cache8* cache, const void* q, const void* k_t, const void* v_t, int32_t n_tokens,
                                 int32_t first_kept, void* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
    (void)hipGetLastError();
    const vs_status st = check_shape8(shape);
    if (st != VS_OK) return st;
    if (!cache || !q || !k_t || !v_t || !out) return VS_ERR_NULL;
    if (cache->capacity < 0 || (cache->capacity > 0 && !capacity_in_range(*shape, cache->capacity)) || cache->len < 0 || n_tokens < 1 || n_tokens > kMaxTokens || first_kept < 0 || first_kept > n_tokens)
        return VS_ERR_SHAPE;
    const int32_t n_kept = n_tokens - first_kept, len = cache->len;
    if ((int64_t)len + n_kept > cache->capacity) return VS_ERR_CAPACITY;
    if ((len > 0 || n_kept > 0) && !cache->data) return VS_ERR_NULL;
    if (!aligned16(cache->data) || !aligned16(q) || !aligned16(k_t) || !aligned16(v_t) || !aligned16(out)) return VS_ERR_ALIGN;
    const size_t ctrl = control_block_bytes(*shape);
    if (!workspace || workspace_bytes < ctrl + prefill8_workspace_need(*shape, n_tokens, len)) return VS_ERR_WORKSPACE;
    if (!aligned16(workspace)) return VS_ERR_ALIGN;
    char* const ws = static_cast<char*>(workspace);
    if (launch_prefill8(*shape, cache->data, len, q, k_t, v_t, n_tokens, first_kept, out, ws + ctrl,
                        static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        return VS_ERR_HIP;
    cache->len += n_kept;
    return VS_OK;
}

}  // extern "C"
