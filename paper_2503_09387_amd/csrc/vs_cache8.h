// Retained rows in 8 bits: how a cache lies in memory, shared by the kernels that write it, read it back and attend over it.
//
// A row x of 128 values (one token, one KV head, K or V) is held as whole numbers q = rint(x / s), ties to even, beside
// s = max(ceil8(max|x| / 127), 2^-126); ceil8 goes up to the next number of 8 significant bits, a bf16.  It stands for q * s.
// x and s both have 8 significant bits, so a quotient that is no tie is further than 2^-17 of itself away from one,
// and the quotient in fp32 rounds to the same whole number as the exact one: what is held does not depend on the arithmetic.
// A row with a value that is not finite gets a scale that is not a number, and stands for nothing else.
//
// 32 rows of a KV head are a block of 8320 bytes: K codes, V codes, 32 scale pairs.  The codes lie as the matrix
// instructions of the decode kernel take them, so that a wavefront moves a block from memory to the multiplier's registers with
// ten loads of 16 bytes per lane and no exchange between lanes:
//   K (A operand of 16 keys x 64 dims, lane = 16 h + key % 16, 16 bytes per lane): [key / 16][dims 64 ds ..][lane][16],
//     bytes 0..7 of a lane: dims 64 ds + 8 h .., bytes 8..15: 64 ds + 32 + 8 h ..; code + 128
//   V (A operand of 16 dims x 32 keys, lane = 16 h + dim / 8): [dim % 8][lane][8], two dims % 8 together in 16 bytes of a
//     lane; bytes 4 kt + r of a lane: key 16 kt + 4 h + r, which is where the product of K leaves that key's score; code + 128
//   scales: [key] (bf16 of K, bf16 of V)
// Blocks are laid [block][KV head]; a cache is ceil(capacity / 32) * Hkv of them, and a cache of another capacity begins
// with the same bytes.
#pragma once
#include "vs_internal.h"

namespace vs {

constexpr int kBlockRows = 32;
constexpr int kBlockV = 4096, kBlockScales = 8192, kBlockBytes = 8320;  // offsets in a block, and its size: a multiple of 128

inline int blocks_of(int32_t rows) { return (int)(((int64_t)rows + kBlockRows - 1) / kBlockRows); }  // (for any number of rows)
inline int64_t cache8_bytes(const vs_shape& s, int32_t capacity) { return (int64_t)blocks_of(capacity) * s.n_kv_heads * kBlockBytes; }

// Where lane c of a row's 16 lanes (dims 8 c .. 8 c + 7) finds its 8 K codes of row `key` of a block.
__device__ __forceinline__ int k_code_offset(int key, int c) {
    return (((key >> 4) * 2 + (c >> 3)) * 64 + (c & 3) * 16 + (key & 15)) * 16 + ((c >> 2) & 1) * 8;
}
// And the V code of dim 8 c + dt of row `key`.
__device__ __forceinline__ int v_code_offset(int key, int c, int dt) {
    return kBlockV + (dt >> 1) * 1024 + (((key & 15) >> 2) * 16 + c) * 16 + (dt & 1) * 8 + (key >> 4) * 4 + (key & 3);
}

// Exchanges in registers (through LDS each would take some 130 cycles): the value of the lane N places on among the 16 of a row,
// and the largest, or the sum, over the lanes 16 and 32 apart.
template <int N>
__device__ __forceinline__ unsigned turned(unsigned x) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, false);  // row_ror
}
template <typename Op>
__device__ __forceinline__ unsigned over_rows(unsigned x, Op op) {
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = op(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return op(b[0], b[1]);
}
__device__ __forceinline__ float max_over_rows(float x) {
    return __uint_as_float(over_rows(__float_as_uint(x), [](unsigned a, unsigned b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ float sum_over_rows(float x) {
    return __uint_as_float(over_rows(__float_as_uint(x), [](unsigned a, unsigned b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// The larger magnitudes of two pairs of bf16 bit patterns without their signs (K below, V above): as whole numbers they are
// ordered as the values are, with infinities and then NaN above all.
__device__ __forceinline__ unsigned max_pairs(unsigned a, unsigned b) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// The scale's bf16 pattern for the largest magnitude's.  (a / 127 to a rounding, and exactly where it is a number of 8 bits: see Divisor.)
__device__ __forceinline__ unsigned scale_bits(unsigned most) {
    const float a = __uint_as_float(most << 16), t = a * (1.0f / 127.0f);
    const unsigned up = (__float_as_uint(fmaf(fmaf(-t, 127.0f, a), 1.0f / 127.0f, t)) + 0xffffu) >> 16;
    return most > 0x7f7fu ? 0x7fc0u : max(up, 0x80u);
}
// The largest magnitudes among 8 K and 8 V values (16 bytes each) of this lane and the row's 15 others.
__device__ __forceinline__ unsigned row_most(const raw16& k, const raw16& v) {
    unsigned a = max_pairs(max_pairs(k[0] & 0x7fff7fffu, k[1] & 0x7fff7fffu), max_pairs(k[2] & 0x7fff7fffu, k[3] & 0x7fff7fffu));
    unsigned b = max_pairs(max_pairs(v[0] & 0x7fff7fffu, v[1] & 0x7fff7fffu), max_pairs(v[2] & 0x7fff7fffu, v[3] & 0x7fff7fffu));
    unsigned m = max_pairs(__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(b, a, 0x07060302u));
    m = max_pairs(m, turned<8>(m));
    m = max_pairs(m, turned<4>(m));
    m = max_pairs(m, turned<2>(m));
    return max_pairs(m, turned<1>(m));
}
// Codes.  x / s to a rounding, or exactly where a product or a tie is: r = 1 / s to a rounding, then t = x r and what the remainder
// x - t s adds.  (The division that the compiler writes takes twice the instructions.)  Below 2^-64 both go up by 2^64, where
// the remainder has all its bits.
struct Divisor {
    float s, r, up;
};
__device__ __forceinline__ Divisor divisor_of(unsigned scale_bits) {
    Divisor d;
    d.s = __uint_as_float(scale_bits << 16);
    d.up = d.s < 0x1p-64f ? 0x1p64f : 1.0f;
    d.s *= d.up;
    const float r = __builtin_amdgcn_rcpf(d.s);
    d.r = fmaf(fmaf(-d.s, r, 1.0f), r, r);
    return d;
}
// The code of one of the two values in a word, plus 128, in the low byte.
__device__ __forceinline__ unsigned code_of(unsigned pair, bool high, const Divisor& d) {
    const float x = __uint_as_float(high ? pair & 0xffff0000u : pair << 16) * d.up, t = x * d.r;
    // (1.5 * 2^23 + 128 on top: the fraction goes, ties to even, and the whole number + 128 stands in the low bits)
    return __float_as_uint(fmaf(fmaf(-t, d.s, x), d.r, t) + 12583040.0f);
}
// The low bytes of four words as one.
__device__ __forceinline__ unsigned bytes_of(unsigned a, unsigned b, unsigned c, unsigned d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// The codes of a row's 16 bytes of K and of V in this lane, K's in two words, V's one a word, and the scale pair.
__device__ __forceinline__ unsigned quantise(const raw16& k, const raw16& v, uint2& k_codes, unsigned (&v_codes)[8]) {
    const unsigned most = row_most(k, v), ks = scale_bits(most & 0xffffu), vs = scale_bits(most >> 16);
    const Divisor kd = divisor_of(ks), vd = divisor_of(vs);
    unsigned w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        w[j] = code_of(k[j >> 1], j & 1, kd);
        v_codes[j] = code_of(v[j >> 1], j & 1, vd);
    }
    k_codes = make_uint2(bytes_of(w[0], w[1], w[2], w[3]), bytes_of(w[4], w[5], w[6], w[7]));
    return ks | (vs << 16);
}

// Rows at .. end - 1 of a cache, as far as they fall into the block at row0, from k, v (this lane's 16 bytes of row `at`, row_bytes apart), by a
// wavefront: lane 16 h + c holds dims 8 c .. of the rows 16 kt + 4 h + r, so that rows are read whole, 256 bytes at a time, a row's
// maximum is four exchanges among 16 lanes, and a lane ends up with all 8 keys that its V operand has side by side.
__device__ __forceinline__ void write_block(char* blk, const char* k, const char* v, int64_t row_bytes, int row0, int at, int end, int lane) {
    const int c = lane & 15, h = lane >> 4;
    raw16 kx[8], vx[8], was[4];
    // what other rows have among this lane's V codes goes back as it was (nobody else writes to the block meanwhile)
    const bool whole = at <= row0 && end >= row0 + kBlockRows;
    if (!whole)
#pragma unroll
        for (int j = 0; j < 4; ++j) was[j] = *reinterpret_cast<const raw16*>(blk + kBlockV + j * 1024 + lane * 16);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int first = row0 + 16 * (u >> 2) + (u & 3);  // of four rows, 4 apart
        if (first + 12 < at || first >= end) continue;
        const int64_t off = (int64_t)(min(max(first + 4 * h, at), end - 1) - at) * row_bytes;  // (rows of others: not stored)
        kx[u] = *reinterpret_cast<const raw16*>(k + off);
        vx[u] = *reinterpret_cast<const raw16*>(v + off);
    }
    unsigned codes[8][8], mask[2] = {0u, 0u};
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int first = row0 + 16 * (u >> 2) + (u & 3), key = 16 * (u >> 2) + 4 * h + (u & 3), row = row0 + key;
        if (first + 12 < at || first >= end) {
#pragma unroll
            for (int j = 0; j < 8; ++j) codes[u][j] = 0;
            continue;
        }
        uint2 k_codes;
        const unsigned pair = quantise(kx[u], vx[u], k_codes, codes[u]);
        if (row >= at && row < end) {
            mask[u >> 2] |= 0xffu << (8 * (u & 3));
            *reinterpret_cast<uint2*>(blk + k_code_offset(key, c)) = k_codes;
            if (c == 0) *reinterpret_cast<unsigned*>(blk + kBlockScales + 4 * key) = pair;
        }
    }
#pragma unroll
    for (int dt = 0; dt < 8; dt += 2) {
        raw16 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = dt + (i >> 1), u = 4 * (i & 1);
            w[i] = bytes_of(codes[u][d], codes[u + 1][d], codes[u + 2][d], codes[u + 3][d]);
            if (!whole) w[i] = (w[i] & mask[i & 1]) | (was[dt >> 1][i] & ~mask[i & 1]);
        }
        *reinterpret_cast<raw16*>(blk + kBlockV + (dt >> 1) * 1024 + lane * 16) = w;
    }
}

// Stores and loads that pass the L2s, which are not coherent with one another.
__device__ __forceinline__ void store_agent(void* dst, unsigned a, unsigned b) {
    __hip_atomic_store(static_cast<unsigned long long*>(dst), (unsigned long long)a | ((unsigned long long)b << 32), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint2 load_agent(const void* src) {
    const unsigned long long v = __hip_atomic_load(static_cast<const unsigned long long*>(src), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_uint2((unsigned)v, (unsigned)(v >> 32));
}

// K and V rows [n_caches][n_tokens][Hkv][128], their rows first_kept .. n_tokens - 1, quantised into the rows behind lens.v[i] of cache i
// (at most kMaxStreamsPerLaunch caches).
hipError_t launch_cache8_append(const vs_shape& s, int32_t n_caches, void* slab, int32_t capacity, const LenTable& lens, const void* k_rows,
                                const void* v_rows, int32_t n_tokens, int32_t first_kept, hipStream_t st);
// Rows first.v[i] .. first.v[i] + n_rows - 1 of cache i as what they stand for, rounded to bf16.
hipError_t launch_cache8_read(const vs_shape& s, int32_t n_caches, const void* slab, int32_t capacity, const LenTable& first, int32_t n_rows,
                              void* k_out, void* v_out, hipStream_t st);
// lens: valid rows, the appended row included.
// counters: the arrival counters of decoding steps at the front of a workspace's control block (see launch_decode_mfma).
size_t decode8_workspace_bytes(const vs_shape& s, int32_t n_streams);
hipError_t launch_decode8(const vs_shape& s, int32_t n_streams, void* slab, int32_t capacity, const LenTable& lens, const void* q,
                          const void* k_new, const void* v_new, void* out, void* counters, void* workspace, hipStream_t st);
// A run's n_tokens over the len rows of one cache and over one another.  Workspace: prefill8_workspace_need; prefill8_workspace_bytes for any run within
// limits.
size_t prefill8_workspace_need(const vs_shape& s, int32_t n_tokens, int32_t len);
size_t prefill8_workspace_bytes(const vs_shape& s, int32_t max_tokens, int32_t max_len);
// Rows first_kept .. of the run are quantised into the cache behind the len rows on the side.
hipError_t launch_prefill8(const vs_shape& s, void* cache, int32_t len, const void* q, const void* k, const void* v, int32_t n_tokens,
                           int32_t first_kept, void* out, void* workspace, hipStream_t st);

}  // namespace vs
