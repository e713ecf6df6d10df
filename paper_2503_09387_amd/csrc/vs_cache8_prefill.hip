// Prefill attention over a cache in 8 bits (Eq. 1 of Section 3.1; Section 3.3): a run's tokens over the retained rows and, causally, over
// one another.
//
//   score(key) = (q . k_codes) * s_k * scale,   out = sum_key p(key) s_v(key) v_codes / sum_key p(key);   scales 1 for the run's own rows
//
// As in the decoding step the products take codes, and the scales of rows go to the scores and the probabilities:
//   * q . (k_codes + 1152): a code + 128 becomes an fp16 by putting 0x64 before its byte (1024 + byte: one permutation for two values);
//     the query is an fp16 after the power of two that brings its largest entry into [2^14, 2^15), which loses nothing down to 2^-28
//     of that entry and 2^-39 of it below; the sums start at -1152 sum q.
//   * p s_v in bf16 (8 bits, as P does over caches in bf16; the denominator sums p before that) times the codes + 128 in bf16, which
//     loses nothing, less 128 times the sum of p s_v, through one more product.
// The G query heads of a KV head are packed into rows (row = token * G + head).  A wavefront holds 32 rows (two sets of 16 columns) and walks
// blocks of 32 keys, which come from memory in the multiplier's own order (vs_cache8.h): nothing is staged, no barrier is met before the
// end.  A workgroup is 8 wavefronts, kRT row tiles x 8 / kRT key groups: the row tiles of a group load the same blocks at about the same
// time (the compute unit's cache serves all but the first), the key groups are added in LDS.
#include "vs_cache8.h"

#include <algorithm>

namespace vs {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int D = 128;
constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kTileRows = 32;  // rows of a wavefront
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazyMax = 8.0f;  // scores may exceed the reference maximum by 2^8 before it is refreshed
constexpr int kMaxSplits = 32;

struct Prefill8Params {
    const char* cache;
    const char* q;
    const char* k;   // the run's own rows
    const char* v;
    __bf16* out;
    _Float16* part_o;  // [split][Hkv][row] normalised, times the power of two that brings the row's largest entry into [2^14, 2^15)
    float* part_ml;    // [split][Hkv][row][4]: reference (log2 units), sum, inverse of the row's scale, unused
    int len, T, G, Hq, Hkv, M;
    int n_cache_blocks;
    int n_groups;      // row groups: kRT * 32 rows each
    int nsplit;
    float scale_log2e;
};

// A block of cached rows in a wavefront's registers.
struct Block {
    raw16 k[4], v[4], s[2];
};
__device__ __forceinline__ void fetch_keys(Block& b, const char* blk, int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j) b.k[j] = *reinterpret_cast<const raw16*>(blk + j * 1024 + lane * 16);
}
__device__ __forceinline__ void fetch_scales(Block& b, const char* blk, int lane) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) b.s[kt] = *reinterpret_cast<const raw16*>(blk + kBlockScales + 64 * kt + 16 * (lane >> 4));
}
__device__ __forceinline__ void fetch_values(Block& b, const char* blk, int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j) b.v[j] = *reinterpret_cast<const raw16*>(blk + kBlockV + j * 1024 + lane * 16);
}

struct State {
    f32x4 o[2][8];    // [columns][dim % 8]: element r of lane (column i16, h): dim 8 (4 h + r) + dim % 8
    f32x4 excess[2];  // 128 times the sum of p s_v, negative
    float m[2], l[2]; // reference (log2 units), this lane's share of the sum
};

// The softmax of a block's scores z f (f: the same for a column's lanes) and the product with V.  Codes: 8 words of V (4 words of 4 codes + 128 for two dims % 8
// each); else 32 words of bf16 pairs.
template <typename VOf>
__device__ __forceinline__ void accumulate(State& st, float (&z)[2][8], const float (&f)[2], const float* sv, VOf v_of) {
    float mx[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
        mx[c] = f[c] * fmaxf(fmaxf(fmaxf(z[c][0], z[c][1]), fmaxf(z[c][2], z[c][3])), fmaxf(fmaxf(z[c][4], z[c][5]), fmaxf(z[c][6], z[c][7])));
    if (__any(mx[0] > st.m[0] + kLazyMax || mx[1] > st.m[1] + kLazyMax)) {  // rare after the first block
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float x = fmaxf(mx[c], __shfl_xor(mx[c], 16));
            x = fmaxf(x, __shfl_xor(x, 32));
            // (-INFINITY: a row that sees none of these keys and has seen none before)
            const float m_new = fmaxf(st.m[c], x), alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m[c] - m_new);
            st.m[c] = m_new;
            st.l[c] *= alpha;
            st.excess[c] *= alpha;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) st.o[c][dt] *= alpha;
        }
    }
    bf16x8 p[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float m = st.m[c] == -INFINITY ? 0.f : st.m[c];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float pe = __builtin_amdgcn_exp2f(fmaf(z[c][e], f[c], -m));
            st.l[c] += pe;
            p[c][e] = (__bf16)(sv ? pe * sv[e] : pe);
        }
    }
    if (sv) {
        const unsigned minus128 = 0xc300c300u;
        const bf16x8 off = __builtin_bit_cast(bf16x8, u32x4{minus128, minus128, minus128, minus128});
#pragma unroll
        for (int c = 0; c < 2; ++c) st.excess[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(off, p[c], st.excess[c], 0, 0, 0);
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        const bf16x8 a = v_of(dt);
#pragma unroll
        for (int c = 0; c < 2; ++c) st.o[c][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[c], st.o[c][dt], 0, 0, 0);
    }
}

// four codes of V as bf16: whole numbers 0..255, whose fp32 has nothing in its lower half
__device__ __forceinline__ void widen(unsigned w, unsigned& lo, unsigned& hi) {
    const unsigned a = __float_as_uint((float)(w & 255u)), b = __float_as_uint((float)((w >> 8) & 255u));
    const unsigned c = __float_as_uint((float)((w >> 16) & 255u)), d = __float_as_uint((float)(w >> 24));
    lo = __builtin_amdgcn_perm(b, a, 0x07060302u);
    hi = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// One block of cached rows, of which `valid` are there; the next block is asked for piece by piece as this one's are used up.
__device__ __forceinline__ void attend_cached(State& st, Block& b, const char* next, const f16x8 (&q)[2][4], const float (&start)[2], const float (&f)[2],
                                              int valid, int lane) {
    const int h = lane >> 4;
    float z[2][8], sv[8];
    f32x4 s[2][2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
        for (int c = 0; c < 2; ++c) s[kt][c] = f32x4{start[c], start[c], start[c], start[c]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned x = b.k[2 * kt + (i >> 1)][2 * (i & 1)] ^ 0x80808080u, y = b.k[2 * kt + (i >> 1)][2 * (i & 1) + 1] ^ 0x80808080u;
            const f16x8 k = __builtin_bit_cast(f16x8, u32x4{__builtin_amdgcn_perm(0x64646464u, x, 0x05010400u), __builtin_amdgcn_perm(0x64646464u, x, 0x07030602u),
                                                            __builtin_amdgcn_perm(0x64646464u, y, 0x05010400u), __builtin_amdgcn_perm(0x64646464u, y, 0x07030602u)});
#pragma unroll
            for (int c = 0; c < 2; ++c) s[kt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[c][i], s[kt][c], 0, 0, 0);
        }
    }
    fetch_keys(b, next, lane);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const unsigned pair = b.s[kt][r];
#pragma unroll
            for (int c = 0; c < 2; ++c) z[c][4 * kt + r] = s[kt][c][r] * __uint_as_float(pair << 16);
            sv[4 * kt + r] = __uint_as_float(pair & 0xffff0000u);
        }
    fetch_scales(b, next, lane);
    if (valid < kBlockRows) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (16 * (e >> 2) + 4 * h + (e & 3) >= valid) {
                z[0][e] = z[1][e] = -INFINITY;
                sv[e] = 0.f;
            }
    }
    accumulate(st, z, f, sv, [&](int dt) {
        u32x4 a;
        unsigned x, y;
        widen(b.v[dt >> 1][2 * (dt & 1)], x, y);
        a[0] = x, a[1] = y;
        widen(b.v[dt >> 1][2 * (dt & 1) + 1], x, y);
        a[2] = x, a[3] = y;
        return __builtin_bit_cast(bf16x8, a);
    });
    fetch_values(b, next, lane);
}

// One block of the run's own rows, keys 32 j ..: column c sees keys up to `last[c]` of them.
__device__ __forceinline__ void attend_own(State& st, const char* k, const char* v, int64_t row_bytes, int j, int T, const bf16x8 (&q)[2][4],
                                           const float (&f)[2], const int (&last)[2], int i16, int h) {
    float z[2][8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        f32x4 s[2];
        s[0] = s[1] = f32x4{0.f, 0.f, 0.f, 0.f};
        const char* const row = k + min(32 * j + 16 * kt + i16, T - 1) * row_bytes + 16 * h;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x8 a = *reinterpret_cast<const bf16x8*>(row + 64 * i);
#pragma unroll
            for (int c = 0; c < 2; ++c) s[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[c][i], s[c], 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 2; ++c) z[c][4 * kt + r] = 32 * j + 16 * kt + 4 * h + r <= last[c] ? s[c][r] : -INFINITY;
    }
    raw16 x[8];  // 8 keys, of each dims 8 i16 ..
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int key = 32 * j + 16 * (e >> 2) + 4 * h + (e & 3);
        x[e] = *reinterpret_cast<const raw16*>(v + min(key, T - 1) * row_bytes + 16 * i16);
    }
    auto columns_of = [](const raw16 (&w)[8], int dt) {  // the 8 keys' values of dim % 8 = dt
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(w[2 * i + 1][dt >> 1], w[2 * i][dt >> 1], dt & 1 ? 0x07060302u : 0x05040100u);
        return __builtin_bit_cast(bf16x8, a);
    };
    // A value that is not finite must not reach the columns that do not see its key (0 times it is NaN): such values go in as 0,
    // and the columns that do see one become NaN there.
    unsigned most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max_pairs(most, x[e][i] & 0x7fff7fffu);
    if (__any(max(most & 0xffffu, most >> 16) > 0x7f7fu)) {
        raw16 odd[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned lo = (x[e][i] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (x[e][i] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
                odd[e][i] = (lo | hi) & 0x3f803f80u;  // 1 for each
                x[e][i] &= ~(lo | hi);
            }
        bf16x8 sees[2];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) sees[c][e] = (__bf16)(32 * j + 16 * (e >> 2) + 4 * h + (e & 3) <= last[c] ? 1.f : 0.f);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(columns_of(odd, dt), sees[c], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n[r] > 0.f) st.o[c][dt][r] = __uint_as_float(0x7fc00000u);
            }
    }
    accumulate(st, z, f, nullptr, [&](int dt) { return columns_of(x, dt); });
}

// Grid: (splits * row groups * Hkv, as workgroups that share the keys of a row group lie side by side).
template <int kRT>
__global__ __launch_bounds__(kThreads, 2) void prefill8_kernel(Prefill8Params p) {
    constexpr int kKG = kWaves / kRT;
    constexpr int kRowStride = D + 4;
    __shared__ __attribute__((aligned(16))) float s_o[kWaves / 2][kTileRows][kRowStride];
    __shared__ float s_m[kWaves / 2][kTileRows], s_l[kWaves / 2][kTileRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, h = lane >> 4;
    const int split = blockIdx.x % p.nsplit, unit = blockIdx.x / p.nsplit, g = unit % p.Hkv, group = unit / p.Hkv;
    const int rt = wave % kRT, kg = wave / kRT;
    const int row0 = (group * kRT + rt) * kTileRows;
    // blocks that rows of the group see: the cache's and the run's own up to its last token
    const int last_row = min((group + 1) * kRT * kTileRows, p.M) - 1;
    const int n_blocks = p.n_cache_blocks + last_row / p.G / 32 + 1;
    const int first = (int)((int64_t)n_blocks * split / p.nsplit), end = (int)((int64_t)n_blocks * (split + 1) / p.nsplit);
    const char* const base = p.cache + (int64_t)g * kBlockBytes;
    const int64_t stride = (int64_t)p.Hkv * kBlockBytes, row_bytes = (int64_t)p.Hkv * 256;

    State st;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) st.o[c][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        st.excess[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        st.m[c] = -INFINITY;
        st.l[c] = 0.f;
    }
    if (row0 < p.M) {
        int b = first + kg;
        const char* q_row[2];
        int last[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int row = min(row0 + 16 * c + i16, p.M - 1), t = row / p.G;
            q_row[c] = p.q + (((int64_t)t * p.Hq + (int64_t)g * p.G + row - t * p.G) * D + 8 * h) * 2;
            last[c] = t;
        }
        if (b < end && b < p.n_cache_blocks) {
            Block x;
            const int stop = min(end, p.n_cache_blocks);
            const char* blk = base + b * stride;
            fetch_keys(x, blk, lane);
            fetch_scales(x, blk, lane);
            fetch_values(x, blk, lane);
            f16x8 q[2][4];
            float start[2], f[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                raw16 w[4];
                unsigned most = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = *reinterpret_cast<const raw16*>(q_row[c] + 64 * i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) most = max_pairs(most, w[i][j] & 0x7fff7fffu);
                }
                most = max(most & 0xffffu, most >> 16);
                most = max(most, (unsigned)__shfl_xor((int)most, 16));
                most = max(most, (unsigned)__shfl_xor((int)most, 32));
                const int up = 14 + 127 - max((int)(most >> 7), 1);
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const unsigned pair = w[i][j >> 1];
                        q[c][i][j] = (_Float16)ldexpf(__uint_as_float(j & 1 ? pair & 0xffff0000u : pair << 16), up);
                        sum += (float)q[c][i][j];
                    }
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                start[c] = -1152.0f * sum;
                // (a query that is not finite gives scores that are not numbers)
                f[c] = most > 0x7f7fu ? __uint_as_float(0x7fc00000u) : fmaxf(ldexpf(p.scale_log2e, -up), 1.17549435e-38f);
            }
            for (; b < stop; b += kKG) {
                if (b + kKG < stop) blk += kKG * stride;  // (behind the last one: that one again)
                attend_cached(st, x, blk, q, start, f, p.len - b * kBlockRows, lane);
            }
        }
        if (b < end) {
            bf16x8 q[2][4];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) q[c][i] = *reinterpret_cast<const bf16x8*>(q_row[c] + 64 * i);
            const float f[2] = {p.scale_log2e, p.scale_log2e};
            for (; b < end; b += kKG)
                attend_own(st, p.k + (int64_t)g * 256, p.v + (int64_t)g * 256, row_bytes, b - p.n_cache_blocks, p.T, q, f, last, i16, h);
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        st.l[c] += __shfl_xor(st.l[c], 16);
        st.l[c] += __shfl_xor(st.l[c], 32);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) st.o[c][dt] += st.excess[c];
    }
    // the key groups, the upper half of them to the lower until one is left
#pragma unroll
    for (int n = kKG / 2; n >= 1; n >>= 1) {
        if (n < kKG / 2) __syncthreads();
        if (kg >= n && kg < 2 * n) {
            const int slot = wave - n * kRT;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (h == 0) {
                    s_m[slot][16 * c + i16] = st.m[c];
                    s_l[slot][16 * c + i16] = st.l[c];
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        f32x4 w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = st.o[c][4 * half + e][r];
                        *reinterpret_cast<f32x4*>(&s_o[slot][16 * c + i16][8 * (4 * h + r) + 4 * half]) = w;
                    }
            }
        }
        __syncthreads();
        if (kg < n) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float m2 = s_m[wave][16 * c + i16], mx = fmaxf(st.m[c], m2);
                const float a = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m[c] - mx), b = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m2 - mx);
                st.m[c] = mx;
                st.l[c] = st.l[c] * a + s_l[wave][16 * c + i16] * b;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const f32x4 w = *reinterpret_cast<const f32x4*>(&s_o[wave][16 * c + i16][8 * (4 * h + r) + 4 * half]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) st.o[c][4 * half + e][r] = st.o[c][4 * half + e][r] * a + w[e] * b;
                    }
            }
        }
    }
    if (kg != 0) return;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int row = row0 + 16 * c + i16;
        const float inv = p.nsplit > 1 && st.l[c] == 0.f ? 0.f : 1.0f / st.l[c];  // (0: none of the split's keys is visible to the row)
        if (p.nsplit == 1) {
            const int t = row / p.G;
            __bf16* const dst = p.out + ((int64_t)t * p.Hq + (int64_t)g * p.G + row - t * p.G) * D + 32 * h;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                bf16x8 w;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (__bf16)(st.o[c][e][r] * inv);
                if (row < p.M) *reinterpret_cast<bf16x8*>(dst + 8 * r) = w;
            }
        } else {
            float big = 0.f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r) big = fmaxf(big, fabsf(st.o[c][dt][r]));
            big *= inv;
            big = fmaxf(big, __shfl_xor(big, 16));
            big = fmaxf(big, __shfl_xor(big, 32));
            const int se = min(max(127 + 14 + 127 - (int)((__float_as_uint(big) >> 23) & 255u), 1), 254);
            const float scale = __uint_as_float((unsigned)se << 23);
            const int64_t pr = ((int64_t)split * p.Hkv + g) * p.M + row;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f16x8 w;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (_Float16)(st.o[c][e][r] * inv * scale);
                if (row < p.M) *reinterpret_cast<f16x8*>(p.part_o + pr * D + 32 * h + 8 * r) = w;
            }
            if (h == 0 && row < p.M)
                *reinterpret_cast<float4*>(p.part_ml + pr * 4) = make_float4(st.m[c], st.l[c], __uint_as_float((unsigned)(254 - se) << 23), 0.f);
        }
    }
}

// The splits of a row added in index order: 16 lanes a row, 8 dims each.
__global__ __launch_bounds__(256) void prefill8_combine_kernel(Prefill8Params p) {
    constexpr int kDepth = 8;
    const int at = blockIdx.x * 16 + (threadIdx.x >> 4), d8 = 8 * (threadIdx.x & 15);
    if (at >= p.M * p.Hkv) return;
    const int g = at / p.M, row = at - g * p.M;
    float m = -INFINITY, l = 0.f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
    for (int s0 = 0; s0 < p.nsplit; s0 += kDepth) {
        float4 ml[kDepth];
        f16x8 x[kDepth];
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            const int64_t pr = ((int64_t)min(s0 + u, p.nsplit - 1) * p.Hkv + g) * p.M + row;
            ml[u] = *reinterpret_cast<const float4*>(p.part_ml + pr * 4);
            x[u] = *reinterpret_cast<const f16x8*>(p.part_o + pr * D + d8);
        }
        float mx = m;
#pragma unroll
        for (int u = 0; u < kDepth; ++u) mx = fmaxf(mx, ml[u].x);
        const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mx);
        l *= f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= f;
        m = mx;
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            if (s0 + u >= p.nsplit) continue;
            const float w = (mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[u].x - mx)) * ml[u].y, wo = w * ml[u].z;
            l += w;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += wo * (float)x[u][e];
        }
    }
    const float inv = 1.0f / l;
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (__bf16)(o[e] * inv);
    const int t = row / p.G;
    *reinterpret_cast<bf16x8*>(p.out + ((int64_t)t * p.Hq + (int64_t)g * p.G + row - t * p.G) * D + d8) = r;
}

// Row tiles per workgroup, row groups, and workgroups that share a group's keys.
struct Plan {
    int rt, groups, nsplit;
};
Plan plan_of(const vs_shape& s, int32_t n_tokens, int32_t len) {
    const int G = s.n_q_heads / s.n_kv_heads, tiles = (n_tokens * G + kTileRows - 1) / kTileRows;
    Plan pl;
    pl.rt = tiles <= 1 ? 1 : tiles <= 2 ? 2 : 4;
    pl.groups = (tiles + pl.rt - 1) / pl.rt;
    // one workgroup per compute unit, and a block for every key group at least
    const int blocks = (len + kBlockRows - 1) / kBlockRows + (n_tokens + 31) / 32, kg = kWaves / pl.rt;
    pl.nsplit = std::max(1, std::min({256 / (pl.groups * s.n_kv_heads), blocks / kg, kMaxSplits}));
    return pl;
}
size_t partial_bytes(const vs_shape& s, int32_t n_tokens, int nsplit) {
    return nsplit <= 1 ? 0 : (size_t)nsplit * n_tokens * s.n_q_heads * (D * sizeof(_Float16) + 4 * sizeof(float));
}

}  // namespace

size_t prefill8_workspace_need(const vs_shape& s, int32_t n_tokens, int32_t len) { return partial_bytes(s, n_tokens, plan_of(s, n_tokens, len).nsplit); }

// What any run of at most max_tokens over at most max_len rows needs (splits come with more rows and go with more tokens).
size_t prefill8_workspace_bytes(const vs_shape& s, int32_t max_tokens, int32_t max_len) {
    size_t most = 0;
    for (int32_t t = 1; t <= max_tokens; ++t) most = std::max(most, prefill8_workspace_need(s, t, max_len));
    return most;
}

hipError_t launch_prefill8(const vs_shape& s, const void* cache, int32_t len, const void* q, const void* k, const void* v, int32_t n_tokens,
                           void* out, void* workspace, hipStream_t st) {
    const Plan pl = plan_of(s, n_tokens, len);
    Prefill8Params p;
    p.cache = (const char*)cache;
    p.q = (const char*)q;
    p.k = (const char*)k;
    p.v = (const char*)v;
    p.out = (__bf16*)out;
    p.len = len;
    p.T = n_tokens;
    p.G = s.n_q_heads / s.n_kv_heads;
    p.Hq = s.n_q_heads;
    p.Hkv = s.n_kv_heads;
    p.M = n_tokens * p.G;
    p.n_cache_blocks = (len + kBlockRows - 1) / kBlockRows;
    p.n_groups = pl.groups;
    p.nsplit = pl.nsplit;
    p.scale_log2e = s.softmax_scale * kLog2e;
    p.part_ml = (float*)workspace;
    p.part_o = (_Float16*)(p.part_ml + (int64_t)pl.nsplit * p.M * p.Hkv * 4);
    const int grid = pl.nsplit * pl.groups * p.Hkv;
    if (pl.rt == 1) prefill8_kernel<1><<<grid, kThreads, 0, st>>>(p);
    else if (pl.rt == 2) prefill8_kernel<2><<<grid, kThreads, 0, st>>>(p);
    else prefill8_kernel<4><<<grid, kThreads, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.nsplit == 1) return e;
    prefill8_combine_kernel<<<(p.M * p.Hkv + 15) / 16, 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace vs
