// Prefill attention over a cache in 8 bits (Eq. 1 of Section 3.1; Section 3.3): a run's tokens over the retained rows and, causally, over
// one another.  The arithmetic is in vs_cache8_attn.h.  The G query heads of a KV head are packed into rows (row = token * G + head).
// A wavefront holds 32 rows (two sets of 16 columns) and walks blocks of 32 keys.  A workgroup is 8 wavefronts, kRT row tiles x 8 / kRT key groups, which are added in LDS at the end:
//   * kRT = 4: two key groups, a wavefront of each on every SIMD.  A block comes from memory once, a quarter by each wavefront of
//     its group, which widens its quarter into LDS for all four (widening costs as many vector instructions as the softmax of 32 rows).
//     The groups take turns, a barrier apart: while one multiplies (the last block's values, the next one's keys), the other works out
//     probabilities and widens, so that matrix and vector instructions of a SIMD run side by side.
//   * kRT = 1: every wavefront has a block of its own, straight from memory into the multiplier, widened as it is multiplied; no merge launch for
//     many sizes.  Bound by vector instructions (237 of a block's turn, beside 34 matrix instructions, two wavefronts a SIMD).
//   Which of the two: plan_of.
// 28/4 heads: 37 tokens over 711 rows 11.4 us, 170 over 4424 30.3 us = 363 TFLOP/s (kRT = 1); 170 over 11016 49.6 us = 545 TFLOP/s, and 4.8 (kRT = 4).
// Some 8 us of each are fixed: launch, first trips to memory, the queries' conversion, the sums' way through LDS, stores.
#include "vs_cache8_attn.h"

#include <algorithm>

namespace vs {
namespace {

constexpr int D = 128;
constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kTileRows = 32;  // rows of a wavefront
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazyMax = 8.0f;     // scores may exceed the reference maximum by 2^8 before it is refreshed
constexpr float kMaxWeight = 15.0f;  // log2 of the largest weight that goes into an fp16
constexpr float kLazyOwn = 20.0f;    // as kLazyMax for a run's own rows, behind cached ones whose weights have set the reference
constexpr int kMaxSplits = 32;
constexpr int kAhead = 5;       // pieces of a block that are on their way from LDS

struct Prefill8Params {
    char* cache;
    const char* q;
    const char* k;   // the run's own rows
    const char* v;
    __bf16* out;
    _Float16* part_o;  // [split][Hkv][row][128] normalised, times the power of two that brings the largest of 32 dims into [2^14, 2^15)
    char* part_ml;     // [split][Hkv][row][16 bytes]: reference (log2 units), sum, the biased exponents of the four powers, unused
    int len, T, G, Hq, Hkv, M;
    int n_cache_blocks;
    int n_groups;      // row groups: kRT * 32 rows each
    int nsplit;
    int first_kept;    // rows of the run from this one on are kept,
    int n_keeping;     // (block, KV head) pairs that they fall into
    unsigned by_G;     // row / G: the upper half of row * by_G (G > 1)
    float scale_log2e;
};

struct State {
    f32x4 o[2][8];     // [columns][dim % 8]: element r of lane (column i16, h): dim 8 (4 h + r) + dim % 8
    f32x4 excess[2];   // what is too much in them, negative
    float m[2], l[2];  // reference (log2 units; 0 until a key has been seen), this lane's share of the sum
    float limit[2];    // what scores (kRT = 1: weights) may come to before the reference is refreshed, log2: -INFINITY until a key has been seen
};

// Scores less the reference become probabilities; the sums take them.
__device__ __forceinline__ void soften(State& st, float (&x)[2][8]) {
    const float mx[2] = {max_of_8(x[0]), max_of_8(x[1])};
    if (__any(mx[0] > st.limit[0] || mx[1] > st.limit[1])) {  // rare after the first block
        asm volatile("s_nop 15\n\ts_nop 15");  // (the last matrix instruction's sums, before assembly that the compiler does not look into)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const bool seen = st.limit[c] != -INFINITY;
            float up = max_over_rows(mx[c]);
            if (seen) up = fmaxf(up, 0.f);
            if (up == -INFINITY) up = 0.f;  // (the column sees none of these keys and has seen none before)
            else st.limit[c] = kLazyMax;
            const float keep = seen ? __builtin_amdgcn_exp2f(-up) : 1.f;
            st.m[c] += up;
            st.l[c] *= keep;
            scale_in_place(st.excess[c], keep);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) scale_in_place(st.o[c][dt], keep);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] -= up;
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[c][e] = __builtin_amdgcn_exp2f(x[c][e]);
            st.l[c] += x[c][e];
        }
}

// The steps of a block of cached rows.  Scores of its keys (k_of(kt, i): 16 keys, 32 dims):
template <typename KOf>
__device__ __forceinline__ void multiply_keys(f32x4 (&s)[2][2], const Queries (&q)[2], KOf k_of) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int c = 0; c < 2; ++c) s[kt][c] = f32x4{q[c].start, q[c].start, q[c].start, q[c].start};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const f16x8 k = k_of(kt, i);
#pragma unroll
            for (int c = 0; c < 2; ++c) s[kt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[c].q[i], s[kt][c], 0, 0, 0);
        }
}
// probabilities times the scales of V, of the first `valid` rows (kRT = 4):
template <typename Then>
__device__ __forceinline__ void weigh(State& st, bf16x8 (&p)[2], const f32x4 (&s)[2][2], const f32x4 (&ks)[2], const f32x4 (&vs)[2], const Queries (&q)[2],
                                      int valid, int h, Then then) {
    float x[2][8], v[8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int c = 0; c < 2; ++c) x[c][4 * kt + r] = fmaf(s[kt][c][r], ks[kt][r] * q[c].f, -st.m[c]);
            v[4 * kt + r] = vs[kt][r];
        }
    if (valid < kBlockRows) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (16 * (e >> 2) + 4 * h + (e & 3) >= valid) {
                x[0][e] = x[1][e] = -INFINITY;
                v[e] = 0.f;
            }
    }
    soften(st, x);
    then();
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) p[c][e] = (__bf16)(x[c][e] * v[e]);
}
// The same for kRT = 1, where every wavefront widens V for itself and it matters that a code becomes an fp16 in a third of the instructions
// that a bf16 takes.  The weights w = p s_v unit are then fp16 too, 11 bits, and it is w that the reference holds in range: at most 2^15, the largest
// 2^6 when it is set; what is below 2^-14 loses bits, 2^-25 a key at most, of what has a key of 2^6.  p is an fp32 of any size up to
// 2^96 (rows of zeros, of the smallest scale, that a query likes best).  unit: see the kernel.
__device__ __forceinline__ void weigh_for_fp16(State& st, f16x8 (&w)[2], const f32x4 (&s)[2][2], const f32x4 (&ks)[2], const f32x4 (&vs)[2], const Queries (&q)[2],
                                               int valid, int h) {
    float x[2][8], v[8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int c = 0; c < 2; ++c) x[c][4 * kt + r] = fmaf(s[kt][c][r], ks[kt][r] * q[c].f, -st.m[c]);
            v[4 * kt + r] = vs[kt][r];
        }
    if (valid < kBlockRows) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (16 * (e >> 2) + 4 * h + (e & 3) >= valid) {
                x[0][e] = x[1][e] = -INFINITY;
                v[e] = 0.f;
            }
    }
    // (log2 of the weights of these 8 keys is at most this; if that passes the limit they are looked at one by one)
    const float top = fmaxf(__builtin_amdgcn_logf(max_of_8(v)), -80.f);
    const float mx[2] = {max_of_8(x[0]) + top, max_of_8(x[1]) + top};
    if (__any(mx[0] > st.limit[0] || mx[1] > st.limit[1])) {  // rare after the first block
        asm volatile("s_nop 15\n\ts_nop 15");  // (as in soften)
        float log_v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) log_v[e] = fmaxf(__builtin_amdgcn_logf(v[e]), -80.f) - 6.f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const bool seen = st.limit[c] != -INFINITY;
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = x[c][e] + log_v[e];
            float up = max_over_rows(max_of_8(z));
            if (seen) up = fmaxf(up, 0.f);
            if (up == -INFINITY) up = 0.f;
            else st.limit[c] = kMaxWeight;
            // (in two steps: scales of V that are far apart take up past 126 and leave the sum a part of the whole all the same)
            const float half = seen ? __builtin_amdgcn_exp2f(-0.5f * up) : 1.f, keep = half * half;
            st.m[c] += up;
            st.l[c] = st.l[c] * half * half;
            scale_in_place(st.excess[c], keep);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) scale_in_place(st.o[c][dt], keep);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] -= up;
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = __builtin_amdgcn_exp2f(x[c][e]);
            st.l[c] += p;
            w[c][e] = (_Float16)(p * v[e]);
        }
}

// The keys of a block of the run's own rows, keys 32 j .., as the products take them.
__device__ __forceinline__ void ask_own_keys(bf16x8 (&to)[2][4], const char* k, int64_t row_bytes, int j, int T, int i16, int h) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        const char* const row = k + min(32 * j + 16 * kt + i16, T - 1) * row_bytes + 16 * h;
#pragma unroll
        for (int i = 0; i < 4; ++i) to[kt][i] = *reinterpret_cast<const bf16x8*>(row + 64 * i);
    }
}
// Such a block: column c sees keys up to `last[c]` of the run; sums in units of 1 / unit.  The keys of block j + step are asked for on the way.
__device__ __forceinline__ void attend_own(State& st, bf16x8 (&keys)[2][4], const char* k, const char* v, int64_t row_bytes, int j, int step, int T,
                                           const raw16 (&q)[2][4], float f, const int (&last)[2], float unit, int i16, int h) {
    raw16 x[8];  // 8 keys, of each dims 8 i16 ..
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int key = 32 * j + 16 * (e >> 2) + 4 * h + (e & 3);
        x[e] = *reinterpret_cast<const raw16*>(v + min(key, T - 1) * row_bytes + 16 * i16);
    }
    float z[2][8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        f32x4 s[2];
        s[0] = s[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 2; ++c) s[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(keys[kt][i], __builtin_bit_cast(bf16x8, q[c][i]), s[c], 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 2; ++c) z[c][4 * kt + r] = 32 * j + 16 * kt + 4 * h + r <= last[c] ? fmaf(s[c][r], f, -st.m[c]) : -INFINITY;
    }
    ask_own_keys(keys, k, row_bytes, j + step, T, i16, h);
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
        bf16x8 sees[2];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) sees[c][e] = (__bf16)(32 * j + 16 * (e >> 2) + 4 * h + (e & 3) <= last[c] ? 1.f : 0.f);
        auto bad = [](unsigned w) {  // ones where a half is not finite
            const unsigned top = ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
            return top | (top - (top >> 15));
        };
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            u32x4 odd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned a = x[2 * i][dt >> 1], b = x[2 * i + 1][dt >> 1];
                odd[i] = bad(dt & 1 ? (a >> 16) | (b & 0xffff0000u) : (a & 0xffffu) | (b << 16)) & 0x3f803f80u;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), sees[c], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n[r] > 0.f) st.o[c][dt][r] = __uint_as_float(0x7fc00000u);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[e][i] &= ~bad(x[e][i]);
    }
    soften(st, z);
    bf16x8 p[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) p[c][e] = (__bf16)(z[c][e] * unit);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        const bf16x8 a = columns_of(x, dt);
#pragma unroll
        for (int c = 0; c < 2; ++c) st.o[c][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[c], st.o[c][dt], 0, 0, 0);
    }
}

// The value of another lane of the same four (kSelect: two bits of each lane's source).
template <int kSelect>
__device__ __forceinline__ float neighbour(float x) {
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), kSelect, 0xf, 0xf, false));
}

// Grid (splits, Hkv, row groups and more): workgroups that read the same keys are Hkv * splits apart.  Those beyond the row groups quantise the
// rows that are kept, a block and KV head each wavefront; whoever attends to the block they go to leaves out rows from len on.
template <int kRT>
__global__ __launch_bounds__(kThreads, 2) void prefill8_kernel(Prefill8Params p) {
    constexpr int kKG = kWaves / kRT;
    constexpr bool kShared = kRT > 1;
    static_assert(!kShared || kKG == 2, "two key groups take turns");
    constexpr int kStaged = 16384 + 256;  // a widened block: K, V, the scales of K, the scales of V
    constexpr int kLds = 16 * (8 * 64 * 4 + 32) * 4;  // both sets of columns of 8 wavefronts
    __shared__ __attribute__((aligned(16))) char smem[kLds];
    static_assert(3 * 2 * kStaged <= kLds, "three blocks of either key group: one each that values, keys and widening are at");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, h = lane >> 4;
    const int split = blockIdx.x, g = blockIdx.y, group = blockIdx.z;
    auto token_of = [&](int row) { return p.G == 1 ? row : (int)__umulhi((unsigned)row, p.by_G); };
    if (group >= p.n_groups) {
        const int item = (((group - p.n_groups) * p.Hkv + g) * p.nsplit + split) * kWaves + wave;
        if (item >= p.n_keeping) return;
        const int kept = p.T - p.first_kept, block = p.len / kBlockRows + item / p.Hkv, head = item % p.Hkv;
        const int64_t row_bytes = (int64_t)p.Hkv * 256, src = p.first_kept * row_bytes + head * 256 + 16 * i16;
        write_block(p.cache + ((int64_t)block * p.Hkv + head) * kBlockBytes, p.k + src, p.v + src, row_bytes, block * kBlockRows, p.len, p.len + kept, lane);
        return;
    }
    const int rt = wave % kRT, kg = wave / kRT;
    const int row0 = (group * kRT + rt) * kTileRows;
    // blocks that rows of the group see: the cache's and the run's own up to its last token
    const int last_row = min((group + 1) * kRT * kTileRows, p.M) - 1;
    // (an own block takes about twice a cached one's time: the shares are even in that measure)
    const unsigned total = p.n_cache_blocks + 2 * (token_of(last_row) / 32 + 1), share = total / p.nsplit, more = total - share * p.nsplit;
    auto border = [&](int s) {
        const int at = s * share + min((unsigned)s, more);
        return at <= p.n_cache_blocks ? at : p.n_cache_blocks + (at - p.n_cache_blocks + 1) / 2;
    };
    const int first = border(split), end = border(split + 1);
    const int stop = min(end, p.n_cache_blocks);
    const char* const base = p.cache + (int64_t)g * kBlockBytes;
    const int64_t stride = (int64_t)p.Hkv * kBlockBytes, row_bytes = (int64_t)p.Hkv * 256;

    State st;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) st.o[c][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        st.excess[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        st.m[c] = st.l[c] = 0.f;
        st.limit[c] = -INFINITY;
    }
    raw16 query[2][4];
    int last[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int row = min(row0 + 16 * c + i16, p.M - 1), t = token_of(row);
        const char* const at = p.q + (((int64_t)t * p.Hq + (int64_t)g * p.G + row - t * p.G) * D + 8 * h) * 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) query[c][i] = *reinterpret_cast<const raw16*>(at + 64 * i);
        last[c] = t;
    }
    // kRT = 1: a power of two that weights carry (and the sums), so that p of rows of V that are very small or large throughout stays in the range of an fp32
    float unit = 1.f;
    // the run's own blocks (kRT = 1: from the last key group on, the first ones have one more of the cache's if any)
    auto own_blocks = [&] {
        int j = max(first, p.n_cache_blocks) + (kShared ? kg : kKG - 1 - kg) - p.n_cache_blocks;
        const int own_end = end - p.n_cache_blocks;
        if (j >= own_end) return;
        const char *const k = p.k + (int64_t)g * 256, *const v = p.v + (int64_t)g * 256;
        bf16x8 keys[2][4];
        ask_own_keys(keys, k, row_bytes, j, p.T, i16, h);
        for (; j < own_end; j += kKG) attend_own(st, keys, k, v, row_bytes, j, kKG, p.T, query, p.scale_log2e, last, kShared ? 1.f : unit, i16, h);
    };
    int b = first + kg;  // the block that this wavefront is at
    if constexpr (kShared) {
        raw16 k{}, v{}, k1{}, v1{};
        unsigned pair = 0, pair1 = 0;
        auto ask = [&](int block) {  // a quarter of a block (behind the last one: that one again)
            const char* const blk = base + min(block, stop - 1) * stride;
            k = *reinterpret_cast<const raw16*>(blk + rt * 1024 + lane * 16);
            v = *reinterpret_cast<const raw16*>(blk + kBlockV + rt * 1024 + lane * 16);
            pair = *reinterpret_cast<const unsigned*>(blk + kBlockScales + 4 * (lane & 31));
        };
        auto widen_into = [&](int buffer) {
            char* const to = smem + (2 * buffer + kg) * kStaged;
            char* const mine = to + rt * 2048 + lane * 16;
            *reinterpret_cast<f16x8*>(mine) = keys_of(k[0], k[1]);
            *reinterpret_cast<f16x8*>(mine + 1024) = keys_of(k[2], k[3]);
            *reinterpret_cast<bf16x8*>(mine + 8192) = values_of(v[0], v[1]);
            *reinterpret_cast<bf16x8*>(mine + 9216) = values_of(v[2], v[3]);
            // (by all four, the same)
            *reinterpret_cast<float*>(to + 16384 + 4 * lane) = __uint_as_float(lane < 32 ? pair << 16 : pair & 0xffff0000u);
        };
        if (first < stop) {
            ask(b + 2);
            k1 = k, v1 = v, pair1 = pair;
            ask(b);
        }
        own_blocks();  // (first: their queries are there as they are needed, and the cache's first blocks come meanwhile)
        if (first < stop) {
            const Queries q[2] = {queries_of(query[0], p.scale_log2e), queries_of(query[1], p.scale_log2e)};
            widen_into(0);
            k = k1, v = v1, pair = pair1;
            __syncthreads();
            if (kg == 1) __syncthreads();  // half a turn behind the other group
            const int turns = (stop - first + 1) / 2;
            f32x4 s[2][2];
            bf16x8 weights[2];
            int next = 1;
            const char* block = smem + kg * kStaged;
            multiply_keys(s, q, [&](int kt, int i) { return *reinterpret_cast<const f16x8*>(block + (4 * kt + i) * 1024 + lane * 16); });
            widen_into(next);
            ask(b + 4);
            for (int turn = 0; turn < turns; ++turn, b += 2) {
                __syncthreads();
                f32x4 ks[2], vs[2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    ks[kt] = *reinterpret_cast<const f32x4*>(block + 16384 + 64 * kt + 16 * h);
                    vs[kt] = *reinterpret_cast<const f32x4*>(block + 16384 + 128 + 64 * kt + 16 * h);
                }
                raw16 piece[16];  // of V, then of the next block's K
                const char* const after = smem + (2 * next + kg) * kStaged;
                auto take = [&](int i) {
                    piece[i] = *reinterpret_cast<const raw16*>(i < 8 ? block + 8192 + i * 1024 + lane * 16 : after + (i - 8) * 1024 + lane * 16);
                };
                weigh(st, weights, s, ks, vs, q, b < stop ? p.len - b * kBlockRows : 0, h, [&] {  // (no block is left: none of its rows count)
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) take(i);
                    __builtin_amdgcn_sched_barrier(0);
                });
                __syncthreads();
                // The products, in this order: pieces come from LDS kAhead steps before they are multiplied, and a word is widened at a step.
                __builtin_amdgcn_s_setprio(1);
                next = next == 2 ? 0 : next + 1;
                char* const to = smem + (2 * next + kg) * kStaged;
                char* const mine = to + rt * 2048 + lane * 16;
                const unsigned minus128 = 0xc300c300u;
                const bf16x8 off = __builtin_bit_cast(bf16x8, u32x4{minus128, minus128, minus128, minus128});
#pragma unroll
                for (int c = 0; c < 2; ++c) st.excess[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(off, weights[c], st.excess[c], 0, 0, 0);
                f32x4 fresh[2][2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) fresh[kt][c] = f32x4{q[c].start, q[c].start, q[c].start, q[c].start};
                u32x4 wide;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    // (K's pieces come in the order (kt, step) 0 0, 0 1, .., 1 3)
                    if (i + kAhead < 16) take(i + kAhead);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (i < 8) st.o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, piece[i]), weights[c], st.o[c][i], 0, 0, 0);
                        else {
                            const int kt = (i - 8) >> 2, step = (i - 8) & 3;
                            fresh[kt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, piece[i]), q[c].q[step], fresh[kt][c], 0, 0, 0);
                        }
                    }
                    if (i < 8) {
                        unsigned lo, hi;
                        if (i < 4) widen_key(k[i], lo, hi);
                        else widen(v[i - 4], lo, hi);
                        wide[2 * (i & 1)] = lo;
                        wide[2 * (i & 1) + 1] = hi;
                        if (i & 1) *reinterpret_cast<u32x4*>(mine + (i < 4 ? 0 : 8192) + ((i >> 1) & 1) * 1024) = wide;
                    } else if (i == 8) {
                        *reinterpret_cast<float*>(to + 16384 + 4 * lane) = __uint_as_float(lane < 32 ? pair << 16 : pair & 0xffff0000u);
                    } else if (i == 9) {
                        ask(b + 6);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) s[kt][c] = fresh[kt][c];
                block = after;
                __builtin_amdgcn_s_setprio(0);
            }
            if (kg == 0) __syncthreads();
        }
    } else {
        // the next block is asked for piece by piece as this one's are used up
        raw16 k[4]{}, v[4]{}, pairs[2]{};
        const char* blk = base + b * stride;
        auto ask_keys = [&] {
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const raw16*>(blk + j * 1024 + lane * 16);
        };
        auto ask_values = [&] {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const raw16*>(blk + kBlockV + j * 1024 + lane * 16);
        };
        auto ask_scales = [&] {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) pairs[kt] = *reinterpret_cast<const raw16*>(blk + kBlockScales + 64 * kt + 16 * h);
        };
        Queries q[2];
        if (b < stop) {
            ask_scales();
            ask_keys();
            ask_values();
            q[0] = queries_of(query[0], p.scale_log2e);
            q[1] = queries_of(query[1], p.scale_log2e);
            unsigned top = 0;  // the largest scale of V in the wavefront's first block (as a bit pattern, K's below it)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = max(top, 16 * kt + 4 * h + r < p.len - b * kBlockRows ? pairs[kt][r] : 0u);
            top = __builtin_amdgcn_readfirstlane(over_rows(top, [](unsigned x, unsigned y) { return max(x, y); }));
            if (top < __float_as_uint(0x1p-60f) && top >= __float_as_uint(0x1p-125f)) unit = 0x1p40f;  // (2^-126: rows of zeros)
            else if (top > __float_as_uint(0x1p60f) && top < 0x7f800000u) unit = 0x1p-40f;
        }
        for (; b < stop; b += kKG) {
            if (b + kKG < stop) blk += kKG * stride;  // (behind the last one: that one again)
            f32x4 s[2][2], ks[2], vs[2];
            f16x8 weights[2];
            multiply_keys(s, q, [&](int kt, int i) { return keys_of(k[2 * kt + (i >> 1)][2 * (i & 1)], k[2 * kt + (i >> 1)][2 * (i & 1) + 1]); });
            ask_keys();
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    ks[kt][r] = __uint_as_float(pairs[kt][r] << 16);
                    vs[kt][r] = __uint_as_float(pairs[kt][r] & 0xffff0000u) * unit;
                }
            weigh_for_fp16(st, weights, s, ks, vs, q, p.len - b * kBlockRows, h);
            const unsigned minus1152 = 0xe480e480u;
            const f16x8 off = __builtin_bit_cast(f16x8, u32x4{minus1152, minus1152, minus1152, minus1152});
#pragma unroll
            for (int c = 0; c < 2; ++c) st.excess[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(off, weights[c], st.excess[c], 0, 0, 0);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                const f16x8 a = keys_of(v[dt >> 1][2 * (dt & 1)], v[dt >> 1][2 * (dt & 1) + 1]);  // (code + 1152, as K's)
#pragma unroll
                for (int c = 0; c < 2; ++c) st.o[c][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, weights[c], st.o[c][dt], 0, 0, 0);
            }
            ask_values();
            ask_scales();
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
            if (st.limit[c] != -INFINITY) st.limit[c] = kLazyOwn;
        own_blocks();
    }

    // ---- the key groups meet in LDS, then 16 rows of a wavefront are done ----
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        st.l[c] = sum_over_rows(st.l[c]);
        if (st.limit[c] == -INFINITY) st.m[c] = -INFINITY;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) st.o[c][dt] += st.excess[c];
    }
    if (!kShared && unit != 1.f) {
        const float back = unit > 1.f ? 0x1p-40f : 0x1p40f;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) st.o[c][dt] *= back;
    }
    __syncthreads();  // (blocks may still be read there)
    float* const box = reinterpret_cast<float*>(smem);
    // a set of columns of a wavefront in LDS: [dim % 8][lane][r], then references and sums
    constexpr int kBox = 8 * 64 * 4 + 32;
    auto put = [&](int slot, const f32x4 (&o)[8], float m, float l) {
        float* const to = box + slot * kBox;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(to + (dt * 64 + lane) * 4) = o[dt];
        if (h == 0) {
            to[2048 + i16] = m;
            to[2064 + i16] = l;
        }
    };
    auto add = [&](f32x4 (&o)[8], float& m, float& l, int slot) {
        const float* const from = box + slot * kBox;
        const float m2 = from[2048 + i16], mx = fmaxf(m, m2);
        const float a = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mx), b2 = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m2 - mx);
        m = mx;
        l = l * a + from[2064 + i16] * b2;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[dt] = o[dt] * a + *reinterpret_cast<const f32x4*>(from + (dt * 64 + lane) * 4) * b2;
    };
    // 8 values of a row, dims 32 hs + 8 r .. (hs: any quarter), times inv, to the output or, times 2^(se - 127), to the split's partial results
    auto store = [&](int row, int hs, int r, const float (&o)[8], float inv, int se) {
        if (row >= p.M) return;
        if (p.nsplit == 1) {
            const int t = token_of(row);
            bf16x8 w;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = (__bf16)(o[e] * inv);
            *reinterpret_cast<bf16x8*>(p.out + ((int64_t)t * p.Hq + (int64_t)g * p.G + row - t * p.G) * D + 32 * hs + 8 * r) = w;
        } else {
            const float scale = __uint_as_float((unsigned)se << 23);
            f16x8 w;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = (_Float16)(o[e] * inv * scale);
            *reinterpret_cast<f16x8*>(p.part_o + (((int64_t)split * p.Hkv + g) * p.M + row) * D + 32 * hs + 8 * r) = w;
        }
    };
    auto store_sums = [&](int row, int hs, float m, float l, int se) {
        if (row >= p.M || p.nsplit == 1) return;
        char* const to = p.part_ml + (((int64_t)split * p.Hkv + g) * p.M + row) * 16;
        to[8 + hs] = (char)se;
        if (hs == 0) *reinterpret_cast<float2*>(to) = make_float2(m, l);
    };
    auto inverse_of = [&](float l) { return l == 0.f && p.nsplit > 1 ? 0.f : 1.0f / l; };  // (0: none of the split's keys is visible to the row)
    auto exponent_of = [](float big) {  // (2^126 at most: its inverse is a number too)
        return min(max(127 + 14 + 127 - (int)((__float_as_uint(big) >> 23) & 255u), 1), 253);
    };
    if constexpr (kShared) {  // each group of two does one set of columns
        if (kg == 0) put(wave, st.o[1], st.m[1], st.l[1]);
        else put(wave, st.o[0], st.m[0], st.l[0]);
        __syncthreads();
        if (kg == 1) {
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) st.o[0][dt] = st.o[1][dt];
            st.m[0] = st.m[1];
            st.l[0] = st.l[1];
        }
        add(st.o[0], st.m[0], st.l[0], (wave + kRT) % kWaves);
        const int row = row0 + 16 * kg + i16;
        float big = 0.f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) big = fmaxf(big, fabsf(st.o[0][dt][r]));
        const float inv = inverse_of(st.l[0]);
        const int se = exponent_of(big * inv);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = st.o[0][e][r];
            store(row, h, r, o, inv, se);
        }
        store_sums(row, h, st.m[0], st.l[0], se);
    } else {
        // every wavefront leaves both, and adds 32 dims of one set in the order of the groups, a lane dims 8 (lane % 4) .. of column lane / 4 (two
        // wavefronts with a set each: 1 us more)
        put(2 * wave, st.o[0], st.m[0], st.l[0]);
        put(2 * wave + 1, st.o[1], st.m[1], st.l[1]);
        __syncthreads();
        const int set = wave & 1, quarter = wave >> 1, column = lane >> 2, row = row0 + 16 * set + column;
        const float* const from = box + set * kBox;
        float m[kWaves], l = 0.f, o[8] = {};
#pragma unroll
        for (int n = 0; n < kWaves; ++n) m[n] = from[2 * n * kBox + 2048 + column];
        float mx = m[0];
#pragma unroll
        for (int n = 1; n < kWaves; ++n) mx = fmaxf(mx, m[n]);
#pragma unroll
        for (int n = 0; n < kWaves; ++n) {
            // (the sum in two steps, as in weigh_for_fp16)
            const float half = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(0.5f * (m[n] - mx)), f = half * half;
            l += half * from[2 * n * kBox + 2064 + column] * half;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[dt] += f * from[2 * n * kBox + dt * 256 + quarter * 64 + lane];
        }
        float big = 0.f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) big = fmaxf(big, fabsf(o[dt]));
        big = fmaxf(big, neighbour<0xb1>(big));  // of the four lanes of a column
        big = fmaxf(big, neighbour<0x4e>(big));
        const float inv = inverse_of(l);
        const int se = exponent_of(big * inv);
        store(row, quarter, lane & 3, o, inv, se);
        if ((lane & 3) == 0) store_sums(row, quarter, mx, l, se);
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
        float2 ml[kDepth];
        unsigned se[kDepth];
        f16x8 x[kDepth];
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            const int64_t pr = ((int64_t)min(s0 + u, p.nsplit - 1) * p.Hkv + g) * p.M + row;
            ml[u] = *reinterpret_cast<const float2*>(p.part_ml + pr * 16);
            se[u] = *reinterpret_cast<const unsigned char*>(p.part_ml + pr * 16 + 8 + (d8 >> 5));
            x[u] = *reinterpret_cast<const f16x8*>(p.part_o + pr * D + d8);
        }
        float mx = m;
#pragma unroll
        for (int u = 0; u < kDepth; ++u) mx = fmaxf(mx, ml[u].x);
        const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(0.5f * (m - mx));
        l = l * f * f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = o[e] * f * f;
        m = mx;
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            if (s0 + u >= p.nsplit) continue;
            // (in two steps, as in weigh_for_fp16)
            const float half = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(0.5f * (ml[u].x - mx)), w = half * ml[u].y * half, wo = w * __uint_as_float((254 - se[u]) << 23);
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
    int most;  // splits that no run of as many tokens over fewer rows passes
};
Plan plan_of(const vs_shape& s, int32_t n_tokens, int32_t len) {
    const int G = s.n_q_heads / s.n_kv_heads, tiles = (n_tokens * G + kTileRows - 1) / kTileRows;
    const int cached = (len + kBlockRows - 1) / kBlockRows, own = (n_tokens + 31) / 32;
    Plan pl{};
    pl.most = 1;
    float least = INFINITY;
    auto consider = [&](int rt, int groups, int nsplit, float us) {
        if (us >= least) return;
        least = us, pl.rt = rt, pl.groups = groups, pl.nsplit = nsplit;
    };
    auto way = [&](int rt, float group, float block, float own_block) {
        const int groups = (tiles + rt - 1) / rt, units = groups * s.n_kv_heads;
        const float blocks = cached + own_block * own;
        const int n = std::max(1, std::min({256 / units, (cached + own) * rt / kWaves, kMaxSplits}));
        consider(rt, groups, 1, 3.5f + ((units + 255) / 256) * (group + block * blocks));
        if (n > 1) consider(rt, groups, n, 3.5f + group + block * blocks / n + 5.0f);
        pl.most = std::max(pl.most, n);
    };
    // What a call takes, in us, from what was measured: a launch, what a workgroup takes besides its blocks, and each of its blocks, as often
    // as workgroups follow one another on a compute unit; or as many splits as run at once, a block for every key group at least,
    // and the launch that adds them.  One tile a workgroup has no merge where four have one; four spend fewer instructions on a block.
    // Attention and merge, us, one tile / four, tokens x rows: 28/4 heads 10x200 8.5 / 12.4, 37x711 11.7 / 18.0, 64x1500 16.1 / 21.0,
    // 100x8000 32.8 / 33.3, 170x352 11.0 / 20.4, 170x2400 20.4 / 26.2, 170x4416 29.1 / 32.1, 170x7000 40.5 / 39.4, 170x11016 58.0 / 50.5,
    // 600x1000 42.7 / 45.6, 1024x0 45.5 / 41.8; 64/8 heads 300x300 28.8 / 24.6, 2048x200 269 / 227; 8/1 heads 170x11016 24.8 / 29.4.
    way(1, 5.1f, 0.144f, 1.0f);
    way(4, 10.2f, 0.525f, 1.25f);  // (causal: the longest of a group's rows count)
    return pl;
}
size_t partial_bytes(const vs_shape& s, int32_t n_tokens, int nsplit) {
    return nsplit <= 1 ? 0 : (size_t)nsplit * n_tokens * s.n_q_heads * (D * sizeof(_Float16) + 16);
}

}  // namespace

size_t prefill8_workspace_need(const vs_shape& s, int32_t n_tokens, int32_t len) { return partial_bytes(s, n_tokens, plan_of(s, n_tokens, len).nsplit); }

// What any run of at most max_tokens over at most max_len rows needs.
size_t prefill8_workspace_bytes(const vs_shape& s, int32_t max_tokens, int32_t max_len) {
    size_t most = 0;
    for (int32_t t = 1; t <= max_tokens; ++t) most = std::max(most, partial_bytes(s, t, plan_of(s, t, max_len).most));
    return most;
}

hipError_t launch_prefill8(const vs_shape& s, void* cache, int32_t len, const void* q, const void* k, const void* v, int32_t n_tokens,
                           int32_t first_kept, void* out, void* workspace, hipStream_t st) {
    const Plan pl = plan_of(s, n_tokens, len);
    Prefill8Params p;
    p.cache = (char*)cache;
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
    p.part_ml = (char*)workspace;
    p.part_o = (_Float16*)(p.part_ml + (int64_t)pl.nsplit * p.M * p.Hkv * 16);
    p.by_G = (unsigned)(0xffffffffu / p.G + 1u);  // exact for row * G < 2^32
    p.first_kept = first_kept;
    p.n_keeping = first_kept < n_tokens ? ((len + n_tokens - first_kept - 1) / kBlockRows - len / kBlockRows + 1) * p.Hkv : 0;
    const int per_plane = pl.nsplit * p.Hkv * kWaves;
    const dim3 grid(pl.nsplit, p.Hkv, pl.groups + (p.n_keeping + per_plane - 1) / per_plane);
    if (pl.rt == 1) prefill8_kernel<1><<<grid, kThreads, 0, st>>>(p);
    else prefill8_kernel<4><<<grid, kThreads, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.nsplit == 1) return e;
    prefill8_combine_kernel<<<(p.M * p.Hkv + 15) / 16, 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace vs
