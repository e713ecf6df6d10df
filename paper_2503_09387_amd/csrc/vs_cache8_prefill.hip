// Prefill attention over a cache in 8 bits (Eq. 1 of Section 3.1; Section 3.3): a run's tokens over the retained rows and, causally, over
// one another.  The arithmetic is in vs_cache8_attn.h.  The G query heads of a KV head are packed into rows (row = token * G + head).
// A wavefront holds 32 rows (two sets of 16 columns) and walks blocks of 32 keys, from memory into the multiplier, widened as they are multiplied.
// A workgroup is 4 wavefronts that take the blocks of the same rows in turn and add their sums in LDS; two workgroups fit a compute unit, so
// that one multiplies while the other starts or ends.  us by workgroup, 28/4 heads, 37 tokens over 711 rows, 170 over 11016, 600 over 1000, 2048 over 200:
//   4 wavefronts 10.4, 47.4, 31.8, 95;  8, one workgroup to a compute unit 11.8, 58.2, 43.2, 125;  2 12.4, 48.8, 35.2, 97;
//   8 of 128 rows that share a block, widened once, through LDS 17.4, 51.2, 45.8, 128.
// A block's turn is one chain (scores, weights, values) of 34 matrix and some 200 vector instructions, 64 of which widen codes, and the two
// wavefronts of a SIMD go through it without filling each other's gaps: of 83 k cycles a SIMD (170 over 11016 in three splits) matrix instructions
// are 28 k and vector ones some 60 k, exponentials at a quarter of the rate.  The sum of the two is what bounds it, neither pipe is full: 45.9 us =
// 590 TFLOP/s, and 4.7 to add the splits.  (The prefill over rows in bf16 widens nothing and overlaps the two: 35.4 us for the same.)  Few blocks are
// bound by some 7 us of start and end: launch, first trips to memory, the queries' conversion, the sums' way through LDS, stores.
#include "vs_cache8_attn.h"

#include <algorithm>

namespace vs {
namespace {

constexpr int D = 128;
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTileRows = 32;  // rows of a workgroup
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazyMax = 8.0f;     // scores may exceed the reference maximum by 2^8 before it is refreshed
constexpr float kMaxWeight = 15.0f;  // log2 of the largest weight that goes into an fp16
constexpr float kLazyOwn = 20.0f;    // as kLazyMax for a run's own rows, behind cached ones whose weights have set the reference
constexpr unsigned kLargeOwn = (127 + 60) << 7;  // 2^60, a bf16
constexpr int kMaxSplits = 32;

struct Prefill8Params {
    char* cache;
    const char* q;
    const char* k;   // the run's own rows
    const char* v;
    __bf16* out;
    _Float16* part_o;  // [split][Hkv][row][128] (half the bytes of an fp32 through memory; 11 bits, where the output has 8) normalised, times the power of two that brings the largest of 32 dims into [2^14, 2^15)
    char* part_ml;     // [split][Hkv][row][16 bytes]: reference (log2 units), sum, the biased exponents of the four powers, unused
    int len, T, G, Hq, Hkv, M;
    int n_cache_blocks;
    int n_tiles;       // of kTileRows rows
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
    float limit[2];    // what weights, of a run's own rows scores, may come to before the reference is refreshed, log2: -INFINITY until a key has been seen
};

// A value that all lanes have, in a scalar register.
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// Scores less the reference become probabilities; the sums take them.  room: log2 of what probabilities may come to beside these values.
__device__ __forceinline__ void soften(State& st, float (&x)[2][8], float room) {
    const float mx[2] = {max_of_8(x[0]), max_of_8(x[1])};
    if (__any(mx[0] > fminf(st.limit[0], room) || mx[1] > fminf(st.limit[1], room))) {  // rare after the first block
        asm volatile("s_nop 15\n\ts_nop 15");  // (the last matrix instruction's sums, before assembly that the compiler does not look into)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const bool seen = st.limit[c] != -INFINITY;
            float up = max_over_rows(mx[c]) - fminf(room, 0.f);
            if (seen) up = fmaxf(up, 0.f);
            if (up == -INFINITY) up = 0.f;  // (the column sees none of these keys and has seen none before)
            else st.limit[c] = kLazyMax;
            // (in two steps, as in weigh)
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
// weights w = p s_v unit of the first `valid` rows, as fp16 like the codes of V: a code becomes an fp16 in a third of the instructions that a bf16
// takes, and a weight has 11 bits.  It is w that the reference holds in range: at most 2^15, the largest 2^6 when it is set; what is below 2^-14 loses
// bits, 2^-25 a key at most, of what has a key of 2^6.  p is an fp32 of any size up to 2^96 (rows of zeros, of the smallest scale, that a
// query likes best).  unit: see the kernel.
__device__ __forceinline__ void weigh(State& st, f16x8 (&w)[2], const f32x4 (&s)[2][2], const f32x4 (&ks)[2], const f32x4 (&vs)[2], const Queries (&q)[2],
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

// The largest scale of V (as a bit pattern, K's below it) of a wavefront's blocks b, b + kWaves, ..: 8 lanes take a block's 32 pairs,
// kScanDepth times 8 blocks from number n on.
constexpr int kScanDepth = 4;
__device__ __forceinline__ int scan_block(int b, int n, int u, int lane) { return b + (n + 8 * u + (lane >> 3)) * kWaves; }
__device__ __forceinline__ void ask_block_scales(raw16 (&to)[kScanDepth], const char* scales, int64_t stride, int b, int n, int stop, int lane) {
#pragma unroll
    for (int u = 0; u < kScanDepth; ++u) to[u] = *reinterpret_cast<const raw16*>(scales + min(scan_block(b, n, u, lane), stop - 1) * stride + 16 * (lane & 7));
}
__device__ __forceinline__ unsigned top_of(const raw16 (&scales)[kScanDepth], int b, int n, int stop, int len, int lane) {
    unsigned top = 0;
#pragma unroll
    for (int u = 0; u < kScanDepth; ++u) {
        const int row = kBlockRows * scan_block(b, n, u, lane) + 4 * (lane & 7);
#pragma unroll
        for (int r = 0; r < 4; ++r) top = max(top, row + r < len ? scales[u][r] : 0u);
    }
    return top;
}
// The largest of all lanes' values, in a scalar register.
__device__ __forceinline__ unsigned over_lanes(unsigned x) {
    x = over_rows(x, [](unsigned a, unsigned b) { return max(a, b); });
    x = max(x, turned<8>(x));
    x = max(x, turned<4>(x));
    x = max(x, turned<2>(x));
    return __builtin_amdgcn_readfirstlane(max(x, turned<1>(x)));
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
// Such a block: column c sees keys up to `last[c]` of the run.  The keys of block j + step are asked for on the way.
__device__ __forceinline__ void attend_own(State& st, bf16x8 (&keys)[2][4], const char* k, const char* v, int64_t row_bytes, int j, int step, int T,
                                           const raw16 (&q)[2][4], float f, const int (&last)[2], int i16, int h) {
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
    auto most_of = [](const raw16 (&w)[8]) {
        unsigned most = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = max_pairs(most, w[e][i] & 0x7fff7fffu);
        return max(most & 0xffffu, most >> 16);
    };
    const unsigned most = most_of(x);
    if (__any(most > 0x7f7fu)) {
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
    // Values of 2^60 and more leave probabilities, which may stand at 2^20 and behind rows of smaller values higher, less room: products of at most
    // 2^100, so that the sums over a run stay numbers.
    float room = kLazyOwn;
    if (__any(most >= kLargeOwn)) room = fminf(room, (float)(100 + 126 - (int)(over_lanes(most_of(x)) >> 7)));
    soften(st, z, room);
    bf16x8 p[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) p[c][e] = (__bf16)z[c][e];
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

// Grid (splits, Hkv, row tiles and more): workgroups that read the same keys are Hkv * splits apart.  Those beyond the tiles quantise the
// rows that are kept, a block and KV head each wavefront; whoever attends to the block they go to leaves out rows from len on.
__global__ __launch_bounds__(kThreads, 2) void prefill8_kernel(Prefill8Params p) {
    // a set of columns of a wavefront: [dim % 8][lane][r], then references and sums
    constexpr int kBox = 8 * 64 * 4 + 32;
    __shared__ __attribute__((aligned(16))) float box[2 * kWaves * kBox];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, h = lane >> 4;
    const int split = blockIdx.x, g = blockIdx.y, tile = blockIdx.z;
    auto token_of = [&](int row) { return p.G == 1 ? row : (int)__umulhi((unsigned)row, p.by_G); };
    if (tile >= p.n_tiles) {
        const int item = (((tile - p.n_tiles) * p.Hkv + g) * p.nsplit + split) * kWaves + wave;
        if (item >= p.n_keeping) return;
        const int kept = p.T - p.first_kept, block = p.len / kBlockRows + item / p.Hkv, head = item % p.Hkv;
        const int64_t row_bytes = (int64_t)p.Hkv * 256, src = p.first_kept * row_bytes + head * 256 + 16 * i16;
        write_block(p.cache + ((int64_t)block * p.Hkv + head) * kBlockBytes, p.k + src, p.v + src, row_bytes, block * kBlockRows, p.len, p.len + kept, lane);
        return;
    }
    const int row0 = tile * kTileRows;
    // blocks that rows of the tile see: the cache's and the run's own up to its last token
    const int last_row = min(row0 + kTileRows, p.M) - 1;
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
    // a power of two that weights over cached rows carry (and the sums), so that their p stay in the range of an fp32, with room for smaller ones, whatever
    // the size of V.  It goes by the largest scale in all of the wavefront's blocks, which are looked through while the first block and the queries
    // are on their way (0.1 .. 0.3 us): small rows may come first and far larger ones behind them.
    float unit = 1.f;
    // the run's own blocks (from the last wavefront on: the first ones have one more of the cache's if any)
    auto own_blocks = [&] {
        int j = max(first, p.n_cache_blocks) + kWaves - 1 - (int)wave - p.n_cache_blocks;
        const int own_end = end - p.n_cache_blocks;
        if (j >= own_end) return;
        const char *const k = p.k + (int64_t)g * 256, *const v = p.v + (int64_t)g * 256;
        bf16x8 keys[2][4];
        ask_own_keys(keys, k, row_bytes, j, p.T, i16, h);
        for (; j < own_end; j += kWaves) attend_own(st, keys, k, v, row_bytes, j, kWaves, p.T, query, p.scale_log2e, last, i16, h);
    };
    int b = first + wave;  // the block that this wavefront is at
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
        raw16 scales[kScanDepth];
        ask_block_scales(scales, base + kBlockScales, stride, b, 0, stop, lane);
        ask_scales();
        ask_keys();
        ask_values();
        q[0] = queries_of(query[0], p.scale_log2e);
        q[1] = queries_of(query[1], p.scale_log2e);
        unsigned top = top_of(scales, b, 0, stop, p.len, lane);
        for (int n = 8 * kScanDepth; b + n * kWaves < stop; n += 8 * kScanDepth) {
            ask_block_scales(scales, base + kBlockScales, stride, b, n, stop, lane);
            top = max(top, top_of(scales, b, n, stop, p.len, lane));
        }
        top = over_lanes(top);
        if (top < __float_as_uint(0x1p-60f)) unit = 0x1p40f;
        else if (top > __float_as_uint(0x1p90f)) unit = 0x1p-40f;
    }
    for (; b < stop; b += kWaves) {
        if (b + kWaves < stop) blk += kWaves * stride;  // (behind the last one: that one again)
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
        weigh(st, weights, s, ks, vs, q, p.len - b * kBlockRows, h);
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
    if (unit != 1.f) {  // (the run's own rows have none)
        asm volatile("s_nop 15\n\ts_nop 15");  // (as in soften)
        const float back = unit > 1.f ? 0x1p-40f : 0x1p40f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            scale_in_place(st.excess[c], back);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) scale_in_place(st.o[c][dt], back);
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (st.limit[c] != -INFINITY) st.limit[c] = kLazyOwn;
    own_blocks();

    // ---- the wavefronts' sums meet in LDS ----
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        st.l[c] = sum_over_rows(st.l[c]);
        if (st.limit[c] == -INFINITY) st.m[c] = -INFINITY;
        float* const to = box + (2 * wave + c) * kBox;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(to + (dt * 64 + lane) * 4) = st.o[c][dt] + st.excess[c];
        if (h == 0) {
            to[2048 + i16] = st.m[c];
            to[2064 + i16] = st.l[c];
        }
    }
    __syncthreads();
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
    // a wavefront adds half the dims of one set in the order of the wavefronts, a lane 8 (lane % 4) .. of a quarter's 32 of column lane / 4
    const int set = wave & 1, column = lane >> 2, row = row0 + 16 * set + column;
    const float* const from = box + set * kBox;
    float f[kWaves], l = 0.f, mx = -INFINITY;
#pragma unroll
    for (int n = 0; n < kWaves; ++n) {
        f[n] = from[2 * n * kBox + 2048 + column];
        mx = fmaxf(mx, f[n]);
    }
#pragma unroll
    for (int n = 0; n < kWaves; ++n) {
        // (the sum in two steps, as in weigh)
        const float half = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(0.5f * (f[n] - mx));
        l += half * from[2 * n * kBox + 2064 + column] * half;
        f[n] = half * half;
    }
    const float inv = inverse_of(l);
#pragma unroll
    for (int quarter = wave >> 1; quarter < 4; quarter += kWaves / 2) {
        float o[8] = {}, big = 0.f;
#pragma unroll
        for (int n = 0; n < kWaves; ++n)
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[dt] += f[n] * from[2 * n * kBox + dt * 256 + quarter * 64 + lane];
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) big = fmaxf(big, fabsf(o[dt]));
        big = fmaxf(big, neighbour<0xb1>(big));  // of the four lanes of a column
        big = fmaxf(big, neighbour<0x4e>(big));
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
            // (in two steps, as in weigh)
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

// Row tiles, and workgroups that share a tile's keys.
struct Plan {
    int tiles, nsplit;
    int most;  // splits that no run of as many tokens over fewer rows passes
};
Plan plan_of(const vs_shape& s, int32_t n_tokens, int32_t len) {
    const int G = s.n_q_heads / s.n_kv_heads, tiles = (n_tokens * G + kTileRows - 1) / kTileRows, units = tiles * s.n_kv_heads;
    const int blocks = blocks_of(len) + blocks_of(n_tokens);
    Plan pl{tiles, 1, std::max(1, std::min({512 / units, blocks / kWaves, kMaxSplits}))};
    // The number of splits by what a call takes, in us, from what was measured: a workgroup alone on a compute unit, or two, by what it takes at all and each
    // of its blocks; and the launch that adds splits.  By splits, 28/4 heads: 37 tokens over 711 rows 10.4 at 1, 12.0 at 3; 64 over 3000 23.3 at 1, 16.6 at
    // 4, 18.4 at 9; 1 over 4000 28.1 at 1, 13.1 at 6, 14.7 at 32; 100 over 4000 29.6 at 1, 24.1 at 2, 22.1 at 5; 170 over 2400 21.6 at 1, 22.4 at 3; over 4416 32.7 at 1, 33.1 at 2, 28.4 at 3.
    float least = INFINITY;
    for (int n = 1; n <= pl.most; ++n) {
        const float us = (units * n <= 256 ? 6.8f + 0.183f * blocks / n : 10.8f + 0.262f * blocks / n) + (n > 1 ? 4.5f + 0.1f * n : 0.0f);
        if (us < least) least = us, pl.nsplit = n;
    }
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
    p.n_cache_blocks = blocks_of(len);
    p.n_tiles = pl.tiles;
    p.nsplit = pl.nsplit;
    p.scale_log2e = s.softmax_scale * kLog2e;
    p.part_ml = (char*)workspace;
    p.part_o = (_Float16*)(p.part_ml + (int64_t)pl.nsplit * p.M * p.Hkv * 16);
    p.by_G = (unsigned)(0xffffffffu / p.G + 1u);  // exact for row * G < 2^32
    p.first_kept = first_kept;
    p.n_keeping = first_kept < n_tokens ? ((len + n_tokens - first_kept - 1) / kBlockRows - len / kBlockRows + 1) * p.Hkv : 0;
    const int per_plane = pl.nsplit * p.Hkv * kWaves;
    const dim3 grid(pl.nsplit, p.Hkv, pl.tiles + (p.n_keeping + per_plane - 1) / per_plane);
    prefill8_kernel<<<grid, kThreads, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.nsplit == 1) return e;
    prefill8_combine_kernel<<<(p.M * p.Hkv + 15) / 16, 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace vs
