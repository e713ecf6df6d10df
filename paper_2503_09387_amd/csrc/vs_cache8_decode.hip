// Decode attention over caches in 8 bits (Eq. 1 of Section 3.1; Section 3.3, decoding phase): one query token per stream.
//
//   score(key) = (q . k_codes) * s_k * scale,   out = sum_key p(key) s_v(key) v_codes / sum_key p(key)
//
// The scales belong to rows, so neither product needs a value of K or V as what it stands for:
//   * q . k_codes: v_mfma_i32_16x16x64_i8 on the codes as they lie in memory.  A query row is held as whole numbers of
//     16 bits, x = 256 hi + lo, with the power of two that brings its largest entry into [2^14, 2^15): entries down
//     to 2^-7 of the largest are exact (a bf16 has 8 bits), smaller ones are off by at most 2^-16 of the largest.  Two
//     products per 64 dims, their sums exact in 32 bits, and no conversion of K at all.
//   * p s_v goes to bf16 (8 bits, as P does over caches in bf16; the denominator sums p before that), V's codes + 128 become
//     bf16 without a rounding (at most 255), and the 128 times the sum of p s_v too much that the product then holds comes off through
//     one more product with a matrix of -128.
// The G query heads of a KV head are the columns of the products, padded to 16.
#include "vs_cache8.h"

#include <algorithm>

namespace vs {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int D = 128;
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRowStride = D + 4;  // of a query head's sums in LDS, in floats
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazyMax = 8.0f;  // scores may exceed the reference maximum by 2^8 before it is refreshed

struct Decode8Params {
    char* slab;
    const char* q;
    const char* k_new;  // may be null
    const char* v_new;
    __bf16* out;
    float* part_o;       // [share][Hkv][G][D], not normalised
    float* part_ml;      // [share][Hkv][G][2]: reference (log2 units), sum
    int64_t cache_bytes;
    int G, Hq, Hkv;
    float scale_log2e;
    LenTable lens;       // valid rows per stream, the appended row included
    int share_end[kMaxStreamsPerLaunch];  // shares of the streams up to and with this one
};

// A block of 32 rows of one KV head in a wavefront's registers.
struct Block {
    raw16 k[4], v[4], s[2];
};

__device__ __forceinline__ raw16 load_once(const char* p) {  // every byte of a cache is read once in a launch
    return __builtin_nontemporal_load(reinterpret_cast<const raw16*>(p));
}
__device__ __forceinline__ void fetch(Block& b, const char* blk, int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j) b.k[j] = load_once(blk + j * 1024 + lane * 16);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) b.s[kt] = load_once(blk + kBlockScales + 64 * kt + 16 * (lane >> 4));
#pragma unroll
    for (int j = 0; j < 4; ++j) b.v[j] = load_once(blk + kBlockV + j * 1024 + lane * 16);
}

// four codes of V as bf16: whole numbers 0..255, whose fp32 has nothing in its lower half
__device__ __forceinline__ void widen(unsigned w, unsigned& lo, unsigned& hi) {
    const unsigned a = __float_as_uint((float)(w & 255u)), b = __float_as_uint((float)((w >> 8) & 255u));
    const unsigned c = __float_as_uint((float)((w >> 16) & 255u)), d = __float_as_uint((float)(w >> 24));
    lo = __builtin_amdgcn_perm(b, a, 0x07060302u);
    hi = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

struct State {
    f32x4 o[8];   // [dim % 8]: element r of lane (query i16, h): dim 8 (4 h + r) + dim % 8, 128 per unit of p s_v too large
    f32x4 excess; // and what is too much
    float m, l;   // reference (log2 units, the same in the lanes of a query), this lane's share of the sum
};

struct Query {
    i32x4 hi[2], lo[2];
    float f;  // scale and log2 e over the power of two of the row's whole numbers
};

// One block.  kPartly: only its first `valid` rows are there.
template <bool kPartly>
__device__ __forceinline__ void attend(State& st, const Block& b, const Query& q, int valid, int h) {
    float z[8], sv[8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        i32x4 hi = {0, 0, 0, 0}, lo = hi;
#pragma unroll
        for (int ds = 0; ds < 2; ++ds) {
            const i32x4 k = __builtin_bit_cast(i32x4, b.k[2 * kt + ds]);
            hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(k, q.hi[ds], hi, 0, 0, 0);
            lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(k, q.lo[ds], lo, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const unsigned pair = b.s[kt][r];
            const bool there = !kPartly || 16 * kt + 4 * h + r < valid;
            const float x = (float)((hi[r] << 8) + lo[r]) * (q.f * __uint_as_float(pair << 16));
            z[4 * kt + r] = there ? x : -INFINITY;
            sv[4 * kt + r] = there ? __uint_as_float(pair & 0xffff0000u) : 0.f;
        }
    }
    float mx = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
    if (__any(mx > st.m + kLazyMax)) {  // rare after the first block
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(st.m, mx), alpha = __builtin_amdgcn_exp2f(st.m - m_new);  // 0 at first
        st.m = m_new;
        st.l *= alpha;
        st.excess *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) st.o[dt] *= alpha;
    }
    bf16x8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float pe = __builtin_amdgcn_exp2f(z[e] - st.m);
        st.l += pe;
        p[e] = (__bf16)(pe * sv[e]);
    }
    const unsigned minus128 = 0xc300c300u;
    const bf16x8 off = __builtin_bit_cast(bf16x8, u32x4{minus128, minus128, minus128, minus128});
    st.excess = __builtin_amdgcn_mfma_f32_16x16x32_bf16(off, p, st.excess, 0, 0, 0);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        u32x4 a;
        unsigned x, y;
        widen(b.v[dt >> 1][2 * (dt & 1)], x, y);
        a[0] = x, a[1] = y;
        widen(b.v[dt >> 1][2 * (dt & 1) + 1], x, y);
        a[2] = x, a[3] = y;
        st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), p, st.o[dt], 0, 0, 0);
    }
}

// Lane (query i16, h) of the columns: dims 32 i + 8 h .. of the row, whole numbers of 16 bits.
__device__ __forceinline__ Query query_of(const char* row, int h, float scale_log2e) {
    raw16 x[4];
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = *reinterpret_cast<const raw16*>(row + 64 * i + 16 * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) most = max_pairs(most, x[i][j] & 0x7fff7fffu);
    }
    most = max(most & 0xffffu, most >> 16);
    most = max(most, (unsigned)__shfl_xor((int)most, 16));
    most = max(most, (unsigned)__shfl_xor((int)most, 32));
    // 2^up brings a largest entry of exponent e into [2^14, 2^15); zeros and subnormal numbers go as if they had the smallest exponent
    const int up = 14 + 127 - max((int)(most >> 7), 1);
    Query q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned hi[2] = {0u, 0u}, lo[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned pair = x[i][j >> 1];
            const float v = ldexpf(__uint_as_float(j & 1 ? pair & 0xffff0000u : pair << 16), up);
            // (hi fits 8 bits up to 32639; 32640, the one number beyond, gives up 2^-15 of itself)
            const int n = (int)rintf(fminf(fmaxf(v, -32639.f), 32639.f)), n_hi = (n + 128) >> 8;
            hi[j >> 2] |= (unsigned)(n_hi & 255) << (8 * (j & 3));
            lo[j >> 2] |= (unsigned)(n & 255) << (8 * (j & 3));
        }
        q.hi[i >> 1][2 * (i & 1)] = (int)hi[0];
        q.hi[i >> 1][2 * (i & 1) + 1] = (int)hi[1];
        q.lo[i >> 1][2 * (i & 1)] = (int)lo[0];
        q.lo[i >> 1][2 * (i & 1) + 1] = (int)lo[1];
    }
    // a query that is not finite gives scores that are not numbers
    q.f = most > 0x7f7fu ? __uint_as_float(0x7fc00000u) : ldexpf(scale_log2e, -up);
    return q;
}

// Grid (shares of all streams, Hkv).  A workgroup is a share of one stream's blocks for one KV head; its wavefronts take the blocks
// in turn and meet in LDS.  A stream of one share is then done; the others leave a partial result for the second kernel.
__global__ __launch_bounds__(kThreads, 2) void decode8_kernel(Decode8Params p) {
    __shared__ __attribute__((aligned(16))) float s_o[kWaves][kMaxGroup][kRowStride];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, h = lane >> 4, g = blockIdx.y, share = blockIdx.x;
    static_assert(kMaxStreamsPerLaunch == 64, "one lane per stream");
    const int end_of = p.share_end[lane], len_of = p.lens.v[lane];
    const int s = __builtin_popcountll(__ballot(end_of <= share));
    const int len = __builtin_amdgcn_readlane(len_of, s);
    const int first_share = s ? __builtin_amdgcn_readlane(end_of, s - 1) : 0;
    const int n_shares = __builtin_amdgcn_readlane(end_of, s) - first_share, j_share = share - first_share;
    const int n_blocks = (len + kBlockRows - 1) / kBlockRows;
    const int first = (int)((int64_t)n_blocks * j_share / n_shares), end = (int)((int64_t)n_blocks * (j_share + 1) / n_shares);
    char* const base = p.slab + s * p.cache_bytes + (int64_t)g * kBlockBytes;
    const int64_t stride = (int64_t)p.Hkv * kBlockBytes;

    // the step's new row, by the wavefront that attends over the block that it falls into
    if (p.k_new && end == n_blocks && wave == (n_blocks - 1 - first) % kWaves) {
        const int key = (len - 1) % kBlockRows;
        const int64_t at = ((int64_t)s * p.Hkv + g) * 256 + 16 * i16;
        const raw16 k = *reinterpret_cast<const raw16*>(p.k_new + at), v = *reinterpret_cast<const raw16*>(p.v_new + at);
        char* const blk = base + (n_blocks - 1) * stride;
        uint2 k_codes;
        unsigned v_codes[8];
        const unsigned pair = quantise(k, v, k_codes, v_codes);
        if (h == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) blk[v_code_offset(key, i16, j)] = (char)v_codes[j];
            *reinterpret_cast<uint2*>(blk + k_code_offset(key, i16)) = k_codes;
            if (i16 == 0) *reinterpret_cast<unsigned*>(blk + kBlockScales + 4 * key) = pair;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");  // the wavefront reads what its lanes have just written
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }

    State st;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) st.o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    st.excess = st.o[0];
    st.m = -INFINITY;
    st.l = 0.f;
    int b = first + wave;
    Block x, y;
    if (b < end) {
        fetch(x, base + b * stride, lane);
        if (b + kWaves < end) fetch(y, base + (b + kWaves) * stride, lane);
        const Query q = query_of(p.q + ((int64_t)s * p.Hq + (int64_t)g * p.G + min(i16, p.G - 1)) * 256, h, p.scale_log2e);
        for (; b < end; b += 2 * kWaves) {
            if (b + 1 == n_blocks) attend<true>(st, x, q, len - b * kBlockRows, h);
            else attend<false>(st, x, q, 0, h);
            if (b + 2 * kWaves < end) fetch(x, base + (b + 2 * kWaves) * stride, lane);
            if (b + kWaves < end) {
                if (b + kWaves + 1 == n_blocks) attend<true>(st, y, q, len - (b + kWaves) * kBlockRows, h);
                else attend<false>(st, y, q, 0, h);
                if (b + 3 * kWaves < end) fetch(y, base + (b + 3 * kWaves) * stride, lane);
            }
        }
    }
    st.l += __shfl_xor(st.l, 16);
    st.l += __shfl_xor(st.l, 32);
    if (h == 0) {
        s_m[wave][i16] = st.m;
        s_l[wave][i16] = st.l;
    }
    __syncthreads();
    if (i16 < p.G) {
        float mx = s_m[0][i16];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) mx = fmaxf(mx, s_m[w][i16]);
        const float f = __builtin_amdgcn_exp2f(st.m - mx);  // 0 for a wavefront without blocks
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (st.o[4 * half + e][r] + st.excess[r]) * f;
                *reinterpret_cast<f32x4*>(&s_o[wave][i16][8 * (4 * h + r) + 4 * half]) = w;
            }
    }
    __syncthreads();
    for (int it = tid; it < p.G * (D / 4); it += kThreads) {
        const int head = it / (D / 4), d = 4 * (it % (D / 4));
        float mx = s_m[0][head];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) mx = fmaxf(mx, s_m[w][head]);
        float l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            l += s_l[w][head] * __builtin_amdgcn_exp2f(s_m[w][head] - mx);
            o += *reinterpret_cast<const f32x4*>(&s_o[w][head][d]);
        }
        if (n_shares == 1) {
            const float inv = 1.0f / l;
            bf16x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = (__bf16)(o[e] * inv);
            *reinterpret_cast<bf16x4*>(p.out + ((int64_t)s * p.Hq + (int64_t)g * p.G + head) * D + d) = r;
        } else {
            const int64_t pr = ((int64_t)share * p.Hkv + g) * p.G + head;
            *reinterpret_cast<f32x4*>(p.part_o + pr * D + d) = o;
            if (d == 0) *reinterpret_cast<float2*>(p.part_ml + pr * 2) = make_float2(mx, l);
        }
    }
}

// The shares of a stream added in index order.  Grid (streams, Hq), a wavefront each: two dims a lane.
__global__ __launch_bounds__(64) void decode8_shares_kernel(Decode8Params p) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    constexpr int kDepth = 8;
    const int s = blockIdx.x, first_share = s ? p.share_end[s - 1] : 0, n_shares = p.share_end[s] - first_share;
    if (n_shares <= 1) return;
    const int g = blockIdx.y / p.G, head = blockIdx.y - g * p.G, dp = 2 * threadIdx.x;
    const int64_t pr0 = ((int64_t)first_share * p.Hkv + g) * p.G + head, step = (int64_t)p.Hkv * p.G;
    float m = -INFINITY, l = 0.f, a = 0.f, b = 0.f;
    for (int j0 = 0; j0 < n_shares; j0 += kDepth) {
        float2 ml[kDepth], o[kDepth];
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            const int64_t pr = pr0 + min(j0 + u, n_shares - 1) * step;
            ml[u] = *reinterpret_cast<const float2*>(p.part_ml + pr * 2);
            o[u] = *reinterpret_cast<const float2*>(p.part_o + pr * D + dp);
        }
        float mx = m;
#pragma unroll
        for (int u = 0; u < kDepth; ++u) mx = fmaxf(mx, ml[u].x);
        const float f = j0 ? __builtin_amdgcn_exp2f(m - mx) : 0.f;
        l *= f;
        a *= f;
        b *= f;
        m = mx;
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            const float w = j0 + u < n_shares ? __builtin_amdgcn_exp2f(ml[u].x - mx) : 0.f;
            if (j0 + u < n_shares) {
                l += w * ml[u].y;
                a += w * o[u].x;
                b += w * o[u].y;
            }
        }
    }
    const float inv = 1.0f / l;
    *reinterpret_cast<bf16x2*>(p.out + ((int64_t)s * p.Hq + blockIdx.y) * D + dp) = bf16x2{(__bf16)(a * inv), (__bf16)(b * inv)};
}

constexpr int kMaxWorkgroups = 512;

// Blocks per share: the fewest, in steps of a block per wavefront, with which all shares run at once, two workgroups
// per compute unit.  Streams that do not fit that way are not shared out.
int blocks_per_share(const LenTable& lens, int n_streams, int n_kv_heads) {
    int64_t total = 0;
    int most = 0;
    for (int i = 0; i < n_streams; ++i) {
        const int n = (lens.v[i] + kBlockRows - 1) / kBlockRows;
        total += n;
        most = std::max(most, n);
    }
    if ((int64_t)n_streams * n_kv_heads >= kMaxWorkgroups) return most;
    int64_t c = total * n_kv_heads / kMaxWorkgroups / kWaves * kWaves;
    for (c = std::max<int64_t>(c, kWaves); c < most; c += kWaves) {
        int64_t n = 0;
        for (int i = 0; i < n_streams; ++i) n += (lens.v[i] + kBlockRows - 1) / kBlockRows / c + ((lens.v[i] + kBlockRows - 1) / kBlockRows % c != 0);
        if (n * n_kv_heads <= kMaxWorkgroups) break;
    }
    return (int)std::min<int64_t>(c, most);
}

}  // namespace

// (shares that leave partial results: at most kMaxWorkgroups of them over all KV heads)
size_t decode8_workspace_bytes(const vs_shape& s, int32_t /*n_streams*/) {
    return (size_t)kMaxWorkgroups * (s.n_q_heads / s.n_kv_heads) * (D + 2) * sizeof(float);
}

hipError_t launch_decode8(const vs_shape& s, int32_t n_streams, void* slab, int32_t capacity, const LenTable& lens, const void* q,
                          const void* k_new, const void* v_new, void* out, void* workspace, hipStream_t st) {
    Decode8Params p;
    p.slab = (char*)slab;
    p.q = (const char*)q;
    p.k_new = (const char*)k_new;
    p.v_new = (const char*)v_new;
    p.out = (__bf16*)out;
    p.cache_bytes = cache8_bytes(s, capacity);
    p.G = s.n_q_heads / s.n_kv_heads;
    p.Hq = s.n_q_heads;
    p.Hkv = s.n_kv_heads;
    p.scale_log2e = s.softmax_scale * kLog2e;
    p.lens = lens;
    const int c = blocks_per_share(lens, n_streams, s.n_kv_heads);
    int n = 0;
    for (int i = 0; i < kMaxStreamsPerLaunch; ++i) {
        if (i < n_streams) n += ((lens.v[i] + kBlockRows - 1) / kBlockRows + c - 1) / c;
        p.share_end[i] = i < n_streams ? n : 0x7fffffff;  // (never "before" a share)
    }
    if (n > n_streams && (int64_t)n * s.n_kv_heads > kMaxWorkgroups) return hipErrorInvalidValue;
    p.part_ml = (float*)workspace;
    p.part_o = p.part_ml + (int64_t)kMaxWorkgroups * p.G * 2;
    decode8_kernel<<<dim3(n, s.n_kv_heads), kThreads, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || n == n_streams) return e;
    decode8_shares_kernel<<<dim3(n_streams, s.n_q_heads), 64, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace vs
