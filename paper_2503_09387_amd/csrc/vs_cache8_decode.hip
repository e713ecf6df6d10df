// Decode attention over caches in 8 bits (Eq. 1 of Section 3.1; Section 3.3, decoding phase): one query token per stream.  The arithmetic
// is in vs_cache8_attn.h; the G query heads of a KV head are the columns of the products, padded to 16.
#include "vs_cache8_attn.h"

#include <algorithm>

namespace vs {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int D = 128;
constexpr int kRowStride = D + 4;  // of a query head's sums in LDS, in floats
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazyMax = 8.0f;  // scores may exceed the reference maximum by 2^8 before it is refreshed
// Where the sums of p s_v come to 2^93, the wavefront begins again with a reference 2^48 up: probabilities are up to 2^8, codes 255 and scales of V
// 2^121, and sums of that over the wavefronts of a stream would pass an fp32.  (What is below 2^-78 of the largest probability then counts as nothing:
// that is at most 2^50 a key, where outputs are 2^93 over the sum of probabilities at least.)
constexpr float kLargeExcess = 0x1p100f, kLift = 48.0f;

struct Decode8Params {
    char* slab;
    const char* q;
    const char* k_new;  // may be null
    const char* v_new;
    __bf16* out;
    float* part_o;       // [share][Hkv][G][D], not normalised
    float* part_ml;      // [share][Hkv][G][2]: reference (log2 units), sum
    unsigned* counters;  // [stream][Hkv], kDecodeCounterStart between launches; null: the shares are added by a second launch
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

struct State {
    f32x4 o[8];   // [dim % 8]: element r of lane (query i16, h): dim 8 (4 h + r) + dim % 8, 128 per unit of p s_v too large
    f32x4 excess; // and what is too much
    float m, l;   // reference (log2 units, the same in the lanes of a query), this lane's share of the sum
};

// One block, of which `valid` rows are there.
__device__ __forceinline__ void attend(State& st, const Block& b, const Queries& q, int valid, int h, float lift) {
    float z[8], sv[8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        f32x4 x = {q.start, q.start, q.start, q.start};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys_of(b.k[2 * kt + (i >> 1)][2 * (i & 1)], b.k[2 * kt + (i >> 1)][2 * (i & 1) + 1]), q.q[i], x, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const unsigned pair = b.s[kt][r];
            z[4 * kt + r] = x[r] * (q.f * __uint_as_float(pair << 16));
            sv[4 * kt + r] = __uint_as_float(pair & 0xffff0000u);
        }
    }
    if (valid < kBlockRows) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (16 * (e >> 2) + 4 * h + (e & 3) >= valid) {
                z[e] = -INFINITY;
                sv[e] = 0.f;
            }
    }
    float mx = max_of_8(z);
    if (__any(mx > st.m + (kLazyMax - lift))) {  // rare after the first block
        mx = max_over_rows(mx) + lift;
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
        st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values_of(b.v[dt >> 1][2 * (dt & 1)], b.v[dt >> 1][2 * (dt & 1) + 1]), p, st.o[dt], 0, 0, 0);
    }
}

// A row's codes in a block as it lies in a wavefront's registers.  k_codes, v_codes, pair: as every lane (i16, any h) has them of its 8 dims.
__device__ __forceinline__ void put_row(Block& b, int key, uint2 k_codes, const unsigned (&v_codes)[8], unsigned pair, int i16, int h) {
    const bool k_mine = i16 == (key & 15), v_mine = h == ((key & 15) >> 2);
    const unsigned byte = 8 * (key & 3), mask = v_mine ? 0xffu << byte : 0u;
    raw16 k[2];  // dims 64 ds + 8 h .. and 64 ds + 32 + 8 h .. of the row
#pragma unroll
    for (int ds = 0; ds < 2; ++ds)
        k[ds] = raw16{(unsigned)__shfl((int)k_codes.x, 8 * ds + h), (unsigned)__shfl((int)k_codes.y, 8 * ds + h), (unsigned)__shfl((int)k_codes.x, 8 * ds + 4 + h),
                      (unsigned)__shfl((int)k_codes.y, 8 * ds + 4 + h)};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        if (kt != key >> 4) continue;
#pragma unroll
        for (int ds = 0; ds < 2; ++ds)
#pragma unroll
            for (int w = 0; w < 4; ++w) b.k[2 * kt + ds][w] = k_mine ? k[ds][w] : b.k[2 * kt + ds][w];
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const unsigned old = b.v[dt >> 1][2 * (dt & 1) + kt];
            b.v[dt >> 1][2 * (dt & 1) + kt] = (old & ~mask) | ((v_codes[dt] << byte) & mask);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) b.s[kt][r] = v_mine && r == (key & 3) ? pair : b.s[kt][r];
    }
}

// The shares of stream s, KV head g, added in index order: dims dp, dp + 1 of query head `head` of the group.  kAgent: the partial
// results were stored in this launch, by other workgroups.
template <bool kAgent>
__device__ __forceinline__ void add_shares(const Decode8Params& p, int s, int g, int first_share, int n_shares, int head, int dp) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    constexpr int kDepth = 8;
    const int64_t pr0 = ((int64_t)first_share * p.Hkv + g) * p.G + head, step = (int64_t)p.Hkv * p.G;
    float m = -INFINITY, l = 0.f, a = 0.f, b = 0.f;
    for (int j0 = 0; j0 < n_shares; j0 += kDepth) {
        float2 ml[kDepth], o[kDepth];
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            const int64_t pr = pr0 + min(j0 + u, n_shares - 1) * step;
            ml[u] = kAgent ? __builtin_bit_cast(float2, load_agent(p.part_ml + pr * 2)) : *reinterpret_cast<const float2*>(p.part_ml + pr * 2);
            o[u] = kAgent ? __builtin_bit_cast(float2, load_agent(p.part_o + pr * D + dp)) : *reinterpret_cast<const float2*>(p.part_o + pr * D + dp);
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
            if (j0 + u >= n_shares) continue;
            const float w = __builtin_amdgcn_exp2f(ml[u].x - mx);
            l += w * ml[u].y;
            a += w * o[u].x;
            b += w * o[u].y;
        }
    }
    const float inv = 1.0f / l;
    *reinterpret_cast<bf16x2*>(p.out + ((int64_t)s * p.Hq + (int64_t)g * p.G + head) * D + dp) = bf16x2{(__bf16)(a * inv), (__bf16)(b * inv)};
}

// Grid (shares of all streams, Hkv).  A workgroup is a share of one stream's blocks for one KV head; its wavefronts take the blocks
// in turn, two of a wavefront's on their way at a time, and meet in LDS.  Where a stream has several shares, they pass fp32 partial results
// through memory at agent scope (the L2s are not coherent with each other), every store acknowledged before the workgroup counts itself in;
// the last to arrive adds the shares in index order, and nobody waits.  The upper 24 bits of a counter are a mark that
// vs_workspace_init puts there; where they are something else the stream's first share does the whole stream.  Streams of many shares (counters
// null) are added by a second launch.
template <int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void decode8_kernel(Decode8Params p) {
    constexpr int kThreads = 64 * kWaves;
    __shared__ __attribute__((aligned(16))) float s_o[kWaves][kMaxGroup][kRowStride];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    __shared__ unsigned s_before;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, h = lane >> 4, g = blockIdx.y, share = blockIdx.x;
    static_assert(kMaxStreamsPerLaunch == 64, "one lane per stream");
    const int end_of = p.share_end[lane], len_of = p.lens.v[lane];
    const int s = __builtin_popcountll(__ballot(end_of <= share));
    const int len = __builtin_amdgcn_readlane(len_of, s);
    const int first_share = s ? __builtin_amdgcn_readlane(end_of, s - 1) : 0;
    const int shares = __builtin_amdgcn_readlane(end_of, s) - first_share, j_share = share - first_share;
    const int n_blocks = (len + kBlockRows - 1) / kBlockRows;
    char* const base = p.slab + s * p.cache_bytes + (int64_t)g * kBlockBytes;
    const int64_t stride = (int64_t)p.Hkv * kBlockBytes;

  // once; a second time only where the first share of a stream does the whole stream
  for (int n_shares = shares;; n_shares = 1) {
    const unsigned per = (unsigned)n_blocks / n_shares, more = n_blocks - per * n_shares;
    const int first = j_share * per + min((unsigned)j_share, more), end = first + per + ((unsigned)j_share < more);
    State st;
    int b;
    for (float lift = 0.f;; lift = kLift) {  // (once, but for values near the largest: 0.1 .. 0.2 us a step)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) st.o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        st.excess = st.o[0];
        st.m = -INFINITY;
        st.l = 0.f;
        b = first + wave;
        if (b < end) {
            // (loads come back in order: the query and the new row before the blocks)
            int64_t from = 0;
            asm volatile("" : "+s"(from));  // (or these loads, and what waits for them, leave the loop and come before the blocks are asked for: 0.2 us)
            const char* const q_row = p.q + from + ((int64_t)s * p.Hq + (int64_t)g * p.G + min(i16, p.G - 1)) * 256 + 16 * h;
            raw16 words[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) words[i] = *reinterpret_cast<const raw16*>(q_row + 64 * i);
            // the step's new row, by the wavefront that attends over the block that it falls into: to memory, and into the block as it is here
            const bool keeps = p.k_new && end == n_blocks && wave == (unsigned)(n_blocks - 1 - first) % kWaves;
            const int64_t at = from + ((int64_t)s * p.Hkv + g) * 256 + 16 * i16;  // (asked for by all: behind a branch it would be waited for)
            const raw16 k_new = *reinterpret_cast<const raw16*>((p.k_new ? p.k_new : p.q) + at), v_new = *reinterpret_cast<const raw16*>((p.k_new ? p.v_new : p.q) + at);
            Block x, y;
            const char* blk = base + b * stride;
            fetch(x, blk, lane);
            blk += kWaves * stride;
            if (b + kWaves < end) fetch(y, blk, lane);
            const Queries q = queries_of(words, p.scale_log2e);
            uint2 k_codes{};
            unsigned v_codes[8] = {}, pair = 0;
            if (keeps) {
                const int key = (len - 1) % kBlockRows;
                pair = quantise(k_new, v_new, k_codes, v_codes);
                if (h == 0) {
                    char* const to = base + (n_blocks - 1) * stride;
#pragma unroll
                    for (int j = 0; j < 8; ++j) to[v_code_offset(key, i16, j)] = (char)v_codes[j];
                    *reinterpret_cast<uint2*>(to + k_code_offset(key, i16)) = k_codes;
                    if (i16 == 0) *reinterpret_cast<unsigned*>(to + kBlockScales + 4 * key) = pair;
                }
            }
            auto turn = [&](Block& here) {
                if (keeps && b + 1 == n_blocks) put_row(here, (len - 1) % kBlockRows, k_codes, v_codes, pair, i16, h);
                attend(st, here, q, len - b * kBlockRows, h, lift);
                b += kWaves;
                blk += kWaves * stride;
                if (b + kWaves < end) fetch(here, blk, lane);
            };
            while (b < end) {
                turn(x);
                if (b < end) turn(y);
            }
        }
        // (the excess is -128 times a column's sum of p s_v; or a row or query was not finite, and nothing changes)
        if (lift > 0.f || !__any(!(st.excess[0] > -kLargeExcess))) break;
    }
    st.l = sum_over_rows(st.l);
    if (h == 0) {
        s_m[wave][i16] = st.m;
        s_l[wave][i16] = st.l;
    }
    if (i16 < p.G)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = st.o[4 * half + e][r] + st.excess[r];
                *reinterpret_cast<f32x4*>(&s_o[wave][i16][8 * (4 * h + r) + 4 * half]) = w;
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
            const float f = __builtin_amdgcn_exp2f(s_m[w][head] - mx);  // 0 for a wavefront without blocks
            l += s_l[w][head] * f;
            o += *reinterpret_cast<const f32x4*>(&s_o[w][head][d]) * f;
        }
        if (n_shares == 1) {
            const float inv = 1.0f / l;
            bf16x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = (__bf16)(o[e] * inv);
            *reinterpret_cast<bf16x4*>(p.out + ((int64_t)s * p.Hq + (int64_t)g * p.G + head) * D + d) = r;
        } else {
            const int64_t pr = ((int64_t)share * p.Hkv + g) * p.G + head;
            store_agent(p.part_o + pr * D + d, __float_as_uint(o[0]), __float_as_uint(o[1]));
            store_agent(p.part_o + pr * D + d + 2, __float_as_uint(o[2]), __float_as_uint(o[3]));
            if (d == 0) store_agent(p.part_ml + pr * 2, __float_as_uint(mx), __float_as_uint(l));
        }
    }
    if (n_shares == 1 || !p.counters) return;

    // ---- the shares of the stream: the last to arrive adds them ----
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's partial results have arrived
    __syncthreads();
    unsigned* const counter = p.counters + s * p.Hkv + g;
    if (tid == 0) s_before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const unsigned before = __builtin_amdgcn_readfirstlane(s_before);
    if ((before & kDecodeCounterMark) != kDecodeCounterStart) {  // not prepared, or overwritten
        if (j_share == 0) continue;
        return;
    }
    if (before - kDecodeCounterStart != (unsigned)(n_shares - 1)) return;
    if (tid == 0) __hip_atomic_store(counter, kDecodeCounterStart, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int it = tid; it < p.G * (D / 2); it += kThreads) add_shares<true>(p, s, g, first_share, n_shares, it / (D / 2), 2 * (it % (D / 2)));
    return;
  }
}

// The shares of a stream added by a launch of their own.  Grid (streams, Hq), a wavefront each.
__global__ __launch_bounds__(64) void decode8_shares_kernel(Decode8Params p) {
    const int s = blockIdx.x, first_share = s ? p.share_end[s - 1] : 0, n_shares = p.share_end[s] - first_share;
    const int g = blockIdx.y / p.G;
    if (n_shares > 1) add_shares<false>(p, s, g, first_share, n_shares, blockIdx.y - g * p.G, 2 * threadIdx.x);
}

constexpr int kMaxWorkgroups = 256;
constexpr int kMaxSharesInside = 12, kMaxBlocksInside = 80, kAloneBlocks = 16;
constexpr int kSmallBlocks = 32, kSmallWorkgroups = 128;

// Wavefronts of a workgroup, and blocks per share.  us a step, 28/4 heads:
//   * up to 16 blocks a stream one share and no merge: 1 x 256 rows 5.8 (in shares 7.0), 1 x 380 6.2 (7.4), 1 x 500 7.1 (7.4); beyond, shares: 1 x 700
//     8.5 as one and 7.3 in shares;
//   * 4 wavefronts and shares of 4 blocks while a stream has 32 at most and that makes 128 workgroups at most: 1 x 700 7.3 (8 wavefronts 7.9),
//     1 x 1000 7.3 (8.0), 4 x 700 7.9 (8.1); beyond, 8: 16 x 700 9.2 (4 wavefronts 10.0), 1 x 1400 8.0 (9.5), 16 ragged 20.9 (24.3);
//   * with 8, the fewest shares, from a block per wavefront on, with which all run at once, a workgroup per compute unit;
//   * but at most 12 shares, which the last to arrive adds, as long as they are no more than 80 blocks: 1 x 8192 12.3 (32 shares and a second
//     launch 15.1), 1 x 16384 15.2 (19.9), 1 x 32768 22.8 (22.9), 1 x 50000 30.2 (25.1).
// (Before the look at the sums of p s_v came in, which is 0.1 .. 0.2 us on each.)
// Streams that do not fit all at once are not shared out.  That is for streams of like lengths, 33 x 8320 57.9 us, 64 x 8320 84.9; a long one among many short
// ones is left to 4 workgroups: 63 x 100 and 1 x 8320 45.7, where 59 x 100 and 1 x 8320 are shared out, 15.4.
// 16 streams of 640..8320 rows (78.9 MB): 19.0 us = 4.2 TB/s, of which some 4 us are the launch, the first trip to memory and the merge; in between
// bytes come at a large copy's rate.
struct Plan {
    int waves, per_share;
};
Plan plan_of(const LenTable& lens, int n_streams, int n_kv_heads) {
    auto blocks_of = [&](int i) { return vs::blocks_of(lens.v[i]); };
    int64_t total = 0;
    int most = 0;
    for (int i = 0; i < n_streams; ++i) {
        total += blocks_of(i);
        most = std::max(most, blocks_of(i));
    }
    if (most <= kSmallBlocks && (int64_t)n_streams * n_kv_heads * ((most + 3) / 4) <= kSmallWorkgroups) return {4, most <= kAloneBlocks ? most : 4};
    if (most <= kAloneBlocks || (int64_t)n_streams * n_kv_heads >= kMaxWorkgroups) return {8, most};
    auto fits = [&](int c) {
        int64_t n = 0;
        for (int i = 0; i < n_streams; ++i) n += (blocks_of(i) + c - 1) / c;
        return n * n_kv_heads <= kMaxWorkgroups;
    };
    int c = (int)std::min<int64_t>(std::max<int64_t>(total * n_kv_heads / kMaxWorkgroups, 8), most);
    while (c < most && !fits(c)) c += 1 + c / 32;
    const int inside = (most + kMaxSharesInside - 1) / kMaxSharesInside;
    return {8, std::min(inside <= kMaxBlocksInside ? std::max(c, inside) : c, most)};
}

}  // namespace

// (shares that leave partial results: at most kMaxWorkgroups of them over all KV heads)
size_t decode8_workspace_bytes(const vs_shape& s, int32_t /*n_streams*/) {
    return (size_t)kMaxWorkgroups * (s.n_q_heads / s.n_kv_heads) * (D + 2) * sizeof(float);
}

hipError_t launch_decode8(const vs_shape& s, int32_t n_streams, void* slab, int32_t capacity, const LenTable& lens, const void* q,
                          const void* k_new, const void* v_new, void* out, void* counters, void* workspace, hipStream_t st) {
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
    const Plan pl = plan_of(lens, n_streams, s.n_kv_heads);
    const int c = pl.per_share;
    int n = 0, most = 0;
    for (int i = 0; i < kMaxStreamsPerLaunch; ++i) {
        const int of = i < n_streams ? (blocks_of(lens.v[i]) + c - 1) / c : 0;
        n += of;
        most = std::max(most, of);
        p.share_end[i] = i < n_streams ? n : 0x7fffffff;  // (never "before" a share)
    }
    if (n > n_streams && (int64_t)n * s.n_kv_heads > kMaxWorkgroups) return hipErrorInvalidValue;
    p.part_ml = (float*)workspace;
    p.part_o = p.part_ml + (int64_t)kMaxWorkgroups * p.G * 2;
    p.counters = most <= kMaxSharesInside ? (unsigned*)counters : nullptr;
    if (pl.waves == 4) decode8_kernel<4><<<dim3(n, s.n_kv_heads), 256, 0, st>>>(p);
    else decode8_kernel<8><<<dim3(n, s.n_kv_heads), 512, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || n == n_streams || p.counters) return e;
    decode8_shares_kernel<<<dim3(n_streams, s.n_q_heads), 64, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace vs
