// Rotary positions with several axes (time, height, width), applied to the rows of Q and K between their projection and the
// attention.  Pair i of a head turns by pos[axis of i] * turns[i] revolutions:
//   (a, b) -> (a cos - b sin, a sin + b cos),
// back with the sign of sin changed: the rotation is orthogonal, so that is also its gradient.
//
// A product of a position and a rate is taken in fp64 and only what is left of a whole revolution goes on in fp32: positions of a long
// stream pass 10^5, and an angle of so many radians in fp32 is off by 10^-2.
//
// Bound by memory: every value is read once and written once.  16384 tokens of 28/4 heads of 128 (269 MB) 40.4 us on the device, 48.3 us a call over
// changing rows = 5.6 TB/s; 16 tokens 3.0 us, which is the launch and the trips to the positions and the rows.  The 256 threads of a workgroup are the pieces
// of a token of 32 heads of 128 in bf16; other layouts leave some idle: 3200 tokens of 4/1 heads of 64 in fp32, 40 threads of 256 with
// data, 4.9 us, three times what its bytes take.  What is left of a revolution is an fp32: 2^-26 of one, which with fp32 rows shows beside
// their rounding (5.3e-8 of a value on average, 4.2e-8 with the angle in fp64) and with bf16 rows does not.
#include "vs_internal.h"

#include <algorithm>

#include <math.h>
#include <string.h>

namespace vs {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 64;

struct RotaryParams {
    const char* q;
    const char* k;
    char* q_out;
    char* k_out;
    const int32_t* pos;  // [3][n_tokens]
    int n_tokens, Hq, Hkv;
    int first;           // token of the launch's first workgroup
    int pairs;           // rotated pairs of a head; the values behind them stay
    int ends[2];         // first pair of the second and of the third axis
    float sign;
    double turns[kMaxPairs];
};

// Grid: tokens, from p.first on.  The first wavefront works out the token's cosines and sines, a pair a lane, while every thread's values are on their
// way.  A thread takes two pieces of 16 bytes of a head that hold whole pairs between them (so that a call may turn rows in place):
// the same piece of both halves (pairs i, i + pairs), or 32 bytes in a row (pairs 2 i, 2 i + 1, and what is not turned).
template <typename T, int D, bool kHalves>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryParams p) {
    constexpr int N = 16 / (int)sizeof(T);
    constexpr int kUnits = D / (2 * N);  // of a head
    __shared__ float s_cos[kMaxPairs], s_sin[kMaxPairs];
    const int t = p.first + blockIdx.x, tid = threadIdx.x, n_units = (p.Hq + p.Hkv) * kUnits;
    raw16 a, b;
    const T* src = nullptr;
    T* dst = nullptr;
    int e0 = 0, apart = N;
    auto locate = [&](int it) {
        const int row = it / kUnits, u = it % kUnits;
        const int64_t at = (row < p.Hq ? (int64_t)t * p.Hq + row : (int64_t)t * p.Hkv + row - p.Hq) * D;
        const bool turned = 2 * N * u < 2 * p.pairs;
        e0 = kHalves && turned ? N * u : 2 * N * u;
        apart = kHalves && turned ? p.pairs : N;
        src = reinterpret_cast<const T*>(row < p.Hq ? p.q : p.k) + at + e0;
        dst = reinterpret_cast<T*>(row < p.Hq ? p.q_out : p.k_out) + at + e0;
        a = *reinterpret_cast<const raw16*>(src);
        b = *reinterpret_cast<const raw16*>(src + apart);
    };
    if (tid < n_units) locate(tid);
    if (tid < p.pairs) {
        const int axis = (tid >= p.ends[0]) + (tid >= p.ends[1]);
        const double r = (double)p.pos[(int64_t)axis * p.n_tokens + t] * p.turns[tid];
        float sn, cs;
        sincospif(2.0f * (float)(r - rint(r)), &sn, &cs);
        s_cos[tid] = cs;
        s_sin[tid] = p.sign * sn;
    }
    __syncthreads();
    for (int it = tid; it < n_units; it += kThreads) {
        if (it != tid) locate(it);
        const T *x = reinterpret_cast<const T*>(&a), *y = reinterpret_cast<const T*>(&b);
        raw16 oa = a, ob = b;
        T *u = reinterpret_cast<T*>(&oa), *v = reinterpret_cast<T*>(&ob);
        if (kHalves) {
            if (e0 < p.pairs) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float c = s_cos[e0 + j], s = s_sin[e0 + j], f = to_f32(x[j]), g = to_f32(y[j]);
                    u[j] = from_f32<T>(f * c - g * s);
                    v[j] = from_f32<T>(f * s + g * c);
                }
            }
        } else if (e0 < 2 * p.pairs) {
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const int i = (e0 + j) / 2;
                float c = s_cos[i], s = s_sin[i], f = to_f32(x[j]), g = to_f32(x[j + 1]);
                u[j] = from_f32<T>(f * c - g * s);
                u[j + 1] = from_f32<T>(f * s + g * c);
                c = s_cos[i + N / 2], s = s_sin[i + N / 2], f = to_f32(y[j]), g = to_f32(y[j + 1]);
                v[j] = from_f32<T>(f * c - g * s);
                v[j + 1] = from_f32<T>(f * s + g * c);
            }
        }
        *reinterpret_cast<raw16*>(dst) = oa;
        *reinterpret_cast<raw16*>(dst + apart) = ob;
    }
}

template <typename T, int D>
void launch(RotaryParams& p, bool halves, hipStream_t st) {
    constexpr int kTokens = 1 << 20;  // of a launch, whose threads a grid counts in 32 bits
    for (p.first = 0; p.first < p.n_tokens; p.first += kTokens) {
        const int n = std::min(p.n_tokens - p.first, kTokens);
        if (halves) rotary_kernel<T, D, true><<<n, kThreads, 0, st>>>(p);
        else rotary_kernel<T, D, false><<<n, kThreads, 0, st>>>(p);
    }
}

constexpr int32_t kMaxTokens = 1 << 26;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool apart(const void* p, int64_t p_bytes, const void* q, int64_t q_bytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a + (uintptr_t)p_bytes <= b || b + (uintptr_t)q_bytes <= a;
}

// pairs of a head that a plan turns, 0 if it is none
int pairs_of(int32_t head_dim, const int32_t* sections) {
    int64_t n = 0;
    for (int i = 0; i < 3; ++i) {
        if (sections[i] < 0) return 0;
        n += sections[i];
    }
    return n >= 8 && n % 8 == 0 && 2 * n <= head_dim && n <= kMaxPairs ? (int)n : 0;
}

}  // namespace
}  // namespace vs

using namespace vs;

extern "C" {

vs_status vs_rotary_plan_make(int32_t head_dim, const int32_t* sections, double theta, int32_t pairing, vs_rotary_plan* plan) {
    if (!sections || !plan) return VS_ERR_NULL;
    if (head_dim != 64 && head_dim != 128) return VS_ERR_UNSUPPORTED;
    const int n = pairs_of(head_dim, sections);
    if (!n || !isfinite(theta) || !(theta > 0.0) || (pairing != VS_ROTARY_HALVES && pairing != VS_ROTARY_ADJACENT)) return VS_ERR_SHAPE;
    vs_rotary_plan made{};
    made.head_dim = head_dim;
    made.pairing = pairing;
    for (int i = 0; i < 3; ++i) made.sections[i] = sections[i];
    for (int i = 0; i < n; ++i) {
        made.turns[i] = pow(theta, -(double)i / n) / (2.0 * M_PI);
        if (!isfinite(made.turns[i])) return VS_ERR_SHAPE;
    }
    *plan = made;
    return VS_OK;
}

vs_status vs_rotary(const vs_shape* shape, const vs_rotary_plan* plan, const int32_t* positions, int32_t n_tokens, const void* q,
                    const void* k, int32_t inverse, void* q_out, void* k_out, void* hip_stream) {
    (void)hipGetLastError();
    const vs_status st = check_shape(shape);
    if (st != VS_OK) return st;
    if (!plan || !positions || (!q && !k) || !q != !q_out || !k != !k_out) return VS_ERR_NULL;
    const int pairs = pairs_of(plan->head_dim, plan->sections);
    if (!pairs || plan->head_dim != shape->head_dim || (plan->pairing != VS_ROTARY_HALVES && plan->pairing != VS_ROTARY_ADJACENT) ||
        n_tokens < 1 || n_tokens > kMaxTokens)
        return VS_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || (reinterpret_cast<uintptr_t>(positions) & 3u))
        return VS_ERR_ALIGN;
    RotaryParams p;
    p.Hq = q ? shape->n_q_heads : 0;
    p.Hkv = k ? shape->n_kv_heads : 0;
    const int64_t head = (int64_t)n_tokens * shape->head_dim * (shape->dtype == VS_F32 ? 4 : 2), nq = p.Hq * head, nk = p.Hkv * head;
    if ((q != q_out && !apart(q, nq, q_out, nq)) || (k != k_out && !apart(k, nk, k_out, nk))) return VS_ERR_SHAPE;
    if (q && k && (!apart(q_out, nq, k_out, nk) || !apart(q_out, nq, k, nk) || !apart(k_out, nk, q, nq))) return VS_ERR_SHAPE;
    const int64_t np = (int64_t)3 * n_tokens * 4;
    if ((q && !apart(q_out, nq, positions, np)) || (k && !apart(k_out, nk, positions, np))) return VS_ERR_SHAPE;
    p.q = (const char*)q;
    p.k = (const char*)k;
    p.q_out = (char*)q_out;
    p.k_out = (char*)k_out;
    p.pos = positions;
    p.n_tokens = n_tokens;
    p.pairs = pairs;
    p.ends[0] = plan->sections[0];
    p.ends[1] = plan->sections[0] + plan->sections[1];
    p.sign = inverse ? -1.0f : 1.0f;
    memcpy(p.turns, plan->turns, sizeof p.turns);
    const bool halves = plan->pairing == VS_ROTARY_HALVES;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (shape->dtype == VS_BF16) launch<__bf16, 128>(p, halves, stream);
    else if (shape->head_dim == 128) launch<float, 128>(p, halves, stream);
    else launch<float, 64>(p, halves, stream);
    return hipGetLastError() == hipSuccess ? VS_OK : VS_ERR_HIP;
}

}  // extern "C"
