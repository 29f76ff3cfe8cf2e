// Rotary positions of queries and keys (include/nova_rope.h).
//
// Memory bound: 4 bytes an element, and a sine and a cosine per token and pair, which all heads of the token share (134 MB in 25.4 us,
// 5.3 TB/s, at B=2, H=12 on 4, T=8192, D=128, 64 of them turned; 50 MB in 9.2 us at B=8, 24 heads, T=1024, D=64, where it took 31.1 with
// each thread making its own angles).  A block has
// a few tokens and all their heads: it makes the tokens' angles once, one or two a thread, into shared memory, while the
// first elements are on their way.  A thread keeps one place in the head (8 dimensions, and in the half layout the 8 that they
// are paired with) of one token and walks over heads with 16-byte accesses, four heads in flight.
#include <algorithm>
#include <cmath>

#include "../../../include/nova_rope.h"
#include "../api.h"
#include "../ptx.cuh"

namespace nova {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxAngles = 2048;  // of a block
// Heads of which a thread has the loads out together: 128 bytes of them in both layouts.
__host__ __device__ constexpr int heads_in_flight(bool interleaved) { return interleaved ? 8 : 4; }

struct RopeArgs {
    const uint16_t* in[2];  // Q, K
    uint16_t* out[2];
    TensorStrides sin[2], sout[2];
    const float* inv_freq;
    const int* positions;
    long long position_stride;
    int heads[2], T, rows, rotary, rot_chunks, chunks, groups, tokens;  // rows: B * T; tokens: of a block
    float amplitude;
    float sign;  // -1: backward
    bool heads_inside;
};

template <int V>
struct Vec;
template <>
struct Vec<8> { using type = uint4; };
template <>
struct Vec<4> { using type = uint2; };
template <>
struct Vec<2> { using type = uint32_t; };
template <>
struct Vec<1> { using type = uint16_t; };

template <int V>
__device__ __forceinline__ void widen(const typename Vec<V>::type& v, float (&f)[V]) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(&v);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = __uint_as_float(static_cast<uint32_t>(p[i]) << 16);
}
template <int V>
__device__ __forceinline__ typename Vec<V>::type narrow(const float (&f)[V]) {
    typename Vec<V>::type v;
    if constexpr (V == 1) {
        v = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
    } else {
        uint32_t* p = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) p[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    }
    return v;
}

// V elements to an access.  Half layout: places d and d + rotary/2 of a pair are V neighbours each; interleaved: V neighbours
// are V/2 pairs.  A unit is a chunk of V places (the last ones are copied), a token and a group of heads; units next to each
// other have the chunks of one head and then, whichever lies closer, the token's other heads or the head's other tokens.
template <int V, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, 3) rope_kernel(const __grid_constant__ RopeArgs a) {
    using T4 = typename Vec<V>::type;
    constexpr int kAngles = kInterleaved ? V / 2 : V;
    constexpr int kHeadsInFlight = heads_in_flight(kInterleaved);
    __shared__ float2 angles[kMaxAngles];  // [token of the block][pair] cosine, sine
    griddep_launch_dependents();
    const int row0 = blockIdx.x * a.tokens, n_tokens = min(a.tokens, a.rows - row0), pairs = a.rotary / 2;
    const int units = n_tokens * a.chunks * a.groups, heads = a.heads[0] + a.heads[1];

    int tok, g, d, d2;  // token of the block, group, first place, and in the half layout that of the other ends of the pairs
    bool turns;
    const uint16_t* in[2];
    uint16_t* out[2];
    T4 x4[kHeadsInFlight], y4[kHeadsInFlight];
    auto locate = [&](int u) {
        const int r = u / a.chunks, c = u - r * a.chunks;
        const int inner = a.heads_inside ? a.groups : n_tokens, y = r / inner, x = r - y * inner;
        tok = a.heads_inside ? y : x, g = a.heads_inside ? x : y;
        const int b = (row0 + tok) / a.T, t = row0 + tok - b * a.T;
        turns = c < a.rot_chunks;
        d = kInterleaved || turns ? c * V : a.rotary + (c - a.rot_chunks) * V;
        d2 = d + pairs;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            in[w] = a.in[w] + b * a.sin[w].b + t * a.sin[w].t - w * a.heads[0] * a.sin[w].h;
            out[w] = a.out[w] + b * a.sout[w].b + t * a.sout[w].t - w * a.heads[0] * a.sout[w].h;
        }
    };
    // heads h0, h0 + groups, ... of both tensors, those of Q first (the pointers of K are those of its head -H)
    auto load = [&](int h0) {
#pragma unroll
        for (int k = 0; k < kHeadsInFlight; ++k) {
            const int h = h0 + k * a.groups;
            if (h >= heads) break;
            const uint16_t* const p = h < a.heads[0] ? in[0] + h * a.sin[0].h : in[1] + h * a.sin[1].h;
            x4[k] = *reinterpret_cast<const T4*>(p + d);
            if (!kInterleaved && turns) y4[k] = *reinterpret_cast<const T4*>(p + d2);
        }
    };

    griddep_wait();
    const bool any = threadIdx.x < units;
    if (any) {
        locate(threadIdx.x);
        load(g);
    }
    for (int x = threadIdx.x; x < n_tokens * pairs; x += kThreads) {
        const int k = x / pairs, i = x - k * pairs;
        const int b = (row0 + k) / a.T, t = row0 + k - b * a.T;
        const double pos = a.positions != nullptr ? __ldg(a.positions + b * a.position_stride + t) : t;
        const double turn = pos * static_cast<double>(__ldg(a.inv_freq + i)) * 0.15915494309189535;  // 1 / 2 pi
        float s, c;
        sincospif(2.0f * static_cast<float>(turn - rint(turn)), &s, &c);
        angles[x] = make_float2(c * a.amplitude, s * a.amplitude * a.sign);
    }
    __syncthreads();

    for (int u = threadIdx.x; u < units; u += kThreads) {
        if (u >= kThreads) {
            locate(u);
            load(g);
        }
        float co[kAngles], si[kAngles];
        if (turns) {
            const float2* const p = angles + tok * pairs + (kInterleaved ? d / 2 : d);
#pragma unroll
            for (int i = 0; i < kAngles; ++i) co[i] = p[i].x, si[i] = p[i].y;
        }
        for (int h0 = g; h0 < heads; h0 += kHeadsInFlight * a.groups) {
            if (h0 != g) load(h0);
#pragma unroll
            for (int k = 0; k < kHeadsInFlight; ++k) {
                const int h = h0 + k * a.groups;
                if (h >= heads) break;
                uint16_t* const to = h < a.heads[0] ? out[0] + h * a.sout[0].h : out[1] + h * a.sout[1].h;
                if (turns) {
                    float p[V];
                    widen<V>(x4[k], p);
                    if constexpr (kInterleaved) {
#pragma unroll
                        for (int i = 0; i < V; i += 2) {
                            const float p0 = p[i];
                            p[i] = p0 * co[i / 2] - p[i + 1] * si[i / 2];
                            p[i + 1] = p[i + 1] * co[i / 2] + p0 * si[i / 2];
                        }
                    } else {
                        float q[V];
                        widen<V>(y4[k], q);
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float p0 = p[i];
                            p[i] = p0 * co[i] - q[i] * si[i];
                            q[i] = q[i] * co[i] + p0 * si[i];
                        }
                        *reinterpret_cast<T4*>(to + d2) = narrow<V>(q);
                    }
                    x4[k] = narrow<V>(p);
                }
                *reinterpret_cast<T4*>(to + d) = x4[k];
            }
        }
    }
}

int rope(const void* Q, const void* K, void* Qo, void* Ko, const float* inv_freq, const int* positions, int B, int H, int H_kv,
         int T, int D, int rotary, int interleaved, float amplitude, long long position_stride, const nova_attn_strides* q,
         const nova_attn_strides* k, const nova_attn_strides* qo, const nova_attn_strides* ko, float sign, void* stream) {
    if (!Q || !Qo || !inv_freq || (K == nullptr) != (Ko == nullptr)) return NOVA_ATTN_ERR_NULL;
    if (!K) H_kv = 0;
    if (B <= 0 || H <= 0 || T <= 0 || (K && H_kv <= 0) || D <= 0 || (D & 7) || D > 1024) return NOVA_ATTN_ERR_SHAPE;
    if (rotary < 2 || (rotary & 1) || rotary > D || position_stride < 0) return NOVA_ATTN_ERR_SHAPE;
    if (static_cast<long long>(H) + H_kv > (1 << 24) || static_cast<long long>(B) * T > (1ll << 30)) return NOVA_ATTN_ERR_SHAPE;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(Qo) || !aligned16(Ko)) return NOVA_ATTN_ERR_ALIGNMENT;
    if ((reinterpret_cast<uintptr_t>(inv_freq) & 3u) || (reinterpret_cast<uintptr_t>(positions) & 3u)) return NOVA_ATTN_ERR_ALIGNMENT;
    if (!std::isfinite(amplitude)) return NOVA_ATTN_ERR_SCALE;
    RopeArgs a{};
    if (int rc = check_strides(q, D, &a.sin[0])) return rc;
    if (int rc = check_strides(qo, D, &a.sout[0])) return rc;
    if (K) {
        if (int rc = check_strides(k, D, &a.sin[1])) return rc;
        if (int rc = check_strides(ko, D, &a.sout[1])) return rc;
    }
    auto same = [](const TensorStrides& x, const TensorStrides& y) { return x.b == y.b && x.h == y.h && x.t == y.t; };
    if ((Q == Qo && !same(a.sin[0], a.sout[0])) || (K && K == Ko && !same(a.sin[1], a.sout[1]))) return NOVA_ATTN_ERR_SHAPE;
    DeviceState* st = nullptr;
    if (int rc = device_state(&st)) return rc;

    a.in[0] = static_cast<const uint16_t*>(Q);
    a.in[1] = static_cast<const uint16_t*>(K);
    a.out[0] = static_cast<uint16_t*>(Qo);
    a.out[1] = static_cast<uint16_t*>(Ko);
    a.inv_freq = inv_freq;
    a.positions = positions;
    a.position_stride = position_stride;
    a.heads[0] = H;
    a.heads[1] = H_kv;
    a.T = T;
    a.rotary = rotary;
    a.amplitude = amplitude;
    a.sign = sign;
    // the widest access that pairs of chunks allow; what is not turned is a multiple of it, too
    const int span = interleaved ? rotary : rotary / 2;
    const int v = span % 8 == 0 ? 8 : span % 4 == 0 ? 4 : span % 2 == 0 ? 2 : 1;
    a.rot_chunks = span / v;
    const bool in_place = Q == Qo && (!K || K == Ko);
    a.chunks = a.rot_chunks + (in_place ? 0 : (D - rotary) / v);
    a.heads_inside = a.sin[0].h < a.sin[0].t;
    // Heads in flight to a thread, if that leaves 512 threads for every SM (24 heads, R=64, half layout, B=8, T=1024: 9.2 us with
    // four, 11.2 with all of them to a thread); tokens for whole blocks, if that leaves a block for every SM.
    const int heads = H + H_kv;
    a.rows = B * T;
    const long long places = static_cast<long long>(a.rows) * a.chunks;
    const int flight = heads_in_flight(interleaved != 0);
    const int per_thread = places * heads >= 512ll * flight * st->num_sms ? flight : 1;
    a.groups = std::max(1, std::min(kThreads / a.chunks, (heads + per_thread - 1) / per_thread));
    int tokens = std::max(1, kThreads / (a.chunks * a.groups));
    tokens = std::min(tokens, std::max(1, kMaxAngles / (rotary / 2)));
    a.tokens = std::max(1, std::min(tokens, (a.rows + st->num_sms - 1) / st->num_sms));
    const int blocks = (a.rows + a.tokens - 1) / a.tokens;
    auto go = [&](auto kernel) {
        return launch_overlapped(kernel, dim3(blocks), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a);
    };
    cudaError_t e;
    if (interleaved)
        e = v == 8 ? go(rope_kernel<8, true>) : v == 4 ? go(rope_kernel<4, true>) : go(rope_kernel<2, true>);
    else
        e = v == 8   ? go(rope_kernel<8, false>)
            : v == 4 ? go(rope_kernel<4, false>)
            : v == 2 ? go(rope_kernel<2, false>)
                     : go(rope_kernel<1, false>);
    return e == cudaSuccess ? NOVA_ATTN_OK : record_cuda_error(e);
}

}  // namespace
}  // namespace nova

extern "C" {

int nova_rope_fwd(const void* Q, const void* K, void* Q_out, void* K_out, const float* inv_freq, const int* positions, int B, int H,
                  int H_kv, int T, int D, int rotary, int interleaved, float amplitude, long long position_stride,
                  const nova_attn_strides* q_strides, const nova_attn_strides* k_strides, const nova_attn_strides* q_out_strides,
                  const nova_attn_strides* k_out_strides, void* stream) {
    return nova::rope(Q, K, Q_out, K_out, inv_freq, positions, B, H, H_kv, T, D, rotary, interleaved, amplitude, position_stride,
                      q_strides, k_strides, q_out_strides, k_out_strides, 1.f, stream);
}

int nova_rope_bwd(const void* dQ_out, const void* dK_out, void* dQ, void* dK, const float* inv_freq, const int* positions, int B, int H,
                  int H_kv, int T, int D, int rotary, int interleaved, float amplitude, long long position_stride,
                  const nova_attn_strides* dq_out_strides, const nova_attn_strides* dk_out_strides,
                  const nova_attn_strides* dq_strides, const nova_attn_strides* dk_strides, void* stream) {
    return nova::rope(dQ_out, dK_out, dQ, dK, inv_freq, positions, B, H, H_kv, T, D, rotary, interleaved, amplitude, position_stride,
                      dq_out_strides, dk_out_strides, dq_strides, dk_strides, -1.f, stream);
}

int nova_rope_frequencies(float* inv_freq, float* amplitude, int rotary, double base, int kind, double factor, long long original,
                          double low, double high) {
    if (!inv_freq || !amplitude) return NOVA_ATTN_ERR_NULL;
    if (rotary < 2 || (rotary & 1) || !std::isfinite(base) || base <= 1.0) return NOVA_ATTN_ERR_SHAPE;
    if (kind < NOVA_ROPE_PLAIN || kind > NOVA_ROPE_YARN) return NOVA_ATTN_ERR_SHAPE;
    const bool bands = kind == NOVA_ROPE_BANDS || kind == NOVA_ROPE_YARN;
    if (kind != NOVA_ROPE_PLAIN && (!std::isfinite(factor) || factor < 1.0)) return NOVA_ATTN_ERR_SHAPE;
    if (kind == NOVA_ROPE_BASE && rotary < 4) return NOVA_ATTN_ERR_SHAPE;
    if (bands && (original < 1 || !std::isfinite(low) || !std::isfinite(high) || low <= 0.0 || high <= low)) return NOVA_ATTN_ERR_SHAPE;
    constexpr double kTwoPi = 6.283185307179586;
    const double R = rotary;
    if (kind == NOVA_ROPE_BASE) base *= std::pow(factor, R / (R - 2.0));
    // the pair's number at which a frequency turns n times in the original context
    auto pair_of = [&](double n) { return R * std::log(original / (n * kTwoPi)) / (2.0 * std::log(base)); };
    const double at_high = bands ? std::fmax(std::floor(pair_of(high)), 0.0) : 0.0;
    double at_low = bands ? std::fmin(std::ceil(pair_of(low)), R - 1.0) : 0.0;
    if (at_low <= at_high) at_low = at_high + 1e-3;  // (where the bounds leave no pair between them)
    const bool none_stays = kind == NOVA_ROPE_YARN && original <= low * kTwoPi;  // the fastest turns `low` times at most
    for (int i = 0; i < rotary / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / R);
        double r = 1.0;  // the part that stays
        if (kind == NOVA_ROPE_LINEAR) r = 0.0;
        if (kind == NOVA_ROPE_BANDS) r = (original * f / kTwoPi - low) / (high - low);
        if (kind == NOVA_ROPE_YARN) r = none_stays ? 0.0 : 1.0 - (i - at_high) / (at_low - at_high);
        r = r < 0.0 ? 0.0 : r > 1.0 ? 1.0 : r;
        inv_freq[i] = static_cast<float>(r == 1.0 ? f : f * (r + (1.0 - r) / factor));
    }
    *amplitude = kind == NOVA_ROPE_YARN ? static_cast<float>(0.1 * std::log(factor) + 1.0) : 1.0f;
    return NOVA_ATTN_OK;
}

}  // extern "C"
