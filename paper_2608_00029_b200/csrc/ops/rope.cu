// Rotary positions of queries and keys (include/nova_rope.h).
//
// Memory bound: 4 bytes an element, and a sine and a cosine per token and pair, which all heads of the token share.  So a thread
// keeps one place in the head (8 dimensions, and in the half layout the 8 that they are paired with) of one token and walks
// over heads: it makes its angles once and then only streams, the 16-byte loads of four heads in flight.
#include <cmath>

#include "../../../include/nova_rope.h"
#include "../api.h"
#include "../ptx.cuh"

namespace nova {
namespace {

constexpr int kThreads = 256;
constexpr int kHeadsInFlight = 4;

struct RopeArgs {
    const uint16_t* in[2];  // Q, K
    uint16_t* out[2];
    TensorStrides sin[2], sout[2];
    const float* inv_freq;
    const int* positions;
    long long position_stride, units;
    int heads[2], T, rotary, rot_chunks, chunks, groups;
    float amplitude;  // its sign is that of the forward
    float sign;       // -1: backward
    bool heads_inside, wide;
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
// are V/2 pairs.  A unit is a chunk of V places (the last ones are copied), a token and a group of heads; where the
// heads of a token lie inside it, units next to each other take its heads in turn.
template <int V, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeArgs a) {
    using T4 = typename Vec<V>::type;
    constexpr int kAngles = kInterleaved ? V / 2 : V;
    griddep_launch_dependents();
    const long long u = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    const bool any = u < a.units;
    int c = 0, t = 0, g = 0, b = 0;
    if (a.wide) {
        long long r = u / a.chunks;
        c = static_cast<int>(u - r * a.chunks);
        const int inner = a.heads_inside ? a.groups : a.T, outer = a.heads_inside ? a.T : a.groups;
        long long r2 = r / inner;
        const int x = static_cast<int>(r - r2 * inner);
        b = static_cast<int>(r2 / outer);
        const int y = static_cast<int>(r2 - static_cast<long long>(b) * outer);
        t = a.heads_inside ? y : x;
        g = a.heads_inside ? x : y;
    } else {
        const uint32_t u32 = static_cast<uint32_t>(u), r = u32 / a.chunks;
        c = static_cast<int>(u32 - r * a.chunks);
        const uint32_t inner = a.heads_inside ? a.groups : a.T, outer = a.heads_inside ? a.T : a.groups;
        const uint32_t r2 = r / inner, x = r - r2 * inner;
        b = static_cast<int>(r2 / outer);
        const uint32_t y = r2 - b * outer;
        t = a.heads_inside ? y : x;
        g = a.heads_inside ? x : y;
    }
    griddep_wait();
    if (!any) return;

    const bool turns = c < a.rot_chunks;
    float co[kAngles], si[kAngles];
    int d = c * V, d2 = d;  // first place, and in the half layout that of the other ends of the pairs
    if (turns) {
        const double pos = a.positions != nullptr ? __ldg(a.positions + b * a.position_stride + t) : t;
        const int pair = kInterleaved ? d / 2 : d;
#pragma unroll
        for (int i = 0; i < kAngles; ++i) {
            const double turn = pos * static_cast<double>(__ldg(a.inv_freq + pair + i)) * 0.15915494309189535;  // 1 / 2 pi
            sincospif(2.0f * static_cast<float>(turn - rint(turn)), &si[i], &co[i]);
            si[i] *= a.amplitude * a.sign;
            co[i] *= a.amplitude;
        }
        if (!kInterleaved) d2 = d + a.rotary / 2;
    } else if (!kInterleaved) {
        d = d2 = a.rotary + (c - a.rot_chunks) * V;
    }

#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const TensorStrides si_ = a.sin[which], so_ = a.sout[which];
        const uint16_t* const in = a.in[which] + b * si_.b + t * si_.t;
        uint16_t* const out = a.out[which] + b * so_.b + t * so_.t;
        // heads are dealt out over the groups through both tensors
        const int first = which == 0 ? g : (g - a.heads[0] % a.groups + a.groups) % a.groups;
        for (int h0 = first; h0 < a.heads[which]; h0 += kHeadsInFlight * a.groups) {
            T4 x[kHeadsInFlight], y[kHeadsInFlight];
#pragma unroll
            for (int k = 0; k < kHeadsInFlight; ++k) {
                const int h = h0 + k * a.groups;
                if (h < a.heads[which]) {
                    x[k] = *reinterpret_cast<const T4*>(in + h * si_.h + d);
                    if (!kInterleaved && turns) y[k] = *reinterpret_cast<const T4*>(in + h * si_.h + d2);
                }
            }
#pragma unroll
            for (int k = 0; k < kHeadsInFlight; ++k) {
                const int h = h0 + k * a.groups;
                if (h >= a.heads[which]) break;
                if (turns) {
                    float p[V];
                    widen<V>(x[k], p);
                    if constexpr (kInterleaved) {
#pragma unroll
                        for (int i = 0; i < V; i += 2) {
                            const float p0 = p[i];
                            p[i] = p0 * co[i / 2] - p[i + 1] * si[i / 2];
                            p[i + 1] = p[i + 1] * co[i / 2] + p0 * si[i / 2];
                        }
                    } else {
                        float q[V];
                        widen<V>(y[k], q);
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float p0 = p[i];
                            p[i] = p0 * co[i] - q[i] * si[i];
                            q[i] = q[i] * co[i] + p0 * si[i];
                        }
                        *reinterpret_cast<T4*>(out + h * so_.h + d2) = narrow<V>(q);
                    }
                    x[k] = narrow<V>(p);
                }
                *reinterpret_cast<T4*>(out + h * so_.h + d) = x[k];
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
    // Groups of heads: threads for two rounds of the chip, if there are heads enough.
    const int heads = H + H_kv;
    const long long places = static_cast<long long>(B) * T * a.chunks, wanted = 2048ll * 2 * st->num_sms;
    long long groups = (wanted + places - 1) / places;
    a.groups = static_cast<int>(groups < heads ? groups : heads);
    a.units = places * a.groups;
    a.wide = a.units >= (1ll << 31);
    const long long blocks = (a.units + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffll) return NOVA_ATTN_ERR_SHAPE;
    auto go = [&](auto kernel) {
        return launch_overlapped(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a);
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
    if (at_low == at_high) at_low += 1e-3;
    for (int i = 0; i < rotary / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / R);
        double r = 1.0;  // the part that stays
        if (kind == NOVA_ROPE_LINEAR) r = 0.0;
        if (kind == NOVA_ROPE_BANDS) r = (original * f / kTwoPi - low) / (high - low);
        if (kind == NOVA_ROPE_YARN) r = 1.0 - (i - at_high) / (at_low - at_high);
        r = r < 0.0 ? 0.0 : r > 1.0 ? 1.0 : r;
        inv_freq[i] = static_cast<float>(r == 1.0 ? f : f * (r + (1.0 - r) / factor));
    }
    *amplitude = kind == NOVA_ROPE_YARN ? static_cast<float>(0.1 * std::log(factor) + 1.0) : 1.0f;
    return NOVA_ATTN_OK;
}

}  // extern "C"
