// One new token per sequence over a cache of keys and values, with a sliding window and sinks (include/nova_window.h).
//
// Memory bound: every kept key and value is read once, 4*D bytes, for the G query heads that share it.  A CTA takes a run of
// `chunk` kept keys of one key/value head of one sequence (so that sequences of all lengths make CTAs of one size), its four
// warps every fourth 16 of them; what a CTA finds, its maximum, sum and weighted sum per query head, is joined with the
// other runs' by a second kernel unless one run holds all.
//
// The two products go through the warp-level tensor instruction (m16n8k16), query heads as the rows: not for its rate, of which
// they need a tenth, but because the dot products of G heads with one key would otherwise be 4 G shuffles.  Its operands come
// straight from global memory, 16 bytes a load: which of the D dimensions, or of the keys, an instruction counts as which is
// free as long as both operands agree.
//   scores  the lane's 16 bytes of a key, dimensions 32 i + 8 (lane % 4) + 0..7, are its shares of two instructions
//   values  the lane's 16 bytes of four keys are columns of eight instructions, keys paired by byte permutes
// The weights enter the second product as two bf16 numbers each, which together keep 16 bits of them: rounded to one, they
// would cost as much accuracy as the rounding of the output does.
#include <cmath>

#include "../api.h"
#include "../ptx.cuh"
#include "window.h"

namespace nova {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kTile = 16;
constexpr int kRows = 16;  // query heads of a CTA at most

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// hi + lo = x to 16 bits, for two numbers at once
__device__ __forceinline__ void split_pair(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = pack_bf16x2(x, y);
    lo = pack_bf16x2(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xffff0000u));
}

// kWide: more than 8 query heads, rows 8 to 15 of the instructions are in use.
template <int D, bool kWide>
__global__ void __launch_bounds__(kThreads) window_decode_kernel(const __grid_constant__ DecodeArgs a) {
    __shared__ float s_o[kWarps][kWide ? 16 : 8][D];
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
    griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3, oct = lane >> 2;
    const int item = blockIdx.x / a.splits, split = blockIdx.x - item * a.splits;
    const int hg = item % a.head_groups, bk = item / a.head_groups;
    const int b = bk / a.H_kv, kv = bk - b * a.H_kv;
    const int h0 = kv * a.group + hg * kRows, rows = min(kRows, a.group - hg * kRows);
    griddep_wait();
    const DecodeKeys keys = decode_keys(a, __ldg(a.lengths + b));
    const int e0 = split * a.chunk, e1 = min(keys.n, e0 + a.chunk);
    if (e0 >= e1 && !(split == 0 && a.splits == 1)) return;  // (a run that is not there is not looked for either)

    // Q as the first operand: rows oct and oct + 8
    uint32_t qa[D / 32][4], qb[D / 32][4];
    const uint16_t* const q = a.q + b * a.sq.b + h0 * a.sq.h + 8 * quad;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        uint4 x = make_uint4(0, 0, 0, 0), y = x;
        if (oct < rows) x = *reinterpret_cast<const uint4*>(q + oct * a.sq.h + 32 * i);
        if (kWide && oct + 8 < rows) y = *reinterpret_cast<const uint4*>(q + (oct + 8) * a.sq.h + 32 * i);
        qa[i][0] = x.x, qa[i][1] = x.y, qa[i][2] = x.z, qa[i][3] = x.w;
        qb[i][0] = y.x, qb[i][1] = y.y, qb[i][2] = y.z, qb[i][3] = y.w;
    }
    const uint16_t* const kp = a.k + b * a.sk.b + kv * a.sk.h + 8 * quad;
    const uint16_t* const vp = a.v + b * a.sv.b + kv * a.sv.h + 8 * oct;

    uint4 kr[2][D / 32];
    auto load_k = [&](int e) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int x = e + 8 * j + oct;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                kr[j][i] = x < e1 ? __ldcs(reinterpret_cast<const uint4*>(kp + keys.token(x) * a.sk.t + 32 * i)) : make_uint4(0, 0, 0, 0);
        }
    };
    float o[D / 64][8][4] = {};
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;  // l: this lane's keys only
    int e = e0 + warp * kTile;
    if (e < e1) load_k(e);
    for (; e < e1; e += kWarps * kTile) {
        uint4 vr[4][D / 64];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int x = e + 2 * quad + (y & 1) + 8 * (y >> 1);
            // (a value that does not count must not reach the product, where 0 times infinity is NaN)
#pragma unroll
            for (int i = 0; i < D / 64; ++i)
                vr[y][i] = x < e1 ? __ldcs(reinterpret_cast<const uint4*>(vp + keys.token(x) * a.sv.t + 64 * i)) : make_uint4(0, 0, 0, 0);
        }
        float s[2][4] = {};
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                mma_16816(s[j], qa[i][0], qb[i][0], qa[i][1], qb[i][1], kr[j][i].x, kr[j][i].y);
                mma_16816(s[j], qa[i][2], qb[i][2], qa[i][3], qb[i][3], kr[j][i].z, kr[j][i].w);
            }
        if (e + kWarps * kTile < e1) load_k(e + kWarps * kTile);
        // base-2 logarithms of the weights; keys past the run weigh nothing
        float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                s[j][y] = e + 8 * j + 2 * quad + (y & 1) < e1 ? s[j][y] * a.scale_log2 : -INFINITY;
                if (y < 2) t0 = fmaxf(t0, s[j][y]);
                else if (kWide) t1 = fmaxf(t1, s[j][y]);
            }
#pragma unroll
        for (int x = 1; x < 4; x <<= 1) {
            t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, x));
            if (kWide) t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, x));
        }
        t0 = fmaxf(t0, m0), t1 = fmaxf(t1, m1);
        if (__any_sync(0xffffffffu, t0 > m0 || t1 > m1)) {
            const float f0 = t0 > m0 ? ex2_approx(m0 - t0) : 1.f, f1 = t1 > m1 ? ex2_approx(m1 - t1) : 1.f;
            m0 = t0, m1 = t1;
            l0 *= f0, l1 *= f1;
#pragma unroll
            for (int i = 0; i < D / 64; ++i)
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    o[i][t][0] *= f0, o[i][t][1] *= f0;
                    if (kWide) o[i][t][2] *= f1, o[i][t][3] *= f1;
                }
        }
        const float r0 = m0 == -INFINITY ? 0.f : m0, r1 = m1 == -INFINITY ? 0.f : m1;
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float p0 = ex2_approx(s[j][0] - r0), p1 = ex2_approx(s[j][1] - r0);
            l0 += p0 + p1;
            split_pair(p0, p1, hi[2 * j], lo[2 * j]);
            hi[2 * j + 1] = lo[2 * j + 1] = 0u;
            if (kWide) {
                const float p2 = ex2_approx(s[j][2] - r1), p3 = ex2_approx(s[j][3] - r1);
                l1 += p2 + p3;
                split_pair(p2, p3, hi[2 * j + 1], lo[2 * j + 1]);
            }
        }
#pragma unroll
        for (int i = 0; i < D / 64; ++i)
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int w = t >> 1;
                const uint32_t sel = (t & 1) ? 0x7632u : 0x5410u;
                auto word = [&](int y) { return w == 0 ? vr[y][i].x : w == 1 ? vr[y][i].y : w == 2 ? vr[y][i].z : vr[y][i].w; };
                const uint32_t b0 = __byte_perm(word(0), word(1), sel), b1 = __byte_perm(word(2), word(3), sel);
                mma_16816(o[i][t], hi[0], hi[1], hi[2], hi[3], b0, b1);
                mma_16816(o[i][t], lo[0], lo[1], lo[2], lo[3], b0, b1);
            }
    }
#pragma unroll
    for (int x = 1; x < 4; x <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, x);
        l1 += __shfl_xor_sync(0xffffffffu, l1, x);
    }

    // ---- the four warps' parts of a row
    if (quad == 0) {
        s_m[warp][oct] = m0, s_l[warp][oct] = l0;
        s_m[warp][oct + 8] = m1, s_l[warp][oct + 8] = l1;
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int z = 0; z < (kWide ? 4 : 2); ++z)  // columns 2 quad + (z & 1) are dimensions 64 i + 8 * column + 0..7
#pragma unroll
            for (int t = 0; t < 8; t += 4)
                *reinterpret_cast<float4*>(&s_o[warp][oct + 8 * (z >> 1)][64 * i + 16 * quad + 8 * (z & 1) + t]) =
                    make_float4(o[i][t][z], o[i][t + 1][z], o[i][t + 2][z], o[i][t + 3][z]);
    __syncthreads();
    for (int x = threadIdx.x; x < rows * (D / 4); x += kThreads) {
        const int r = x / (D / 4), d = x % (D / 4) * 4;
        float m = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m = fmaxf(m, s_m[w][r]);
        float l = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float f = s_m[w][r] == -INFINITY ? 0.f : ex2_approx(s_m[w][r] - m);
            const float4 v = *reinterpret_cast<const float4*>(&s_o[w][r][d]);
            l += f * s_l[w][r];
            sum.x += f * v.x, sum.y += f * v.y, sum.z += f * v.z, sum.w += f * v.w;
        }
        const long long row = static_cast<long long>(b) * a.H + h0 + r;
        if (a.splits == 1) {
            const float inv = keys.n > 0 ? 1.f / l : 0.f;
            *reinterpret_cast<uint2*>(a.o + b * a.so.b + (h0 + r) * a.so.h + d) =
                make_uint2(pack_bf16x2(sum.x * inv, sum.y * inv), pack_bf16x2(sum.z * inv, sum.w * inv));
            if (d == 0) a.lse[row] = keys.n > 0 ? (m + log2f(l)) * kLn2 : -INFINITY;
        } else {
            const long long at = row * a.splits + split;
            *reinterpret_cast<float4*>(a.part_o + at * D + d) = sum;
            if (d == 0) a.part_ml[at] = make_float2(m, l);
        }
    }
}

// Joins the runs of a row (a block): its warps take runs in turn, a lane D/32 dimensions.
template <int D>
__global__ void __launch_bounds__(256) window_join_kernel(const __grid_constant__ DecodeArgs a) {
    constexpr int kPer = D / 32, kJoinWarps = 8;
    __shared__ float s_o[kJoinWarps][D];
    __shared__ float2 s_ml[kJoinWarps];
    griddep_launch_dependents();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H;
    const DecodeKeys keys = decode_keys(a, __ldg(a.lengths + b));
    const int runs = (keys.n + a.chunk - 1) / a.chunk;
    const long long at = static_cast<long long>(blockIdx.x) * a.splits;
    float m = -INFINITY, l = 0.f, o[kPer] = {};
    constexpr int kDeep = 4;
    for (int s = warp; s < runs; s += kJoinWarps * kDeep) {
        float2 ml[kDeep];
        float v[kDeep][kPer];
#pragma unroll
        for (int x = 0; x < kDeep; ++x) {
            const int run = s + x * kJoinWarps;
            ml[x] = make_float2(-INFINITY, 0.f);
            if (run < runs) ml[x] = a.part_ml[at + run];
#pragma unroll
            for (int i = 0; i < kPer; ++i) v[x][i] = run < runs ? a.part_o[(at + run) * D + lane * kPer + i] : 0.f;
        }
#pragma unroll
        for (int x = 0; x < kDeep; ++x) {
            const float t = fmaxf(m, ml[x].x), r = t == -INFINITY ? 0.f : t;
            const float f = ex2_approx(m - r), w = ex2_approx(ml[x].x - r);
            m = t;
            l = l * f + ml[x].y * w;
#pragma unroll
            for (int i = 0; i < kPer; ++i) o[i] = o[i] * f + v[x][i] * w;
        }
    }
    if (lane == 0) s_ml[warp] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < kPer; ++i) s_o[warp][lane * kPer + i] = o[i];
    __syncthreads();
    if (threadIdx.x >= D / 2) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, s_ml[w].x);
    const float r = top == -INFINITY ? 0.f : top;
    float sum = 0.f, x0 = 0.f, x1 = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
        const float f = ex2_approx(s_ml[w].x - r);
        sum += f * s_ml[w].y;
        x0 += f * s_o[w][2 * threadIdx.x];
        x1 += f * s_o[w][2 * threadIdx.x + 1];
    }
    const float inv = keys.n > 0 ? 1.f / sum : 0.f;
    *reinterpret_cast<uint32_t*>(a.o + b * a.so.b + h * a.so.h + 2 * threadIdx.x) = pack_bf16x2(x0 * inv, x1 * inv);
    if (threadIdx.x == 0) a.lse[blockIdx.x] = keys.n > 0 ? (top + log2f(sum)) * kLn2 : -INFINITY;
}

}  // namespace

DecodePlan decode_plan(int B, int H, int H_kv, int T_max, int window, int sinks) {
    DecodePlan p;
    const long long most = static_cast<long long>(window) + sinks;
    const int n = static_cast<int>(most < T_max ? most : T_max), group = H / H_kv;
    p.head_groups = (group + kRows - 1) / kRows;
    const long long items = static_cast<long long>(B) * H_kv * p.head_groups;
    // Runs of equal size: eight CTAs for each of the 148 SMs if the runs stay long enough for it, one tile a warp at least.
    long long chunk = (n * items + 148 * 8 - 1) / (148 * 8);
    constexpr int kLeast = kWarps * kTile;
    chunk = (chunk + kLeast - 1) / kLeast * kLeast;
    p.chunk = static_cast<int>(chunk < kLeast ? kLeast : chunk);
    p.splits = (n + p.chunk - 1) / p.chunk;
    p.items = items;
    return p;
}

cudaError_t launch_window_decode(const DecodeArgs& a, int D, long long items, int B, cudaStream_t stream) {
    const dim3 grid(static_cast<unsigned>(items * a.splits));
    auto go = [&](auto kernel) { return launch_overlapped(kernel, grid, dim3(kThreads), 0, stream, a); };
    const bool wide = a.group > 8;
    const cudaError_t e = D == 64 ? (wide ? go(window_decode_kernel<64, true>) : go(window_decode_kernel<64, false>))
                                  : (wide ? go(window_decode_kernel<128, true>) : go(window_decode_kernel<128, false>));
    if (e != cudaSuccess || a.splits == 1) return e;
    auto join = [&](auto kernel) {
        return launch_overlapped(kernel, dim3(static_cast<unsigned>(B) * a.H), dim3(256), 0, stream, a);
    };
    return D == 64 ? join(window_join_kernel<64>) : join(window_join_kernel<128>);
}

}  // namespace nova
