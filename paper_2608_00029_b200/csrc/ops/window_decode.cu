// One new token per sequence over a cache of keys and values, with a sliding window and sinks (include/nova_window.h).
//
// Memory bound: every kept key and value is read once, 4*D bytes, for the G query heads that share it (775 MB in 127 us, 6.1 TB/s, at
// B=64, H=32 on 8, D=128, ragged lengths up to 8192, window 4096).  A CTA takes a run of
// `chunk` kept keys of one key/value head of one sequence (so that sequences of all lengths make CTAs of one size), its four
// warps every fourth 16 of them; what a CTA finds, its maximum, sum and weighted sum per query head, is joined with the
// other runs' by a second kernel, or where there are few CTAs and a row's runs fit a cluster by these CTAs themselves.
//
// The two products go through the warp-level tensor instruction (m16n8k16), keys or dimensions as its 16 rows, query heads as its 8
// columns: not for its rate, of which they need a tenth, but because the dot products of G heads with one key would otherwise be
// 4 G shuffles.  Its operands come straight from global memory, 16 bytes a load: which of the D dimensions, or of the keys, an
// instruction counts as which is free as long as both operands agree.
//   scores  S^T = K Q^T: the lane's 16 bytes of a key, dimensions 32 i + 8 (lane % 4) + 0..7, are its shares of two instructions
//   values  O^T = V^T P^T: the lane's 16 bytes of four keys are two rows each of four instructions, keys paired by byte permutes;
//           P^T is the transpose of what the first product leaves in the lanes (movmatrix)
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
constexpr int kMaxCluster = 8;
// CTAs of the kernel below that an SM holds, cols: groups of 8 query heads.
__host__ __device__ constexpr int resident(int D, int cols) { return cols == 1 ? (D == 64 ? 5 : 3) : (D == 64 ? 3 : 2); }

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

// 8x8 matrix of 16-bit numbers, a row in four lanes: its transpose.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same shared-memory address in the CTA of the cluster with number `rank`.
__device__ __forceinline__ uint32_t peer_address(const void* p, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float4 load_peer4(uint32_t at) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float2 load_peer2(uint32_t at) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}

// kCols: groups of 8 query heads.  kCluster: the runs of a row are a cluster (no CTA leaves before the others have read from it).
template <int D, int kCols, bool kCluster>
__global__ void __launch_bounds__(kThreads, resident(D, kCols))
window_decode_kernel(const __grid_constant__ DecodeArgs a) {
    __shared__ float s_o[kWarps][8 * kCols][D + 4];  // (rows of a warp's eight lanes in different banks)
    __shared__ float s_m[kWarps][8 * kCols], s_l[kWarps][8 * kCols];
    __shared__ float4 s_run[kCluster ? 8 * kCols : 1][D / 4];  // kCluster: the CTA's sums, and their maxima and weights
    __shared__ float2 s_run_ml[8 * kCols];
    griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3, oct = lane >> 2;
    const int item = blockIdx.x / a.splits, split = blockIdx.x - item * a.splits;
    const int hg = item % a.head_groups, bk = item / a.head_groups;
    const int b = bk / a.H_kv, kv = bk - b * a.H_kv;
    const int h0 = kv * a.group + hg * kRows, rows = min(kRows, a.group - hg * kRows);
    griddep_wait();
    const DecodeKeys keys = decode_keys(a, __ldg(a.lengths + b));
    const int e0 = split * a.chunk, e1 = min(keys.n, e0 + a.chunk);
    if (!kCluster && e0 >= e1 && !(split == 0 && a.splits == 1)) return;  // (a run that is not there is not looked for either)

    // Q^T as the second operand: column oct of each group of heads
    uint4 qr[kCols][D / 32];
    const uint16_t* const q = a.q + b * a.sq.b + h0 * a.sq.h + 8 * quad;
#pragma unroll
    for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
            qr[n][i] = 8 * n + oct < rows ? *reinterpret_cast<const uint4*>(q + (8 * n + oct) * a.sq.h + 32 * i) : make_uint4(0, 0, 0, 0);
    const uint16_t* const kp = a.k + b * a.sk.b + kv * a.sk.h + 8 * quad;
    const uint16_t* const vp = a.v + b * a.sv.b + kv * a.sv.h + 8 * oct;

    uint4 kr[2][D / 32];  // keys oct and oct + 8 of the next sixteen
    auto load_k = [&](int e) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int x = e + 8 * j + oct;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                kr[j][i] = x < e1 ? __ldcs(reinterpret_cast<const uint4*>(kp + keys.token(x) * a.sk.t + 32 * i)) : make_uint4(0, 0, 0, 0);
        }
    };
    // o: dimensions 64 i + 8 oct + 2 t (+ 1: the second half) of heads 8 n + 2 quad and + 1; m, l: of the same two heads
    float o[kCols][D / 64][4][4] = {};
    float m[kCols][2], l[kCols][2];  // l: this lane's keys only
#pragma unroll
    for (int n = 0; n < kCols; ++n) m[n][0] = m[n][1] = -INFINITY, l[n][0] = l[n][1] = 0.f;
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
        float s[kCols][4] = {};  // keys oct (0, 1) and oct + 8 (2, 3), heads 2 quad and 2 quad + 1
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
                mma_16816(s[n], kr[0][i].x, kr[1][i].x, kr[0][i].y, kr[1][i].y, qr[n][i].x, qr[n][i].y);
                mma_16816(s[n], kr[0][i].z, kr[1][i].z, kr[0][i].w, kr[1][i].w, qr[n][i].z, qr[n][i].w);
            }
        if (e + kWarps * kTile < e1) load_k(e + kWarps * kTile);
        uint32_t hi[kCols][2], lo[kCols][2];
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
            // base-2 logarithms of the weights; keys past the run weigh nothing
            float t[2];
#pragma unroll
            for (int y = 0; y < 4; ++y) s[n][y] = e + oct + 8 * (y >> 1) < e1 ? s[n][y] * a.scale_log2 : -INFINITY;
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                t[z] = fmaxf(s[n][z], s[n][z + 2]);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) t[z] = fmaxf(t[z], __shfl_xor_sync(0xffffffffu, t[z], x));
                t[z] = fmaxf(t[z], m[n][z]);
            }
            if (__any_sync(0xffffffffu, t[0] > m[n][0] || t[1] > m[n][1])) {
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const float f = t[z] > m[n][z] ? ex2_approx(m[n][z] - t[z]) : 1.f;
                    m[n][z] = t[z];
                    l[n][z] *= f;
#pragma unroll
                    for (int i = 0; i < D / 64; ++i)
#pragma unroll
                        for (int w = 0; w < 4; ++w) o[n][i][w][z] *= f, o[n][i][w][z + 2] *= f;
                }
            }
            const float r0 = m[n][0] == -INFINITY ? 0.f : m[n][0], r1 = m[n][1] == -INFINITY ? 0.f : m[n][1];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float p0 = ex2_approx(s[n][2 * j] - r0), p1 = ex2_approx(s[n][2 * j + 1] - r1);
                l[n][0] += p0;
                l[n][1] += p1;
                split_pair(p0, p1, hi[n][j], lo[n][j]);
                hi[n][j] = transpose_8x8(hi[n][j]);
                lo[n][j] = transpose_8x8(lo[n][j]);
            }
        }
#pragma unroll
        for (int i = 0; i < D / 64; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                auto word = [&](int y) { return w == 0 ? vr[y][i].x : w == 1 ? vr[y][i].y : w == 2 ? vr[y][i].z : vr[y][i].w; };
                const uint32_t a0 = __byte_perm(word(0), word(1), 0x5410u), a1 = __byte_perm(word(0), word(1), 0x7632u);
                const uint32_t a2 = __byte_perm(word(2), word(3), 0x5410u), a3 = __byte_perm(word(2), word(3), 0x7632u);
#pragma unroll
                for (int n = 0; n < kCols; ++n) {
                    mma_16816(o[n][i][w], a0, a1, a2, a3, hi[n][0], hi[n][1]);
                    mma_16816(o[n][i][w], a0, a1, a2, a3, lo[n][0], lo[n][1]);
                }
            }
    }

    // ---- the four warps' parts of a row
#pragma unroll
    for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l[n][z] += __shfl_xor_sync(0xffffffffu, l[n][z], x);
            const int r = 8 * n + 2 * quad + z;
            if (oct == 0) s_m[warp][r] = m[n][z], s_l[warp][r] = l[n][z];
#pragma unroll
            for (int i = 0; i < D / 64; ++i)
#pragma unroll
                for (int w = 0; w < 4; w += 2)
                    *reinterpret_cast<float4*>(&s_o[warp][r][64 * i + 8 * oct + 2 * w]) =
                        make_float4(o[n][i][w][z], o[n][i][w][z + 2], o[n][i][w + 1][z], o[n][i][w + 1][z + 2]);
        }
    __syncthreads();
    for (int x = threadIdx.x; x < rows * (D / 4); x += kThreads) {
        const int r = x / (D / 4), d = x % (D / 4) * 4;
        float top = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top = fmaxf(top, s_m[w][r]);
        float sum_l = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float f = s_m[w][r] == -INFINITY ? 0.f : ex2_approx(s_m[w][r] - top);
            const float4 v = *reinterpret_cast<const float4*>(&s_o[w][r][d]);
            sum_l += f * s_l[w][r];
            sum.x += f * v.x, sum.y += f * v.y, sum.z += f * v.z, sum.w += f * v.w;
        }
        const long long row = static_cast<long long>(b) * a.H + h0 + r;
        if (kCluster) {
            s_run[r][d / 4] = sum;
            if (d == 0) s_run_ml[r] = make_float2(top, sum_l);
        } else if (a.splits == 1) {
            const float inv = keys.n > 0 ? 1.f / sum_l : 0.f;
            *reinterpret_cast<uint2*>(a.o + b * a.so.b + (h0 + r) * a.so.h + d) =
                make_uint2(pack_bf16x2(sum.x * inv, sum.y * inv), pack_bf16x2(sum.z * inv, sum.w * inv));
            if (d == 0) a.lse[row] = keys.n > 0 ? (top + log2f(sum_l)) * kLn2 : -INFINITY;
        } else {
            const long long at = row * a.splits + split;
            *reinterpret_cast<float4*>(a.part_o + at * D + d) = sum;
            if (d == 0) a.part_ml[at] = make_float2(top, sum_l);
        }
    }
    if constexpr (kCluster) {  // the CTAs share the row's columns
        cluster_sync();
        for (int x = split * kThreads + threadIdx.x; x < rows * (D / 4); x += a.splits * kThreads) {
            const int r = x / (D / 4), d = x % (D / 4) * 4;
            float2 ml[kMaxCluster];
            float4 v[kMaxCluster];
#pragma unroll
            for (int k = 0; k < kMaxCluster; ++k) {
                ml[k] = make_float2(-INFINITY, 0.f);
                v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k < a.splits) {
                    ml[k] = load_peer2(peer_address(&s_run_ml[r], k));
                    v[k] = load_peer4(peer_address(&s_run[r][d / 4], k));
                }
            }
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < kMaxCluster; ++k) top = fmaxf(top, ml[k].x);
            float sum_l = 0.f;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kMaxCluster; ++k) {
                if (k >= a.splits) break;
                const float f = ml[k].x == -INFINITY ? 0.f : ex2_approx(ml[k].x - top);
                sum_l += f * ml[k].y;
                sum.x += f * v[k].x, sum.y += f * v[k].y, sum.z += f * v[k].z, sum.w += f * v[k].w;
            }
            const float inv = keys.n > 0 ? 1.f / sum_l : 0.f;
            *reinterpret_cast<uint2*>(a.o + b * a.so.b + (h0 + r) * a.so.h + d) =
                make_uint2(pack_bf16x2(sum.x * inv, sum.y * inv), pack_bf16x2(sum.z * inv, sum.w * inv));
            if (d == 0) a.lse[static_cast<long long>(b) * a.H + h0 + r] = keys.n > 0 ? (top + log2f(sum_l)) * kLn2 : -INFINITY;
        }
        cluster_sync();
    }
}

// Joins the runs of a row: kPer warps to a row take its runs in turn, a lane D/32 dimensions; 8 / kPer rows (kPer <= 8) to a block.
template <int D, int kPer>
__global__ void __launch_bounds__(kPer > 8 ? 32 * kPer : 256) window_join_kernel(const __grid_constant__ DecodeArgs a, int n_rows) {
    constexpr int kDims = D / 32, kBlockWarps = kPer > 8 ? kPer : 8, kBlockRows = kBlockWarps / kPer;
    __shared__ float s_o[kPer > 1 ? kBlockWarps : 1][D];
    __shared__ float2 s_ml[kBlockWarps];
    griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % kPer;
    const int row = static_cast<int>(blockIdx.x) * kBlockRows + warp / kPer, b = min(row, n_rows - 1) / a.H, h = row - b * a.H;
    griddep_wait();
    const DecodeKeys keys = decode_keys(a, __ldg(a.lengths + b));
    const int runs = row < n_rows ? (keys.n + a.chunk - 1) / a.chunk : 0;
    const long long at = static_cast<long long>(row) * a.splits;
    float m = -INFINITY, l = 0.f, o[kDims] = {};
    constexpr int kDeep = 8;
    for (int s = part; s < runs; s += kPer * kDeep) {
        float2 ml[kDeep];
        float v[kDeep][kDims];
#pragma unroll
        for (int x = 0; x < kDeep; ++x) {
            const int run = s + x * kPer;
            ml[x] = make_float2(-INFINITY, 0.f);
            if (run < runs) ml[x] = a.part_ml[at + run];
#pragma unroll
            for (int i = 0; i < kDims; ++i) v[x][i] = run < runs ? a.part_o[(at + run) * D + lane * kDims + i] : 0.f;
        }
#pragma unroll
        for (int x = 0; x < kDeep; ++x) {
            const float t = fmaxf(m, ml[x].x), r = t == -INFINITY ? 0.f : t;
            const float f = ex2_approx(m - r), w = ex2_approx(ml[x].x - r);
            m = t;
            l = l * f + ml[x].y * w;
#pragma unroll
            for (int i = 0; i < kDims; ++i) o[i] = o[i] * f + v[x][i] * w;
        }
    }
    if constexpr (kPer > 1) {
        if (lane == 0) s_ml[warp] = make_float2(m, l);
#pragma unroll
        for (int i = 0; i < kDims; ++i) s_o[warp][lane * kDims + i] = o[i];
        __syncthreads();
        if (part != 0) return;
        float top = -INFINITY;
        for (int w = 0; w < kPer; ++w) top = fmaxf(top, s_ml[warp + w].x);
        const float r = top == -INFINITY ? 0.f : top;
        m = top;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < kDims; ++i) o[i] = 0.f;
#pragma unroll 8
        for (int w = 0; w < kPer; ++w) {
            const float f = ex2_approx(s_ml[warp + w].x - r);
            l += f * s_ml[warp + w].y;
#pragma unroll
            for (int i = 0; i < kDims; ++i) o[i] += f * s_o[warp + w][lane * kDims + i];
        }
    }
    if (row >= n_rows) return;
    const float inv = keys.n > 0 ? 1.f / l : 0.f;
    uint16_t* const to = a.o + b * a.so.b + h * a.so.h + lane * kDims;
    if constexpr (kDims == 2)
        *reinterpret_cast<uint32_t*>(to) = pack_bf16x2(o[0] * inv, o[1] * inv);
    else
        *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    if (lane == 0) a.lse[row] = keys.n > 0 ? (m + log2f(l)) * kLn2 : -INFINITY;
}

}  // namespace

DecodePlan decode_plan(int B, int H, int H_kv, int T_max, int D, int window, int sinks) {
    DecodePlan p;
    const long long most = static_cast<long long>(window) + sinks;
    const long long n = most < T_max ? most : T_max;
    const int group = H / H_kv;
    p.head_groups = (group + kRows - 1) / kRows;
    p.items = static_cast<long long>(B) * H_kv * p.head_groups;
    constexpr int kLeast = kWarps * kTile;
    auto rounded = [](long long chunk) { return (chunk + kLeast - 1) / kLeast * kLeast; };
    // Where it leaves no run longer than 1280 keys: as many runs to a row as leave no more CTAs than the GPU holds at once, so that all start
    // together and the last is done when the first is (us against eight CTAs to an SM: B=16, H=32 on 8, D=128, 1024 keys: 14.8, 20.4; B=8,
    // 4096 keys: 24.9, 31.2; B=1, 8192 keys: 11.9, 15.7; B=8, H=12, D=64, 1024 keys: 9.2, 11.2).  In clusters if they can be a few longer
    // runs: B=4, H=32 on 8, D=128, 2048 keys: 11.4 with 8 to a row, 12.2 with 11 and a kernel to join them.
    // From half of those CTAs on that is one run to a row.  H=32 on 8, D=128, 1024 keys, with one run, with three and with six: B=28 (224 of
    // 444 CTAs) 27.6, 28.9, 28.8, B=36 29.8, 32.1, 35.0, B=55 37.4, 45.5, 47.4; lengths up to 1024, where some rows end early, B=28 21.9,
    // 17.2, 17.7, B=36 23.8, 21.2, 21.1, B=55 26.5, 29.0, 28.5.
    const long long at_once = 148ll * resident(D, group > 8 ? 2 : 1) / p.items;
    long long splits = at_once > 1 ? at_once : 1;
    if (splits > kMaxCluster && n <= kMaxCluster * 256) splits = kMaxCluster;
    long long chunk = rounded((n + splits - 1) / splits);
    // Longer: twelve CTAs to an SM, which evens out sequences of different lengths.  (Time over that of the bytes, three draws of lengths
    // each, with twelve and with eight: B=64, H=32 on 8, D=128, lengths up to 8192, of which 4100 keys are kept: 1.05, 1.08; B=16, all
    // kept: 1.15, 1.23; H=64 on 4, D=64, B=32: 1.83, 2.00; B=2, up to 131072: 1.18, 1.20; B=4, up to 32768: 1.23, 1.14; all
    // B=64 of full length 1.01, 1.04.)
    if (chunk > 1280) chunk = rounded((n * p.items + 148 * 12 - 1) / (148 * 12));
    p.chunk = static_cast<int>(chunk);
    p.splits = static_cast<int>((n + chunk - 1) / chunk);
    return p;
}

cudaError_t launch_window_decode(const DecodeArgs& a, int D, long long items, int B, cudaStream_t stream) {
    const dim3 grid(static_cast<unsigned>(items * a.splits));
    auto go = [&](auto kernel) { return launch_overlapped(kernel, grid, dim3(kThreads), 0, stream, a); };
    const bool two = a.group > 8;
    // A cluster holds its places until its longest run is through, which does not matter where there are places for all.
    if (a.splits > 1 && a.splits <= kMaxCluster && items * a.splits <= 148 * resident(D, two ? 2 : 1)) {
        auto together = [&](auto kernel) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = grid;
            cfg.blockDim = dim3(kThreads);
            cfg.stream = stream;
            cudaLaunchAttribute attr[2];
            attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[0].val.programmaticStreamSerializationAllowed = 1;
            attr[1].id = cudaLaunchAttributeClusterDimension;
            attr[1].val.clusterDim = {static_cast<unsigned>(a.splits), 1, 1};
            cfg.attrs = attr;
            cfg.numAttrs = 2;
            return cudaLaunchKernelEx(&cfg, kernel, a);
        };
        return D == 64 ? (two ? together(window_decode_kernel<64, 2, true>) : together(window_decode_kernel<64, 1, true>))
                       : (two ? together(window_decode_kernel<128, 2, true>) : together(window_decode_kernel<128, 1, true>));
    }
    const cudaError_t e = D == 64 ? (two ? go(window_decode_kernel<64, 2, false>) : go(window_decode_kernel<64, 1, false>))
                                  : (two ? go(window_decode_kernel<128, 2, false>) : go(window_decode_kernel<128, 1, false>));
    if (e != cudaSuccess || a.splits == 1) return e;
    // Warps to a row: all of its runs in flight at once.
    const int n_rows = B * a.H;
    auto join = [&](auto kernel, int per) {
        const int rows = per > 8 ? 1 : 8 / per;
        return launch_overlapped(kernel, dim3((n_rows + rows - 1) / rows), dim3(per > 8 ? 32 * per : 256), 0, stream, a, n_rows);
    };
    if (a.splits <= 8) return D == 64 ? join(window_join_kernel<64, 1>, 1) : join(window_join_kernel<128, 1>, 1);
    if (a.splits <= 64) return D == 64 ? join(window_join_kernel<64, 8>, 8) : join(window_join_kernel<128, 8>, 8);
    return D == 64 ? join(window_join_kernel<64, 32>, 32) : join(window_join_kernel<128, 32>, 32);
}

}  // namespace nova
