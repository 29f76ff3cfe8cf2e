// How the dK/dV kernels' work with a window is cut into items (KvParts), and the sum of what the parts of a key tile found.
#include <algorithm>

#include "../api.h"
#include "../ptx.cuh"

namespace nova {
namespace {

constexpr int kThreads = 256;

// Eight columns of one row of dV or dK per thread: the parts' sums in order, 32 bits, rounded once.  Memory bound, and small beside the
// pass: 4.5 us cold, 2 parts of 8 tiles at D=128.
template <int D>
__global__ void __launch_bounds__(kThreads) window_sum_kernel(const float* __restrict__ partial, const KvParts parts, uint16_t* __restrict__ dK,
                                                              uint16_t* __restrict__ dV, const TensorStrides sdk, const TensorStrides sdv,
                                                              int BH, int H, int T, float scale) {
    constexpr int kPerRow = D / 8, kRows = kThreads / kPerRow, kBlocks = 2 * kBlockK / kRows;  // blocks of a tile: dV, dK
    griddep_launch_dependents();
    const int tile_bh = blockIdx.x / kBlocks, in = blockIdx.x - tile_bh * kBlocks;
    const int first = parts.sink_parts > 1 ? 0 : parts.sink_tiles;  // the first tile that is in parts
    const int kt = first + tile_bh / BH, bh = tile_bh - (kt - first) * BH;
    const int n = kt < parts.sink_tiles ? parts.sink_parts : parts.parts;
    const int vr = in * kRows + threadIdx.x / kPerRow, which = vr / kBlockK, r = vr - which * kBlockK, c = threadIdx.x % kPerRow * 8;
    // the slots of a tile lie BH apart
    const long long before = kt < parts.sink_tiles ? static_cast<long long>(kt) * n * BH
                                                   : (parts.sink_parts > 1 ? static_cast<long long>(parts.sink_tiles) * parts.sink_parts * BH : 0) +
                                                         static_cast<long long>(kt - parts.sink_tiles) * n * BH;
    const float* p = partial + ((before + bh) * 2 * kBlockK + vr) * D + c;
    const size_t step = static_cast<size_t>(BH) * 2 * kBlockK * D;
    const int row = kt * kBlockK + r;
    griddep_wait();
    if (row >= T) return;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
#pragma unroll 4
    for (int i = 0; i < n; ++i, p += step) {
        const float4 x = __ldcs(reinterpret_cast<const float4*>(p)), y = __ldcs(reinterpret_cast<const float4*>(p) + 1);
        a.x += x.x, a.y += x.y, a.z += x.z, a.w += x.w;
        b.x += y.x, b.y += y.y, b.z += y.z, b.w += y.w;
    }
    const float f = which ? scale : 1.f;
    const TensorStrides& s = which ? sdk : sdv;
    const int batch = bh / H, head = bh - batch * H;
    *reinterpret_cast<uint4*>((which ? dK : dV) + batch * s.b + head * s.h + row * s.t + c) =
        make_uint4(pack_bf16x2(a.x * f, a.y * f), pack_bf16x2(a.z * f, a.w * f), pack_bf16x2(b.x * f, b.y * f), pack_bf16x2(b.z * f, b.w * f));
}

}  // namespace

KvParts kv_parts(int BH, int T, int D, const Window& win) {
    constexpr int kSms = 148;
    KvParts p;
    p.n_tiles = (T + kBlockK - 1) / kBlockK;
    p.sink_tiles = std::min(p.n_tiles, (win.sinks + kBlockK - 1) / kBlockK);
    p.sink_parts = p.parts = 1;
    auto list = [&](int kt) { return static_cast<long long>(win.group) * query_steps(win, kt * kBlockK, kBlockK, T, kKeyStep); };
    // Steps of all lists, per SM: those with sinks end with the sequence, the others are of one length until they do, too.
    const long long n_q = (T + kKeyStep - 1) / kKeyStep, per_tile = kBlockK / kKeyStep;
    const long long whole = (static_cast<long long>(win.window) + kBlockK - 2) / kKeyStep + 1;
    auto to_end = [&](long long first, long long last) {  // tiles first .. last - 1
        return first < last ? (last - first) * n_q - per_tile * (last * (last - 1) - first * (first - 1)) / 2 : 0ll;
    };
    const long long cut_from = std::min<long long>(p.n_tiles, std::max<long long>(p.sink_tiles, n_q >= whole ? (n_q - whole) / per_tile + 1 : 0));
    const long long all = to_end(0, p.sink_tiles) + (cut_from - p.sink_tiles) * whole + to_end(cut_from, p.n_tiles);
    const long long total = all * win.group * BH, per_sm = total / kSms, tiles = static_cast<long long>(p.n_tiles) * BH;
    // Parts of tiles whose longest list is the first, the shortest the last.  One count for all of them, so that an item's tile is found by
    // a division, and no more than the shortest list has steps: the sequence's last tile has `group` of them or twice that, so without
    // shared heads nothing is cut, or in two, whatever is said below.  With counts by ranges of tiles the look-up cost more than that
    // mostly gave.  Backward (us), one count and ranges: H=2 on 1, T=64, window 16, D=64 7.4, 8.1; B=8, H=12, T=1024, window 256, D=64 54, 58;
    // H=16 on 2, T=768, window 475, D=128 31, 35; H=2, T=4097, window 1024, D=128 27, 40; where it gave, whole triangles on few heads: H=1,
    // T=8193, D=128 140, 124; H=4 on 2, T=1025, D=128 30, 23.
    auto cut = [&](int first, int last, long long most) -> int {
        const long long n = (list(first) + most - 1) / most;
        return static_cast<int>(std::max(1ll, std::min(n, list(last))));
    };
    // Small problems: the items of dQ and these run side by side as long as there is an SM for each.  Three quarters of what dQ leaves,
    // because each part costs memory traffic, too (backward, H=8 on 1, T=1024, window 256: at D=64 17.7 us with parts of 12 steps, 16.1
    // with 6; at D=128 with 4 sinks 25 with 8, 26 with 12; T=512, window 128, D=64, H=2 on 1: 15.0 with 12, 13.1 with 4).
    const long long spare = 3 * (kSms - win.group * tiles - tiles) / 4;
    const long long few = spare > 0 ? std::max(4ll, (total + spare - 1) / spare) : total;
    const long long rest = static_cast<long long>(p.n_tiles - p.sink_tiles) * BH;
    if (D == 128) {
        // dQ comes behind and fills up what these leave: as far as `cut` goes no part longer than an SM's share of the steps of both (a
        // step of dQ takes two thirds of one here).  B=2, H=12 on 4, T=8192, window 1024, 4 sinks, a list of 384 steps, a share of 349:
        // 419 us in one item, 370 in 2; H=12 on 4, T=4096, window 300, 1 sink, 192 and 38: 220, 61 in 6, 66 in 16; H=16 on 4, T=4096, window 512, all lists of
        // 40, 55: 80, 93 in 2; H=16 on 2, T=768, window 475, 1 sink, 96 and 80, 8: 104, 31 in 12 and 8, 35 in 6 and 6.  Parts without
        // sinks, which come later and are more, may be a third longer: H=16 on 4, T=1024, window 1024, 64 steps, 12: 34 in 4, 40 in 5.
        const long long most = std::max(std::min(few, 8ll), 5 * total / (3 * kSms));
        if (p.sink_tiles > 0) p.sink_parts = cut(0, p.sink_tiles - 1, most);
        if (rest > 0) p.parts = cut(p.sink_tiles, p.n_tiles - 1, most * 4 / 3);
        return p;
    }
    // dQ goes ahead, and the last of these to end should not be a long one.  A tile with sinks that is longer than an SM's share of all
    // steps: into parts of that share (H=8 on 8, T=16384, window 512, 4 sinks, a list of 256 steps, a share of 82: 214 us in one item, 103
    // in 4, 107 in 8).  Shorter ones go first and hold nobody up (B=8, H=12, T=1024, window 256, 4 sinks, 16 steps of 30: 55 us, 63
    // in two parts).  The others only where there are fewer of them than SMs.
    const long long least = std::min(few, 12ll), sink_least = few < 12 ? few : 16;  // below that the ends of an item cost more than its steps
    if (p.sink_tiles > 0 && list(0) > per_sm) p.sink_parts = cut(0, p.sink_tiles - 1, std::max(sink_least, per_sm));
    if (rest > 0 && rest < kSms) p.parts = cut(p.sink_tiles, p.n_tiles - 1, std::max(least, list(p.sink_tiles) * rest / kSms));
    return p;
}

cudaError_t launch_window_sum(const float* partial, const KvParts& parts, __nv_bfloat16* dK, __nv_bfloat16* dV, const TensorStrides& sdk,
                              const TensorStrides& sdv, int B, int H_kv, int T, int D, float scale, cudaStream_t stream) {
    const int BH = B * H_kv;
    const long long tiles = static_cast<long long>(parts.sink_parts > 1 ? parts.sink_tiles : 0) + (parts.parts > 1 ? parts.n_tiles - parts.sink_tiles : 0);
    const dim3 grid(static_cast<unsigned>(tiles * BH * (2 * kBlockK * (D / 8) / kThreads)));
    auto go = [&](auto kernel) {
        return launch_overlapped(kernel, grid, dim3(kThreads), 0, stream, partial, parts, reinterpret_cast<uint16_t*>(dK),
                                 reinterpret_cast<uint16_t*>(dV), sdk, sdv, BH, H_kv, T, scale);
    };
    return D == 64 ? go(window_sum_kernel<64>) : go(window_sum_kernel<128>);
}

}  // namespace nova
