// dQ of the attention with a window at D = 128: the roles of attn_dq.cu on the steps in reach of an item (KeySpan), K and V with the
// heads that query heads share.  Of a pair of tiles B leaves out the steps that only A's window reaches.
//
// Started while dK/dV runs, of which it needs nothing (ptx.cuh), and behind it rather than ahead because its items are the shorter
// ones: they fill up what the other's lists with sinks leave.  Backward (us), dQ behind dK/dV and ahead of it: B=2, H=12 on 4,
// T=8192, window 1024, 4 sinks: 367, 380; H=32 on 8, T=4096: 241, 255; H=16 on 4, T=1024, window 1024: 42.4, 43.7; H=4 on 2, T=993, window
// 93, 150 sinks: 17.9, 19.0.
#include <type_traits>

#include "../attn_dq.cuh"

namespace nova {
namespace {

template <int kTiles, bool kStrided>
__global__ void __launch_bounds__(kThreads, 1)
window_dq_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmdO,
                 const __grid_constant__ CUtensorMap tmdQ, const float* __restrict__ LSE, const float* __restrict__ Delta, int T, int BH,
                 int H, uint32_t orders, int n_blocks, int chunk, float scale, int* __restrict__ dev_status, const Window win) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    DqBars* bars = reinterpret_cast<DqBars*>(smem + DqCfg<128, kTiles>::kOffBar);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const DqWork<128, kTiles, true> wk{BH, n_blocks, chunk, T, H, orders, true, win};

    if (threadIdx.x == 0 || warp >= 4) griddep_taken_over();  // the threads that will read global memory
    const uint32_t tmem_base = dq_set_up<128, kTiles, false>(bars, &tmQ, &tmK, &tmV, &tmdO, &tmdQ, warp);
    griddep_launch_dependents();
    dq_roles<128, kTiles, true, kStrided, false, true>(smem, bars, tmem_base, &tmQ, &tmK, &tmV, &tmdO, &tmdQ, LSE, Delta, nullptr, wk, scale,
                                                       warp, lane);

    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, kTmemCols);
    griddep_wait();  // what waits for this kernel waits for dK/dV too
    if (threadIdx.x == 0 && bars->abort_flag != 0) atomicExch(dev_status, kDevTimeout);
}

}  // namespace

cudaError_t configure_window_dq() {
    auto set = [](auto kernel, int smem) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); };
    cudaError_t e = set(window_dq_kernel<1, false>, DqCfg<128, 1>::kSmemBytes);
    if (e == cudaSuccess) e = set(window_dq_kernel<1, true>, DqCfg<128, 1>::kSmemBytes);
    if (e == cudaSuccess) e = set(window_dq_kernel<2, false>, DqCfg<128, 2>::kSmemBytes);
    if (e == cudaSuccess) e = set(window_dq_kernel<2, true>, DqCfg<128, 2>::kSmemBytes);
    return e;
}

cudaError_t launch_window_dq(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const CUtensorMap& tmdO,
                             const CUtensorMap& tmdQ, bool strided, uint32_t orders, const float* LSE, const float* Delta,
                             const AttnShape& s, const Window& win, int num_sms, int* dev_status, cudaStream_t stream) {
    // Single tiles or pairs by the weights of attn_dq.cu; beyond a few rounds all items count as the last block's.  Backward, pairs and
    // single tiles: B=2, H=12 on 4, T=8192, window 1024, 4 sinks: 369, 383 us; B=4, H=32 on 8, T=2048, window 512: 281, 287; H=8 on 2,
    // T=2048, window 512: 44.1, 38.8; H=9 on 3, T=2304, window 700: 47.4, 43.2; H=16 on 4, T=4096, window 512, where the rule is wrong:
    // 80.0, 77.1.
    const int n_tiles = (s.T + kBlockQ - 1) / kBlockQ, n_pairs = (n_tiles + 1) / 2, BH = s.B * s.H;
    auto until_done = [&](int tiles, int n) -> long long {
        auto steps = [&](long long i) {
            return 2ll + key_span(win, (n - 1 - static_cast<int>(i / BH)) * tiles * kBlockQ, tiles * kBlockQ, s.T, kStep).n;
        };
        const long long items = static_cast<long long>(n) * BH;
        return items <= 8ll * num_sms ? steps_until_done(items, num_sms, steps) : (items + num_sms - 1) / num_sms * steps(0);
    };
    const bool single = 5 * until_done(1, n_tiles) < 8 * until_done(2, n_pairs);
    const int n_blocks = single ? n_tiles : n_pairs, chunk = heads_per_chunk(BH, n_blocks, s.T, s.D, num_sms);
    const dim3 grid(static_cast<unsigned>(n_blocks) * BH);
    auto go = [&](auto kernel, int smem) {
        return launch_overlapped(kernel, grid, dim3(kThreads), smem, stream, tmQ, tmK, tmV, tmdO, tmdQ, LSE,
                                 Delta, s.T, BH, s.H, orders, n_blocks, chunk, s.scale, dev_status, win);
    };
    if (single)
        return strided ? go(window_dq_kernel<1, true>, DqCfg<128, 1>::kSmemBytes)
                       : go(window_dq_kernel<1, false>, DqCfg<128, 1>::kSmemBytes);
    return strided ? go(window_dq_kernel<2, true>, DqCfg<128, 2>::kSmemBytes)
                   : go(window_dq_kernel<2, false>, DqCfg<128, 2>::kSmemBytes);
}

}  // namespace nova
