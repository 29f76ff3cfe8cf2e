// dK and dV of the attention with a window at D = 128: the roles of attn_dkdv.cu.  The heads are those of K and V; an item is a tile's
// list of steps in reach of all query heads that share its head, or a part of it (KvParts).  B=2, H=12 on 4, T=8192, window 1024, 4
// sinks: 258 us under ncu, the tensor pipe 52 % busy.
// dQ (window_dq.cu) starts while this kernel runs: where the one waited for the other, the backward of H=4 on 2, T=993, window 93, 150
// sinks took 28.2 us, now 17.9; of H=8 on 1, T=1024, window 256, 4 sinks 33.9, now 24.2; the training pass of the shape above 540, now 517.
#include "../attn_dkdv.cuh"

namespace nova {
namespace {

template <bool kStrided>
__global__ void __launch_bounds__(kThreads, 1)
window_dkdv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmdO,
                   const __grid_constant__ CUtensorMap tmdK, const __grid_constant__ CUtensorMap tmdV,
                   const float* __restrict__ LSE, const float* __restrict__ Delta, int T, int BH, int H, uint32_t orders, float scale,
                   int* __restrict__ dev_status, const Window win, const KvParts parts, float* __restrict__ partial) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    if (smem != smem_raw) {
        // No room to realign: give up before anything is set up, but only once the predecessor in the stream
        // has completed (the status word is global memory, and this grid must not finish ahead of it).
        griddep_wait();
        if (threadIdx.x == 0) atomicExch(dev_status, kDevTimeout);
        return;
    }
    KvBars* bars = reinterpret_cast<KvBars*>(smem + kOffBar);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const KvWork<true> wk{BH, parts.n_tiles, BH, T, H, orders, true, win, parts};

    const uint32_t tmem_base = kv_set_up(bars, tmQ, tmK, tmV, tmdO, tmdK, tmdV, warp);
    griddep_wait();  // everything above overlaps the previous kernel of the stream
    griddep_launch_dependents();  // the dQ kernel, which needs nothing of dK and dV, but what was there before (ptx.cuh)
    kv_roles<true, kStrided, true>(smem, bars, tmem_base, tmQ, tmK, tmV, tmdO, tmdK, tmdV, partial, LSE, Delta, scale, wk, warp, lane);

    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, kTmemCols);
    if (threadIdx.x == 0 && bars->abort_flag != 0) atomicExch(dev_status, kDevTimeout);
}

}  // namespace

cudaError_t configure_window_dkdv() {
    const cudaError_t e =
        cudaFuncSetAttribute(window_dkdv_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(window_dkdv_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
}

cudaError_t launch_window_dkdv(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const CUtensorMap& tmdO,
                               const CUtensorMap& tmdK, const CUtensorMap& tmdV, bool strided, uint32_t orders, const float* LSE,
                               const float* Delta, const AttnShape& s, const Window& win, const KvParts& parts, float* partial,
                               int* dev_status, cudaStream_t stream) {
    const int H = s.H / win.group, BH = s.B * H;
    const dim3 grid(static_cast<unsigned>(parts.items(BH)));
    auto go = [&](auto kernel) {
        return launch_overlapped(kernel, grid, dim3(kThreads), kSmemBytes, stream, tmQ, tmK, tmV, tmdO, tmdK, tmdV, LSE, Delta,
                                 s.T, BH, H, orders, s.scale, dev_status, win, parts, partial);
    };
    return strided ? go(window_dkdv_kernel<true>) : go(window_dkdv_kernel<false>);
}

}  // namespace nova
