// dK and dV of the two-kernel backward at D = 128 (paper Section 4.2, "The Backward Pass": one kernel reduces dQ over
// keys, the other reduces dK and dV over queries; the probability matrix is rebuilt from the saved log-sum-exp, never
// stored; the causal loop bound is raised so that queries above the diagonal are never visited).
//
// A work item is one 128-key tile of one head; its queries go by in steps of 64.  As in the fused kernel everything is
// transposed, keys on the lanes of tensor memory, so that P^T and dS^T feed the tensor cores from where they are made:
//   S^T  = K_j Q_s^T,  dP^T = V_j dO_s^T                       (smem x smem -> one of two buffers in TMEM)
//   P^T  = exp2(S^T*c - LSE*log2e),  dS^T = P^T * (dP^T - Delta)   (bf16, over the S^T and dP^T they came from)
//   dV  += P^T dO_s,  dK += dS^T Q_s                           (TMEM x smem, dO and Q read MN-major)
// Items are handed out dynamically (WorkRing), heaviest first within a chunk of heads whose tensors stay in L2
// together.  512 threads:
//   warp 0      TMA producer: K_j double-buffered, V_j, and Q_s and dO_s through a ring of 64-query stages
//   warp 1      UMMA issuer: S^T and dP^T run two steps ahead of dV and dK, across item boundaries
//   warp 2      row loader: -LSE*log2e and -Delta of a step into shared memory
//   warps 4-7   compute group 0, warps 8-11 group 1: the steps alternate between the groups; a thread has one key
//               row and the 64 queries of its step
//   warps 12-15 send dV and dK of a finished item out, through the item's own K buffer, which nothing reads any more,
//               while the compute warps are in the next item
#include "attn_dkdv.cuh"

namespace nova {
namespace {

template <bool kCausal, bool kStrided>
__global__ void __launch_bounds__(kThreads, 1)
attn_dkdv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmdO,
                 const __grid_constant__ CUtensorMap tmdK, const __grid_constant__ CUtensorMap tmdV,
                 const float* __restrict__ LSE, const float* __restrict__ Delta, int T, int BH, int H, uint32_t orders,
                 int n_tiles, int chunk, float scale, int* __restrict__ dev_status) {
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
    const KvWork<false> wk{BH, n_tiles, chunk, T, H, orders, kCausal, Window{}, KvParts{}};

    const uint32_t tmem_base = kv_set_up(bars, tmQ, tmK, tmV, tmdO, tmdK, tmdV, warp);
    griddep_launch_dependents();
    griddep_wait();  // everything above overlaps the previous kernel of the stream
    kv_roles<kCausal, kStrided, false>(smem, bars, tmem_base, tmQ, tmK, tmV, tmdO, tmdK, tmdV, nullptr, LSE, Delta, scale, wk, warp, lane);

    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, kTmemCols);
    if (threadIdx.x == 0 && bars->abort_flag != 0) atomicExch(dev_status, kDevTimeout);
}

}  // namespace

cudaError_t configure_attn_dkdv() {
    auto set = [](auto kernel) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    };
    cudaError_t e = set(attn_dkdv_kernel<true, false>);
    if (e == cudaSuccess) e = set(attn_dkdv_kernel<true, true>);
    if (e == cudaSuccess) e = set(attn_dkdv_kernel<false, false>);
    if (e == cudaSuccess) e = set(attn_dkdv_kernel<false, true>);
    return e;
}

cudaError_t launch_attn_dkdv(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                             const CUtensorMap& tmdO, const CUtensorMap& tmdK, const CUtensorMap& tmdV, bool strided,
                             uint32_t orders, const float* LSE, const float* Delta, const AttnShape& s, int num_sms,
                             int* dev_status, cudaStream_t stream) {
    const int n_tiles = (s.T + kBlockK - 1) / kBlockK, BH = s.B * s.H;
    const int chunk = heads_per_chunk(BH, n_tiles, s.T, D, num_sms);
    const dim3 grid(static_cast<unsigned>(n_tiles) * BH);  // one CTA per item; those that do not start are taken over
    auto go = [&](auto kernel) {
        return launch_overlapped(kernel, grid, dim3(kThreads), kSmemBytes, stream, tmQ, tmK, tmV, tmdO, tmdK, tmdV, LSE, Delta,
                                 s.T, BH, s.H, orders, n_tiles, chunk, s.scale, dev_status);
    };
    if (s.causal) return strided ? go(attn_dkdv_kernel<true, true>) : go(attn_dkdv_kernel<true, false>);
    return strided ? go(attn_dkdv_kernel<false, true>) : go(attn_dkdv_kernel<false, false>);
}

}  // namespace nova
