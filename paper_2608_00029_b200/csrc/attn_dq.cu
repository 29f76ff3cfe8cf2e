// Query-major passes of the backward (paper Section 4.2, "The Backward Pass": one kernel reduces dQ over keys, the
// other reduces dK and dV over queries; the probability matrix is rebuilt from the saved log-sum-exp, never stored):
//   attn_dq_kernel     dQ_i = scale * sum_j dS_ij K_j,  dS = exp2(S*c - LSE*log2e) * (dP - Delta).  Every dQ row is
//                      summed by one thread block in key order: no atomics, no workspace, bitwise reproducible.
//   attn_delta_kernel  Delta_i = sum_j P_ij (dO_i . V_j): the exact softmax-Jacobian row term.  The cheap route to the
//                      same quantity, rowsum(dO * O), inherits the bf16 rounding of the stored O, which with sharply
//                      peaked rows (|O| ~ |V|) is the largest term in dQ and dK.
// dQ at D=128 only, the exact Delta there and, in the smallest and the largest problems, at D=64 (elsewhere: attn_dq64.cu).
// Both form S = Q K_j^T and dP = dO V_j^T tile by tile and differ in what becomes of the tile, so they are two builds of
// one kernel.
//
// A work item is a block of 256 query rows of one head: two 128-row tiles, A and B, that share every K and V tile
// they both need; in small problems one tile (plan_of).  The keys go by in steps of 64.  Items are handed out dynamically,
// heaviest first, as in the forward (WorkRing).  384 threads:
//   warp 0      TMA producer: Q and dO per tile of an item, K and V through a ring of 64-key stages
//   warps 1, 3  UMMA issuers, one per query tile, so that neither tile waits for the other's products and A may be in
//               the next item while B finishes this one
//   warps 4-7   rows of tile A, warps 8-11 rows of tile B: one thread per query row takes 64 keys of S and dP out of
//               tensor memory and writes dS back as bf16 (or adds P*dP into its Delta)
// (with single tiles, tile B's warps have nothing to do)
//
// What bounds it: one tile in flight is a serial chain (products -> tensor memory -> arithmetic -> tensor memory ->
// product), during which the tensor cores idle; two tiles fill each other's gaps.  64 keys per step is what tensor memory
// allows two tiles at D=128: dQ takes 128 of a tile's 256 columns, S and dP 64 each.  A product of N=64 with both
// operands in shared memory costs 49 clocks per 16 k elements against 65 for twice the keys, so a 128 x 128 block takes
// 2100 clocks of tensor time at D=128 (1560 with N=128).
#include <algorithm>
#include <type_traits>

#include "attn_dq.cuh"

namespace nova {
namespace {

// Set-up and roles, shared by the two builds below.
template <int D, int kTiles, bool kCausal, bool kStrided, bool kDelta>
__device__ __forceinline__ void dq_body(const CUtensorMap* tmQ, const CUtensorMap* tmK, const CUtensorMap* tmV,
                                        const CUtensorMap* tmdO, const CUtensorMap* tmdQ, const float* __restrict__ LSE,
                                        const float* __restrict__ Delta, float* __restrict__ Delta_out,
                                        const DqWork<D, kTiles, false>& wk, float scale, int* __restrict__ dev_status) {
    using Cfg = DqCfg<D, kTiles>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    DqBars* bars = reinterpret_cast<DqBars*>(smem + Cfg::kOffBar);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    const uint32_t tmem_base = dq_set_up<D, kTiles, kDelta>(bars, tmQ, tmK, tmV, tmdO, tmdQ, warp);
    griddep_launch_dependents();
    griddep_wait();  // everything above overlaps the previous kernel of the stream
    dq_roles<D, kTiles, kCausal, kStrided, kDelta, false>(smem, bars, tmem_base, tmQ, tmK, tmV, tmdO, tmdQ, LSE, Delta, Delta_out, wk, scale,
                                                          warp, lane);

    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, kTmemCols);
    if (threadIdx.x == 0 && bars->abort_flag != 0) atomicExch(dev_status, kDevTimeout);
}

template <int D, int kTiles, bool kCausal, bool kStrided>
__global__ void __launch_bounds__(kThreads, 1)
attn_dq_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
               const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmdO,
               const __grid_constant__ CUtensorMap tmdQ, const float* __restrict__ LSE, const float* __restrict__ Delta,
               int T, int BH, int H, uint32_t orders, int n_blocks, int chunk, float scale, int* __restrict__ dev_status) {
    dq_body<D, kTiles, kCausal, kStrided, false>(&tmQ, &tmK, &tmV, &tmdO, &tmdQ, LSE, Delta, nullptr,
                                                 DqWork<D, kTiles, false>{BH, n_blocks, chunk, T, H, orders, kCausal, Window{}}, scale,
                                                 dev_status);
}

template <int D, int kTiles, bool kCausal>
__global__ void __launch_bounds__(kThreads, 1)
attn_delta_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmdO,
                  const float* __restrict__ LSE, float* __restrict__ Delta, int T, int BH, int n_blocks, int chunk, float scale,
                  int* __restrict__ dev_status) {
    dq_body<D, kTiles, kCausal, false, true>(&tmQ, &tmK, &tmV, &tmdO, nullptr, LSE, nullptr, Delta,
                                             DqWork<D, kTiles, false>{BH, n_blocks, chunk, T, 1, 0u, kCausal, Window{}}, scale,
                                             dev_status);
}

// Key steps after which the last SM is done.  Every item costs two besides its own.
long long span_of(const AttnShape& s, int tiles, int n_blocks, int num_sms) {
    const long long BH = static_cast<long long>(s.B) * s.H, n_all = (s.T + kStep - 1) / kStep;
    return steps_until_done(n_blocks * BH, num_sms, [&](long long idx) {
        const long long blk = n_blocks - 1 - idx / BH;
        return 2 + (s.causal ? std::min(tiles * (blk + 1) * (kBlockQ / kStep), n_all) : n_all);
    });
}

// How many tiles an item has, and what follows from it.
//
// Two tiles share their K and V and fill each other's gaps, which is worth 30 to 40 % of the work where there is enough of
// it; a tile alone takes a step in 0.6 of a pair's time, so it wins where the longest chain or the last round of items
// decides.  The weights 5:8 are fitted to both forms' times over 688 shapes (T = 129 to 8192, 40 to 1200 tiles, with and
// without the mask, both head dimensions): the slower form is taken at a mean cost of 0.3 %.  Pairs against single tiles,
// exact Delta: H=8, T=4096: 69.4, 41.8 us.  (What comes here at D=64 is either one tile a head or many pairs.)
struct Plan {
    int tiles, n_blocks, chunk;
    dim3 grid;  // one CTA per item; those that do not start at once are taken over by those that did
};
Plan plan_of(const AttnShape& s, int num_sms) {
    Plan p;
    const int n_tiles = (s.T + kBlockQ - 1) / kBlockQ, n_pairs = (n_tiles + 1) / 2, BH = s.B * s.H;
    p.tiles = 2;
    if (static_cast<long long>(n_pairs) * BH <= 4ll * num_sms) {  // (beyond that pairs always win, and the sum stays short)
        const long long one = span_of(s, 1, n_tiles, num_sms), two = span_of(s, 2, n_pairs, num_sms);
        if (5 * one < 8 * two) p.tiles = 1;
    }
    p.n_blocks = (n_tiles + p.tiles - 1) / p.tiles;
    p.chunk = heads_per_chunk(BH, p.n_blocks, s.T, s.D, num_sms);
    p.grid = dim3(static_cast<unsigned>(p.n_blocks) * BH);
    return p;
}

// Calls f with the head dimension, the tiles of an item and the mask as compile-time constants.
template <typename F>
cudaError_t dispatch(int D, int tiles, bool causal, F&& f) {
    auto with_d = [&](auto d) {
        auto with_tiles = [&](auto t) { return causal ? f(d, t, std::true_type{}) : f(d, t, std::false_type{}); };
        return tiles == 1 ? with_tiles(std::integral_constant<int, 1>{}) : with_tiles(std::integral_constant<int, 2>{});
    };
    return D == 64 ? with_d(std::integral_constant<int, 64>{}) : with_d(std::integral_constant<int, 128>{});
}

}  // namespace

cudaError_t configure_attn_dq() {
    cudaError_t e = cudaSuccess;
    for (int k = 0; k < 8 && e == cudaSuccess; ++k)
        e = dispatch(k & 1 ? 64 : 128, k & 2 ? 1 : 2, (k & 4) != 0, [](auto d, auto t, auto causal) {
            constexpr int D = decltype(d)::value, kTiles = decltype(t)::value;
            constexpr bool kCausal = decltype(causal)::value;
            auto set = [](auto kernel) {
                return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, DqCfg<D, kTiles>::kSmemBytes);
            };
            cudaError_t r = set(attn_delta_kernel<D, kTiles, kCausal>);
            if constexpr (D == 128) {
                if (r == cudaSuccess) r = set(attn_dq_kernel<D, kTiles, kCausal, false>);
                if (r == cudaSuccess) r = set(attn_dq_kernel<D, kTiles, kCausal, true>);
            }
            return r;
        });
    return e;
}

cudaError_t launch_attn_dq(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                           const CUtensorMap& tmdO, const CUtensorMap& tmdQ, bool strided, uint32_t orders,
                           const float* LSE, const float* Delta, const AttnShape& s, int num_sms, int* dev_status,
                           cudaStream_t stream) {
    const Plan p = plan_of(s, num_sms);
    return dispatch(s.D, p.tiles, s.causal, [&](auto d, auto t, auto causal) {
        constexpr int D = decltype(d)::value, kTiles = decltype(t)::value;
        constexpr bool kCausal = decltype(causal)::value;
        if constexpr (D == 64) {
            return cudaErrorNotSupported;  // (attn_dq64.cu)
        } else {
            auto go = [&](auto kernel) {
                return launch_overlapped(kernel, p.grid, dim3(kThreads), DqCfg<D, kTiles>::kSmemBytes, stream, tmQ, tmK, tmV,
                                         tmdO, tmdQ, LSE, Delta, s.T, s.B * s.H, s.H, orders, p.n_blocks, p.chunk, s.scale,
                                         dev_status);
            };
            return strided ? go(attn_dq_kernel<D, kTiles, kCausal, true>) : go(attn_dq_kernel<D, kTiles, kCausal, false>);
        }
    });
}

cudaError_t launch_attn_delta(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                              const CUtensorMap& tmdO, const float* LSE, float* Delta, const AttnShape& s,
                              int num_sms, int* dev_status, cudaStream_t stream) {
    const Plan p = plan_of(s, num_sms);
    return dispatch(s.D, p.tiles, s.causal, [&](auto d, auto t, auto causal) {
        constexpr int D = decltype(d)::value, kTiles = decltype(t)::value;
        constexpr bool kCausal = decltype(causal)::value;
        return launch_overlapped(attn_delta_kernel<D, kTiles, kCausal>, p.grid, dim3(kThreads), DqCfg<D, kTiles>::kSmemBytes,
                                 stream, tmQ, tmK, tmV, tmdO, LSE, Delta, s.T, s.B * s.H, p.n_blocks, p.chunk, s.scale,
                                 dev_status);
    });
}

}  // namespace nova
