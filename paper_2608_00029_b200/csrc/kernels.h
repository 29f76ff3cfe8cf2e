// Internal launch interface between the C ABI (api.cu) and the kernels.  Not installed.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace nova {

constexpr int kBlockQ = 128;        // query rows per tile (UMMA M)
constexpr int kBlockK = 128;        // keys per tile
constexpr int kBoxCols = 64;        // bf16 elements per 128-byte swizzled row (TMA box inner extent)
constexpr int kHalfTileBytes = 128 * 128;  // one [128 rows x 64 bf16] box

struct AttnShape {
    int B, H, T, D;
    int causal;
    float scale;
};

// Strides, in elements, of a bf16 tensor indexed [b, h, t, d]; d is contiguous.  [B,H,T,D] storage has
// (H*T*D, T*D, D); the Q slice of a fused projection output [B, T, 3, H, D] has (T*3*H*D, D, 3*H*D).
struct TensorStrides {
    long long b, h, t;
};

// The window of nova_window.h: query i keeps key j if j <= i and (i - j < window or j < sinks).  Both at most T; `group` query heads
// share a key/value head.  The attention kernels have builds of their own for it (kWindow).
struct Window {
    int window, sinks, group;
};

// The key tiles of `unit` keys that the queries q0 .. q0 + rows - 1 of T keep anything of, numbered: those of the sinks that lie
// before the window, then the window's.
struct KeySpan {
    int sinks, skip, n;
    __host__ __device__ __forceinline__ int at(int j) const { return j < sinks ? j : j + skip; }
};
__host__ __device__ __forceinline__ KeySpan key_span(const Window& w, int q0, int rows, int T, int unit) {
    const int last = (q0 + rows < T ? q0 + rows : T) - 1, first = q0 - w.window + 1;
    const int lo = first > 0 ? first / unit : 0, hi = last / unit + 1;
    const int all = (w.sinks + unit - 1) / unit, sinks = all < lo ? all : lo;
    return KeySpan{sinks, lo - sinks, sinks + hi - lo};
}
// The query steps of `unit` rows of which anything keeps a key of the tile k0 .. k0 + keys - 1: the first, and how many.
__host__ __device__ __forceinline__ int query_steps(const Window& w, int k0, int keys, int T, int unit) {
    const int reach = (k0 + keys < T ? k0 + keys : T) - 1 + w.window;  // past the last query that a key outside the sinks has
    const int end = k0 < w.sinks || reach > T ? T : reach;
    return (end - 1) / unit + 1 - k0 / unit;
}

// Items of the dK/dV kernels with the window.  A key tile's list of steps (all query heads that share its head, one after another) is
// dealt out to `parts` items of equal length, or with sinks in the tile `sink_parts`: those lists end with the sequence.  Where there
// is more than one part each writes its sums, in 32 bits, to a slot of the workspace ([2][128][D]: dV, dK), and
// launch_window_sum adds them up.  One order of sums for all of a shape's calls.
struct KvParts {
    int n_tiles, sink_tiles, sink_parts, parts;  // tiles of a head; the first ones, which hold sinks
    __host__ __device__ __forceinline__ long long items(long long BH) const {
        return BH * (static_cast<long long>(sink_tiles) * sink_parts + static_cast<long long>(n_tiles - sink_tiles) * parts);
    }
    __host__ __device__ __forceinline__ long long slots(long long BH) const {
        return BH * ((sink_parts > 1 ? static_cast<long long>(sink_tiles) * sink_parts : 0) +
                     (parts > 1 ? static_cast<long long>(n_tiles - sink_tiles) * parts : 0));
    }
};
// How many parts the tile of item `idx` has.
__host__ __device__ __forceinline__ int kv_parts_of(const KvParts& p, int BH, int idx) {
    return idx < p.sink_tiles * p.sink_parts * BH ? p.sink_parts : p.parts;
}
struct KvItem {
    int kt, bh, part, parts, slot;  // slot: -1 without one
};
// Item `idx` of a problem with BH heads of K and V: tile by tile, the first (longest) ones first.
__host__ __device__ __forceinline__ KvItem kv_item(const KvParts& p, int BH, int idx) {
    const int first = p.sink_tiles * p.sink_parts * BH;
    const bool sink = idx < first;
    KvItem it;
    it.parts = sink ? p.sink_parts : p.parts;
    const int in = sink ? idx : idx - first, per_tile = it.parts * BH, tile = in / per_tile, rem = in - tile * per_tile;
    it.kt = (sink ? 0 : p.sink_tiles) + tile;
    it.part = it.parts == 1 ? 0 : rem / BH;
    it.bh = rem - it.part * BH;
    it.slot = it.parts == 1 ? -1 : sink ? idx : in + (p.sink_parts > 1 ? first : 0);
    return it;
}
// Steps [first, first + n) of a list of `all` that a part has.
__host__ __device__ __forceinline__ void kv_part(int all, int part, int parts, int* first, int* n) {
    *first = 0;
    *n = all;
    if (parts == 1) return;
    *first = static_cast<int>(static_cast<long long>(all) * part / parts);
    *n = static_cast<int>(static_cast<long long>(all) * (part + 1) / parts) - *first;
}
// BH: heads of K and V in all.  Of the shape alone.
KvParts kv_parts(int BH, int T, int D, const Window& win);
cudaError_t launch_window_sum(const float* partial, const KvParts& parts, __nv_bfloat16* dK, __nv_bfloat16* dV, const TensorStrides& sdk,
                              const TensorStrides& sdv, int B, int H_kv, int T, int D, float scale, cudaStream_t stream);

#ifdef __CUDACC__
// Bits 0 .. n - 1 of 64.
__device__ __forceinline__ uint64_t bits_below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }
// Which of the 64 keys from k0 on query `row` keeps (bit i: key k0 + i).
__device__ __forceinline__ uint64_t kept_keys(const Window& w, int row, int k0) {
    return bits_below(row + 1 - k0) & (~bits_below(row + 1 - w.window - k0) | bits_below(w.sinks - k0));
}
// The same of 32.
__device__ __forceinline__ uint32_t bits_below_32(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }
__device__ __forceinline__ uint32_t kept_keys_32(const Window& w, int row, int k0) {
    return bits_below_32(row + 1 - k0) & (~bits_below_32(row + 1 - w.window - k0) | bits_below_32(w.sinks - k0));
}
// Is there anything among the 64 keys from k0 on that one of the queries q0 .. q1 does not keep?
__device__ __forceinline__ bool any_dropped(const Window& w, int q0, int q1, int k0) {
    return k0 + 63 > q0 || (q1 - k0 >= w.window && k0 + 64 > w.sinks);
}
// Is there anything among the 64 queries from q0 on that does not keep one of the keys k0 .. k0 + 127?
__device__ __forceinline__ bool any_dropping(const Window& w, int k0, int q0) {
    return q0 < k0 + kBlockK - 1 || (q0 + 63 - k0 >= w.window && k0 + kBlockK > w.sinks);
}
// Which of the 64 queries from q0 on keep `key`.
__device__ __forceinline__ uint64_t keeping_queries(const Window& w, int key, int q0) {
    return ~bits_below(key - q0) & (key < w.sinks ? ~0ull : bits_below(key + w.window - q0));
}
#endif

// Records a CUDA error code for nova_attn_last_cuda_error() of the calling thread and returns
// NOVA_ATTN_ERR_CUDA; for the entry points that live outside api.cu.
int record_cuda_error(int code);

// The argument checks every backward entry point makes before anything else (NULL pointers, shape, 16-byte
// alignment of the tensors, scale); returns NOVA_ATTN_OK or the error nova_attn_bwd would report.
int validate_bwd_args(const void* Q, const void* K, const void* V, const void* dO, const float* LSE,
                      const float* Delta, const void* dQ, const void* dK, const void* dV, int B, int H, int T, int D,
                      float scale);

// Launches `kernel` allowing it to overlap the tail of the previous kernel in `stream` (programmatic
// dependent launch); the kernel must call griddep_wait() before it touches global memory.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_overlapped(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem_bytes,
                                     cudaStream_t stream, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem_bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Forward.  Two builds of every kernel.  Plain (`strided` false): all bf16 tensors have batch stride =
// H * head stride, so their maps are 3-D [D, T, B*H]; box of 64 x 128 tokens, 128-byte swizzle.  Strided:
// the maps are 4-D [D, x, y, z] with token / head / batch in order of increasing stride, and `orders`
// holds, four bits per tensor in the order Q, K, V, O, which of the three sits where (see
// tma_load_tile).  `tmO` describes the output and is used for TMA stores.  Persistent: launches at most
// `num_sms` CTAs.  `wait_limit`: cycle limit of every device-side wait; `inject`: test aid, 1 makes the
// loader leave out its first K-tile request so that a wait runs out (0 in normal use).
cudaError_t launch_attn_fwd(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                            const CUtensorMap& tmO, bool strided, uint32_t orders, float* LSE, const AttnShape& s,
                            int num_sms, long long wait_limit, int inject, int* dev_status, cudaStream_t stream);
cudaError_t configure_attn_fwd();

// `rest`: what rounding took from O, with its strides, or null.
cudaError_t launch_attn_bwd_preprocess(const __nv_bfloat16* O, const __nv_bfloat16* rest, const __nv_bfloat16* dO, float* Delta,
                                       const AttnShape& s, const TensorStrides& so, const TensorStrides& sdo,
                                       int num_sms, cudaStream_t stream);

// The query-major passes of the backward (attn_dq.cu; dQ at D = 128 only): K and V maps with boxes of kKeyStep rows.
constexpr int kKeyStep = 64;
// Exact Delta_i = sum_j P_ij (dO_i . V_j) with P rebuilt from LSE (two contractions + exp2 per tile).
cudaError_t launch_attn_delta(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                              const CUtensorMap& tmdO, const float* LSE, float* Delta, const AttnShape& s,
                              int num_sms, int* dev_status, cudaStream_t stream);
// Deterministic dQ (the dQ half of the paper's two-kernel backward): one CTA per pair of 128-row query tiles walks
// the keys in order and writes dQ = bf16(scale * sum_j dS_j K_j) through `tmdQ`.  `strided`, `orders`: as in the
// forward, for Q, K, V, dO, dQ.
cudaError_t launch_attn_dq(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                           const CUtensorMap& tmdO, const CUtensorMap& tmdQ, bool strided, uint32_t orders,
                           const float* LSE, const float* Delta, const AttnShape& s, int num_sms, int* dev_status,
                           cudaStream_t stream);
// With the window (D = 128): K and V maps have B * H / win.group heads.
cudaError_t launch_window_dq(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const CUtensorMap& tmdO,
                             const CUtensorMap& tmdQ, bool strided, uint32_t orders, const float* LSE, const float* Delta,
                             const AttnShape& s, const Window& win, int num_sms, int* dev_status, cudaStream_t stream);
cudaError_t configure_attn_dq();
// The same two at D = 64, with their operands in tensor memory (attn_dq64.cu).  The same bits of Delta.
cudaError_t launch_attn_delta64(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                                const CUtensorMap& tmdO, const float* LSE, float* Delta, const AttnShape& s, int* dev_status,
                                cudaStream_t stream);
cudaError_t launch_attn_dq64(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                             const CUtensorMap& tmdO, const CUtensorMap& tmdQ, bool strided, uint32_t orders,
                             const float* LSE, const float* Delta, const AttnShape& s, int* dev_status, cudaStream_t stream);
cudaError_t launch_window_dq64(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const CUtensorMap& tmdO,
                               const CUtensorMap& tmdQ, bool strided, uint32_t orders, const float* LSE, const float* Delta,
                               const AttnShape& s, const Window& win, int* dev_status, cudaStream_t stream);
cudaError_t configure_attn_dq64();

// The dK/dV half of the two-kernel backward at D = 128 (attn_dkdv.cu): Q and dO maps with boxes of kKeyStep rows, the
// others of 128.  `orders` for Q, K, V, dO, dK, dV.
cudaError_t launch_attn_dkdv(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                             const CUtensorMap& tmdO, const CUtensorMap& tmdK, const CUtensorMap& tmdV, bool strided,
                             uint32_t orders, const float* LSE, const float* Delta, const AttnShape& s, int num_sms,
                             int* dev_status, cudaStream_t stream);
// With the window (ops/window_dkdv.cu): dK and dV have the heads of K and V, an item all query heads that share its key/value head.
cudaError_t launch_window_dkdv(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const CUtensorMap& tmdO,
                               const CUtensorMap& tmdK, const CUtensorMap& tmdV, bool strided, uint32_t orders, const float* LSE,
                               const float* Delta, const AttnShape& s, const Window& win, const KvParts& parts, float* partial,
                               int* dev_status, cudaStream_t stream);
cudaError_t configure_attn_dkdv();
// The same at D = 64 (attn_dkdv64.cu).  `terms`: the row terms of every query as launch_row_terms64 leaves them (32 bytes for
// each of B * H * ceil(T / 64) * 64 rows, 16-byte aligned), or null: the kernel makes them itself (plain layout only).  Goes out
// right after the dQ kernel, whose end it does not wait for (ptx.cuh).
cudaError_t launch_row_terms64(const float* LSE, const float* Delta, void* terms, const AttnShape& s, cudaStream_t stream);
cudaError_t launch_attn_dkdv64(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                               const CUtensorMap& tmdO, const CUtensorMap& tmdK, const CUtensorMap& tmdV, bool strided,
                               uint32_t orders, const float* LSE, const float* Delta, const void* terms, const AttnShape& s,
                               int* dev_status, cudaStream_t stream);
cudaError_t launch_window_dkdv64(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const CUtensorMap& tmdO,
                                 const CUtensorMap& tmdK, const CUtensorMap& tmdV, bool strided, uint32_t orders, const float* LSE,
                                 const float* Delta, const AttnShape& s, const Window& win, const KvParts& parts, float* partial,
                                 int* dev_status, cudaStream_t stream);
cudaError_t configure_attn_dkdv64();

// Heads that the items of the kernels at D=128 are taken in together: enough items for two rounds of the SMs, and no more
// than about 48 MB of Q, K, V and dO, so that what the tiles of a head share stays in L2 (the forward re-reads K and V only,
// half of that).  All heads in one list, chunks, in us, forward / exact Delta / deterministic backward: B=16, H=32, T=1024
// 200, 174 / 173, 157 / 604, 547; B=4, H=32, T=2048 without the mask 280, 241 / 264, 240 / 908, 814.  Budgets of 24 and 96 MB
// are within 3 % of it, most within 1 %, in either direction (the forward at the first shape 184 and 176).  All heads where
// everything fits anyway (96 of the 126 MB): at 83 MB (B=16, H=16, T=333) 89.7 in one list, 92.2 us in two chunks, lost to
// the uneven end of the first; at 100 to 128 MB the two differ by at most 3 %.
inline int heads_per_chunk(int BH, int items_per_head, long long T, int D, int num_sms) {
    const long long per_head = T * D * 8;
    long long c = (48ll << 20) / per_head;
    const long long c_min = (2ll * num_sms + items_per_head - 1) / items_per_head;
    if (c < c_min) c = c_min;
    if (per_head * BH <= (96ll << 20) || c * 3 / 2 >= BH) return BH;
    const long long n = (BH + c - 1) / c;
    return static_cast<int>((BH + n - 1) / n);
}

// Steps after which the last SM is done with `items` work items that go out heaviest first, about: the longest item, or one
// item after another, the smallest of the first round with the largest of each later one.  steps(i): those of item i, with
// what an item costs besides.  For a few rounds of items (it adds them up).
template <typename F>
long long steps_until_done(long long items, int num_sms, F&& steps) {
    if (items <= num_sms) return steps(0);
    long long sum = steps(num_sms - 1);
    for (long long k = num_sms; k < items; k += num_sms) sum += steps(k);
    return steps(0) > sum ? steps(0) : sum;
}

// What the backward main kernel does with its partial tiles of dQ.
enum class DqMode {
    kAccumulate,  // adds them, unscaled, into the fp32 accumulator
    kDirect,      // T <= kBlockK, a head has one key tile: its dQ tile is complete and is written scaled, as bf16
};

// Backward main kernel: adds unscaled dQ partial tiles into the fp32 accumulator [B,H,T,D] (zero on
// entry) described by `tmAcc` (fp32 [D, T, B*H], box [32, 128, 1], 128-byte swizzle) and writes dK and dV
// through TMA stores (`tmdK`, `tmdV`: the bf16 maps of the outputs).  `strided`, `orders`: as in the forward, for
// Q, K, V, dO, dK, dV (and dQ).  `dq`: see above; `tmAcc` is the bf16 map of dQ with kDirect.
// Persistent: launches at most `num_sms` CTAs.
cudaError_t launch_attn_bwd(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                            const CUtensorMap& tmdO, const CUtensorMap& tmAcc, const CUtensorMap& tmdK,
                            const CUtensorMap& tmdV, bool strided, uint32_t orders, DqMode dq, const float* LSE,
                            const float* Delta, const AttnShape& s, int num_sms, int* dev_status, cudaStream_t stream);
cudaError_t configure_attn_bwd();

// Loss head (lmhead.cu): `tmX` is the 2-D map of X [K, M] with box [64, 128], `tmW` that of W [K, N] with box
// [64, 256], `tmL` that of the logits [N, M] with box [64, 32] (any valid map if `store_logits` is false), all
// bf16 with 128-byte swizzle.  Enqueues the fused contraction + statistics kernel and the merge.
cudaError_t launch_lmhead(const CUtensorMap& tmX, const CUtensorMap& tmW, const CUtensorMap& tmWh, const CUtensorMap& tmL,
                          bool store_logits, const int* targets, float* lse, float* loss, int M, int N, int K,
                          void* workspace, int num_sms, int* dev_status, cudaStream_t stream);
cudaError_t configure_lmhead();
size_t lmhead_workspace_bytes(int M, int N);
float* lmhead_target_logits(void* workspace, int M, int N);  // the part of the workspace behind the partial pairs
// Rows of the X and W boxes; returns the box width in k elements.
int lmhead_boxes(int* box_rows_x, int* box_rows_w);

// The same for at most kLmHeadFewRows rows (lmhead_rows.cu).  lmhead_rows_plan says whether this kernel is the faster one and
// chooses the number of CTAs, the height of a W tile (rows of the box of `tmW`) and the rows of the box of `tmX`; both boxes
// are 64 k elements wide.
constexpr int kLmHeadFewRows = 64;
cudaError_t configure_lmhead_rows();
bool lmhead_rows_plan(int M, int N, int num_sms, int* ctas, int* tile_h, int* m_pad);
cudaError_t launch_lmhead_rows(const CUtensorMap& tmX, const CUtensorMap& tmW, const int* targets, void* logits,
                               float* lse, float* loss, int M, int N, int K, int ctas, int tile_h, int m_pad,
                               void* workspace, float* tgt_logit, int* dev_status, cudaStream_t stream);

// The forward of the attention with a window (ops/window_fwd.cu).
cudaError_t configure_window_fwd();
// ops/window_dkdv.cu, ops/window_dq.cu
cudaError_t configure_window_dkdv();
cudaError_t configure_window_dq();

// Clears `bytes` (a multiple of 16) at the 16-byte aligned `ptr`.
cudaError_t launch_zero(void* ptr, size_t bytes, int num_sms, cudaStream_t stream);

// dQ = bf16(scale * dq_acc); the accumulator is contiguous [B,H,T,D], dQ has strides `sdq`.
cudaError_t launch_dq_convert(const float* dq_acc, __nv_bfloat16* dQ, const AttnShape& s, const TensorStrides& sdq,
                              float scale, int num_sms, cudaStream_t stream);

}  // namespace nova
