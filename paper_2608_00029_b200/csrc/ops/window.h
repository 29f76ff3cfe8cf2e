// The attention with a sliding window and sinks between the entry points and the kernels.  Not installed.
#pragma once

#include "../kernels.h"

namespace nova {

// K and V maps have B * H / win.group heads and boxes of kKeyStep rows; O and `rest` (which may be null) have strides `so`.
cudaError_t launch_window_fwd(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, bool strided, uint32_t orders,
                              __nv_bfloat16* O, __nv_bfloat16* rest, float* LSE, const TensorStrides& so, const AttnShape& s,
                              const Window& win, int* dev_status, cudaStream_t stream);

struct DecodeArgs {
    const uint16_t *q, *k, *v;
    uint16_t* o;
    TensorStrides sq, sk, sv, so;  // elements; the token strides of q and o are not used
    const int* lengths;
    float* lse;
    float* part_o;    // [B*H][splits][D] weighted sums relative to the maximum of their run
    float2* part_ml;  // [B*H][splits] maximum (base-2 logarithm) and sum
    int H, H_kv, group, head_groups, T_max, window, sinks, chunk, splits;
    float scale_log2;
};

// The keys that the query of a sequence of `length` tokens keeps, numbered: the sinks before the window, the window.
struct DecodeKeys {
    int n, sinks, skip;
    __device__ __forceinline__ long long token(int e) const { return e < sinks ? e : e + skip; }
};
__device__ __forceinline__ DecodeKeys decode_keys(const DecodeArgs& a, int length) {
    const int len = min(max(length, 0), a.T_max);
    const int first = max(0, len - a.window);
    const int sinks = min(a.sinks, first);
    return DecodeKeys{sinks + len - first, sinks, first - sinks};
}

struct DecodePlan {
    int head_groups, chunk, splits;
    long long items;  // sequences x key/value heads x groups of 16 query heads
};
// Of the shape alone: the size of the workspace and the order of the sums follow from it.
DecodePlan decode_plan(int B, int H, int H_kv, int T_max, int D, int window, int sinks);
cudaError_t launch_window_decode(const DecodeArgs& a, int D, long long items, int B, cudaStream_t stream);

}  // namespace nova
