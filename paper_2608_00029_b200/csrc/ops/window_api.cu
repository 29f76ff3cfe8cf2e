// Entry points of include/nova_window.h: argument checks, tensor maps, launches on the caller's stream.
#include <algorithm>
#include <cmath>

#include "../../../include/nova_window.h"
#include "../api.h"
#include "window.h"

using namespace nova;

namespace {

int check_window(int B, int H, int H_kv, int T, int D, int window, int sinks) {
    if (int rc = check_shape(B, H, T, D)) return rc;
    if (H_kv <= 0 || H % H_kv != 0 || window < 1 || sinks < 0) return NOVA_ATTN_ERR_SHAPE;
    return NOVA_ATTN_OK;
}

bool scale_ok(float scale) { return std::isfinite(scale) && scale > 0.f; }

size_t decode_bytes(const DecodePlan& p, int B, int H, int D) {
    return p.splits == 1 ? 0 : static_cast<size_t>(B) * H * p.splits * (D + 2) * sizeof(float);
}

Window window_of(int H, int H_kv, int T, int window, int sinks) { return Window{std::min(window, T), std::min(sinks, T), H / H_kv}; }

// The slots of the key tiles that are summed in parts.
size_t bwd_bytes(int B, int H_kv, int D, const KvParts& parts) {
    return std::max<size_t>(256, static_cast<size_t>(parts.slots(static_cast<long long>(B) * H_kv)) * 2 * kBlockK * D * sizeof(float));
}

}  // namespace

extern "C" {

int nova_window_fwd(const void* Q, const void* K, const void* V, void* O, void* O_rest, float* LSE, int B, int H, int H_kv, int T,
                    int D, int window, int sinks, const nova_attn_strides* q_strides, const nova_attn_strides* k_strides,
                    const nova_attn_strides* v_strides, const nova_attn_strides* o_strides, float scale, void* stream) {
    if (!Q || !K || !V || !O || !LSE) return NOVA_ATTN_ERR_NULL;
    if (int rc = check_window(B, H, H_kv, T, D, window, sinks)) return rc;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(O_rest) || !aligned16(LSE))
        return NOVA_ATTN_ERR_ALIGNMENT;
    if (!scale_ok(scale)) return NOVA_ATTN_ERR_SCALE;
    TensorStrides sq, sk, sv, so;
    if (int rc = check_strides(q_strides, D, &sq)) return rc;
    if (int rc = check_strides(k_strides, D, &sk)) return rc;
    if (int rc = check_strides(v_strides, D, &sv)) return rc;
    if (int rc = check_strides(o_strides, D, &so)) return rc;
    DeviceState* st = nullptr;
    if (int rc = device_state(&st)) return rc;
    const AttnShape s{B, H, T, D, 1, scale}, s_kv{B, H_kv, T, D, 1, scale};
    const Window win = window_of(H, H_kv, T, window, sinks);
    CUtensorMap tmQ, tmK, tmV;
    uint32_t oq, ok, ov;
    const bool strided = !(merges(s, sq) && merges(s_kv, sk) && merges(s_kv, sv));
    if (int rc = get_bf16_map(Q, s, sq, strided, &tmQ, &oq)) return rc;
    if (int rc = get_bf16_map(K, s_kv, sk, strided, &tmK, &ok, kKeyStep)) return rc;
    if (int rc = get_bf16_map(V, s_kv, sv, strided, &tmV, &ov, kKeyStep)) return rc;
    const uint32_t orders = oq | (ok << 4) | (ov << 8);
    const cudaError_t e = launch_window_fwd(tmQ, tmK, tmV, strided, orders, static_cast<__nv_bfloat16*>(O), static_cast<__nv_bfloat16*>(O_rest),
                                            LSE, so, s, win, st->dev_status, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? NOVA_ATTN_OK : record_cuda_error(e);
}

int nova_window_bwd_preprocess(const void* O, const void* O_rest, const void* dO, float* Delta, int B, int H, int T, int D,
                               const nova_attn_strides* o_strides, const nova_attn_strides* do_strides, void* stream) {
    if (!O || !dO || !Delta) return NOVA_ATTN_ERR_NULL;
    if (int rc = check_shape(B, H, T, D)) return rc;
    if (!aligned16(O) || !aligned16(O_rest) || !aligned16(dO) || !aligned16(Delta)) return NOVA_ATTN_ERR_ALIGNMENT;
    TensorStrides so, sdo;
    if (int rc = check_strides(o_strides, D, &so)) return rc;
    if (int rc = check_strides(do_strides, D, &sdo)) return rc;
    DeviceState* st = nullptr;
    if (int rc = device_state(&st)) return rc;
    const AttnShape s{B, H, T, D, 1, 1.f};
    const cudaError_t e = launch_attn_bwd_preprocess(static_cast<const __nv_bfloat16*>(O), static_cast<const __nv_bfloat16*>(O_rest),
                                                     static_cast<const __nv_bfloat16*>(dO), Delta, s, so, sdo, st->num_sms,
                                                     static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? NOVA_ATTN_OK : record_cuda_error(e);
}

size_t nova_window_bwd_workspace_bytes(int B, int H, int H_kv, int T, int D, int window, int sinks) {
    if (check_window(B, H, H_kv, T, D, window, sinks) != NOVA_ATTN_OK) return 0;
    return bwd_bytes(B, H_kv, D, kv_parts(B * H_kv, T, D, window_of(H, H_kv, T, window, sinks)));
}

int nova_window_bwd(const void* Q, const void* K, const void* V, const void* dO, const float* LSE, const float* Delta, void* dQ, void* dK,
                    void* dV, int B, int H, int H_kv, int T, int D, int window, int sinks, const nova_attn_strides* q_strides,
                    const nova_attn_strides* k_strides, const nova_attn_strides* v_strides, const nova_attn_strides* do_strides,
                    const nova_attn_strides* dq_strides, const nova_attn_strides* dk_strides, const nova_attn_strides* dv_strides,
                    float scale, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = validate_bwd_args(Q, K, V, dO, LSE, Delta, dQ, dK, dV, B, H, T, D, scale)) return rc;
    if (int rc = check_window(B, H, H_kv, T, D, window, sinks)) return rc;
    TensorStrides sq, sk, sv, sdo, sdq, sdk, sdv;
    if (int rc = check_strides(q_strides, D, &sq)) return rc;
    if (int rc = check_strides(k_strides, D, &sk)) return rc;
    if (int rc = check_strides(v_strides, D, &sv)) return rc;
    if (int rc = check_strides(do_strides, D, &sdo)) return rc;
    if (int rc = check_strides(dq_strides, D, &sdq)) return rc;
    if (int rc = check_strides(dk_strides, D, &sdk)) return rc;
    if (int rc = check_strides(dv_strides, D, &sdv)) return rc;
    const Window win = window_of(H, H_kv, T, window, sinks);
    const KvParts parts = kv_parts(B * H_kv, T, D, win);
    if (!workspace || workspace_bytes < bwd_bytes(B, H_kv, D, parts)) return NOVA_ATTN_ERR_WORKSPACE;
    if (parts.items(static_cast<long long>(B) * H_kv) > 0x7fffffffll) return NOVA_ATTN_ERR_SHAPE;
    if (!aligned16(workspace)) return NOVA_ATTN_ERR_ALIGNMENT;
    DeviceState* st = nullptr;
    if (int rc = device_state(&st)) return rc;
    const AttnShape s{B, H, T, D, 1, scale}, s_kv{B, H_kv, T, D, 1, scale};
    const bool strided = !(merges(s, sq) && merges(s_kv, sk) && merges(s_kv, sv) && merges(s, sdo) && merges(s, sdq) &&
                           merges(s_kv, sdk) && merges(s_kv, sdv));
    // Each kernel takes what it streams in boxes of kKeyStep rows and what it holds in boxes of 128.
    CUtensorMap tmQ, tmK, tmV, tmdO, tmQs, tmKs, tmVs, tmdOs, tmdQ, tmdK, tmdV;
    uint32_t oq, ok, ov, odo, odq, odk, odv;
    if (int rc = get_bf16_map(Q, s, sq, strided, &tmQ, &oq)) return rc;
    if (int rc = get_bf16_map(K, s_kv, sk, strided, &tmK, &ok)) return rc;
    if (int rc = get_bf16_map(V, s_kv, sv, strided, &tmV, &ov)) return rc;
    if (int rc = get_bf16_map(dO, s, sdo, strided, &tmdO, &odo)) return rc;
    if (int rc = get_bf16_map(K, s_kv, sk, strided, &tmKs, &ok, kKeyStep)) return rc;
    if (int rc = get_bf16_map(V, s_kv, sv, strided, &tmVs, &ov, kKeyStep)) return rc;
    if (int rc = get_bf16_map(Q, s, sq, strided, &tmQs, &oq, kKeyStep)) return rc;
    if (int rc = get_bf16_map(dO, s, sdo, strided, &tmdOs, &odo, kKeyStep)) return rc;
    if (int rc = get_bf16_map(dQ, s, sdq, strided, &tmdQ, &odq)) return rc;
    if (int rc = get_bf16_map(dK, s_kv, sdk, strided, &tmdK, &odk)) return rc;
    if (int rc = get_bf16_map(dV, s_kv, sdv, strided, &tmdV, &odv)) return rc;
    const uint32_t orders = oq | (ok << 4) | (ov << 8) | (odo << 12);
    const uint32_t orders_dq = orders | (odq << 16), orders_kv = orders | (odk << 16) | (odv << 20);
    const cudaStream_t cs = static_cast<cudaStream_t>(stream);
    float* const partial = static_cast<float*>(workspace);
    cudaError_t e;
    if (D == 64) {
        e = launch_window_dq64(tmQ, tmKs, tmVs, tmdO, tmdQ, strided, orders_dq, LSE, Delta, s, win, st->dev_status, cs);
        if (e == cudaSuccess)
            e = launch_window_dkdv64(tmQs, tmK, tmV, tmdOs, tmdK, tmdV, strided, orders_kv, LSE, Delta, s, win, parts, partial,
                                     st->dev_status, cs);
    } else {
        e = launch_window_dkdv(tmQs, tmK, tmV, tmdOs, tmdK, tmdV, strided, orders_kv, LSE, Delta, s, win, parts, partial, st->dev_status,
                               cs);
        if (e == cudaSuccess)
            e = launch_window_dq(tmQ, tmKs, tmVs, tmdO, tmdQ, strided, orders_dq, LSE, Delta, s, win, st->num_sms, st->dev_status, cs);
    }
    if (e == cudaSuccess && parts.slots(1) > 0)
        e = launch_window_sum(partial, parts, static_cast<__nv_bfloat16*>(dK), static_cast<__nv_bfloat16*>(dV), sdk, sdv, B, H_kv, T, D, scale, cs);
    return e == cudaSuccess ? NOVA_ATTN_OK : record_cuda_error(e);
}

size_t nova_window_decode_workspace_bytes(int B, int H, int H_kv, int T_max, int D, int window, int sinks) {
    if (check_window(B, H, H_kv, T_max, D, window, sinks) != NOVA_ATTN_OK) return 0;
    return decode_bytes(decode_plan(B, H, H_kv, T_max, D, window, sinks), B, H, D);
}

int nova_window_decode(const void* Q, const void* K, const void* V, const int* lengths, void* O, float* LSE, int B, int H, int H_kv,
                       int T_max, int D, int window, int sinks, const nova_attn_strides* q_strides, const nova_attn_strides* k_strides,
                       const nova_attn_strides* v_strides, const nova_attn_strides* o_strides, float scale, void* workspace,
                       size_t workspace_bytes, void* stream) {
    if (!Q || !K || !V || !lengths || !O || !LSE) return NOVA_ATTN_ERR_NULL;
    if (int rc = check_window(B, H, H_kv, T_max, D, window, sinks)) return rc;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return NOVA_ATTN_ERR_ALIGNMENT;
    if ((reinterpret_cast<uintptr_t>(LSE) & 3u) || (reinterpret_cast<uintptr_t>(lengths) & 3u)) return NOVA_ATTN_ERR_ALIGNMENT;
    if (!scale_ok(scale)) return NOVA_ATTN_ERR_SCALE;
    DecodeArgs a{};
    if (int rc = check_strides(q_strides, D, &a.sq)) return rc;
    if (int rc = check_strides(k_strides, D, &a.sk)) return rc;
    if (int rc = check_strides(v_strides, D, &a.sv)) return rc;
    if (int rc = check_strides(o_strides, D, &a.so)) return rc;
    const DecodePlan p = decode_plan(B, H, H_kv, T_max, D, window, sinks);
    if (p.items * p.splits > 0x7fffffffll) return NOVA_ATTN_ERR_SHAPE;
    const size_t need = decode_bytes(p, B, H, D);
    if (need > 0 && (!workspace || workspace_bytes < need)) return NOVA_ATTN_ERR_WORKSPACE;
    if (need > 0 && !aligned16(workspace)) return NOVA_ATTN_ERR_ALIGNMENT;
    DeviceState* st = nullptr;
    if (int rc = device_state(&st)) return rc;
    a.q = static_cast<const uint16_t*>(Q);
    a.k = static_cast<const uint16_t*>(K);
    a.v = static_cast<const uint16_t*>(V);
    a.o = static_cast<uint16_t*>(O);
    a.lengths = lengths;
    a.lse = LSE;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + static_cast<size_t>(B) * H * p.splits * D);
    a.H = H;
    a.H_kv = H_kv;
    a.group = H / H_kv;
    a.head_groups = p.head_groups;
    a.T_max = T_max;
    a.window = std::min(window, T_max);
    a.sinks = std::min(sinks, T_max);
    a.chunk = p.chunk;
    a.splits = p.splits;
    a.scale_log2 = scale * 1.4426950408889634f;
    const cudaError_t e = launch_window_decode(a, D, p.items, B, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? NOVA_ATTN_OK : record_cuda_error(e);
}

}  // extern "C"
