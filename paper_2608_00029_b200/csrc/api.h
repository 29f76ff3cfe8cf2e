// What the files with entry points of the C ABI share (api.cu defines it): set-up of a device, argument checks, tensor maps.
// Not installed.
#pragma once

#include "../../include/nova_attn.h"
#include "kernels.h"

namespace nova {

struct DeviceState {
    bool ready = false;
    int status = NOVA_ATTN_OK;  // sticky result of the one-time set-up
    int num_sms = 0;
    int* dev_status = nullptr;
};

// One-time set-up of the current device: capability check, opt-in shared memory sizes, address of
// the device status word, tensor-map encoder entry point.
int device_state(DeviceState** out);

int check_shape(int B, int H, int T, int D);
bool aligned16(const void* p);

// Strides are in elements; every one a multiple of 8 (16 bytes, which TMA and the 16-byte accesses of the
// helper kernels need), the token stride at least D, none so large that a byte offset leaves 2^40.
int check_strides(const nova_attn_strides* p, int D, TensorStrides* out);

// Heads and batches of the tensor merge into one dimension (the [B,H,T,D] family): 3-D maps, plain kernels.
bool merges(const AttnShape& s, const TensorStrides& st);

// The map of a bf16 tensor for the plain (3-D) or the strided (4-D) build of the kernels.
int get_bf16_map(const void* ptr, const AttnShape& s, const TensorStrides& st, bool strided, CUtensorMap* out,
                 uint32_t* order, int box_rows = kBlockQ);

}  // namespace nova
