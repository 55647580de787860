// Internal launch interface of what surrounds a layer's products: the norm (norm.hip), the product of 8-bit rows (gemm_a8.hip) and the
// requests' adapters (lora.hip); layer_api.hip checks arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kernels.h"

namespace mxfp4 {

// h = x + r, y = h / sqrt(mean(h^2) + eps) * w; what is null is not read or not written.
struct NormArgs {
    const uint16_t* x;
    const uint16_t* r;
    const uint16_t* w;
    uint16_t* sum;
    uint16_t* y;
    uint8_t* q8;        // E4M3 codes [M, K] and scale bytes [M, K / 32]
    uint8_t* s;
    int64_t ldx, ldr, lds, ldy;
    int m, k;
    float eps;
};
hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream);

// y = x8 * dequant(W)^T and what follows it.
struct A8Args {
    const uint8_t* x;   // E4M3 codes [M, K]
    const uint8_t* xs;  // their scale bytes [M, K / 32]
    const uint8_t* q;
    const uint8_t* s;
    uint16_t* y;
    int64_t ldy, ldr;
    Epilogue epi;       // (its ldr is not used)
    int m, n, k;
};
hipError_t launch_w4a8(const A8Args& a, const DeviceInfo& dev, hipStream_t stream);

// y[m] = base[m] + scale[i] * B_i (A_i x[m]) with i = ids[m]; rows with no such adapter: base[m].
struct LoraArgs {
    const uint16_t* x;
    const uint16_t* a;  // [adapters, R, K]
    const uint16_t* b;  // [adapters, N, R]
    const int32_t* ids;
    const float* scales;
    const uint16_t* base;
    uint16_t* y;
    float* part;        // [splits, M, R]: sums of A_i x over parts of K
    int64_t ldx, ldb, ldy;
    int m, n, k, r, adapters, splits;
};
constexpr int kMostAdapters = 8192;     // (four numbers of each lie in the LDS)
size_t lora_workspace(int64_t m, int64_t k, int64_t r);
hipError_t launch_lora(const LoraArgs& a, const DeviceInfo& dev, hipStream_t stream);

}  // namespace mxfp4
