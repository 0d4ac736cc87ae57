// Argument block and launchers of the linear with adapters of many requests
// (lora_linear.hip, lora_gemm.hip).
#pragma once

#include "qmlp_internal.h"

namespace qmlp {

struct LoraArgs {
    const uint32_t *codes, *meta;        // W [n][k], `bits` wide in groups of g
    const uint16_t* x;                   // [M][k] activation type, rows ldx elements apart
    uint16_t* y;                         // [M][n], rows ldy elements apart
    const uint16_t *A, *B;               // [T][R][k], [T][n][R] activation type
    const float* scale;                  // [T] or null (1.0)
    const int32_t* ids;                  // [M]: adapter of a row, none outside [0, T)
    long ldx, ldy;
    int M, n, k, bits, g, T, R;
    int bf;                              // activations are bfloat16 (else binary16)
    // workspace
    float* t;                            // [M][R] scale[a] A_a x, fp32; zeros where there is no adapter
    uint16_t* x16;                       // bfloat16 rows as binary16 x 2^e (rows k apart), or null
    float* xf;                           // [M] 2^-e, or null
};

constexpr int kLoraFewTokens = 16;       // rows of the one-shot kernel (a matrix operand's)

// Whether the one-shot kernel takes the call: its rows fit one operand and its
// arrays 32-bit offsets.
inline bool lora_few_fits(const LoraArgs& a) {
    constexpr long most = 1l << 31;
    return a.M <= kLoraFewTokens && (long)a.n * a.k * a.bits / 8 < most && (long)a.n * (a.k / a.g) * 4 < most &&
           (a.x16 ? a.k : a.ldx) < most / 2 / kLoraFewTokens;
}
hipError_t launch_lora_prep(const LoraArgs& a, hipStream_t st);
hipError_t launch_lora_few(const LoraArgs& a, hipStream_t st);
hipError_t launch_lora_gemm(const LoraArgs& a, hipStream_t st);

}  // namespace qmlp
