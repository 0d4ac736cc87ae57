// Argument block and launchers of the linear with adapters of many requests
// (lora_linear.hip, lora_gemm.hip).
#pragma once

#include "oneshot_plan.h"
#include "qmlp_internal.h"
#include "tokens_plan.h"

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
    int shares, cus;                     // of k, past 16 rows; compute units of the device
    // workspace
    int* known;                          // up to 16 rows: [16] adapter of a row, -1: none
    float* t;                            // up to 16 rows: [M][R] scale[a] A_a x, fp32; zeros where there is no adapter
    uint16_t* xo;                        // up to 16 rows: x in operand order, rows side by side (oneshot.h), or null
    float* xs;                           // and its group sums
    uint16_t* x16;                       // more: bfloat16 rows as binary16 x 2^e (rows k apart), or null
    float* xf;                           // [M] 2^-e (bfloat16)
    uint16_t* tb;                        // more than 16 rows: t as two bfloat16 terms [2][M][R]
    int* slots;                          // [M / 32, rounded up]: which of the mixed sets, or -1; then [kMixedSets]: their places
    float* parts;                        // [shares][M][n] sums of the shares of k, where lora_join() adds up; or null
    float* mixed;                        // [kMixedSets 32][n] adapter terms of the mixed sets' rows
};

// Sets of 32 rows with more than kMixedFrom adapters between them (rows without one
// count as one more) have their terms formed beforehand, up to kMixedSets of them.
constexpr int kMixedSets = 128, kMixedFrom = 3;
inline int lora_mixed_most(int M) { return (M + 31) / 32 < kMixedSets ? (M + 31) / 32 : kMixedSets; }

// Whether the one-shot kernel takes M rows: they fit one operand, and W's arrays
// 32-bit offsets.
inline bool lora_few_rows(int M, const qmlp_qweight* w) {
    return M <= kLoraFewTokens && (long)w->n_out * w->k_in * w->bits / 8 < (1l << 31) &&
           (long)w->n_out * (w->k_in / w->group) * 4 < (1l << 31);
}
hipError_t launch_lora_prep(const LoraArgs& a, hipStream_t st);
hipError_t launch_lora_mixed(const LoraArgs& a, hipStream_t st);
hipError_t launch_lora_few(const LoraArgs& a, hipStream_t st);
// (Into parts, and without the adapters, where those are not null: launch_lora_join adds up.)
hipError_t launch_lora_gemm(const LoraArgs& a, hipStream_t st);
hipError_t launch_lora_join(const LoraArgs& a, hipStream_t st);

}  // namespace qmlp
