// Argument block and launchers of the router and the whole MoE layer
// (moe_route.hip, moe_layer.hip).
#pragma once

#include "oneshot_plan.h"
#include "qmlp_internal.h"
#include "tokens_plan.h"

namespace qmlp {

constexpr int kMoeExperts = 512, kMoeTopk = 16, kMoeTokens = 64;

struct RouteArgs {
    const uint16_t* x;       // [M][d]
    const uint16_t* router;  // [E][d]
    const float* bias;       // [E] or null
    int32_t* idx;            // [M][k]
    float* w;                // [M][k]
    double* logits;          // workspace: [M][E], and for many tokens the rows' norms [M], [E]
    float *xnorm, *wnorm;
    int M, d, E, k, score, bf;
};
hipError_t launch_route(const RouteArgs& a, hipStream_t st);
hipError_t launch_route_logits(const RouteArgs& a, hipStream_t st);

// A block of work of the experts' launches: up to 16 instances (a token and one
// of its slots) of one expert.
constexpr int kBlkInts = 64, kBlkInst = 16, kBlkTok = 32;    // ints: [0] expert, [1] instances, [2] its first row of h, [16..] their numbers, [32..] their tokens

struct MoeArgs {
    const uint32_t *cg, *mg, *cu, *mu, *cd, *md;             // [E] matrices each, one after another
    const uint16_t *Ag, *Bg, *Au, *Bu;                       // [E][r][d], [E][f][r], or null
    const uint16_t* x;
    uint16_t* y;
    int32_t* idx;            // [M][k], -1: slot not used
    float* w;
    const double* logits;    // [M][E]
    int* blocks;             // moe_blocks_most() blocks, those past the last with no instances
    float* t;                // [M k][2 r]
    uint16_t* h;             // M k rows in operand order, those of a block side by side (oneshot.h), in the blocks' order
    uint16_t* xo;            // x in operand order
    float* xs;               // and its group sums
    float* part;             // [M k][d]
    int M, d, f, r, E, k, score, gb, gg, db, dg;
    float lora_scale;
};
// The most blocks n instances of E experts can make.
__host__ __device__ inline int moe_blocks_most(int n, int E) { return n < E + n / 16 ? n : E + n / 16; }
// Behind launch_route_logits: chooses, runs the experts and adds up.
hipError_t launch_moe_experts(const MoeArgs& a, hipStream_t st);

}  // namespace qmlp
