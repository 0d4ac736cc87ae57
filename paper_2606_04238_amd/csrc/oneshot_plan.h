// Sizes of the one-shot kernels (oneshot.h): waves of a workgroup, and rows of
// activations in the operands' order.
#pragma once

#include <hip/hip_runtime.h>

namespace qmlp {

// Steps of a row (64 bytes of codes), and the waves that share them: twice as many as
// long as a wave would have more than four, up to 8, so two to four steps each and
// more past 32.  (us, 4-bit rows of 2880, 23 steps, 21 experts:
// 4 waves 29.2, 6 30.9, 8 25.5; of 768, 6 steps, 104 experts: 2 waves 18.2, 4 20.2,
// 6 30.7; 2-bit gate and up of 2880, 12 steps, 21 experts: 3 waves 40.2, 4 37.2, 6
// 46.4, 8 41.5.)
__host__ __device__ constexpr int oneshot_steps(int K, int bits) { return (K * bits + 511) / 512; }
inline int oneshot_waves(int steps) {
    int kw = 1;
    while (kw < 8 && steps > 4 * kw) kw *= 2;
    return kw;
}

// Elements of a row in operand order, padded to whole steps, and its group sums.
__host__ __device__ inline int operand_row(int K, int bits) { return oneshot_steps(K, bits) * (512 / bits); }
__host__ __device__ inline int operand_sums(int K, int bits, int g) { return operand_row(K, bits) / g * 2; }

}  // namespace qmlp
