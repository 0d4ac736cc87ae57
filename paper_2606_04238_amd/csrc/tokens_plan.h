// How linear_lora and moe_layer split their products: rows of the few-token kernels,
// shares of k, tiles.  Plain host C++ over sizes and compute units, so that the rules
// can be checked without a device.  The times are of a whole MI355X (256 units).
#pragma once

namespace qmlp {

constexpr int kLoraFewTokens = 16;       // rows of the one-shot kernel (a matrix operand's)
constexpr int kLoraMidRows = 64;         // rows up to which lora_mid_kernel multiplies

// Tiles of 16 outputs of a workgroup, up to 16 rows.  Two tiles share its operands, one
// makes twice the workgroups: one where those are no more than the compute units (us, 4
// bits, one and two tiles: 2560 x 2560, 160 tiles, M = 1 4.9 and 6.1, M = 16 7.1 and
// 8.4; 6144 x 4096, 384 tiles, 9.5 and 8.9, 16.4 and 12.0; 28672 x 4096 25.9 and 24.9,
// 51.9 and 38.9).
inline int lora_few_tiles(int n, int cus) { return (n + 15) / 16 <= cus ? 1 : 2; }

// Shares of k for 17 to 512 rows, where tiles of 128 outputs (and 128 rows) leave half
// the compute units or more without one: as many as there are units for, of at
// least eight steps of 64.  (us, the product's launches with one share and with
// the rule's: 17 x 6144 x 4096, 48 tiles, 35.7 and 16.9; 67 rows 50.5 and 23.4; 200 x
// 2560 x 2560 36.9 and 20.6; 128 x 2560 x 9728 97 and 26; rank 64: 256 x 4096 x 4096
// 67 and 52, 512 84 and 71.)
inline int lora_shares(int M, int n, int k, int cus) {
    const long tiles = (long)((M + 127) / 128) * ((n + 127) / 128);
    if (M < 1 || M > 512 || tiles > cus / 2)
        return 1;
    const int most = k / 64 / 8, fill = (int)(cus / tiles);
    return most < 1 ? 1 : fill < most ? fill : most;
}
// Whether launch_lora_join follows launch_lora_gemm, for several shares or for the adapters.
inline bool lora_join(int M, int shares, bool adapters) { return shares > 1 || (M <= kLoraMidRows && adapters); }

// Whether more rows, in one share, run in tiles of 256 x 192 instead of 128 x 128.  The
// large ones take 2.2 times as long for three times the work; both run in rounds over
// the compute units (us, large and small: 600 x 2560 x 9728 236 and 116, 1024 x 6144 x
// 4096 141 and 117, 2048 x 2560 x 2560 110 and 86, 512 x 28672 x 4096 218 and 202;
// 4096 x 2560 x 2560 123 and 153, 520 x 14336 x 4096 114 and 146).
inline bool lora_large_tiles(int M, int n, int cus) {
    const auto rounds = [&](int BM, int BN) { return ((long)((M + BM - 1) / BM) * ((n + BN - 1) / BN) + cus - 1) / cus; };
    return 11 * rounds(256, 192) < 5 * rounds(128, 128);
}

// Whether a workgroup of moe_layer's gate and up, `inst` instances (a token and one of
// its experts) of E experts, f rows each, takes two tiles, which share its operands: not
// where that left compute units without a workgroup (us, 4 bits, d = 4096, f = 1536, one
// token's 2 experts: one tile 8.4, two 13.1), and for 2 bits, whose two tiles leave
// registers for two waves a SIMD, from an average of two instances an expert (d = f =
// 2880, 4 of 32 experts, one tile and two: M = 1 10.6 and 12.7, 8 37.3 and 40.4, 16 52.3
// and 52.9, 32 65.0 and 62.7, 64 80.5 and 68.8; 4 bits, d = 2048, f = 768, 8 of 128: M =
// 4 18.0 and 16.8, 13 37.2 and 35.3, 64 71.0 and 62.8).
inline bool moe_two_tiles(int inst, int E, int f, int bits, int cus) {
    return (long)inst * (f / 32) >= cus && (bits == 4 || inst > 2 * E);
}

}  // namespace qmlp
