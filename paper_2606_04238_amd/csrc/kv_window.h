// The window of the attention kernels over the 4-bit cache: plain C++, so that its arithmetic can be checked without a device.
#pragma once

namespace qmlp {

// The first token that a row at position `pos` sees: max(0, pos - window + 1), or 0 without a window (0).  Positions go
// below 0 where a request has more new tokens than cached ones, and a window may be any int that is not negative: the
// difference is formed only where it is not negative either.
constexpr int first_seen(int pos, int window) { return window && pos >= window ? pos - window + 1 : 0; }

}  // namespace qmlp
