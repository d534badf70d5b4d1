// Sixteen bytes of a lane moved up or down by a number of bytes that differs from
// lane to lane.  Only 32-bit shifts: on gfx950 a 64-bit shift whose amount lies in
// the last vector register that the wavefront holds now and then gives a wrong
// result (6% of the lanes of a kernel of 128 registers with the amount in v127; none
// with it in v126, none where the kernel held 136), and the compiler puts it there.
#pragma once

#include <hip/hip_runtime.h>

namespace fqvit {

struct Bytes16 {
    uint32_t w[4];
};

// Byte n of `b` becomes byte 0, zeros come in at the top; n in [0, 16].
__device__ __forceinline__ Bytes16 bytes_down(Bytes16 b, int n) {
    if (n & 16) b = Bytes16{{0, 0, 0, 0}};
    if (n & 8) b = Bytes16{{b.w[2], b.w[3], 0, 0}};
    if (n & 4) b = Bytes16{{b.w[1], b.w[2], b.w[3], 0}};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        b.w[i] = __builtin_amdgcn_alignbyte(i < 3 ? b.w[i + 1] : 0, b.w[i], n & 3);
    return b;
}

// Byte 0 of `b` becomes byte n, zeros come in below; n in [0, 16].
__device__ __forceinline__ Bytes16 bytes_up(Bytes16 b, int n) {
    if (n & 16) b = Bytes16{{0, 0, 0, 0}};
    if (n & 8) b = Bytes16{{0, 0, b.w[0], b.w[1]}};
    if (n & 4) b = Bytes16{{0, b.w[0], b.w[1], b.w[2]}};
    if (n & 3) {
#pragma unroll
        for (int i = 3; i >= 0; --i)
            b.w[i] = __builtin_amdgcn_alignbyte(b.w[i], i > 0 ? b.w[i - 1] : 0, 4 - (n & 3));
    }
    return b;
}

}  // namespace fqvit
