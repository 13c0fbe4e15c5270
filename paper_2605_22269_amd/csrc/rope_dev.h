// Device helpers of the kernels that rotate rows on their way: elements of 16-byte pieces, the turn of a pair.
#pragma once

#include "attend_dev.h"
#include "paged_internal.h"

namespace mukv {

template <typename T>
__device__ __forceinline__ float piece_get(const raw16 &x, int e) {
    if constexpr (sizeof(T) == 4)
        return __uint_as_float(x[e]);
    else
        return __uint_as_float(e & 1 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16);
}
template <typename T>
__device__ __forceinline__ void piece_put(raw16 &x, int e, float y0, float y1) { // elements e, e + 1
    if constexpr (sizeof(T) == 4) {
        x[e] = __float_as_uint(y0);
        x[e + 1] = __float_as_uint(y1);
    } else {
        x[e / 2] = bf16_pair(y0, y1);
    }
}

// Past the caches: what is written here is read by other launches, on other XCDs (1568 tokens, 28/4 heads of 128: 7.6 us a launch, 8.8
// without; 24 prompts of 64/8 heads, 0.45 GB: 90, 95).
__device__ __forceinline__ void put_piece(unsigned char *p, raw16 x) { __builtin_nontemporal_store(x, reinterpret_cast<raw16 *>(p)); }

// Cosine and sine of pair p of a token.
__device__ __forceinline__ float2 turn_of(const RopeArgs &a, int token, int p) {
    // (up to three axes: all positions of the token, so that nothing waits for which one it is)
    const int ax = a.axis ? a.axis[p] : 0;
    const int32_t *at = a.positions + token;
    int pos = at[0];
    if (a.n_axes <= 3) {
        const int second = a.n_axes > 1 ? at[a.n_tokens] : 0, third = a.n_axes > 2 ? at[2 * (int64_t)a.n_tokens] : 0;
        pos = ax == 0 ? pos : ax == 1 ? second : ax == 2 ? third : 0;
    } else {
        pos = (unsigned)ax < (unsigned)a.n_axes ? at[(int64_t)ax * a.n_tokens] : 0;
    }
    double turns = (double)pos * a.inv_freq[p] * 0.15915494309189533577; // 1 / 2 pi
    turns -= rint(turns);
    float s, c;
    sincospif((float)(2.0 * turns), &s, &c);
    return float2{c, a.inverse ? -s : s};
}

} // namespace mukv
