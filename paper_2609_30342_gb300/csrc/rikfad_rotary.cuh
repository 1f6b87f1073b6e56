// rikfad_rotary.cuh -- a token's position and the cosine and sine of its pairs, for
// the operators that turn heads.
#pragma once
#include <stdint.h>

namespace rikfad {

// positions: position_bytes (4 or 8) bytes each, NULL: start + token.
__device__ __forceinline__ int64_t token_position(const void *positions, int position_bytes, int64_t position_batch,
                                                  int64_t start, int64_t batch, int64_t token)
{
    if (positions == nullptr)
        return start + token;
    const int64_t k = batch * position_batch + token;
    return position_bytes == 4 ? (int64_t)static_cast<const int32_t *>(positions)[k] : static_cast<const int64_t *>(positions)[k];
}

// Cosine and sine of position times `turns` / 2^64 turns: the product's fraction of a
// turn in [-1/2, 1/2), in half turns for sincospi.
__device__ __forceinline__ float2 cosine_sine(int64_t position, uint64_t turns)
{
    const uint64_t turn = (uint64_t)position * turns;
    float c, s;
    sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &s, &c);
    return make_float2(c, s);
}

}  // namespace rikfad
