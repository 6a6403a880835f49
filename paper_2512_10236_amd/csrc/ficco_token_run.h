// Which tokens a workgroup of the balance kernels has. Plain C++, so that the host can go through the whole range of sizes. Not installed.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define FICCO_TOKEN_RUN_FN static __host__ __device__ __forceinline__
#else
#define FICCO_TOKEN_RUN_FN static inline
#endif

namespace ficco {

// Tokens [begin, end). There may be 2^31 - 1 of them, and a thread steps past its run's end (and starts behind it, in a run of
// none), so that a token's number has 64 bits everywhere.
struct TokenRun {
    int32_t group;
    int64_t begin, end;
};

// Chunk c: the (c % per_group)-th run of chunk_tokens tokens of group c / per_group; what is behind the group's or the last token is not there.
FICCO_TOKEN_RUN_FN TokenRun token_run(int32_t chunk, int32_t per_group, int32_t chunk_tokens, int32_t group_tokens, int32_t tokens)
{
    const int32_t group = chunk / per_group;
    const int64_t group_end = (int64_t)(group + 1) * group_tokens, last = group_end < tokens ? group_end : tokens;
    const int64_t b = (int64_t)group * group_tokens + (int64_t)(chunk % per_group) * chunk_tokens, e = b + chunk_tokens;
    const int64_t begin = b < last ? b : last;
    return {group, begin, e < last ? e : last};
}

}  // namespace ficco
