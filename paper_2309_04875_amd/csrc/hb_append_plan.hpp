// How appended tokens are shared out to workgroups and launches.  Whole numbers alone, for the host and the kernel.
#pragma once

#include <stdint.h>

namespace hb {

constexpr int kAppendBlock = 256;

// Workgroups of one kind (keys, values or queries) of a launch.
struct AppendShape {
    uint32_t blocks;
    uint32_t groups;            // of 2 N numbers of a token
    uint32_t per_token;         // workgroups of a token, or 0:
    uint32_t together;          // tokens of a workgroup
};

// groups: of a token's numbers of this kind.
constexpr AppendShape append_shape(uint64_t tokens, uint64_t groups)
{
    const uint64_t per = kAppendBlock;
    if (groups == 0) return AppendShape{};
    const uint64_t each = groups >= per ? (groups + per - 1) / per : 0, together = groups < per ? per / groups : 0;
    const uint64_t blocks = each != 0 ? tokens * each : (tokens + together - 1) / together;
    return AppendShape{(uint32_t)blocks, (uint32_t)groups, (uint32_t)each, (uint32_t)together};
}

// Tokens that one launch takes, for groups of a token's keys (and values) and of its queries: a grid has fewer than 2^32 threads, and what is more goes
// into further launches.
constexpr uint64_t append_launch_tokens(uint64_t stored, uint64_t asked)
{
    // workgroups of 256 tokens, rounded up; and one of each kind that is not full
    const uint64_t tokens = 256, of_each = append_shape(tokens, stored).blocks, of_queries = append_shape(tokens, asked).blocks;
    return (0xffffffffull / kAppendBlock - 3) / (2 * of_each + of_queries) * tokens;
}

}  // namespace hb
