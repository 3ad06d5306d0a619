// Which kernels a call of attention takes: rules on its sizes alone, on the host.
#pragma once

#include <algorithm>
#include <cstdint>

namespace heddle {
namespace attn {

struct Sizes {
    int64_t sequences, q_rows, k_rows;        // rows of all sequences; sequences >= 1
    int32_t heads, kv_heads;
};

// split: split_kernel, 32 rows of a key head a workgroup and the keys divided over `parts`; else forward_kernel of `rows` rows
struct ForwardPlan {
    bool split;
    int rows, parts;
};
inline ForwardPlan plan_forward(const Sizes &z)
{
    // rows of a key head in a sequence, on average
    const int64_t n = z.sequences, rows = std::max<int64_t>(1, z.q_rows * (z.heads / z.kv_heads) / n), keys = z.k_rows / n;
    // Whether the keys are divided over workgroups, by an estimate in us of both kernels. Measured, 8 sequences of 4000 keys, 32
    // heads on 8: 2, 16, 32, 64 queries 27, 39, 59, 115 us divided, 83, 82, 84, 85 not; 32 of 200 keys, 16 queries: 18 and 14; one of
    // 16000 keys, 64 queries: 72 and 312; 2 of 600, 600 queries, 8 heads: 21.5 and 19.3.
    const double tiles128 = (double)n * ((rows + 127) / 128) * z.kv_heads, tiles32 = (double)n * ((rows + 31) / 32) * z.kv_heads;
    if (8 + 0.0125 * keys * std::max(1.0, tiles32 / 256) < 2 + 0.0205 * keys * std::max(1.0, tiles128 / 360)) {
        const int64_t used = std::max<int64_t>(1, n * ((rows + 31) / 32) * z.kv_heads);
        // One workgroup a CU at a time. Two rounds of them where there are many anyway: the sequences' lengths differ (32 of up
        // to 8192 keys, 8 key heads: 126 us, 142 with one part each); one round else (8 of up to 4000: 23.5 us, 26.5 with twice the parts).
        return {true, 32, (int)std::max<int64_t>(1, std::min<int64_t>({(used >= 128 ? 512 : 256) / used, keys / 128, 64}))};
    }
    // 256 rows a workgroup read each tile of keys half as often as 128, but want two rounds of workgroups (2 sequences of 2048, 32
    // heads: 88 us with 256 rows, 111 with 128; one of 2000, 8 heads: 64 and 50; 3 of 333, 12 heads: 18 and 15)
    return {false, rows >= 512 && n * ((rows + 255) / 256) * z.kv_heads >= 512 ? 256 : 128, 1};
}

// Keys a workgroup of dk and dv takes: 32 (few_keys_kernel) where there would not be one of 128 keys for every CU (one sequence of 2000,
// 8 heads: 54 us, 66 with pairs of 128); pairs of 128 where that leaves few rounds (4 of 2048, 64 heads on 8: 563 us, 603 with 128; 4 of 1000, 32 heads: 91 and 87).
inline int plan_keys(const Sizes &z)
{
    const int64_t keys = std::max<int64_t>(1, z.k_rows / z.sequences), singles = z.sequences * ((keys + 127) / 128) * z.kv_heads;
    return singles < 256 ? 32 : singles < 1024 && keys >= 512 ? 256 : 128;
}

}  // namespace attn
}  // namespace heddle
