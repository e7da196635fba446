// How many CTAs share a tile of the 8-bit product (host code without CUDA, so that it can be tested anywhere).
#pragma once
#include <cstddef>
#include <cstdint>

namespace sqnn {

// CTAs with tensor memory that fit on an SM: 228 KB, of which a CTA takes 1 KB and its static variables besides, and 512 columns.
constexpr uint32_t ctas_per_sm(size_t smem, uint32_t tmem_cols)
{
    const uint32_t by_smem = (uint32_t)(228 * 1024 / (smem + 1536)), by_tmem = 512 / tmem_cols;
    return by_smem < by_tmem ? by_smem : by_tmem;
}

// Clusters that run at once.  The runtime was seen to count one CTA with tensor memory per SM where shared and tensor memory allow more; if it
// counts more of them, `counted`, its number already has them in it.
constexpr uint32_t clusters_at_once(uint32_t runtime_says, uint32_t cluster, uint32_t sms, uint32_t per_sm)
{
    const uint32_t counted = (runtime_says * cluster + sms - 1) / sms;
    return counted < per_sm && counted > 0 ? runtime_says * per_sm / counted : runtime_says;
}

// CTAs (or pairs) per tile: enough for `wanted` of them in all, as far as all clusters run at once (a second wave costs more than the split
// gains: 4096 x 9216 batch 64 by clusters of four, 128 CTAs, 12.7 us; of six and eight, in two waves, 19 and 25).
template <typename F>
uint32_t split_for(uint32_t tiles, uint32_t wanted, uint32_t most, const F &at_once)
{
    uint32_t split = 1;
    while (tiles * split < wanted && split < most && tiles <= at_once(split + 1)) ++split;
    return split;
}

}  // namespace sqnn
