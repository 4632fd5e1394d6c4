// tile_order.h -- in which order the XCDs take a grouped GEMM's tiles (find_tile of
// moe_prefill.hip).
#pragma once

namespace moe {

// Narrow matrices are one list of the experts' tiles, an eighth of it for each XCD,
// so that most experts' weights and token rows are read through one L2 (dealt in
// groups of eight feature tiles every XCD reads every expert's: 32 experts of d 512, f
// 4096, 4000 tokens, down 149 us against 103; 16 of d 1024, f 4096, 1900 tokens, 112
// against 98).  Of wider ones the XCDs stay with one expert at a time (8 experts of d
// 2048, f 8192, 4000 tokens, down 304 us against 354 from a list).  Whole layer, 8
// experts, top-2, d 256, f 512, 32768 tokens: 505 us with tile ft on XCD ft % 8, now 335.
constexpr int kNarrow = 2048;          // features

// The same on the small tiles of e4m3 weights, where an expert's weights are half of
// the bytes and its tiles fewer: a list up to here (groups -> list; plain products, 4096
// to 2304 features, 300 tokens 23.8 -> 22.3 us, 1000 tokens 39.9 -> 34.0; whole layers, 4
// experts of d 2304, f 1152, top-2, 2000 tokens 113 -> 108; 32 of d 2048, f 4096, top-4,
// 1000 tokens, 305 -> 299; 16 of d 6144, f 10752, top-4, 700 tokens 1264 -> 1247, but 4 of the
// 16 326 -> 336).  Gate and up of 8192 and more packed features in a list too: 200 tokens
// through the 16 experts 626 -> 644, 4 of them 179 -> 185; 8 of d 2048, f 8192, top-2, 300
// tokens 140 -> 146.
constexpr int kNarrowSmallE4m3 = 8192;

constexpr bool one_list(int features, bool small_e4m3)
{
    return features < (small_e4m3 ? kNarrowSmallE4m3 : kNarrow);
}

}  // namespace moe
