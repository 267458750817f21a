// psd_adjust_plan.hpp -- how adjusted logits are cut into workgroups (host; internal to libpsd).
#pragma once

namespace psd {

// A workgroup's stretch where there are many: 16 KB of bfloat16 or float32, four pieces a thread.
constexpr int adjust_stretch(bool bf16) { return bf16 ? 8192 : 4096; }
constexpr int adjust_short_stretch(bool bf16) { return adjust_stretch(bf16) / 4; }

// Workgroups: a long stretch and all rows of a sequence each, so that its text is counted once a stretch; fewer
// rows, then a short stretch, while there are fewer than kAdjustFill, three a CU.  us with 256, 512, 768, 1024 and 1536
// (bfloat16, V=128256, texts to 2048): 1 path of 16 sequences 21, 16, 14, 16, 20, of 8 15, 10, 13, 13, 14; 4 paths of 8 37, 24, 21, 23,
// 25, of 32 94, 93, 77, 77, 78; V=50257, 4 paths of 24 49, 35, 34, 34, 32.  Over 21 calls 512 is 1 % ahead in the mean and up to 21 %
// behind, the others are 16, 2 and 6 % behind.
struct AdjustCut {
    int seg, segments, per;
    long wgs(int B, int R) const { return (long)segments * B * ((R + per - 1) / per); }
};
constexpr long kAdjustFill = 768;
inline AdjustCut adjust_cut(int B, int R, int V, bool bf16) {
    AdjustCut c;
    c.seg = adjust_stretch(bf16);
    c.segments = (V + c.seg - 1) / c.seg;
    c.per = R;
    while (c.per > 1 && c.wgs(B, R) < kAdjustFill) c.per = (c.per + 1) / 2;
    if (c.per == 1 && c.wgs(B, R) < kAdjustFill) {
        c.seg = adjust_short_stretch(bf16);
        c.segments = (V + c.seg - 1) / c.seg;
    }
    return c;
}

}  // namespace psd
