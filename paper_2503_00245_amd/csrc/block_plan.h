// How rows of the block around a layer are dealt out, by sizes (internal; host only, so that a test can hold the tested sizes to every plan).
#pragma once

#include <algorithm>

namespace moe {

// Waves that share a row, chunks of 512 values that one of them holds.  Rows of more than 4096 values: eight waves with two chunks have twice the registers
// of sixteen with one (us, 16 x 1 / 8 x 2, 16384 rows of 8192: bf16 forward 276 / 225, back 395 / 374, fp32 back 1291 / 697; 3000 of 5120 45 / 34 and 60 / 61).
// Two chunks of fp32 are too many to keep beside the next row's (back 882 so).
struct RowPlan {
    int waves, chunks;
};
inline RowPlan row_plan(int d) {
    const int chunks = (d + 511) / 512;
    return chunks <= 4 ? RowPlan{chunks, 1} : chunks <= 16 ? RowPlan{8, (chunks + 7) / 8} : RowPlan{16, (chunks + 15) / 16};
}
inline int row_groups(int T, int d) { return row_plan(d).waves == 1 ? (T + 3) / 4 : T; }  // workgroups that have a row at all
// Most workgroups of a pass.  Forward: 16384 rows of 2048, dropout, 1024 / 2048 / 4096 / 16384 of them 58.7 / 62.0 / 55.1 / 57.3 us.  Backward, four
// waves of 132 registers each: 256 / 512 / 768 / 1024 of them 151 / 95.5 / 86 / 91 us; as many waves of narrower rows.  Of eight waves and more a CU holds one
// workgroup: 256 of them (4096 rows of 4096 384 / 256 of them 72 / 58 us; 1024 of 16384, 16 waves, 192 / 256 124 / 112, 512 of
// 32768 254 / 282 in bf16 and 445 / 406 in fp32).
constexpr int kGroups = 4096, kGradWaves = 12 * 256;
inline int most_grad_groups(int d) {
    const int waves = row_plan(d).waves;
    return waves > 4 ? 256 : kGradWaves / (waves == 1 ? 4 : waves);
}
inline int grad_groups(int T, int d) { return std::min(most_grad_groups(d), row_groups(T, d)); }

}  // namespace moe
