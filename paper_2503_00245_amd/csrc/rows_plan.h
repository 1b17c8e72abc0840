// Which forms the kernels between tokens and experts' rows take, by sizes (internal; host only but for the constants, so that a test can hold the tested
// sizes to every one of them).
#pragma once

#include <algorithm>

namespace moe {

// ---- counting the pairs of each expert (dispatch_kernel)
// Pairs up to which every workgroup counts all keys itself, and counting needs no launch of its own (us, so / with that launch: 96 pairs of 16 experts
// 5.6 / 8.1, 2048 pairs of 8 6.8 / 8.8, 4096 of 8 10.0 / 10.7, of 64 8.2 / 11.8, 8192 of 64 11.6 / 14.0, of 8 15.2 / 13.9, 16384 of 8 20.2 / 14.3)
constexpr int kKeysAlone = 8192;
// Experts up to which it does so by ballots: LDS additions of a wave to one address come one after the other (8192 pairs, us, with them / by ballots: one expert
// 28.5 / 9.1, two 18.3 / 10.6, eight 15.2 / 23.3)
constexpr int kBallotExperts = 4;
constexpr int kMaxCounts = 16384;  // counts that a workgroup adds up beyond

enum DispatchCount { COUNT_BALLOTS, COUNT_ADDS, COUNT_LAUNCH };
inline DispatchCount dispatch_count(long long P, int E) { return P > kKeysAlone ? COUNT_LAUNCH : E <= kBallotExperts ? COUNT_BALLOTS : COUNT_ADDS; }

// Chunks of whole tokens: about two workgroups a CU, no more chunks than their counts may be
struct DispatchPlan {
    int tokens;  // of a chunk
    int chunks;
};
inline DispatchPlan dispatch_plan(long long T, int E) {
    const long long most = std::min(512, kMaxCounts / E);
    const long long tokens = std::max<long long>(4, (T + most - 1) / most);
    return DispatchPlan{(int)tokens, (int)((T + tokens - 1) / tokens)};
}

// ---- rows to tokens and tokens to rows (collect_kernel, spread_kernel)
// A wave for every 512 values, up to four (us, one wave / four / so: collect of 16384 tokens of 432, two experts, 7.8 / 9.6 / 7.8, 2048 of 2048 4.8 / 4.1 / 4.2;
// its gradient at 16384 of 2048 68.0 / 65.0 / 62.8, 8192 of 1024 14.4 / 15.6 / 14.7, 2048 of 720, eight experts, 11.5 / 13.6 / 10.4)
struct RowsForm {
    int waves;  // that share a token: 1, 2, 4
    int pairs;  // of a token, held in registers: 1, 2, 4, 8; 0: any number, their dot products in LDS
};
inline RowsForm rows_form(int d, int k) {
    return RowsForm{d <= 512 ? 1 : d <= 1024 ? 2 : 4, k == 1 ? 1 : k == 2 ? 2 : k <= 4 ? 4 : k <= 8 ? 8 : 0};
}

}  // namespace moe
