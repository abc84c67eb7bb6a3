// Among how many tokens a workgroup of an append looks for the beginning of runs (kv_cache.hip, kv_rotary.hip): a rule on the host, by sizes alone.
#pragma once
#include <cstdint>

namespace abft {

constexpr int kAppendHeads = 2;    // of a workgroup
constexpr int kMaxWindow = 64;

// A workgroup looks for runs among so many tokens: few, so that single tokens do not wait for each other, while that makes up to 2048
// workgroups; of more tokens most lie inside runs, and the workgroups that find none would hold up the others (us, 1 / 2 / 4 / 8 /
// 16 tokens: 6000 of one request 94 / 86 / 30 / 16 / 11, 64 single tokens 4.2 / 4.8 / 7.3 / 11.8 / 21, 1169 of 40 requests 8.8 / 8.2 / 8.7 /
// 10.6 / 12.6).
inline int append_window(int64_t n_tokens, int heads, int64_t groups = 2048, int most = 16) {
    const int64_t all = n_tokens * ((heads + kAppendHeads - 1) / kAppendHeads);
    int window = 1;
    while (window < most && all > groups * window) window *= 2;
    return window;
}
// Of a prompt in blocks of 32 and more, few tokens begin a run, and workgroups that find none cost more here than for an append, since they need more
// registers: windows up to a block, of fewer workgroups.  Blocks of 16 have runs enough for the appends' rule.  (us, windows of 4 / 8 / 16 / 32 / 64 tokens:
// 2000 of one request, 8 heads of 128, blocks of 64 23.5 / 14.6 / 12.9 / 12.2 / 11.9, 400 runs of 5 28.6 / 28.0 / 27.7 / 37.9 / 65.3; 1458 of one request,
// 16 heads of 32, blocks of 32 22.3 / 21.6 / 23.7 / 18.7 / 18.5; 6000 in blocks of 16 49.1 / 34.3 / 30.2 / 27.8 / 27.7, 1722 of 40 requests the kernel
// alone 10.4 / - / 14.1 / - / -.)
inline int rotary_window(int64_t n_tokens, int heads, int block) {
    return append_window(n_tokens, heads, block > 16 ? 512 : 2048, block < kMaxWindow ? block : kMaxWindow);
}

}  // namespace abft
