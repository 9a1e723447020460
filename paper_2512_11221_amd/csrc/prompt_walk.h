// How a launch over packed prompts goes about its rows (prompt.hip): which walk, and in
// what order its workgroups take their blocks.  Plain arithmetic on the host, apart from
// the kernel so that it is checked without a GPU.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define ASRKF_WALK_HD __host__ __device__
#else
#define ASRKF_WALK_HD
#endif

namespace asrkf {

// kTeam: a workgroup's waves take 32 rows each and share the tiles of keys, two buffers
// of them behind a barrier a tile.  kSplit: its waves take the same 32 rows and every
// fourth tile each, without a barrier, and their states are merged at the end.  kHalves:
// as kTeam, but two waves take the same 32 rows, with the first and the second half of
// every tile's keys, and their states are merged.
enum Walk { kTeam, kSplit, kHalves };

struct PromptWalk {
    Walk walk;
    int waves;              // of a workgroup
    int rows() const { return 32 * (walk == kSplit ? 1 : walk == kHalves ? waves / 2 : waves); }
};

// Keys of a tile in LDS, at most, and bytes from one token to the next of packed rows, at
// most: offsets within a tile are 32-bit.
constexpr int kPromptTileKeys = 128;
constexpr int64_t kMaxTokenStride = (int64_t)16 << 20;
static_assert(kPromptTileKeys * kMaxTokenStride <= (int64_t)1 << 31, "a tile's offsets, its last row included");

constexpr int kPromptSeqs = 128;           // sequences of a launch, whose table is a kernel argument
constexpr int kPromptStoreTokens = 16;     // tokens of a workgroup that writes rows into the cache

// Tokens of a launch over several packed prompts, at most, for the 2^32 threads of a grid.
// (A sequence has below 2^24 tokens: 2 GiB in 128-byte rows.)
constexpr int64_t kPromptTokens = (int64_t)1 << 24;
// Threads of a launch, at most: workgroups of 512, one for 256 query rows of a KV head
// (launches of fewer rows have below 2^12 units) and one for the store.
constexpr int64_t prompt_threads(int64_t tokens, int q_heads, int n_kv_heads) {
    return 512 * ((tokens * q_heads / 256 + kPromptSeqs * n_kv_heads) + (tokens / kPromptStoreTokens + kPromptSeqs));
}
static_assert(prompt_threads(kPromptTokens, 64, 32) < (int64_t)1 << 32, "the grid of the longest launch");

// waves of a SIMD that the registers leave room for
constexpr int prompt_waves(bool bf16, int head_dim, int waves, Walk walk) {
    const int row = head_dim * (bf16 ? 2 : 4);
    return waves == 8 || row < 256 || (walk == kTeam && row == 256) ? 2 : 1;
}

// Which walk, by the launch's work: units of 32 rows of a KV head.  The times are of one
// run over every walk, in us; heads are query / KV heads, of 128 where not said.
//  kSplit  with so few units that they leave compute units idle, a unit's keys are split
//          over four waves.  bf16 rows of 128 up to 256 units (1024 tokens of 8/8 heads:
//          18.9, in halves 24.6; 512 units, 512 tokens of 32/8: 21.9 and 17.7), rows of 64,
//          two workgroups a CU, up to 1024 (2048 tokens of 16/2: 25.6 and 26.6; 2500: 31.8
//          and 31.5); fp32 rows, whose products take 16 times as long, up to 1024 (700
//          tokens of 32/8: 72 and 99; 1100: 142 and 153, past the limit; 2000: 383 and
//          295).  Rows of 256 bf16 have no registers left for it, nor for halves.
//  kHalves where the launch would wait for the longest workgroup of four waves, alone on its
//          CU: prompts of 512 tokens or more with that workgroup's tiles 1.2 times the mean of
//          a CU's (32/8 heads: 1024 tokens 27.0, with four waves 31.1; 1280: 31.8 and 39.6;
//          1536: 37.8 and 45.2; 2048: 59.0 and 58.3; two prompts of 512: 19.1 and 20.5; of
//          1024: 42.8 and 36.6; four of 375: 25.5 and 22.6).  fp32 rows, whose products hide
//          the merge, always (2000 tokens of 32/8: 295, with eight waves 501; 4000: 1059
//          and 1053).
//  kTeam   four waves until every CU has its eight at least twice over, then eight, which
//          read a tile once for 256 rows (32/8 heads: 2048 tokens 58.3 with four, 67.9 with
//          eight; 4096 tokens 181 and 168).  The limit knows the units alone and is not the
//          best one for every batch: four prompts of 1024, past it, take 64 with four and
//          70 with eight, and rows of 256, with one workgroup of four waves on a CU, are
//          faster with eight well below it (16/8 heads: one prompt of 2048 110 and 117, two
//          142 and 122, five of 700 72 and 50; 1000 to 4000 tokens, past it, 447 and 313).
inline PromptWalk prompt_walk(bool bf16, int head_dim, int group, int n_kv_heads, const int32_t* len, int n) {
    int64_t units = 0, pairs = 0;
    int longest = 0;
    for (int i = 0; i < n; ++i) {
        units += ((int64_t)len[i] * group + 31) / 32 * n_kv_heads;
        pairs += (int64_t)len[i] * (len[i] + 64);
        longest = len[i] > longest ? len[i] : longest;
    }
    if (!(bf16 && head_dim == 256) && units <= (bf16 && head_dim == 128 ? 256 : 1024)) return {kSplit, 4};
    if (units >= 4096) return {kTeam, 8};
    if (!bf16) return {kHalves, 8};
    // workgroups of 128 rows and tiles of 64 keys: longest / 64 against
    // pairs / 2 / 64 * Hq / 128 / 256 CUs
    if (head_dim < 256 && longest >= 512 && (int64_t)longest * 65536 * 5 > pairs * group * n_kv_heads * 6) return {kHalves, 8};
    return {kTeam, 4};
}

// The longest blocks come first.  Where every CU gets two workgroups at once, the second
// half goes the other way, so that a CU's two are a long and a short one: the units from
// here on are in reverse (two prompts of 1024, 32/8 heads of 128: 42 us without, 35 with).
// A CU with room for one takes its second when the first ends, the longest first then too:
// rows of 256, 16/8 heads, two prompts of 2048 191 us in reverse and 151 without, one of
// 4000 280 and 229, five of 700 75 and 72.
inline int prompt_fold(const PromptWalk& w, bool bf16, int head_dim, int blocks, int n_kv_heads) {
    constexpr int kCUs = 256;
    const int workgroups = blocks * n_kv_heads;
    const bool pairs = w.walk == kTeam && w.waves == 4 && prompt_waves(bf16, head_dim, w.waves, w.walk) >= 2;
    return pairs && workgroups > kCUs && workgroups <= 2 * kCUs ? blocks / 2 : blocks;
}

// The unit that the workgroups of place `unit` take, of `blocks` units.
ASRKF_WALK_HD inline int prompt_unit(int unit, int fold, int blocks) {
    return unit < fold ? unit : blocks - 1 - (unit - fold);
}

}  // namespace asrkf
