// The walk and the order of a launch over packed prompts (prompt_walk.h) over plain
// arrays, for the CPU test.
#include "../../paper_2512_11221_amd/csrc/prompt_walk.h"

using namespace asrkf;

extern "C" {

// walk: 0 team, 1 split, 2 halves; returns the waves of a workgroup.
int prompt_choice(int bf16, int head_dim, int group, int n_kv_heads, const int32_t* len, int n, int* walk, int* rows) {
    const PromptWalk w = prompt_walk(bf16 != 0, head_dim, group, n_kv_heads, len, n);
    *walk = w.walk;
    *rows = w.rows();
    return w.waves;
}

// units: the unit of every place, for `blocks` blocks of one KV head; returns the fold.
int prompt_order(int bf16, int head_dim, int walk, int waves, int blocks, int n_kv_heads, int32_t* units) {
    const int fold = prompt_fold(PromptWalk{(Walk)walk, waves}, bf16 != 0, head_dim, blocks, n_kv_heads);
    for (int i = 0; i < blocks; ++i) units[i] = prompt_unit(i, fold, blocks);
    return fold;
}

int64_t prompt_max_tokens() { return kPromptTokens; }
int64_t prompt_max_stride() { return kMaxTokenStride; }
int prompt_max_tile() { return kPromptTileKeys; }

}  // extern "C"
