// Prints plan_window's choice for descriptors read from stdin, one per line:
//   R block Hq Hkv d f32 max_kv_len window sinks kv_split  ->  waves block_rows row_blocks splits split_tiles by_rows few
#include <cstdio>

#include "sv_host.h"

int main() {
    sv_window_desc w{};
    sv_attn_desc& d = w.attn;
    int f32;
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d", &d.num_reqs, &d.block, &d.num_q_heads, &d.num_kv_heads, &d.head_dim,
                      &f32, &d.max_kv_len, &w.window, &w.sinks, &d.kv_split) == 10) {
        d.dtype = f32 ? SV_F32 : SV_BF16;
        d.total_q_max = d.num_reqs * d.block;
        d.page_size = 16;
        d.max_pages_per_req = (d.max_kv_len + 15) / 16;
        d.num_pages = 10;
        if (sv::check_window(&w) != SV_OK) {
            std::fprintf(stderr, "refused: %s\n", sv::last_error());
            return 1;
        }
        const sv::WindowPlan p = sv::plan_window(w);
        std::printf("%d %d %d %d %d %d %d\n", p.waves, p.block_rows, p.row_blocks, p.splits, p.split_tiles, p.by_rows, p.few);
    }
    return 0;
}
