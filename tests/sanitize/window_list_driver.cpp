// Drives the key list of windowed attention (csrc/window_list.h) and the plan made for it (sv_host.cpp) on the
// host, under AddressSanitizer and UndefinedBehaviorSanitizer without recovery: the list holds every
// key that a row sees exactly once, no list is longer than the host's bound, and splits and workspace
// cover the longest.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "sv_host.h"
#include "window_list.h"

namespace {

void expect(bool ok, const char* what, long long a, long long b, long long c, long long d) {
    if (!ok) {
        std::fprintf(stderr, "FAILED: %s (%lld, %lld, %lld, %lld)\n", what, a, b, c, d);
        std::exit(2);
    }
}

uint64_t g_state = 0x9E3779B97F4A7C15ull;
uint64_t next_u64() {  // splitmix64
    uint64_t z = (g_state += 0x9E3779B97F4A7C15ull);
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

long lists = 0;

void check_list(int W, int S, int block, int L, int k) {
    const sv::KeyList x = sv::key_list(W, S, L, k);
    const int n = L + k;
    expect(x.nt >= 1 && x.ns >= 0 && x.ns <= x.nt, "sizes", W, S, L, k);
    for (int max_kv : {n, n + 1, n + 100, 1 << 22})
        expect(x.nt <= sv::longest_list(W, S, block, max_kv), "the host's bound", W, S, L, k);
    int before = -1;
    for (int t = 0; t < x.nt; t++) {
        const int tile = sv::list_tile(x, t);
        expect(tile > before && tile * 64 < n, "tiles ascend and begin inside the request", W, S, L, k);
        // every tile between two of the list holds nothing that a row sees
        for (long long s = (before + 1) * 64LL; s < tile * 64LL; s++)
            expect(s >= S && s <= (long long)L - W, "a key that is left out", W, S, s, L);
        before = tile;
    }
    expect(n <= (before + 1) * 64, "the last row's own key", W, S, L, k);
    lists++;
}

}  // namespace

int main() {
    const int windows[] = {1, 2, 3, 15, 16, 48, 49, 50, 63, 64, 65, 66, 100, 127, 128, 129, 1000, INT_MAX - 1, INT_MAX};
    const int sinks[] = {0, 1, 4, 63, 64, 65, 100, 128, 129, 500, INT_MAX - 1, INT_MAX};
    for (int W : windows)
        for (int S : sinks)
            for (int L = 0; L < 420; L++)
                for (int k : {1, 2, 5, 16}) check_list(W, S, k == 5 ? 8 : k, L, k);
    for (int n = 0; n < 20000; n++) {
        const int W = 1 + (int)(next_u64() % 9000), S = (int)(next_u64() % 400), block = 1 + (int)(next_u64() % 16);
        check_list(W, S, block, (int)(next_u64() % 30000), 1 + (int)(next_u64() % block));
    }
    long plans = 0;
    for (int n = 0; n < 20000; n++) {
        sv_window_desc w{};
        sv_attn_desc& d = w.attn;
        d.num_reqs = 1 + (int)(next_u64() % 300);
        d.block = 1 + (int)(next_u64() % 16);
        d.total_q_max = 1 + (int)(next_u64() % (d.num_reqs * d.block));
        d.num_kv_heads = 1 + (int)(next_u64() % 9);
        d.num_q_heads = d.num_kv_heads * (1 + (int)(next_u64() % 64));
        d.head_dim = n % 2 ? 64 : 128;
        d.page_size = 1 << (next_u64() % 9);
        d.max_kv_len = 1 + (int)(next_u64() % (n % 5 ? 20000 : 1 << 22));
        d.max_pages_per_req = (d.max_kv_len + d.page_size - 1) / d.page_size;
        d.num_pages = 10;
        d.dtype = n % 7 ? SV_BF16 : SV_F32;
        d.kv_split = n % 3 ? 0 : 64 * (int)(next_u64() % 100);
        w.window = n % 11 ? 1 + (int)(next_u64() % 9000) : INT_MAX;
        w.sinks = n % 13 ? (int)(next_u64() % 200) : INT_MAX;
        if (sv::check_window(&w) != SV_OK) continue;
        plans++;
        const sv::WindowPlan p = sv::plan_window(w);
        const long long most = sv::longest_list(w.window, w.sinks, d.block, d.max_kv_len);
        expect(p.splits >= 1 && p.split_tiles >= 1 && (long long)p.splits * p.split_tiles >= most &&
                   (p.splits - 1LL) * p.split_tiles < most,
               "splits cover the longest list, none is empty", p.splits, p.split_tiles, most, n);
        const long long rows = (long long)(d.num_q_heads / d.num_kv_heads) * d.block;
        expect((long long)p.row_blocks * p.block_rows >= rows, "row blocks", p.row_blocks, p.block_rows, rows, n);
        expect(d.dtype == SV_F32 || p.block_rows == 32 * p.waves, "rows of a block", p.block_rows, p.waves, n, 0);
        const size_t parts = (size_t)p.splits * d.total_q_max * d.num_q_heads;
        if (p.splits > 1)
            expect(p.part_o_bytes >= parts * d.head_dim * 4 && p.ws_bytes >= p.part_o_bytes + parts * 4 &&
                       p.part_o_bytes % 16 == 0,
                   "workspace", p.splits, d.total_q_max, n, 0);
    }
    expect(plans > 5000, "plans", plans, 0, 0, 0);
    std::printf("ok: %ld lists, %ld plans\n", lists, plans);
    return 0;
}
