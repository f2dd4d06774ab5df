// The keys that the rows of a request see in windowed attention, as a list of tiles of 64 positions. The
// host sizes splits and workspace by the longest list, the kernels walk it; one definition for both.
#pragma once
#ifndef __HIP__
#define __device__
#define __host__
#endif

namespace sv {

constexpr int kWindowTile = 64;

struct KeyList {
    int ns;  // tiles 0 .. ns-1 hold the first positions
    int ft;  // then tiles from ft on
    int nt;  // tiles in all
};

// k >= 1 rows after L >= 0 committed positions; window >= 1, sinks >= 0
__device__ __host__ inline KeyList key_list(int window, int sinks, int L, int k) {
    const int first = L - window + 1 > 0 ? L - window + 1 : 0;  // of the first row's window
    const int head = sinks < first ? sinks : first;
    const int ns = (int)(((unsigned)head + kWindowTile - 1) / kWindowTile);
    const int ft = first / kWindowTile > ns ? first / kWindowTile : ns;
    return KeyList{ns, ft, ns + (L + k - 1) / kWindowTile - ft + 1};
}
__device__ __host__ inline int list_tile(const KeyList& x, int t) { return t < x.ns ? t : x.ft + (t - x.ns); }

// the most tiles of any list with k <= block rows and L + k <= max_kv_len positions: those of the first positions,
// and of span = window + block - 1 positions that may begin at a tile's end; and no more than all positions have
__host__ inline long long longest_list(int window, int sinks, int block, int max_kv_len) {
    constexpr long long T = kWindowTile;
    const long long all = (max_kv_len + T - 1) / T;
    const long long span = (long long)window + block - 1;
    const long long most = (sinks + T - 1) / T + (span + T - 2) / T + 1;
    return most < all ? most : all;
}

}  // namespace sv
