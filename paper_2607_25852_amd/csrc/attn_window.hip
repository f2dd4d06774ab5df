// Attention with a sliding window and visible first tokens over the paged cache (sv_window_attn).
// The row at position p sees the keys s <= p with s < S or s > p - W:
//     z_s = scale <q, K_s>,  lse = ln sum exp(z_s),  o = sum exp(z_s - lse) V_s.
//
// The keys that any row of a request sees are a list of tiles: those of the first S positions, then
// those from the first row's window to the last row. Window and S are the host's, so the longest
// list is known there: a list may be divided into splits of whole tiles (partial results merged
// by a second kernel) without a plan on the device.
#include <algorithm>

#include "attn_tile.h"
#include "rows.h"
#include "sv_internal.h"
#include "window_list.h"

namespace sv {
namespace {

struct WindowArgs {
    const void* q;
    const void* kc;
    const void* vc;
    const int32_t* page_table;
    const int32_t* qo;
    const int32_t* kv_lens;
    void* out;
    float* lse;
    float* part_o;    // [splits, total_q, Hq, d], of the splits of divided lists
    float* part_lse;  // [splits, total_q, Hq], log2 domain
    int R, total_q, Hq, Hkv, G, block, HD;
    int log2P, maxp, num_pages, max_kv_len;
    int window, sinks;
    int splits, split_tiles;  // of every list; tiles per split
    int nrb, per_xcd;         // row blocks per (request, kv-head); (request, split, kv-head)s per XCD
    int by_rows;              // requests in the order of their rows (R <= 64)
    float scale, scale_log2;  // sm_scale, sm_scale * log2(e)
};

// the request's packing and key count; false: not sound
__device__ inline bool load_request(const WindowArgs& a, int i, int& q0, int& k_i, int& kv_len) {
    q0 = a.qo[i];
    k_i = a.qo[i + 1] - q0;
    kv_len = min(a.kv_lens[i], a.max_kv_len);
    return rows_in_batch(q0, k_i, a.block, a.total_q) && kv_len >= k_i;
}

template <typename T> struct Vec4;
template <> struct Vec4<float> {
    static __device__ f32x4 get(const float* p) { return *(const f32x4*)p; }
    static __device__ void put(float* p, f32x4 x) { *(f32x4*)p = x; }
};
template <> struct Vec4<uint16_t> {
    static __device__ f32x4 get(const uint16_t* p) {
        const uint2 w = *(const uint2*)p;
        return f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xFFFF0000u)};
    }
    static __device__ void put(uint16_t* p, f32x4 x) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = (__bf16)x[e];
        *(bf16x4*)p = v;
    }
};

// Whether any of keys s0 .. s1 is seen by some rows of a request (at positions L .. last) and not by others: a key behind
// the first row, or one that the first rows' windows begin with.
__device__ inline bool some_shared(const WindowArgs& a, int L, int last, int s0, int s1) {
    return (last > L) & (((s1 > L) & (s0 <= last)) | ((s1 > L - a.window) & (s0 <= last - a.window) & (s1 >= a.sinks)));
}
// There are at most 15 of either (a block has 16 rows). A value of theirs that is not finite must not meet the weights 0 of
// the rows that do not see it (0 * NaN is NaN), so it is taken for 0 and its key's bit set; the rows that do see it
// get it at the end. All other values that are not finite are seen by every row of the request, whose results they are.
// Against no such check at all: 4 requests of one token 14.8 and 14.1 us, 64 requests of up to 16 60.2 and 58.5 us; with a
// NaN in every request's last value 70 us (its rows computed again one by one: 28.5 ms).
static_assert(SV_MAX_BLOCK <= 16, "bits of the keys");
__device__ inline uint32_t shared_bit(const WindowArgs& a, int L, int s) {
    return 1u << (s > L ? s - L - 1 : 16 + s - (L - a.window + 1));
}
// infinity or NaN
__device__ inline bool odd(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }
__device__ inline bool odd(uint16_t x) { return (x & 0x7F80u) == 0x7F80u; }
// The values of the keys `bits` to the result of the row at position p, which is at out: to 4 dims each from d on, in steps
// of `step` below d1. Of bf16 values those that are not finite were taken for 0, of fp32 ones all. lse2 is the row's
// in the log2 domain. Rolled loops: this is cold, and unrolled it cost a call of a few microseconds half a microsecond.
template <typename T, typename O>
__device__ __forceinline__ void give_back(const WindowArgs& a, uint32_t bits, const T* q, O* out, const int32_t* pt, int h, int L,
                                          int p, float lse2, int d, int d1, int step) {
    for (; bits; bits &= bits - 1) {
        const int b = __builtin_ctz(bits), s = b < 16 ? L + 1 + b : L - a.window + 1 + (b - 16);
        if (s > p || (s >= a.sinks && s <= p - a.window)) continue;
        const int pg = pt[s >> a.log2P];
        if ((unsigned)pg >= (unsigned)a.num_pages) continue;
        const size_t off = ((((size_t)pg * a.Hkv + h) << a.log2P) + (s & ((1 << a.log2P) - 1))) * a.HD;
        float z = 0.0f;
#pragma unroll 1
        for (int e = 0; e < a.HD; e += 4) {
            const f32x4 x = Vec4<T>::get((const T*)a.kc + off + e), y = Vec4<T>::get(q + e);
            z += x[0] * y[0] + x[1] * y[1] + x[2] * y[2] + x[3] * y[3];
        }
        const float weight = exp2f(z * a.scale_log2 - lse2);
#pragma unroll 1
        for (int e = d; e < d1; e += step) {
            const f32x4 v = Vec4<T>::get((const T*)a.vc + off + e);
            f32x4 o = Vec4<O>::get(out + e);
#pragma unroll
            for (int c = 0; c < 4; c++)
                if (sizeof(T) == 4 || odd(v[c])) o[c] += weight * v[c];
            Vec4<O>::put(out + e, o);
        }
    }
}

// What a workgroup works on. Neighbouring workgroups go to the XCDs in turn. Each XCD takes a run of (request, split,
// kv-head)s, whose heads share pages, and the row blocks of one follow each other. With by_rows (blocks of up to 64
// requests) the requests with the most rows come first and are dealt to the XCDs in turn, so that all XCDs have as
// much to do and the last items are short ones. Requests of 1 to 16 positions, in their own order and by rows:
// 32 with windows of 32768 (512 items of 8 waves, 256 at a time) 630 and 584 us, 48 with windows of 4000
// (384 items, all at once) 183 and 157 us, 64 with windows of 1024 66.6 and 61.8 us.
struct Item {
    int i, h, sp, row0, M;  // request, kv-head, split, first row of the kv-head group, rows
    int q0, L, last;        // the request's first row; positions of its first and last row
    int t0, t1;
    KeyList list;
};
__device__ __forceinline__ bool find_item(const WindowArgs& a, int block_rows, Item& x) {
    // (the quotients of vector divisions, back in scalar registers: the copies' addresses need them there)
    auto scalar = [](unsigned v) { return __builtin_amdgcn_readfirstlane((int)v); };
    const unsigned slot = blockIdx.x / 8, xcd = blockIdx.x % 8;
    const int ux = scalar(slot / (unsigned)a.nrb), rb = scalar(slot % (unsigned)a.nrb);
    int is;
    if (a.by_rows) {
        is = scalar((unsigned)ux / (unsigned)a.Hkv * 8 + xcd);
        x.h = scalar((unsigned)ux % (unsigned)a.Hkv);
    } else {
        const unsigned unit = xcd * (unsigned)a.per_xcd + (unsigned)ux;
        is = scalar(unit / (unsigned)a.Hkv);
        x.h = scalar(unit % (unsigned)a.Hkv);
    }
    if (ux >= a.per_xcd || (unsigned)is >= (unsigned)a.R * (unsigned)a.splits) return false;
    x.sp = scalar((unsigned)is % (unsigned)a.splits);
    x.i = scalar((unsigned)is / (unsigned)a.splits);
    if (a.by_rows) {  // the x.i-th request by rows, descending (at most 64 requests: one per lane)
        const int lane = threadIdx.x & 63, k = lane < a.R ? a.qo[lane + 1] - a.qo[lane] : 0;
        int rank = 0;
        for (int j = 0; j < a.R; j++) {
            const int kj = __builtin_amdgcn_readlane(k, j);
            rank += (kj > k) | ((kj == k) & (j < lane));
        }
        x.i = (int)__builtin_ctzll(__ballot(lane < a.R && rank == x.i));
    }
    x.row0 = rb * block_rows;
    int k_i, kv_len;
    if (!load_request(a, x.i, x.q0, k_i, kv_len)) return false;
    x.M = min(a.G * k_i - x.row0, block_rows);
    if (x.M <= 0) return false;
    x.L = kv_len - k_i;
    x.last = kv_len - 1;
    x.list = key_list(a.window, a.sinks, x.L, k_i);
    x.t0 = x.sp * a.split_tiles;
    x.t1 = min(x.list.nt, x.t0 + a.split_tiles);
    return x.t0 < x.t1;
}

// ---------------------------------------------------------------------------------
// fp32 MFMA kernel
// ---------------------------------------------------------------------------------
// A workgroup of four waves takes one item of RG groups of 16 query rows; wave w has keys 16 w .. + 15 of every tile.
// v_mfma_f32_16x16x4_f32 multiplies and adds in fp32. Its k index is free as long as both operands agree, which
// lets every lane load 16 bytes at a time straight into the operands (lane = 16 q + n):
//   scores S^T = K Q^T: step (b, c) takes dim 16 b + 4 q + c of key n and of row n;
//   lane 16 q + n gets the scores of row n with keys 4 q + e, e = 0..3;
//   O^T = V^T P^T: step e takes key 4 q + e, so P^T is where the scores were left; tile (g, c) of the
//   output has dims 64 g + 4 n + c, and lane 16 q + n gets dims 64 g + 16 q + 4 e + c of row n.
// Keys that no row sees are not loaded. Bound by the latency of a tile's loads (page, K and V) and by the chain of
// its products (fp32 products run at a sixteenth of the bf16 rate). With two groups of rows (twice the
// products per load, half the waves) 8 requests of 5 positions and windows of 512 take 22.5 us, with one
// 19.8 us; they pay where one would take more rounds of workgroups (plan_window). With the next tile's keys loaded ahead 21.7 instead of 20.7 us, 32 requests 47 instead of 43 us.
// So what hides the latency is workgroups: the rows stay in LDS, which leaves room for three of them (147 registers) where
// rows in registers left two (45 requests 57 us, then 77 us). Four (128 registers) spill: 24 instead of 21 us.
template <int DG, int RG>
__global__ __launch_bounds__(256, DG * RG >= 4 ? 2 : 3) void window_f32_kernel(WindowArgs a) {
    constexpr int NW = 4, NB = 4 * DG;  // waves; 16-dim blocks of the scores' sum
    __shared__ union {
        f32x4 q[RG][NB][64];  // the rows, as every wave's lanes take them
        float o[NW][DG * 4][4][64];
    } u;
    __shared__ float s_ml[NW][2][64];
    __shared__ uint32_t s_odd;  // keys whose values were taken for 0 (shared_bit)
    Item x;
    if (!find_item(a, 16 * RG, x)) return;
    if (threadIdx.x == 0) s_odd = 0;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n = lane & 15, q = lane >> 4, HD = a.HD;
    const int32_t* __restrict__ pt = a.page_table + (size_t)x.i * a.maxp;
    // the page of this lane's key (n) of tile t; -1: no row sees it, or it does not exist
    auto page_of = [&](int t) {
        const int s = list_tile(x.list, t) * kTile + 16 * w + n, col = s >> a.log2P;
        const bool seen = (s <= x.last) & ((s < a.sinks) | (s > x.L - a.window)) & (col < a.maxp);
        const int pg = seen ? pt[col] : -1;
        return pg < a.num_pages ? pg : -1;
    };
    int pg = page_of(x.t0);
    // row n of group g: its place in the kv-head group
    auto row_of = [&](int g) { return x.row0 + (16 * g + n < x.M ? 16 * g + n : 0); };
    auto out_row = [&](int g) { return (size_t)(x.q0 + row_of(g) / a.G) * a.Hq + x.h * a.G + row_of(g) % a.G; };
    int p[RG];  // the rows' positions
#pragma unroll
    for (int g = 0; g < RG; g++) {
        p[g] = x.L + row_of(g) / a.G;
        const float* src = (const float*)a.q + out_row(g) * HD;
#pragma unroll
        for (int b = w; b < NB; b += NW) {
            const int d = 16 * b + 4 * q;
            u.q[g][b][lane] = 16 * g + n < x.M && d < HD ? *(const f32x4*)(src + d) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    __syncthreads();
    f32x4 o[RG][DG * 4];
    float m[RG], l[RG];
#pragma unroll
    for (int g = 0; g < RG; g++) {
#pragma unroll
        for (int d = 0; d < DG * 4; d++) o[g][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        m[g] = -INFINITY, l[g] = 0.0f;
    }
    for (int t = x.t0; t < x.t1; t++) {
        const int s0 = list_tile(x.list, t) * kTile + 16 * w;
        const int next = t + 1 < x.t1 ? page_of(t + 1) : -1;
        auto row_at = [&](int page, int key) {
            return ((((size_t)page * a.Hkv + x.h) << a.log2P) + ((s0 + key) & ((1 << a.log2P) - 1))) * HD;
        };
        f32x4 kf[NB], vf[4][DG];
        const float* kp = (const float*)a.kc + row_at(max(pg, 0), n);
#pragma unroll
        for (int b = 0; b < NB; b++) {
            const int d = 16 * b + 4 * q;
            kf[b] = pg >= 0 && d < HD ? *(const f32x4*)(kp + d) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
        int vpg[4];
        auto load_v = [&](unsigned gone) {  // gone: keys (by e) whose value is taken for 0
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float* vp = (const float*)a.vc + row_at(max(vpg[e], 0), 4 * q + e);
#pragma unroll
                for (int c = 0; c < DG; c++) {
                    const int d = 64 * c + 4 * n;
                    vf[e][c] = vpg[e] >= 0 && d < HD && !(gone >> e & 1) ? *(const f32x4*)(vp + d) : f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
        };
#pragma unroll
        for (int e = 0; e < 4; e++) vpg[e] = __shfl(pg, 4 * q + e, 64);
        load_v(0);
        const bool any = __any(pg >= 0);
        pg = next;
        if (!any) continue;
#pragma unroll
        for (int g = 0; g < RG; g++) {
            if (g > 0 && x.M <= 16 * g) break;
            f32x4 s = {0.f, 0.f, 0.f, 0.f}, s2 = s;  // two chains
#pragma unroll
            for (int b = 0; b < NB; b++) {
                const f32x4 qf = u.q[g][b][lane];
#pragma unroll
                for (int c = 0; c < 4; c += 2) {
                    s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[b][c], qf[c], s, 0, 0, 0);
                    s2 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[b][c + 1], qf[c + 1], s2, 0, 0, 0);
                }
            }
            // keys s0 + 4 q + e of row n
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int key = s0 + 4 * q + e;
                const bool ok = (vpg[e] >= 0) & (key <= p[g]) & ((key < a.sinks) | (key > p[g] - a.window));
                s[e] = ok ? (s[e] + s2[e]) * a.scale_log2 : -INFINITY;
                mx = fmaxf(mx, s[e]);
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_new = fmaxf(m[g], mx), ref = m_new == -INFINITY ? 0.0f : m_new;
            const float alpha = m[g] == -INFINITY ? (l[g] != 0.0f ? 1.0f : 0.0f) : exp2f(m[g] - m_new);
            m[g] = m_new;
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                s[e] = exp2f(s[e] - ref);
                sum += s[e];
            }
            l[g] = l[g] * alpha + sum;
            if (g == 0 && some_shared(a, x.L, x.last, s0, s0 + 15)) {
                unsigned gone = 0;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int key = s0 + 4 * q + e;
                    bool take = false;
#pragma unroll
                    for (int c = 0; c < DG; c++)
#pragma unroll
                        for (int y = 0; y < 4; y++) take |= odd(vf[e][c][y]);
                    take &= some_shared(a, x.L, x.last, key, key);
                    if ((__ballot(take) >> (16 * q) & 0xFFFF) != 0) {  // in any lane of the key
                        gone |= 1u << e;
                        if (n == 0) atomicOr(&s_odd, shared_bit(a, x.L, key));
                    }
                }
                // (loaded again rather than changed in place, which costs registers)
                if (__builtin_expect(__any(gone != 0), 0)) load_v(gone);
            }
#pragma unroll
            for (int d = 0; d < DG * 4; d++) o[g][d] *= alpha;
#pragma unroll
            for (int e = 0; e < 4; e++)
#pragma unroll
                for (int d = 0; d < DG * 4; d++)
                    o[g][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[e][d / 4][d % 4], s[e], o[g][d], 0, 0, 0);
        }
    }
    // merge the waves' states; wave w finishes every fourth block of 16 dims
    const bool whole = a.splits == 1 || x.t1 - x.t0 == x.list.nt;
#pragma unroll
    for (int g = 0; g < RG; g++) {
        if (g > 0 && x.M <= 16 * g) break;
        const bool row_ok = 16 * g + n < x.M;
        const size_t orow = out_row(g);
        l[g] += __shfl_xor(l[g], 16, 64);
        l[g] += __shfl_xor(l[g], 32, 64);
        __syncthreads();  // (the rows, or the states of the group before, are no longer read)
        s_ml[w][0][lane] = m[g];
        s_ml[w][1][lane] = l[g];
#pragma unroll
        for (int d = 0; d < DG * 4; d++)
#pragma unroll
            for (int e = 0; e < 4; e++) u.o[w][d][e][lane] = o[g][d][e];
        __syncthreads();
        float M = -INFINITY, lt = 0.0f, wt[NW];
#pragma unroll
        for (int y = 0; y < NW; y++) M = fmaxf(M, s_ml[y][0][lane]);
#pragma unroll
        for (int y = 0; y < NW; y++) {
            const float my = s_ml[y][0][lane], ly = s_ml[y][1][lane];
            // (a part whose scores are all NaN has no maximum, but its sum counts)
            wt[y] = my == -INFINITY ? (ly != 0.0f ? 1.0f : 0.0f) : exp2f(my - M);
            lt += ly * wt[y];
        }
        const float inv = 1.0f / lt;
        const size_t prow = (size_t)x.sp * a.total_q * a.Hq + orow;
        float* out = whole ? (float*)a.out + orow * HD : a.part_o + prow * HD;
        for (int y = w; y < DG * 4; y += NW) {  // dims 64 (y / 4) + 16 q + 4 (y % 4) + c
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 4; c++)
#pragma unroll
                for (int z = 0; z < NW; z++) v[c] += u.o[z][y / 4 * 4 + c][y % 4][lane] * wt[z];
            const int d = 64 * (y / 4) + 16 * q + 4 * (y % 4);
            if (row_ok && d < HD) *(f32x4*)(out + d) = lt == 0.0f ? f32x4{0.f, 0.f, 0.f, 0.f} : v * inv;
        }
        const float lse2 = lt == 0.0f ? -INFINITY : M + log2f(lt);
        if (__builtin_expect(s_odd != 0 && row_ok && lt != 0.0f, 0))
            give_back<float>(a, s_odd, (const float*)a.q + orow * HD, out, pt, x.h, x.L, p[g], lse2, 16 * q + 4 * w, HD, 64);
        if (w == 0 && q == 0 && row_ok) {
            if (!whole) a.part_lse[prow] = lse2;
            else if (a.lse) a.lse[orow] = lse2 * kLn2;
        }
    }
}

// ---------------------------------------------------------------------------------
// bf16 MFMA kernel
// ---------------------------------------------------------------------------------
// A workgroup of NW waves takes one (request, split, kv-head, row block): up to NW * 32 query rows of the
// kv-head group (row r: position j = r / G, head r % G) against the split's tiles of 64 keys. Where the rows
// fill half of the waves or less, two waves share 32 rows and take the halves of every tile
// (PARTS = 2), else a wave takes both halves; up to 32 rows are shared by all four waves, which take two tiles
// at a time (PARTS = 4). As in attn.hip, S^T = K Q^T puts
// the scores of a query row into one lane pair, and P^T is then in the operand layout of
// O^T = V^T P^T, with V read transposed from LDS. K and V tiles come through the page table into an LDS
// ring by direct loads while earlier tiles are multiplied; the parts of a row are merged at the end.
// The weights go to the second product as the sum of two bf16 numbers: the upper half of the fp32 weight's bits, and the
// rest rounded to bf16, which together are off by at most 2^-15 of the weight. V is read from LDS once for both, but has
// two products instead of one. With weights rounded to one bf16 number (off by up to 2^-8) the results are 0.0023 off
// (rms, relative, against 64 bits) instead of the 0.0017 that their own rounding costs; that form took 54.0 instead of 56.6 us for
// 64 requests with windows of 1024 and, where the products bound it (32 requests, windows of 32768), 465 instead of 575 us.
// Maximum, sum (of the fp32 weights) and outputs stay in fp32.
// Bound: 64 requests of 1 to 16 rows, 8 kv-heads of 128 dims, windows of 1024 (282 MB, two waves on 32 rows): 60 us,
// 4.7 TB/s, of which 6 us go by before the first tile is there (packing, page ids, first copies).
// 32 requests, 16 heads per kv-head, windows of 32768 (2.16 GB, waves with whole tiles): 550 to 585 us, 3.8 TB/s, the
// tile's dependent steps (LDS reads, exponents, and the products, 48 per wave, of which two share a matrix unit: 1.3 us of the 2 us of
// a tile). 4 requests of one row, windows of 1024 (17 MB, 5 splits): 12 us and 3 to 4 us of merge, all of it latency.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kPageSlots = 1024;  // page ids staged at a time

// How a tile's addresses are found: one page holds the whole tile, one page holds each 1 KB segment of
// it, or every lane looks its token's page up.
enum class Pages { kTile, kSegment, kLane };

template <int HD, int NW, int NBUF>
struct WindowLds {
    union {
        struct {
            uint16_t k[NBUF][kTile * HD];  // [buffer][token * HD + d], swizzled (attn_tile.h)
            uint16_t v[NBUF][kTile * HD];
        };
        float park[NW * HD * 32];  // the waves' partial outputs
    };
    float ml[NW][2][64];
    int32_t pid[kPageSlots];
    int32_t holes;  // a page that the list needs is missing
    uint32_t odd;   // keys with values that were taken for 0 (shared_bit)
};

// wait until at most min(newer, MAX) tiles of IPW loads each are outstanding
template <int MAX, int IPW>
__device__ inline void wait_tiles(int newer) {
    if constexpr (MAX == 0) {
        wait_vm<0>();
    } else {
        if (newer >= MAX) wait_vm<MAX * IPW>();
        else wait_tiles<MAX - 1, IPW>(newer);
    }
}

// One item, its waves divided into row groups of PARTS waves
template <int HD, int NW, int NBUF, Pages PM, int PARTS>
__device__ __forceinline__ void window_item(const WindowArgs& a, WindowLds<HD, NW, NBUF>& lds, const Item& x) {
    const int i = x.i, h = x.h, sp = x.sp, row0 = x.row0, q0 = x.q0, L = x.L, M = x.M, last = x.last, t0 = x.t0, t1 = x.t1;
    const KeyList list = x.list;
    constexpr int CPR = HD / 8;             // 16-byte chunks per token row
    constexpr int TPS = 1024 / (HD * 2);    // tokens per 1 KB DMA segment
    constexpr int NSEG = kTile / TPS;       // segments per tensor per tile
    constexpr int IPW = 2 * NSEG / NW;      // DMA instructions per wave per tile
    static_assert(IPW * NW == 2 * NSEG && (NSEG % IPW) == 0, "DMA split: a wave moves one tensor");
    constexpr int KK = HD / 16;             // MFMA k-steps over the head dim
    constexpr int DT = HD / 32;             // output d-tiles
    constexpr int log2T64 = 6;
    static_assert(kTile == 1 << log2T64 && kTile == kWindowTile, "tile");
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int32_t* __restrict__ pt = a.page_table + (size_t)i * a.maxp;
    const int log2S = min(a.log2P, log2T64), log2T = log2T64 - log2S;  // tokens per page slot, slots per tile
    const int chunk_tiles = kPageSlots >> log2T;
    // page ids of tiles c0 .. c1-1 into LDS; a missing page is flagged where a row sees the slot
    auto stage = [&](int c0, int c1) {
        bool hole = false;
        for (int e = tid; e < (c1 - c0) << log2T; e += NW * 64) {
            const int s = list_tile(list, c0 + (e >> log2T)) * kTile + ((e & ((1 << log2T) - 1)) << log2S);
            const int col = s >> a.log2P, pg = col < a.maxp ? pt[col] : -1;
            const bool ok = pg >= 0 && pg < a.num_pages;
            hole |= !ok && s <= last && (s < a.sinks || s + (1 << log2S) > L - a.window + 1);
            lds.pid[e] = ok ? pg : -1;
        }
        if (hole) lds.holes = 1;
    };
    if (tid == 0) lds.holes = 0, lds.odd = 0;

    const int rg = w / PARTS, th = w % PARTS;
    // with PARTS = 4 a step takes two tiles: the wave's tile of the step, and its half of that tile
    constexpr int STEP = PARTS == 4 ? 2 : 1;
    static_assert(NBUF % STEP == 0, "the tiles of a step are neighbours in the ring");
    const int dt = PARTS == 4 ? th >> 1 : 0, hh = PARTS == 4 ? th & 1 : th;
    const int r = rg * 32 + (lane & 31), half = lane >> 5;
    const bool row_ok = r < M;
    const int rr = row0 + (row_ok ? r : 0);  // row within the request's kv-head group
    const int jq = rr / a.G, head = h * a.G + rr % a.G;
    const int p = L + jq;  // the row's position

    // per-lane byte offsets of the V^T transpose reads (attn.hip)
    int vofs[2][DT];
    {
        const int g = lane >> 4, jl = lane & 15;
#pragma unroll
        for (int qh = 0; qh < 2; qh++) {
            const int tl = 8 * qh + 4 * (g >> 1) + (jl >> 2);  // token mod 16
#pragma unroll
            for (int t = 0; t < DT; t++) {
                const int dd = 32 * t + 16 * (g & 1) + 4 * (jl & 3);
                vofs[qh][t] = (hh * 32 * HD + tl * HD + (((dd >> 3) ^ (swz(tl) & (CPR - 1))) << 3) + (dd & 7)) * 2;
            }
        }
    }
    bf16x8 qf[KK];
    {
        const uint16_t* src = (const uint16_t*)a.q + ((size_t)(q0 + jq) * a.Hq + head) * HD;
#pragma unroll
        for (int kk = 0; kk < KK; kk++) {
            const u16x8 v = row_ok ? *(const u16x8*)(src + kk * 16 + half * 8) : u16x8{0, 0, 0, 0, 0, 0, 0, 0};
            qf[kk] = __builtin_bit_cast(bf16x8, v);
        }
    }
    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; t++) o[t] = f32x16{};
    float m_run = -INFINITY, l_run = 0.0f;  // log2 domain
    bool far = false;                       // an m_run of the wave is 2^28 or further from 0

    // DMA: wave w moves segments w*IPW .. +IPW-1 of the 2*NSEG of a tile (K first). Lane l of a segment moves
    // position l % CPR of token row seg*TPS + l/CPR, fetching chunk (l % CPR) ^ swz(token). A missing
    // page reads page 0 (which exists); tokens that no row sees are masked out of the scores and
    // zeroed in V, whatever was read.
    const int seg0 = (w * IPW) % NSEG, my_tensor = (w * IPW) / NSEG;
    // (the swizzle repeats every 16 tokens)
    constexpr int NV = 16 / TPS < IPW ? 16 / TPS : IPW;
    uint32_t voff[NV];  // bytes from the tile's first segment of this wave (kTile) or the segment
#pragma unroll
    for (int k = 0; k < NV; k++)
        voff[k] = (uint32_t)(((PM == Pages::kTile ? k * TPS : 0) + lane / CPR) * HD +
                             (((lane % CPR) ^ (swz((seg0 + k) * TPS + lane / CPR) & (CPR - 1))) << 3)) * 2u;
    auto token = [&](int k) { return (seg0 + k) * TPS + lane / CPR; };  // of segment k, in the tile
    const char* cbase = (const char*)(my_tensor ? a.vc : a.kc);
    const uint32_t my_ring = (uint32_t)(uintptr_t)(my_tensor ? &lds.v[0][0] : &lds.k[0][0]) + (uint32_t)(seg0 * 1024);
    const int pmask = (1 << a.log2P) - 1;
    const uint64_t page_bytes = ((uint64_t)a.Hkv << a.log2P) * (HD * 2);
    const uint64_t head_bytes = ((uint64_t)h << a.log2P) * (HD * 2);
    int ibuf = 0;
    // The page ids of a tile are read from LDS one tile before its copies are issued: lane k has that of segment
    // k (kLane: every lane has its tokens'), so the look-up's latency is off the path.
    constexpr int NPG = PM == Pages::kLane ? IPW : 1;
    int pgs[STEP][NPG];
    auto find_pages = [&](int t, int c0, int (&pgv)[NPG]) {
        const int32_t* ids = lds.pid + ((t - c0) << log2T);
        if constexpr (PM == Pages::kLane) {
            int x = seg0 * TPS + lane / CPR;
            asm volatile("" : "+v"(x));  // (the addresses of all segments, kept through the loop, would not fit the registers)
#pragma unroll
            for (int k = 0; k < IPW; k++) pgv[k] = ids[(x + k * TPS) >> log2S];
        } else if constexpr (PM == Pages::kSegment) {
            pgv[0] = ids[((seg0 + (lane & (IPW - 1))) * TPS) >> log2S];
        } else {
            pgv[0] = ids[0];
        }
    };
    // what a tile at token tb needs: 0 nothing (every row sees all of it), 1 the mask, 2 mask and page look-up
    bool holes = false;
    auto tile_edge = [&](int tb) {
        return holes ? 2 : (tb + kTile - 1 <= L) & ((tb + kTile <= a.sinks) | (tb > last - a.window)) ? 0 : 1;
    };
    // Segments that no row sees are not fetched from memory: the first one of the cache is read again in
    // their place (which keeps the count of loads per tile).
    auto dead = [&](int s0, int s1) { return (s0 > last) | ((s0 >= a.sinks) & (s1 <= L - a.window)); };
    auto issue_tile = [&](int t, const int (&pgv)[NPG]) {
        const int tb = list_tile(list, t) * kTile;
        const bool edge = tile_edge(tb) != 0;
        const uint32_t lbuf = my_ring + (uint32_t)(ibuf * kTile * HD * 2);
        ibuf = ibuf + 1 == NBUF ? 0 : ibuf + 1;
        if constexpr (PM == Pages::kTile) {
            const unsigned pg = max(__builtin_amdgcn_readfirstlane(pgv[0]), 0);
            const char* base = cbase + pg * page_bytes + head_bytes + (uint32_t)((tb & pmask) + seg0 * TPS) * (HD * 2);
            if (edge) {
#pragma unroll
                for (int k = 0; k < IPW; k++) {
                    const int s0 = tb + (seg0 + k) * TPS;
                    dma16s(voff[k % NV], dead(s0, s0 + TPS - 1) ? cbase : base + k / NV * (NV * TPS * HD * 2),
                           lbuf + 1024 * k);
                }
            } else {
#pragma unroll
                for (int k = 0; k < IPW; k++) dma16s(voff[k % NV], base + k / NV * (NV * TPS * HD * 2), lbuf + 1024 * k);
            }
        } else {
            int x = seg0 * TPS + lane / CPR;
            if constexpr (PM == Pages::kLane) asm volatile("" : "+v"(x));
#pragma unroll
            for (int k = 0; k < IPW; k++) {
                const int s0 = tb + (seg0 + k) * TPS;
                const bool skip = edge && dead(s0, s0 + TPS - 1);
                if constexpr (PM == Pages::kLane) {
                    const char* src = cbase;
                    if (pgv[k] >= 0 && !skip)
                        src += (unsigned)pgv[k] * page_bytes + head_bytes + (uint32_t)((tb + x + k * TPS) & pmask) * (HD * 2) +
                               (voff[k % NV] - (uint32_t)(lane / CPR) * (HD * 2));
                    dma16(src, lbuf + 1024 * k);
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    const unsigned pg = max(__builtin_amdgcn_readlane(pgv[0], k), 0);
                    const char* base = cbase + pg * page_bytes + head_bytes + (uint32_t)(s0 & pmask) * (HD * 2);
                    dma16s(voff[k % NV], skip ? cbase : base, lbuf + 1024 * k);
                }
            }
        }
    };

    // Before the barrier that publishes an edge tile, the lanes that copied V rows zero those that no row sees, and of those
    // that only some rows see what is not finite (shared_bit).
    auto clean_tile = [&](int t, int c0, int buf, int edge) {
        const int tb = list_tile(list, t) * kTile;
#pragma unroll 1
        for (int k = 0; k < IPW; k++) {
            const int s0 = tb + (seg0 + k) * TPS, s1 = s0 + TPS - 1;  // the segment's keys
            const bool shared = some_shared(a, L, last, s0, s1);
            if (edge == 1 && !shared && (s1 <= last) & ((s1 < a.sinks) | (s0 > L - a.window))) continue;
            const int s = tb + token(k);
            u16x8* at = (u16x8*)((char*)lds.v[buf] + (seg0 + k) * 1024 + 16 * lane);
            bool zero = (s > last) | ((s >= a.sinks) & (s <= L - a.window));
            if (edge == 2) zero |= lds.pid[((t - c0) << log2T) + (token(k) >> log2S)] < 0;
            if (zero) *at = u16x8{};
            if (!shared) continue;
            // an exponent of ones carries into the sign bit's place
            const u32x4 x = *(const u32x4*)at;
            unsigned any = 0;
#pragma unroll
            for (int e = 0; e < 4; e++) any |= (x[e] & 0x7F807F80u) + 0x00800080u;
            if (__builtin_expect((any & 0x80008000u) != 0 && some_shared(a, L, last, s, s), 0)) {
                u16x8 v = *at;
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = odd(v[e]) ? 0 : v[e];
                *at = v;
                atomicOr(&lds.odd, shared_bit(a, L, s));
            }
        }
    };

    // LDS byte offsets of the operands inside a tile: K of k-step j of this lane's key, V^T (attn.hip)
    uint32_t kofs[KK];
#pragma unroll
    for (int j = 0; j < KK; j++)
        kofs[j] = (uint32_t)((hh * 32 + (lane & 31)) * HD + (((2 * j + half) ^ (swz(lane & 31) & (CPR - 1))) << 3)) * 2u;
    // One online-softmax step: this wave's NSB halves (32 keys each) of a tile. The products' operands are read
    // from LDS a few products ahead; the scheduling barriers keep that order. With two halves, the
    // exponents of the second are computed between the first half's products with V.
    constexpr int NSB = PARTS == 1 ? 2 : 1;
    auto compute_tile = [&](int t, int c0, int buf, int edge) {
        const char* kt = (const char*)lds.k[buf];
        const char* vt = (const char*)lds.v[buf];
        constexpr int HB = 32 * HD * 2;  // bytes of half a tile
        // S^T = K Q^T: the two halves are two chains
        f32x16 s[NSB];
        {
            constexpr int NF = NSB * KK, KPD = 4;
            auto kread = [&](int j) {
                return __builtin_bit_cast(bf16x8, *(const u16x8*)(kt + kofs[j / NSB] + (j % NSB) * HB));
            };
            bf16x8 kb[KPD + 1];
#pragma unroll
            for (int x = 0; x < NSB; x++) s[x] = f32x16{};
#pragma unroll
            for (int j = 0; j < KPD; j++) kb[j] = kread(j);
#pragma unroll
            for (int j = 0; j < NF; j++) {
                if (j + KPD < NF) kb[(j + KPD) % (KPD + 1)] = kread(j + KPD);
                __builtin_amdgcn_sched_barrier(0);
                s[j % NSB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[j % (KPD + 1)], qf[j / NSB], s[j % NSB], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // register e of half x holds key base + 32 x + y, y = 8 (e / 4) + e % 4
        if (edge) {
            const int base = list_tile(list, t) * kTile + 32 * hh + 4 * half;
            const int hi = p - base, past = p - a.window - base, first = a.sinks - base;
#pragma unroll
            for (int x = 0; x < NSB; x++)
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const int y = 32 * x + 8 * (e >> 2) + (e & 3);
                    s[x][e] = (y <= hi) & ((y > past) | (y < first)) ? s[x][e] : -INFINITY;
                }
            if (edge == 2) {
                const int32_t* ids = lds.pid + ((t - c0) << log2T);
#pragma unroll
                for (int x = 0; x < NSB; x++)
#pragma unroll
                    for (int e = 0; e < 16; e++) {
                        s[x][e] = ids[(32 * (hh + x) + 4 * half + 8 * (e >> 2) + (e & 3)) >> log2S] < 0 ? -INFINITY : s[x][e];
                        if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (few at a time: registers)
                    }
            }
        }
        // The row's maximum: lane-local, then across the lane halves. Weights are relative to m_run, which lies 8 (log2
        // units) above a maximum and moves only when a score of the row passes it, so they stay at 1 or below, and no row's
        // bits depend on another's scores.
        float mx = fmaxf(fmaxf(s[0][0], s[0][1]), s[0][2]);
#pragma unroll
        for (int e = 3; e < 15; e += 2) mx = fmaxf(fmaxf(mx, s[0][e]), s[0][e + 1]);
        mx = fmaxf(mx, s[0][15]);
        if constexpr (NSB == 2) {
#pragma unroll
            for (int e = 0; e < 16; e += 2) mx = fmaxf(fmaxf(mx, s[1][e]), s[1][e + 1]);
        }
        {
            const auto sw2 = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(sw2[0]), __uint_as_float(sw2[1]));
        }
        mx *= a.scale_log2;
        if (__any(mx > m_run)) {  // (from -inf: the first visible key)
            const float m_new = mx > m_run ? mx + 8.0f : m_run;
            far = __any(fabsf(m_new) >= 0x1p28f && m_new != -INFINITY);
            const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_new);
            l_run *= alpha;
#pragma unroll
            for (int t2 = 0; t2 < DT; t2++) o[t2] *= alpha;
            m_run = m_new;
        }
        float nm = m_run == -INFINITY ? 0.0f : -m_run, factor = a.scale_log2;
        // A score's product with the scale is not rounded before m_run, which is, is taken from it: a factor of 2^8 at most
        // while m_run is below 2^28. Beyond, the row's scores are rounded first.
        if (__builtin_expect(far, 0)) {
            if (fabsf(nm) >= 0x1p28f) {
#pragma unroll
                for (int x = 0; x < NSB; x++)
#pragma unroll
                    for (int e = 0; e < 16; e++) {
                        float z = s[x][e] * factor;
                        asm volatile("" : "+v"(z));  // (rounded)
                        s[x][e] = z + nm;
                    }
                nm = 0.0f, factor = 1.0f;
            }
        }
        // O^T += V^T P^T: products j (of both parts of the weights) of half j / NJ, 16-key chunk (j % NJ) / DT, d-tile j % DT
        constexpr int NJ = 2 * DT, NT = NSB * NJ, VPD = 4;
        auto vread = [&](int j) {
            i16x4 vq[2];
#pragma unroll
            for (int qh = 0; qh < 2; qh++)
                vq[qh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_i16x4*)(vt + vofs[qh][j % DT] + (j / NJ) * HB + ((j % NJ) / DT) * (16 * HD * 2)));
            return __builtin_shufflevector(vq[0], vq[1], 0, 1, 2, 3, 4, 5, 6, 7);
        };
        i16x8 vb[VPD + 1];
#pragma unroll
        for (int j = 0; j < VPD; j++) vb[j] = vread(j);
        __builtin_amdgcn_sched_barrier(0);
        float psum[NSB];
        bf16x8 phi[NSB][2], plo[NSB][2];
        auto weight = [&](int x, int e) {
            s[x][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e], factor, nm));
            psum[x] += s[x][e];
        };
        // the weights of half x as hi + lo. 2^-20 of hi is left in lo: with lo = 0 an infinite value would give 0 * inf.
        auto pack = [&](int x) {
            constexpr float kRest = -(1.0f - 0x1p-20f);
#pragma unroll
            for (int cc = 0; cc < 2; cc++) {
                u32x4 hi;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const uint32_t w0 = __float_as_uint(s[x][8 * cc + e]), w1 = __float_as_uint(s[x][8 * cc + e + 1]);
                    hi[e / 2] = __builtin_amdgcn_perm(w1, w0, 0x07060302);  // the upper halves of both
                    plo[x][cc][e] = (__bf16)__builtin_fmaf(__uint_as_float(w0 & 0xFFFF0000u), kRest, s[x][8 * cc + e]);
                    plo[x][cc][e + 1] = (__bf16)__builtin_fmaf(__uint_as_float(w1 & 0xFFFF0000u), kRest, s[x][8 * cc + e + 1]);
                }
                phi[x][cc] = __builtin_bit_cast(bf16x8, hi);
            }
        };
#pragma unroll
        for (int x = 0; x < NSB; x++) psum[x] = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; e++) weight(0, e);
        pack(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < NT; j++) {
            if (j + VPD < NT) vb[(j + VPD) % (VPD + 1)] = vread(j + VPD);
            __builtin_amdgcn_sched_barrier(0);
            o[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vb[j % (VPD + 1)]),
                                                                phi[j / NJ][(j % NJ) / DT], o[j % DT], 0, 0, 0);
            o[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vb[j % (VPD + 1)]),
                                                                plo[j / NJ][(j % NJ) / DT], o[j % DT], 0, 0, 0);
            if constexpr (NSB == 2) {
                if (j < NJ) {
#pragma unroll
                    for (int x = 0; x < 16 / NJ; x++) weight(1, j * (16 / NJ) + x);
                    if (j == NJ - 1) pack(1);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int x = 0; x < NSB; x++) l_run += psum[x];
    };

    // Tile t: wait for its copies (and only those), barrier (tile visible; the buffer that the next copies
    // fill no longer read), start those of the tiles that they take, multiply. (The first NBUF start together.)
    const bool active = rg * 32 < M;
    int buf = 0;
    for (int c0 = t0; c0 < t1; c0 += chunk_tiles) {
        const int c1 = min(t1, c0 + chunk_tiles);
        __syncthreads();  // (holes cleared; page ids of the chunk before read)
        stage(c0, c1);
        __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): no other load pending when the ring starts
        __syncthreads();
        holes = __builtin_amdgcn_readfirstlane(lds.holes) != 0;
#pragma unroll
        for (int x = 0; x < NBUF; x++)
            if (c0 + x < c1) {
                find_pages(c0 + x, c0, pgs[x % STEP]);
                issue_tile(c0 + x, pgs[x % STEP]);
            }
#pragma unroll
        for (int x = 0; x < STEP; x++)
            if (c0 + NBUF + x < c1) find_pages(c0 + NBUF + x, c0, pgs[x]);
        for (int t = c0; t < c1; t += STEP) {
            int edge[STEP];
#pragma unroll
            for (int x = 0; x < STEP; x++) edge[x] = t + x < c1 ? tile_edge(list_tile(list, t + x) * kTile) : 0;
            const int end = min(t + STEP, c1);  // tiles issued after these: up to the ring's length ahead of the last step
            wait_tiles<NBUF - STEP, IPW>(min(c1, (t == c0 ? t : t - STEP) + NBUF) - end);
            if (my_tensor == 1) {
#pragma unroll
                for (int x = 0; x < STEP; x++)
                    if (edge[x] != 0) clean_tile(t + x, c0, buf + x, edge[x]);
            }
            __syncthreads();
            if (t > c0) {
#pragma unroll
                for (int x = 0; x < STEP; x++) {
                    const int next = t + NBUF - STEP + x;
                    if (next >= c1) break;
                    issue_tile(next, pgs[x]);
                    if (next + STEP < c1) find_pages(next + STEP, c0, pgs[x]);
                }
            }
            if (active && t + dt < c1) compute_tile(t + dt, c0, buf + dt, STEP == 2 && dt ? edge[STEP - 1] : edge[0]);
            buf = buf + STEP == NBUF ? 0 : buf + STEP;
        }
        ibuf = buf;
    }

    // The parts of a row group hold the same (row, dim) elements in the same lanes and registers; each finishes DO of
    // the d-tiles and parks the others in the ring.
    float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    constexpr int DO = DT >= PARTS ? DT / PARTS : 1;
    if constexpr (PARTS > 1) {
        __syncthreads();  // (the ring is free)
        f32x4* park = (f32x4*)lds.park + lane;
        lds.ml[w][0][lane] = m_run;
        lds.ml[w][1][lane] = l_tot;
#pragma unroll
        for (int t = 0; t < DT; t++) {
            if (t / DO == th) continue;
#pragma unroll
            for (int g = 0; g < 4; g++)
                park[((w * DT + t) * 4 + g) * 64] = f32x4{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]};
        }
        __syncthreads();
        float mm = m_run, wt[PARTS];
#pragma unroll
        for (int x = 0; x < PARTS; x++) mm = fmaxf(mm, lds.ml[rg * PARTS + x][0][lane]);
        l_tot = 0.0f;
#pragma unroll
        for (int x = 0; x < PARTS; x++) {
            const float mx = lds.ml[rg * PARTS + x][0][lane], lx = lds.ml[rg * PARTS + x][1][lane];
            // (a part whose scores are all NaN has no maximum, but its sum counts)
            wt[x] = mx == -INFINITY ? (lx != 0.0f ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f(mx - mm);
            l_tot += lx * wt[x];
        }
        m_run = mm;
#pragma unroll
        for (int t = 0; t < DT; t++) {
            if (t / DO != th) continue;
            float mine = wt[0];
#pragma unroll
            for (int x = 1; x < PARTS; x++) mine = x == th ? wt[x] : mine;
            o[t] *= mine;
#pragma unroll
            for (int x = 0; x < PARTS; x++) {
                if (x == th) continue;
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    const f32x4 v = park[(((rg * PARTS + x) * DT + t) * 4 + g) * 64];
#pragma unroll
                    for (int e = 0; e < 4; e++) o[t][4 * g + e] += v[e] * wt[x];
                }
            }
        }
    }
    // (the row's place once more, from a thread id that the compiler cannot relate to the one above: kept through the
    // loop, it would cost registers there)
    int tid2 = threadIdx.x;
    asm volatile("" : "+v"(tid2));
    const int r2 = row0 + min(rg * 32 + (tid2 & 31), M - 1), half2 = (tid2 >> 5) & 1;
    const size_t orow = (size_t)(q0 + r2 / a.G) * a.Hq + h * a.G + r2 % a.G;
    if (active && row_ok) {
        const float inv = 1.0f / l_tot;
        const bool whole = a.splits == 1 || t1 - t0 == list.nt;
        const int d0 = PARTS > 1 ? th * DO * 32 : 0, d1 = PARTS > 1 ? min(d0 + DO * 32, HD) : HD;  // this wave's dims
        // dims 32 t + 8 g + 4 half .. + 3
        auto each = [&](auto put) {
#pragma unroll
            for (int t = 0; t < DT; t++) {
                if (PARTS > 1 && t / DO != th) continue;
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; e++) v[e] = l_tot == 0.0f ? 0.0f : o[t][4 * g + e] * inv;
                    put(t * 32 + 8 * g, v);
                }
            }
        };
        const float lse2 = l_tot == 0.0f ? -INFINITY : (m_run - 8.0f) + __log2f(256.0f * l_tot);
        if (whole) {
            uint16_t* out = (uint16_t*)a.out + orow * HD + 4 * half2;
            each([&](int d, f32x4 v) { Vec4<uint16_t>::put(out + d, v); });
            if (__builtin_expect(lds.odd != 0 && l_tot != 0.0f, 0))
                give_back(a, lds.odd, (const uint16_t*)a.q + orow * HD, out - 4 * half2, pt, h, L, L + r2 / a.G, lse2,
                          d0 + 4 * half2, d1, 8);
            if (a.lse && half2 == 0 && th == 0) a.lse[orow] = lse2 * kLn2;
        } else {
            const size_t prow = (size_t)sp * a.total_q * a.Hq + orow;
            float* out = a.part_o + prow * HD + 4 * half2;
            each([&](int d, f32x4 v) { Vec4<float>::put(out + d, v); });
            if (__builtin_expect(lds.odd != 0 && l_tot != 0.0f, 0))
                give_back(a, lds.odd, (const uint16_t*)a.q + orow * HD, out - 4 * half2, pt, h, L, L + r2 / a.G, lse2,
                          d0 + 4 * half2, d1, 8);
            if (half2 == 0 && th == 0) a.part_lse[prow] = lse2;
        }
    }
}

// FEW: at most 32 rows (of every request)
template <int HD, int NW, int NBUF, Pages PM, bool FEW>
__global__ __launch_bounds__(NW * 64, 2) void window_bf16_kernel(WindowArgs a) {
    __shared__ __attribute__((aligned(16))) WindowLds<HD, NW, NBUF> lds;
    Item x;
    if (!find_item(a, FEW ? 32 : NW * 32, x)) return;
    if constexpr (FEW) window_item<HD, NW, NBUF, PM, 4>(a, lds, x);
    else if (x.M <= NW * 16) window_item<HD, NW, NBUF, PM, 2>(a, lds, x);
    else window_item<HD, NW, NBUF, PM, 1>(a, lds, x);
}

// The splits of the divided lists: one thread per (row, 4 dims).
template <typename T>
__global__ __launch_bounds__(256) void window_merge_kernel(WindowArgs a) {
    const int SL = a.HD / 4, i = blockIdx.y;
    int q0, k_i, kv_len;
    if (!load_request(a, i, q0, k_i, kv_len)) return;
    const KeyList list = key_list(a.window, a.sinks, kv_len - k_i, k_i);
    if (list.nt <= a.split_tiles) return;
    const int n = (list.nt + a.split_tiles - 1) / a.split_tiles;
    const long long u = (long long)blockIdx.x * 256 + threadIdx.x;
    if (u >= (long long)k_i * a.Hq * SL) return;
    const size_t orow = (size_t)q0 * a.Hq + (size_t)(u / SL);
    const int sl = (int)(u % SL);
    float mx = -INFINITY, wsum = 0.0f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n; s0 += 8) {  // 8 partial results in flight
        float lw[8];
        f32x4 v[8];
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const size_t prow = (size_t)min(s0 + k, n - 1) * a.total_q * a.Hq + orow;
            lw[k] = s0 + k < n ? a.part_lse[prow] : -INFINITY;
            v[k] = *(const f32x4*)(a.part_o + prow * a.HD + sl * 4);
        }
        float bm = mx;
#pragma unroll
        for (int k = 0; k < 8; k++) bm = fmaxf(bm, lw[k]);
        const float sc = mx == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mx - bm);
        wsum *= sc;
        acc *= sc;
#pragma unroll
        for (int k = 0; k < 8; k++) {
            if (lw[k] == -INFINITY) continue;  // (NaN goes on: its row's result is NaN)
            const float wgt = __builtin_amdgcn_exp2f(lw[k] - bm);
            wsum += wgt;
            acc += wgt * v[k];
        }
        mx = bm;
    }
    const float inv = wsum == 0.0f ? 0.0f : 1.0f / wsum;
    Vec4<T>::put((T*)a.out + orow * a.HD + sl * 4, acc * inv);
    if (a.lse && sl == 0) a.lse[orow] = wsum == 0.0f ? -INFINITY : (mx + __log2f(wsum)) * kLn2;
}

int ilog2(int x) {
    int r = 0;
    while ((1 << r) < x) r++;
    return r;
}

}  // namespace

hipError_t launch_window(const sv_window_desc& w, const WindowPlan& plan, const void* q, const void* k_cache,
                         const void* v_cache, const int32_t* page_table, const int32_t* qo_indptr,
                         const int32_t* kv_lens, void* out, float* lse, void* ws, hipStream_t stream) {
    const sv_attn_desc& d = w.attn;
    WindowArgs a{};
    a.q = q;
    a.kc = k_cache;
    a.vc = v_cache;
    a.page_table = page_table;
    a.qo = qo_indptr;
    a.kv_lens = kv_lens;
    a.out = out;
    a.lse = lse;
    a.part_o = (float*)ws;
    a.part_lse = (float*)((char*)ws + plan.part_o_bytes);
    a.R = d.num_reqs;
    a.total_q = d.total_q_max;
    a.Hq = d.num_q_heads;
    a.Hkv = d.num_kv_heads;
    a.G = d.num_q_heads / d.num_kv_heads;
    a.block = d.block;
    a.HD = d.head_dim;
    a.log2P = ilog2(d.page_size);
    a.maxp = d.max_pages_per_req;
    a.num_pages = d.num_pages;
    a.max_kv_len = d.max_kv_len;
    // (no position is as far: differences with them stay inside 32 bits)
    a.window = std::min(w.window, d.max_kv_len);
    a.sinks = std::min(w.sinks, d.max_kv_len);
    a.splits = plan.splits;
    a.split_tiles = plan.split_tiles;
    a.nrb = plan.row_blocks;
    const long long units = (long long)d.num_reqs * plan.splits * d.num_kv_heads;
    a.by_rows = plan.by_rows;
    a.per_xcd = a.by_rows ? (d.num_reqs * plan.splits + 7) / 8 * d.num_kv_heads : (int)((units + 7) / 8);
    a.scale = d.sm_scale > 0.0f ? d.sm_scale : 1.0f / sqrtf((float)d.head_dim);
    a.scale_log2 = a.scale * kLog2e;
    const dim3 grid(8 * a.per_xcd * plan.row_blocks);
#define SV_WINDOW(HD, NW, NB, PM, FEW) \
    hipLaunchKernelGGL((window_bf16_kernel<HD, NW, NB, Pages::PM, FEW>), grid, dim3(NW * 64), 0, stream, a)
#define SV_WINDOW_PAGES(HD, NW, NB, FEW) \
    if (d.page_size >= kTile) SV_WINDOW(HD, NW, NB, kTile, FEW); \
    else if (d.page_size >= 512 / HD) SV_WINDOW(HD, NW, NB, kSegment, FEW); \
    else SV_WINDOW(HD, NW, NB, kLane, FEW)
    if (d.dtype == SV_F32) {
        const bool two = plan.block_rows == 32;
        if (d.head_dim > 128) hipLaunchKernelGGL((window_f32_kernel<4, 1>), grid, dim3(256), 0, stream, a);
        else if (d.head_dim > 64 && two) hipLaunchKernelGGL((window_f32_kernel<2, 2>), grid, dim3(256), 0, stream, a);
        else if (d.head_dim > 64) hipLaunchKernelGGL((window_f32_kernel<2, 1>), grid, dim3(256), 0, stream, a);
        else if (two) hipLaunchKernelGGL((window_f32_kernel<1, 2>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((window_f32_kernel<1, 1>), grid, dim3(256), 0, stream, a);
    } else if (plan.few) {
        if (d.head_dim == 128) { SV_WINDOW_PAGES(128, 4, 4, true); }
        else { SV_WINDOW_PAGES(64, 4, 4, true); }
    } else if (plan.waves == 4) {
        if (d.head_dim == 128) { SV_WINDOW_PAGES(128, 4, 2, false); }
        else { SV_WINDOW_PAGES(64, 4, 4, false); }
    } else {
        if (d.head_dim == 128) { SV_WINDOW_PAGES(128, 8, 4, false); }
        else { SV_WINDOW_PAGES(64, 8, 4, false); }
    }
#undef SV_WINDOW_PAGES
#undef SV_WINDOW
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.splits == 1) return e;
    const long long slices = (long long)d.block * d.num_q_heads * (d.head_dim / 4);
    const dim3 mgrid((unsigned)((slices + 255) / 256), d.num_reqs);
    if (d.dtype == SV_F32) hipLaunchKernelGGL(window_merge_kernel<float>, mgrid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(window_merge_kernel<uint16_t>, mgrid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sv
