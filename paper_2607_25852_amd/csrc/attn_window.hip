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
    int nrb, per_xcd;         // row blocks per (request, kv-head); (request, split, kv-head) per XCD
    float scale, scale_log2;  // sm_scale, sm_scale * log2(e)
};

// The keys of a request with k rows after L committed tokens, in tiles of TT tokens
struct KeyList {
    int ns;  // tiles 0 .. ns-1 hold the first positions
    int ft;  // then tiles from ft on
    int nt;  // tiles in all
};
__device__ inline KeyList key_list(int window, int sinks, int TT, int L, int k) {
    const int first = max(0, L - window + 1);
    const int ns = (int)(((unsigned)min(sinks, first) + (unsigned)TT - 1) / (unsigned)TT);
    const int ft = max(first / TT, ns);
    return KeyList{ns, ft, ns + (L + k - 1) / TT - ft + 1};
}
__device__ inline int list_tile(const KeyList& x, int t) { return t < x.ns ? t : x.ft + (t - x.ns); }

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
};
template <> struct Vec4<uint16_t> {
    static __device__ f32x4 get(const uint16_t* p) {
        const uint2 w = *(const uint2*)p;
        return f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xFFFF0000u)};
    }
};
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ inline void store1(float* p, float f) { *p = f; }
__device__ inline void store1(uint16_t* p, float f) { *p = f2bf(f); }

// One wave: the row of query qp at position p (kv-head h, page table row pt) against tiles t, t +
// step, .. < t1 of its request's list. Leaves the softmax state (m, l) and o[e] for dim lane + 64 e.
// Every key is used by itself: what a row does not see is not read.
template <typename T>
__device__ void wave_row(const WindowArgs& a, const T* qp, const int32_t* pt, int h, int p, const KeyList& list, int TT,
                         int t, int t1, int step, float& m, float& l, float (&o)[4]) {
    const int lane = threadIdx.x & 63, HD = a.HD, P = 1 << a.log2P;
    m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = 0.0f;
    for (; t < t1; t += step)
        for (int at = 0; at < TT; at += 64) {
            const int s = list_tile(list, t) * TT + at + lane;
            float z = -INFINITY;
            size_t off = 0;
            bool ok = at + lane < TT && s <= p && (s < a.sinks || s > p - a.window);
            if (ok) {
                const int col = s >> a.log2P, pg = col < a.maxp ? pt[col] : -1;
                ok = pg >= 0 && pg < a.num_pages;
                if (ok) {
                    off = ((((size_t)pg * a.Hkv + h) << a.log2P) + (s & (P - 1))) * HD;
                    float dot = 0.0f;
                    for (int e = 0; e < HD; e += 4) {
                        const f32x4 x = Vec4<T>::get((const T*)a.kc + off + e), y = Vec4<T>::get(qp + e);
                        dot += x[0] * y[0] + x[1] * y[1] + x[2] * y[2] + x[3] * y[3];
                    }
                    z = dot * a.scale;
                }
            }
            float mx = z;
            for (int x = 32; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x, 64));
            const float m_new = fmaxf(m, mx);
            if (m_new == -INFINITY && !__any(ok && z != z)) continue;
            const float alpha = m == -INFINITY ? 0.0f : expf(m - m_new);
            const float w = ok ? expf(z - m_new) : 0.0f;
            float ws = w;
            for (int x = 32; x > 0; x >>= 1) ws += __shfl_xor(ws, x, 64);
            l = l * alpha + ws;
            m = m_new;
#pragma unroll
            for (int e = 0; e < 4; e++) o[e] *= alpha;
            uint64_t todo = __ballot(ok);
            while (todo) {
                const int j = __builtin_ctzll(todo);
                todo &= todo - 1;
                const float wj = __shfl(w, j, 64);
                const size_t offj = ((size_t)(uint32_t)__shfl((int)(off >> 32), j, 64) << 32) |
                                    (uint32_t)__shfl((int)(uint32_t)off, j, 64);
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (lane + 64 * e < HD) o[e] += wj * load1((const T*)a.vc + offj + lane + 64 * e);
            }
        }
}

// fp32: one workgroup of four waves per (query row, head); wave w takes every fourth tile of 64 keys,
// and the waves' softmax states are merged at the end.
template <typename T>
__global__ __launch_bounds__(256) void window_rows_kernel(WindowArgs a) {
    __shared__ float s_o[4][4][64];
    __shared__ float s_ml[4][2];
    const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63, HD = a.HD;
    const int row = blockIdx.x / a.Hq, head = blockIdx.x % a.Hq;
    if (row >= a.qo[a.R]) return;
    int lo = 0, hi = a.R - 1;  // the last request whose rows start at or before this one
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.qo[mid] <= row) lo = mid; else hi = mid - 1;
    }
    int q0, k_i, kv_len;
    if (!load_request(a, lo, q0, k_i, kv_len) || row < q0 || row >= q0 + k_i) return;
    const int p = kv_len - k_i + (row - q0);
    const KeyList list = key_list(a.window, a.sinks, 64, p, 1);
    float o[4], m, l;
    wave_row<T>(a, (const T*)a.q + ((size_t)row * a.Hq + head) * HD, a.page_table + (size_t)lo * a.maxp, head / a.G, p,
                list, 64, wv, list.nt, 4, m, l, o);
#pragma unroll
    for (int e = 0; e < 4; e++) s_o[wv][e][lane] = o[e];
    if (lane == 0) {
        s_ml[wv][0] = m;
        s_ml[wv][1] = l;
    }
    __syncthreads();
    if (wv != 0) return;
    float M = -INFINITY, lt = 0.0f, ot[4] = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < 4; w++) M = fmaxf(M, s_ml[w][0]);
    for (int w = 0; w < 4; w++) {
        const float mw = s_ml[w][0], wt = mw == -INFINITY ? (s_ml[w][1] != 0.0f ? 1.0f : 0.0f) : expf(mw - M);
        lt += s_ml[w][1] * wt;
#pragma unroll
        for (int e = 0; e < 4; e++) ot[e] += s_o[w][e][lane] * wt;
    }
    const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
    T* op = (T*)a.out + ((size_t)row * a.Hq + head) * HD;
#pragma unroll
    for (int e = 0; e < 4; e++)
        if (lane + 64 * e < HD) store1(op + lane + 64 * e, ot[e] * inv);
    if (a.lse && lane == 0) a.lse[(size_t)row * a.Hq + head] = lt == 0.0f ? -INFINITY : M + logf(lt);
}

// ---------------------------------------------------------------------------------
// bf16 MFMA kernel
// ---------------------------------------------------------------------------------
// A workgroup of RG * TS waves takes one (request, split, kv-head, row block): up to RG * 32 query rows of
// the kv-head group (row r: position j = r / G, head r % G) against the split's tiles of TS * 32
// keys. Wave w has rows 32 (w / TS) .. + 31 and keys 32 (w % TS) .. + 31 of every tile. As in
// attn.hip, S^T = K Q^T puts the scores of a query row into one lane pair, and P^T is then
// in the operand layout of O^T = V^T P^T, with V read transposed from LDS. K and V tiles come
// through the page table into an LDS ring by direct loads while earlier tiles are multiplied;
// the TS parts of a row are merged at the end.
constexpr int kPageSlots = 1024;  // page ids staged at a time

template <int HD, int RG, int TS, int NBUF>
struct WindowLds {
    static constexpr int TT = 32 * TS;
    union {
        struct {
            uint16_t k[NBUF][TT * HD];  // [buffer][token * HD + d], swizzled (attn_tile.h)
            uint16_t v[NBUF][TT * HD];
        };
        float park[TS == 1 ? 1 : RG * TS * HD * 32];  // the waves' partial outputs
    };
    float ml[RG * TS][2][64];
    int32_t pid[kPageSlots];
    int32_t holes;  // a page that the list needs is missing
    int32_t dirty;  // a value that only some rows see was not finite
};

// the rows of a row block one by one (rare: see `dirty`)
template <int HD>
__device__ __noinline__ void redo_rows(WindowArgs a, int i, int h, int sp, int row0, int M, int q0, int L,
                                       KeyList list, int TT, int t0, int t1) {
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    for (int r = threadIdx.x >> 6; r < M; r += waves) {
        const int rr = row0 + r, jq = rr / a.G, head = h * a.G + rr % a.G;
        const size_t orow = (size_t)(q0 + jq) * a.Hq + head;
        float o[4], m, l;
        wave_row<uint16_t>(a, (const uint16_t*)a.q + orow * HD, a.page_table + (size_t)i * a.maxp, h, L + jq, list, TT,
                           t0, t1, 1, m, l, o);
        const float inv = l == 0.0f ? 0.0f : 1.0f / l, lse = l == 0.0f ? -INFINITY : m + logf(l);
        const bool whole = t1 - t0 == list.nt;
        const size_t prow = (size_t)sp * a.total_q * a.Hq + orow;
        for (int e = 0; e < HD / 64; e++) {
            if (whole) ((uint16_t*)a.out)[orow * HD + lane + 64 * e] = f2bf(o[e] * inv);
            else a.part_o[prow * HD + lane + 64 * e] = o[e] * inv;
        }
        if (lane == 0) {
            if (!whole) a.part_lse[prow] = lse * kLog2e;
            else if (a.lse) a.lse[orow] = lse;
        }
    }
}

// LANE: pages below a 1 KB segment of a tile, every lane looks its token's page up
template <int HD, int RG, int TS, int NBUF, bool LANE>
__global__ __launch_bounds__(RG * TS * 64, 2) void window_bf16_kernel(WindowArgs a) {
    constexpr int NW = RG * TS, TT = 32 * TS;
    constexpr int CPR = HD / 8;             // 16-byte chunks per token row
    constexpr int TPS = 1024 / (HD * 2);    // tokens per 1 KB DMA segment
    constexpr int NSEG = TT / TPS;          // segments per tensor per tile
    constexpr int IPW = 2 * NSEG / NW;      // DMA instructions per wave per tile
    static_assert(IPW * NW == 2 * NSEG && IPW >= 1 && (NSEG % IPW) == 0, "DMA split: a wave moves one tensor");
    constexpr int KK = HD / 16;             // MFMA k-steps over the head dim
    constexpr int DT = HD / 32;             // output d-tiles
    constexpr int PF = NBUF - 1;            // prefetch distance in tiles
    __shared__ __attribute__((aligned(16))) WindowLds<HD, RG, TS, NBUF> lds;

    // neighbouring workgroups go to the XCDs in turn: each takes a run of (request, split, kv-head)s, whose heads
    // share pages, and the row blocks of one follow each other
    // (the quotients of vector divisions, back in scalar registers: the copies' addresses need them there)
    auto scalar = [](unsigned x) { return __builtin_amdgcn_readfirstlane((int)x); };
    const unsigned slot = blockIdx.x / 8;
    const int ux = scalar(slot / (unsigned)a.nrb), rb = scalar(slot % (unsigned)a.nrb);
    const unsigned unit = (blockIdx.x % 8) * (unsigned)a.per_xcd + (unsigned)ux;
    if (ux >= a.per_xcd || unit >= (unsigned)a.R * (unsigned)a.splits * (unsigned)a.Hkv) return;
    const int h = scalar(unit % (unsigned)a.Hkv), is = scalar(unit / (unsigned)a.Hkv);
    const int sp = scalar((unsigned)is % (unsigned)a.splits), i = scalar((unsigned)is / (unsigned)a.splits);
    const int row0 = rb * RG * 32;
    int q0, k_i, kv_len;
    if (!load_request(a, i, q0, k_i, kv_len)) return;
    const int M = min(a.G * k_i - row0, RG * 32);
    if (M <= 0) return;
    const int L = kv_len - k_i, last = kv_len - 1;  // the first and the last row's position
    const KeyList list = key_list(a.window, a.sinks, TT, L, k_i);
    const int t0 = sp * a.split_tiles, t1 = min(list.nt, t0 + a.split_tiles);
    if (t0 >= t1) return;

    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int32_t* __restrict__ pt = a.page_table + (size_t)i * a.maxp;
    const int log2S = a.log2P < 31 - __builtin_clz(TT) ? a.log2P : 31 - __builtin_clz(TT);  // tokens per slot
    const int log2T = 31 - __builtin_clz(TT) - log2S;                                      // slots per tile
    const int chunk_tiles = kPageSlots >> log2T;
    // page ids of tiles c0 .. c1-1 into LDS; a missing page is flagged where a row sees the slot
    auto stage = [&](int c0, int c1) {
        bool hole = false;
        for (int e = tid; e < (c1 - c0) << log2T; e += NW * 64) {
            const int s = (list_tile(list, c0 + (e >> log2T)) * TT) + ((e & ((1 << log2T) - 1)) << log2S);
            const int col = s >> a.log2P, pg = col < a.maxp ? pt[col] : -1;
            const bool ok = pg >= 0 && pg < a.num_pages;
            hole |= !ok && s <= last && (s < a.sinks || s + (1 << log2S) > L - a.window + 1);
            lds.pid[e] = ok ? pg : -1;
        }
        if (hole) lds.holes = 1;
    };
    if (tid == 0) lds.holes = lds.dirty = 0;

    const int rg = w / TS, th = w % TS;
    const int r = rg * 32 + (lane & 31), half = lane >> 5;
    const bool row_ok = r < M;
    const int rr = row0 + (row_ok ? r : 0);  // row within the request's kv-head group
    const int jq = rr / a.G, head = h * a.G + rr % a.G;
    const int p = L + jq;  // the row's position

    // per-lane element offsets of the V^T transpose reads (attn.hip)
    int vofs[2][DT];
    {
        const int g = lane >> 4, jl = lane & 15;
#pragma unroll
        for (int qh = 0; qh < 2; qh++) {
            const int tl = 8 * qh + 4 * (g >> 1) + (jl >> 2);  // token mod 16
#pragma unroll
            for (int t = 0; t < DT; t++) {
                const int dd = 32 * t + 16 * (g & 1) + 4 * (jl & 3);
                vofs[qh][t] = th * 32 * HD + tl * HD + (((dd >> 3) ^ (swz(tl) & (CPR - 1))) << 3) + (dd & 7);
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
    float m_run = -INFINITY, l_run = 0.0f;  // the maximum of the unscaled scores

    // DMA: wave w moves segments w*IPW .. +IPW-1 of the 2*NSEG of a tile (K first). Lane l of a segment moves
    // position l % CPR of token row seg*TPS + l/CPR, fetching chunk (l % CPR) ^ swz(token). A missing
    // page, or a segment that no row sees, reads page 0 (which exists); such tokens are masked
    // out of the scores and zeroed in V.
    uint32_t voff[IPW];
    int tk[IPW], sg[IPW];
#pragma unroll
    for (int k = 0; k < IPW; k++) {
        const int seg = (w * IPW + k) % NSEG;
        const int t = seg * TPS + lane / CPR;
        tk[k] = t;
        sg[k] = __builtin_amdgcn_readfirstlane(seg * TPS);
        voff[k] = (uint32_t)((lane / CPR) * HD + (((lane % CPR) ^ (swz(t) & (CPR - 1))) << 3)) * 2u;
    }
    const int my_tensor = __builtin_amdgcn_readfirstlane((w * IPW) / NSEG);
    const uint16_t* cbase = (const uint16_t*)(my_tensor ? a.vc : a.kc);
    const uint32_t my_ring = (uint32_t)(uintptr_t)(my_tensor ? &lds.v[0][0] : &lds.k[0][0]) +
                             (uint32_t)__builtin_amdgcn_readfirstlane(((w * IPW) % NSEG) * 1024);
    const int pmask = (1 << a.log2P) - 1;
    int ibuf = 0;
    auto issue_tile = [&](int t, int c0) {
        const int tb = list_tile(list, t) * TT;
        const uint32_t lbuf = my_ring + (uint32_t)(ibuf * TT * HD * 2);
        ibuf = ibuf + 1 == NBUF ? 0 : ibuf + 1;
        const int32_t* ids = lds.pid + ((t - c0) << log2T);
#pragma unroll
        for (int k = 0; k < IPW; k++) {
            if constexpr (LANE) {
                const int tok = tb + tk[k], pg = ids[tk[k] >> log2S];
                const uint16_t* src = cbase;
                if (pg >= 0)
                    src += ((((size_t)pg * a.Hkv + h) << a.log2P) + (size_t)(tok & pmask)) * HD +
                           (voff[k] / 2 - (lane / CPR) * HD);
                dma16(src, lbuf + 1024 * k);
            } else {
                const int tok = tb + sg[k], pg = max(__builtin_amdgcn_readfirstlane(ids[sg[k] >> log2S]), 0);
                dma16s(voff[k], cbase + ((((size_t)pg * a.Hkv + h) << a.log2P) + (size_t)(tok & pmask)) * HD,
                       lbuf + 1024 * k);
            }
        }
    };

    // what a tile at token tb needs: 0 nothing (every row sees all of it), 1 the mask, 2 mask and page look-up
    auto tile_edge = [&](int tb) {
        if (lds.holes) return 2;
        return tb + TT - 1 <= L && (tb + TT <= a.sinks || tb > last - a.window) ? 0 : 1;
    };
    // before the barrier that publishes an edge tile: the lanes that copied V rows which no row sees zero them (P
    // is 0 there, but 0 * NaN is not), and rows that only some see are zeroed if they are not finite: the
    // row block is then done again row by row
    auto clean_tile = [&](int t, int c0, int buf) {
        const int tb = list_tile(list, t) * TT;
        const int edge = tile_edge(tb);
        if (edge == 0 || my_tensor == 0) return;
#pragma unroll
        for (int k = 0; k < IPW; k++) {
            const int s = tb + tk[k];
            u16x8* at = (u16x8*)((char*)lds.v[buf] + ((w * IPW) % NSEG + k) * 1024 + 16 * lane);
            bool zero = s > last || (s >= a.sinks && s <= L - a.window);
            if (edge == 2) zero |= lds.pid[((t - c0) << log2T) + (tk[k] >> log2S)] < 0;
            if (!zero && (s > L || (s >= a.sinks && s <= last - a.window))) {
                const u16x8 v = *at;
#pragma unroll
                for (int e = 0; e < 8; e++) zero |= (v[e] & 0x7F80) == 0x7F80;
                if (zero) lds.dirty = 1;
            }
            if (zero) *at = u16x8{};
        }
    };

    auto compute_tile = [&](int t, int c0, int buf) {
        const uint16_t* kt = lds.k[buf];
        const uint16_t* vt = lds.v[buf];
        const int tb = list_tile(list, t) * TT;
        // S^T = K Q^T of this wave's 32 keys in two chains, operands read KPD products ahead
        f32x16 s;
        {
            const int sw = swz(lane & 31) & (CPR - 1);
            const uint16_t* krow = kt + (th * 32 + (lane & 31)) * HD;
            constexpr int KPD = 4;
            auto kread = [&](int j) { return __builtin_bit_cast(bf16x8, *(const u16x8*)(krow + (((2 * j + half) ^ sw) << 3))); };
            bf16x8 kb[KPD + 1];
            f32x16 c0a = f32x16{}, c1a = f32x16{};
#pragma unroll
            for (int j = 0; j < KPD; j++) kb[j] = kread(j);
#pragma unroll
            for (int j = 0; j < KK; j++) {
                if (j + KPD < KK) kb[(j + KPD) % (KPD + 1)] = kread(j + KPD);
                __builtin_amdgcn_sched_barrier(0);
                if (j & 1) c1a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[j % (KPD + 1)], qf[j], c1a, 0, 0, 0);
                else c0a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[j % (KPD + 1)], qf[j], c0a, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            s = c0a + c1a;
        }
        // register e holds key tb + 32 th + 4 half + x, x = 8 (e / 4) + e % 4
        const int edge = tile_edge(tb);
        if (edge) {
            const int base = tb + 32 * th + 4 * half;
            const int hi = p - base, past = p - a.window - base, first = a.sinks - base;
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const int x = 8 * (e >> 2) + (e & 3);
                if (!(x <= hi && (x > past || x < first))) s[e] = -INFINITY;
            }
            if (edge == 2) {
                const int32_t* ids = lds.pid + ((t - c0) << log2T);
#pragma unroll
                for (int e = 0; e < 16; e++)
                    if (ids[(32 * th + 4 * half + 8 * (e >> 2) + (e & 3)) >> log2S] < 0) s[e] = -INFINITY;
            }
        }
        // the row's maximum: lane-local, then across the lane halves; the running maximum moves only when a
        // score passes it by more than 8 in log2 units, so the weights stay below 2^8
        float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
        for (int e = 3; e < 15; e += 2) mx = fmaxf(fmaxf(mx, s[e]), s[e + 1]);
        mx = fmaxf(mx, s[15]);
        {
            const auto sw2 = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(sw2[0]), __uint_as_float(sw2[1]));
        }
        if (__any((mx - m_run) * a.scale_log2 > 8.0f)) {  // (from -inf: the first visible key)
            const float m_new = fmaxf(m_run, mx);
            const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run - m_new) * a.scale_log2);
            l_run *= alpha;
#pragma unroll
            for (int t2 = 0; t2 < DT; t2++) o[t2] *= alpha;
            m_run = m_new;
        }
        const float ref = m_run == -INFINITY ? 0.0f : m_run;
        constexpr int NJ = 2 * DT, VPD = 4;
        auto vread = [&](int j) {
            const int c = j / DT, t2 = j % DT;  // 16-token chunk of the wave's keys, d-tile
            i16x4 vq[2];
#pragma unroll
            for (int qh = 0; qh < 2; qh++)
                vq[qh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vt + 16 * c * HD + vofs[qh][t2]));
            return __builtin_shufflevector(vq[0], vq[1], 0, 1, 2, 3, 4, 5, 6, 7);
        };
        i16x8 vb[VPD + 1];
#pragma unroll
        for (int j = 0; j < VPD; j++) vb[j] = vread(j);
        __builtin_amdgcn_sched_barrier(0);
        float psum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; e++) {
            s[e] = __builtin_amdgcn_exp2f((s[e] - ref) * a.scale_log2);
            psum += s[e];
        }
        l_run += psum;
        bf16x8 pb[2];
#pragma unroll
        for (int cc = 0; cc < 2; cc++)
#pragma unroll
            for (int e = 0; e < 8; e++) pb[cc][e] = (__bf16)s[8 * cc + e];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < NJ; j++) {
            if (j + VPD < NJ) vb[(j + VPD) % (VPD + 1)] = vread(j + VPD);
            __builtin_amdgcn_sched_barrier(0);
            o[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vb[j % (VPD + 1)]), pb[j / DT],
                                                                o[j % DT], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // Tile t: wait for its copies (and only those), barrier (tile visible; the buffer that the next copies
    // fill no longer read), start those of tile t + PF, multiply.
    const bool active = __builtin_amdgcn_readfirstlane(rg) * 32 < M;
    int buf = 0;
    for (int c0 = t0; c0 < t1; c0 += chunk_tiles) {
        const int c1 = min(t1, c0 + chunk_tiles);
        __syncthreads();  // (holes, dirty cleared; page ids of the chunk before read)
        stage(c0, c1);
        __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): no other load pending when the ring starts
        __syncthreads();
#pragma unroll
        for (int x = 0; x < PF; x++)
            if (c0 + x < c1) issue_tile(c0 + x, c0);
        for (int t = c0; t < c1; t++) {
            const int newer = min(PF - 1, c1 - 1 - t);
            if (newer >= 2) wait_vm<2 * IPW>();
            else if (newer == 1) wait_vm<IPW>();
            else wait_vm<0>();
            clean_tile(t, c0, buf);
            __syncthreads();
            if (t + PF < c1) issue_tile(t + PF, c0);
            if (active) compute_tile(t, c0, buf);
            buf = buf + 1 == NBUF ? 0 : buf + 1;
        }
        ibuf = buf;
    }
    static_assert(PF <= 3, "the waits above");

    float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    // merge the TS parts of a row group; wave th finishes d-tiles th, th + TS, ..
    constexpr int DO = (DT + TS - 1) / TS;
    f32x16 of[DO];
    if constexpr (TS > 1) {
        __syncthreads();  // (the ring is free)
        f32x4* park = (f32x4*)lds.park + lane;
        if (active) {
#pragma unroll
            for (int t = 0; t < DT; t++)
#pragma unroll
                for (int g = 0; g < 4; g++)
                    park[((w * DT + t) * 4 + g) * 64] = f32x4{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]};
            lds.ml[w][0][lane] = m_run;
            lds.ml[w][1][lane] = l_tot;
        }
        __syncthreads();
        if (active) {
            float mm = -INFINITY, wt[TS];
            l_tot = 0.0f;
#pragma unroll
            for (int x = 0; x < TS; x++) mm = fmaxf(mm, lds.ml[rg * TS + x][0][lane]);
#pragma unroll
            for (int x = 0; x < TS; x++) {
                const float mx = lds.ml[rg * TS + x][0][lane], lx = lds.ml[rg * TS + x][1][lane];
                // (a part whose scores are all NaN has no maximum, but its sum counts)
                wt[x] = mx == -INFINITY ? (lx != 0.0f ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f((mx - mm) * a.scale_log2);
                l_tot += lx * wt[x];
            }
            m_run = mm;
#pragma unroll
            for (int k = 0; k < DO; k++) {
                of[k] = f32x16{};
                const int t = th + k * TS;
                if (t >= DT) continue;
#pragma unroll
                for (int x = 0; x < TS; x++)
#pragma unroll
                    for (int g = 0; g < 4; g++) {
                        const f32x4 v = park[(((rg * TS + x) * DT + t) * 4 + g) * 64];
#pragma unroll
                        for (int e = 0; e < 4; e++) of[k][4 * g + e] += v[e] * wt[x];
                    }
            }
        }
    } else {
#pragma unroll
        for (int t = 0; t < DT; t++) of[t] = o[t];
    }
    if (active && row_ok) {
        const float inv = l_tot == 0.0f ? 0.0f : 1.0f / l_tot;
        const float lse2 = l_tot == 0.0f ? -INFINITY : m_run * a.scale_log2 + __log2f(l_tot);
        const size_t orow = (size_t)(q0 + jq) * a.Hq + head;
        const bool whole = t1 - t0 == list.nt;
        const size_t prow = (size_t)sp * a.total_q * a.Hq + orow;
#pragma unroll
        for (int k = 0; k < DO; k++) {
            const int t = th + k * TS;
            if (t >= DT) continue;
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const int d0 = t * 32 + 8 * g + 4 * half;
                if (whole) {
                    bf16x4 v;
#pragma unroll
                    for (int e = 0; e < 4; e++) v[e] = (__bf16)(of[k][4 * g + e] * inv);
                    *(bf16x4*)((uint16_t*)a.out + orow * HD + d0) = v;
                } else {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; e++) v[e] = of[k][4 * g + e] * inv;
                    *(f32x4*)(a.part_o + prow * HD + d0) = v;
                }
            }
        }
        if (half == 0 && th == 0) {
            if (!whole) a.part_lse[prow] = lse2;
            else if (a.lse) a.lse[orow] = lse2 * kLn2;
        }
    }
    if (lds.dirty) {  // (written before a barrier that all have passed)
        __syncthreads();
        redo_rows<HD>(a, i, h, sp, row0, M, q0, L, list, TT, t0, t1);
    }
}

// The splits of the divided lists: one thread per (row, 4 dims).
__global__ __launch_bounds__(256) void window_merge_kernel(WindowArgs a, int TT) {
    const int SL = a.HD / 4, i = blockIdx.y;
    int q0, k_i, kv_len;
    if (!load_request(a, i, q0, k_i, kv_len)) return;
    const KeyList list = key_list(a.window, a.sinks, TT, kv_len - k_i, k_i);
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
    uint64_t pk = 0;
#pragma unroll
    for (int e = 0; e < 4; e++) pk |= (uint64_t)f2bf(acc[e] * inv) << (16 * e);
    *(uint64_t*)((uint16_t*)a.out + orow * a.HD + sl * 4) = pk;
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
    a.window = w.window;
    a.sinks = w.sinks;
    a.splits = plan.splits;
    a.split_tiles = plan.split_tiles;
    a.nrb = plan.row_blocks;
    const long long units = (long long)d.num_reqs * plan.splits * d.num_kv_heads;
    a.per_xcd = (int)((units + 7) / 8);
    a.scale = d.sm_scale > 0.0f ? d.sm_scale : 1.0f / sqrtf((float)d.head_dim);
    a.scale_log2 = a.scale * kLog2e;
    if (d.dtype == SV_F32) {
        hipLaunchKernelGGL(window_rows_kernel<float>, dim3(d.total_q_max * d.num_q_heads), dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    const dim3 grid(8 * a.per_xcd * plan.row_blocks);
    const int tps = 512 / d.head_dim;  // tokens per 1 KB segment
#define SV_WINDOW(HD, RG, TS, NB, LANE) \
    hipLaunchKernelGGL((window_bf16_kernel<HD, RG, TS, NB, LANE>), grid, dim3(RG * TS * 64), 0, stream, a)
#define SV_WINDOW_SHAPE(HD, LANE) \
    if (plan.row_groups == 1) SV_WINDOW(HD, 1, 4, 2, LANE); \
    else if (plan.row_groups == 2) SV_WINDOW(HD, 2, 2, 3, LANE); \
    else SV_WINDOW(HD, 4, 1, 4, LANE)
    if (d.head_dim == 128) {
        if (d.page_size >= tps) { SV_WINDOW_SHAPE(128, false); }
        else { SV_WINDOW_SHAPE(128, true); }
    } else {
        if (d.page_size >= tps) { SV_WINDOW_SHAPE(64, false); }
        else { SV_WINDOW_SHAPE(64, true); }
    }
#undef SV_WINDOW_SHAPE
#undef SV_WINDOW
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.splits == 1) return e;
    const long long slices = (long long)d.block * d.num_q_heads * (d.head_dim / 4);
    hipLaunchKernelGGL(window_merge_kernel, dim3((unsigned)((slices + 255) / 256), d.num_reqs), dim3(256), 0, stream, a,
                       plan.tile);
    return hipGetLastError();
}

}  // namespace sv
