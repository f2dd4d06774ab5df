// The work of the page-table calls (pages.hip) on one entry or by one workgroup. Integer index
// arithmetic only; every id read from a table, list or workspace is range-checked before it is used
// as an index. The header also builds for the host, where the sanitizer test runs it.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace sv {

constexpr int kPageChunk = 4096;      // pages per workgroup of the kernels that walk the counts
constexpr int kReserveReqs = 4096;    // requests whose entry offsets fit the LDS of sv_reserve_pages
constexpr int32_t kNeverServed = 0x7FFFFFFF;

// a value that other waves of the workgroup changed with atomics (which bypass this CU's cache)
__device__ inline int load_counted(const int32_t* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// sum of v over lanes 0 .. lane of the wave
__device__ inline uint32_t wave_scan(uint32_t v) {
#ifdef __AMDGCN__
    // within rows of 16 lanes by 1, 2, 4, 8, then the last lane of a row (of two) to the rows after it
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);
#else
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t u = __shfl_up(v, off, 64);
        if ((int)(threadIdx.x & 63) >= off) v += u;
    }
#endif
    return v;
}

// sum of v over the threads before this one; total: over all. wsum: NT / 64 entries of LDS.
template <int NT>
__device__ inline uint32_t block_scan(uint32_t v, uint32_t* wsum, uint32_t& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t incl = wave_scan(v);
    __syncthreads();  // (wsum may still be read by an earlier scan)
    if (lane == 63) wsum[w] = incl;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
    for (int k = 0; k < NT / 64; k++) {
        if (k < w) before += wsum[k];
        total += wsum[k];
    }
    return before + incl - v;
}

// ---- fork ----------------------------------------------------------------------------
struct ForkArgs {
    const int32_t* table_in;  // [rows_in, maxp]
    const int32_t* lens_in;   // [rows_in]
    const int32_t* parent;    // [R]
    int32_t* table_out;       // [R, maxp]
    int32_t* lens_out;        // [R]
    int32_t* ref;             // [num_pages]
    int R, rows_in, maxp, num_pages, log2P;
};

// entry e: the entries of table_out, then those of table_in, whose holds end
__device__ inline void fork_entry(const ForkArgs& a, long long e) {
    const long long n_out = (long long)a.R * a.maxp;
    if (e >= n_out) {
        e -= n_out;
        if (e >= (long long)a.rows_in * a.maxp) return;
        const int pg = a.table_in[e];
        if ((unsigned)pg < (unsigned)a.num_pages) atomicAdd(&a.ref[pg], -1);
        return;
    }
    const int i = (int)((unsigned)e / (unsigned)a.maxp), c = (int)((unsigned)e % (unsigned)a.maxp);
    const int p = a.parent[i];
    const int len = (unsigned)p < (unsigned)a.rows_in ? max(a.lens_in[p], 0) : 0;
    int pg = -1;
    if ((long long)c << a.log2P < len) {
        pg = a.table_in[(size_t)p * a.maxp + c];
        if ((unsigned)pg < (unsigned)a.num_pages) atomicAdd(&a.ref[pg], 1);
        else pg = -1;
    }
    a.table_out[e] = pg;
    if (c == 0) a.lens_out[i] = len;
}

// ---- release -------------------------------------------------------------------------
struct ReleaseArgs {
    int32_t* table;       // [R, maxp]
    int32_t* ref;         // [num_pages]
    const int32_t* lens;  // [R]
    int R, maxp, num_pages, log2P, window, sinks;
};

__device__ inline void release_entry(const ReleaseArgs& a, long long e) {
    if (e >= (long long)a.R * a.maxp) return;
    const int i = (int)((unsigned)e / (unsigned)a.maxp), c = (int)((unsigned)e % (unsigned)a.maxp);
    const long long len = a.lens[i];
    const long long first = (long long)c << a.log2P, past = (long long)(c + 1) << a.log2P;
    const bool passed = a.window > 0 && first >= a.sinks && past <= len - a.window + 1;
    if (first < len && !passed) return;
    const int pg = a.table[e];
    if ((unsigned)pg >= (unsigned)a.num_pages) return;
    a.table[e] = -1;
    atomicAdd(&a.ref[pg], -1);
}

// ---- reserve -------------------------------------------------------------------------
struct ReserveArgs {
    int32_t* table;            // [R, maxp]
    int32_t* ref;              // [num_pages]
    const int32_t* ctx;        // [R]
    const int32_t* new_lens;   // [R]
    int32_t* copy_src;         // [R]
    int32_t* copy_dst;
    int32_t* copy_tokens;
    int32_t* info;             // [4]
    int R, maxp, num_pages, log2P, chunks;
    // workspace
    int32_t* writers;     // [num_pages] entries of this call that want to write a shared page ...
    int32_t* last;        // [num_pages] ... and the last of them
    int32_t* demand;      // [num_pages] table entry that takes the k-th lowest free page
    int32_t* copy_of;     // [num_pages] its index in the copy list, or -1
    int32_t* upto;        // [R] demands of requests 0 .. i
    int32_t* copies;      // [R] copies of requests 0 .. i
    int32_t* chunk_free;  // [chunks] free pages of each chunk
    const int32_t* was;   // [num_pages] ref, or a copy of it from before the call
};

// the last request whose first entry is at or before e (start[0] = 0, non-decreasing)
__device__ inline int request_of(const int32_t* start, int R, int e) {
    int lo = 0, hi = R - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start[mid] <= e) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <int NT>
struct ReserveLds {
    int32_t start[kReserveReqs + 1];  // first entry of each request, entries in (request, column) order
    uint32_t wsum[NT / 64];
    int32_t limit;  // the first request that can never be served
    int32_t shared;
};

// The demands of the batch, by one workgroup: which entries take a free page, in order. An entry
// that holds a shared page gives it up unless every holder of the page writes it here and
// this is the last: in order, the r-th writer meets ref - r holders.
template <int NT>
__device__ inline void reserve_demands(const ReserveArgs& a, ReserveLds<NT>& lds) {
    const int tid = threadIdx.x;
    if (tid == 0) {
        lds.limit = a.R;
        lds.shared = 0;
    }
    __syncthreads();
    uint32_t E = 0;
    for (int i0 = 0; i0 < a.R; i0 += NT) {
        const int i = i0 + tid;
        uint32_t n = 0;
        if (i < a.R) {
            const int ctx = a.ctx[i], len = a.new_lens[i];
            if (ctx < 0) {
                atomicMin(&lds.limit, i);
            } else if (len > ctx) {
                const unsigned past = ((unsigned)len + (1u << a.log2P) - 1) >> a.log2P;
                if (past > (unsigned)a.maxp) atomicMin(&lds.limit, i);
                else n = past - ((unsigned)ctx >> a.log2P);
            }
        }
        uint32_t total;
        const uint32_t before = block_scan<NT>(n, lds.wsum, total);
        if (i < a.R) lds.start[i] = (int)(E + before);
        E += total;
    }
    if (tid == 0) lds.start[a.R] = (int)E;
    __syncthreads();
    const int limit = lds.limit;
    E = (uint32_t)lds.start[limit];
    struct Entry {
        int i, c, at, page, holders;  // holders: of a valid page, else 0
    };
    auto entry = [&](uint32_t e) {
        Entry x;
        x.i = request_of(lds.start, a.R, (int)e);
        x.c = (a.ctx[x.i] >> a.log2P) + ((int)e - lds.start[x.i]);
        x.at = x.i * a.maxp + x.c;
        x.page = a.table[x.at];
        x.holders = (unsigned)x.page < (unsigned)a.num_pages ? max(a.was[x.page], 1) : 0;
        return x;
    };
    // each thread's first entry is read once (a round's batch rarely has more)
    const Entry first = (uint32_t)tid < E ? entry(tid) : Entry{};
    bool any = false;
    for (uint32_t e = tid; e < E; e += NT) {
        const Entry x = e < NT ? first : entry(e);
        if (x.holders > 1) {
            a.writers[x.page] = 0;
            a.last[x.page] = -1;
            any = true;
        }
    }
    if (any) lds.shared = 1;
    __syncthreads();
    const bool shared = lds.shared != 0;
    if (shared) {
        for (uint32_t e = tid; e < E; e += NT) {
            const Entry x = e < NT ? first : entry(e);
            if (x.holders > 1) {
                atomicAdd(&a.writers[x.page], 1);
                atomicMax(&a.last[x.page], (int)e);
            }
        }
        __syncthreads();
    }
    uint32_t W = 0, C = 0;  // demands and copies so far
    for (uint32_t e0 = 0; e0 < E; e0 += NT) {
        const uint32_t e = e0 + tid;
        bool want = false, copy = false;
        Entry x{};
        if (e < E) {
            x = e < NT ? first : entry(e);
            want = x.holders == 0;
            if (x.holders > 1)
                want = !(load_counted(&a.writers[x.page]) == x.holders && load_counted(&a.last[x.page]) == (int)e);
            const int ctx = a.ctx[x.i];
            copy = want && x.holders > 0 && x.c == ctx >> a.log2P && (ctx & ((1 << a.log2P) - 1)) > 0;
        }
        uint32_t total;
        const uint32_t before = block_scan<NT>((want ? 1u : 0u) | (copy ? 1u << 16 : 0u), lds.wsum, total);
        const uint32_t rank = W + (before & 0xFFFF), crank = C + (before >> 16);
        if (want && rank < (uint32_t)a.num_pages) {
            a.demand[rank] = x.at;
            a.copy_of[rank] = copy ? (int)crank : -1;
        }
        if (e < E && (int)e + 1 == lds.start[x.i + 1]) {  // the request's last entry
            a.upto[x.i] = (int)(rank + want);
            a.copies[x.i] = (int)(crank + copy);
        }
        W += total & 0xFFFF;
        C += total >> 16;
    }
    __syncthreads();
    // requests without entries, and those that are never served
    for (int i = tid; i < a.R; i += NT) {
        if (i >= limit) {
            a.upto[i] = kNeverServed;
            a.copies[i] = 0;
        } else if (lds.start[i + 1] == lds.start[i]) {
            const int j = lds.start[i] > 0 ? request_of(lds.start, a.R, lds.start[i] - 1) : -1;
            a.upto[i] = j < 0 ? 0 : a.upto[j];
            a.copies[i] = j < 0 ? 0 : a.copies[j];
        }
    }
}

// pages of chunk b with (live) or without a holder
template <int NT>
__device__ inline void count_chunk(const int32_t* ref, int num_pages, int b, bool live, int32_t* out, uint32_t* wsum) {
    uint32_t n = 0;
    for (int k = threadIdx.x; k < kPageChunk; k += NT) {
        const int p = b * kPageChunk + k;
        if (p < num_pages) n += (ref[p] > 0) == live && (live || ref[p] == 0);
    }
    uint32_t total;
    block_scan<NT>(n, wsum, total);
    if (threadIdx.x == 0) out[b] = (int)total;
}

// sums of v[0 .. n): before index b, and all
template <int NT>
__device__ inline void sum_chunks(const int32_t* v, int n, int b, uint32_t* wsum, uint32_t& before, uint32_t& all) {
    uint32_t x = 0, y = 0;
    for (int k = threadIdx.x; k < n; k += NT) {
        const uint32_t u = (uint32_t)v[k];
        if (k < b) x += u;
        y += u;
    }
    block_scan<NT>(x, wsum, before);
    block_scan<NT>(y, wsum, all);
}

// with F free pages: the requests that are served and their demands; thread 0 writes info if asked to
template <int NT>
__device__ inline uint32_t reserve_served(const ReserveArgs& a, uint32_t F, bool report, uint32_t* wsum) {
    uint32_t n = 0, served;
    for (int i = threadIdx.x; i < a.R; i += NT) n += a.upto[i] <= (int)F;  // (non-decreasing)
    block_scan<NT>(n, wsum, served);
    const uint32_t S = served ? (uint32_t)a.upto[served - 1] : 0;
    if (report && threadIdx.x == 0) {
        a.info[0] = (int)served;
        a.info[1] = (int)S;
        a.info[2] = served ? a.copies[served - 1] : 0;
        a.info[3] = (int)(F - S);
    }
    return S;
}

// The free pages of chunk b, of which `base` lie before it, to the first S demands. Returns the free pages up to
// its end (or to the last one taken).
template <int NT>
__device__ inline uint32_t reserve_chunk(const ReserveArgs& a, int b, uint32_t base, uint32_t S, uint32_t* wsum) {
    const int tid = threadIdx.x;
    // pages 4 at a time per thread, in the order of their ids
    for (int k0 = 0; k0 < kPageChunk && base < S; k0 += 4 * NT) {
        const int p0 = b * kPageChunk + k0 + 4 * tid;
        int r[4];
        uint32_t m = 0;
        for (int x = 0; x < 4; x++) r[x] = p0 + x < a.num_pages && k0 + 4 * tid + x < kPageChunk ? a.was[p0 + x] : 1;
        for (int x = 0; x < 4; x++) m += r[x] == 0;
        uint32_t total, rank = base + block_scan<NT>(m, wsum, total);
        for (int x = 0; x < 4; x++) {
            if (r[x] != 0) continue;
            if (rank < S && rank < (uint32_t)a.num_pages) {
                const int page = p0 + x, at = a.demand[rank], copy = a.copy_of[rank];
                const int old = a.table[at];
                a.table[at] = page;
                a.ref[page] = 1;
                if ((unsigned)old < (unsigned)a.num_pages) atomicAdd(&a.ref[old], -1);
                if (copy >= 0) {
                    a.copy_src[copy] = old;
                    a.copy_dst[copy] = page;
                    a.copy_tokens[copy] = a.ctx[at / a.maxp] & ((1 << a.log2P) - 1);
                }
            }
            rank++;
        }
        base += total;
    }
    return base;
}

// the assignment by a workgroup per chunk
template <int NT>
__device__ inline void reserve_assign(const ReserveArgs& a, int b, uint32_t* wsum) {
    uint32_t base, F;
    sum_chunks<NT>(a.chunk_free, a.chunks, b, wsum, base, F);
    const uint32_t S = reserve_served<NT>(a, F, b == 0, wsum);
    reserve_chunk<NT>(a, b, base, S, wsum);
}

// All of it by one workgroup. The walk ends with the last page taken, the count needs all.
template <int NT>
__device__ inline void reserve_alone(const ReserveArgs& a, ReserveLds<NT>& lds) {
    uint32_t n = 0, F;
    for (int p = threadIdx.x; p < a.num_pages; p += NT) n += a.was[p] == 0;
    reserve_demands<NT>(a, lds);
    block_scan<NT>(n, lds.wsum, F);
    __syncthreads();  // (the demands are in memory)
    const uint32_t S = reserve_served<NT>(a, F, true, lds.wsum);
    uint32_t base = 0;
    for (int b = 0; b < a.chunks && base < S; b++) base = reserve_chunk<NT>(a, b, base, S, lds.wsum);
}

// ---- compact -------------------------------------------------------------------------
struct CompactArgs {
    int32_t* table;     // [R, maxp]
    int32_t* ref;       // [num_pages]
    int32_t* move_src;  // [limit]
    int32_t* move_dst;
    int32_t* info;      // [2]
    int R, maxp, num_pages, chunks, limit;
    // workspace
    int32_t* chunk_live;  // [chunks]
    int32_t* move_of;     // [num_pages] the move of a page at or above the count of live ones, or -1
};

// With N pages in use, the free pages below N are the lowest free ones, as many as the pages in
// use at or above N, which are the highest: the k-th of either are a move.
template <int NT>
__device__ inline void compact_pair(const CompactArgs& a, int b, uint32_t* wsum) {
    const int tid = threadIdx.x;
    uint32_t base, N;
    sum_chunks<NT>(a.chunk_live, a.chunks, b, wsum, base, N);
    if (b == 0 && tid == 0) {
        a.info[1] = (int)N;
        if (N == (uint32_t)a.num_pages || N == 0) a.info[0] = 0;
    }
    for (int k0 = 0; k0 < kPageChunk; k0 += 4 * NT) {
        const int p0 = b * kPageChunk + k0 + 4 * tid;
        const int room = min(4, min(a.num_pages - p0, kPageChunk - (k0 + 4 * tid)));
        int r[4];
        uint32_t m = 0;
        for (int x = 0; x < 4; x++) r[x] = x < room ? a.ref[p0 + x] : 0;
        for (int x = 0; x < 4; x++) m += r[x] > 0;
        uint32_t total, before = base + block_scan<NT>(m, wsum, total);  // pages in use below p0
        for (int x = 0; x < 4; x++) {
            if (x >= room) continue;
            const uint32_t p = (uint32_t)(p0 + x);
            if (p == N && N > 0) a.info[0] = min((int)(N - before), a.limit);  // free pages below N
            if (p < N) {
                const uint32_t k = p - before;
                if (r[x] <= 0 && k < (uint32_t)a.limit) a.move_dst[k] = (int)p;
            } else {
                const uint32_t k = N - 1 - before;  // pages in use above p
                const bool moves = r[x] > 0 && k < (uint32_t)a.limit;
                if (moves) a.move_src[k] = (int)p;
                a.move_of[p] = moves ? (int)k : -1;
            }
            before += r[x] > 0;
        }
        base += total;
    }
}

// entry e: the table's entries, then the moves' counts
__device__ inline void compact_entry(const CompactArgs& a, long long e) {
    const long long n = (long long)a.R * a.maxp;
    const int N = a.info[1];
    if (e < n) {
        const int pg = a.table[e];
        if (pg < N || pg >= a.num_pages) return;
        const int k = a.move_of[pg];
        if (k >= 0) a.table[e] = a.move_dst[k];
    } else if (e - n < a.info[0]) {
        const int src = a.move_src[e - n], dst = a.move_dst[e - n];
        a.ref[dst] = a.ref[src];
        a.ref[src] = 0;
    }
}

}  // namespace sv
