// Pages of the cache between rounds: fork, reserve (with copy-on-write), release and compact work on
// the page table and the counts (pages_ops.h), sv_copy_pages moves the data. All of it is integer
// arithmetic and copies, so results do not depend on the order the GPU works in: counts change by
// atomic sums, and everything that has an order (which page, which move) comes from scans.
#include <algorithm>

#include "pages_ops.h"
#include "sv_internal.h"

namespace sv {
namespace {

constexpr int kWalkThreads = 1024;
static_assert(kPageChunk == kPageChunkSize && kReserveReqs == SV_MAX_RESERVE_REQS, "the host sizes the workspace");

__global__ __launch_bounds__(256) void fork_kernel(ForkArgs a) {
    fork_entry(a, (long long)blockIdx.x * 256 + threadIdx.x);
}

__global__ __launch_bounds__(256) void release_kernel(ReleaseArgs a) {
    release_entry(a, (long long)blockIdx.x * 256 + threadIdx.x);
}

// workgroup 0: the demands; the others: the free pages of a chunk each
__global__ __launch_bounds__(kWalkThreads) void reserve_demand_kernel(ReserveArgs a) {
    __shared__ ReserveLds<kWalkThreads> lds;
    if (blockIdx.x == 0) reserve_demands<kWalkThreads>(a, lds);
    else count_chunk<kWalkThreads>(a.ref, a.num_pages, blockIdx.x - 1, false, a.chunk_free, lds.wsum);
}

__global__ __launch_bounds__(kWalkThreads) void reserve_assign_kernel(ReserveArgs a) {
    __shared__ uint32_t wsum[kWalkThreads / 64];
    reserve_assign<kWalkThreads>(a, blockIdx.x, wsum);
}

// At most one chunk of pages: the counts and all that lies in the workspace otherwise fit the LDS, which takes most
// round trips to memory out of the chain (a round's reserve and release with 4000 pages 11.9 us; with the workspace in
// memory 12.4 us).
__global__ __launch_bounds__(kWalkThreads) void reserve_alone_kernel(ReserveArgs a) {
    __shared__ ReserveLds<kWalkThreads> lds;
    __shared__ int32_t was[kPageChunk], writers[kPageChunk], last[kPageChunk], demand[kPageChunk], copy_of[kPageChunk];
    __shared__ int32_t upto[kReserveReqs], copies[kReserveReqs];
    if (a.num_pages > kPageChunk) return;  // (plan_reserve takes this kernel for one chunk only; the arrays above hold no more)
    for (int p = threadIdx.x; p < a.num_pages; p += kWalkThreads) was[p] = a.ref[p];
    a.was = was, a.writers = writers, a.last = last, a.demand = demand, a.copy_of = copy_of, a.upto = upto, a.copies = copies;
    __syncthreads();
    reserve_alone<kWalkThreads>(a, lds);
}

__global__ __launch_bounds__(kWalkThreads) void compact_count_kernel(CompactArgs a) {
    __shared__ uint32_t wsum[kWalkThreads / 64];
    count_chunk<kWalkThreads>(a.ref, a.num_pages, blockIdx.x, true, a.chunk_live, wsum);
}

__global__ __launch_bounds__(kWalkThreads) void compact_pair_kernel(CompactArgs a) {
    __shared__ uint32_t wsum[kWalkThreads / 64];
    compact_pair<kWalkThreads>(a, blockIdx.x, wsum);
}

__global__ __launch_bounds__(256) void compact_entry_kernel(CompactArgs a) {
    compact_entry(a, (long long)blockIdx.x * 256 + threadIdx.x);
}

// ---- copies ----------------------------------------------------------------------------
struct CopyArgs {
    const int32_t* src;     // [max_copies]
    const int32_t* dst;
    const int32_t* tokens;  // [max_copies] or NULL
    const int32_t* count;   // [1]
    char* kc;
    char* vc;
    size_t layer_bytes;
    int max_copies, layers, heads, P, num_pages;
    unsigned row_vecs;   // 16-byte vectors per token and head
    unsigned pieces;     // pieces per page and cache
};

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
constexpr int kCopyLoads = 4;                   // vectors in flight per thread
constexpr unsigned kPiece = 256 * kCopyLoads;   // vectors per piece (16 KB)
static_assert(kPiece * 16 == kCopyPieceBytes, "the host bounds the pieces of a copy");

// Bound by HBM: every byte is read and written once, past the caches (3930 pages of 32 KB in two layers and two
// caches, 1.03 GB: 209 us with ordinary loads and stores, 193 us so; a large plain copy runs at 4.9 TB/s). A workgroup
// walks (copy, layer, cache, piece) items; the vectors of the live tokens alone are numbered, head
// after head. Eight vectors per thread instead of four took 1.5 times as long.
__global__ __launch_bounds__(256) void copy_pages_kernel(CopyArgs a) {
    const long long n = min(*a.count, a.max_copies);
    const long long per_copy = 2LL * a.layers * a.pieces;
    for (long long item = blockIdx.x; item < n * per_copy; item += gridDim.x) {
        const int e = (int)(item / per_copy);
        const unsigned rest = (unsigned)(item % per_copy);
        const unsigned piece = rest % a.pieces, lt = rest / a.pieces;
        const int src = a.src[e], dst = a.dst[e];
        if ((unsigned)src >= (unsigned)a.num_pages || (unsigned)dst >= (unsigned)a.num_pages) continue;
        const int live = a.tokens ? min(max(a.tokens[e], 0), a.P) : a.P;
        const unsigned head_live = (unsigned)live * a.row_vecs, head_vecs = (unsigned)a.P * a.row_vecs;
        const unsigned nv = head_live * (unsigned)a.heads;
        const unsigned v0 = piece * kPiece + threadIdx.x;
        if (piece * kPiece >= nv) continue;
        char* base = (lt & 1 ? a.vc : a.kc) + (size_t)(lt >> 1) * a.layer_bytes;
        const size_t page_vecs = (size_t)head_vecs * a.heads;
        const u32x4* from = (const u32x4*)base + (size_t)src * page_vecs;
        u32x4* to = (u32x4*)base + (size_t)dst * page_vecs;
        u32x4 x[kCopyLoads];
        unsigned at[kCopyLoads];
#pragma unroll
        for (int k = 0; k < kCopyLoads; k++) {
            const unsigned v = v0 + 256 * k;
            at[k] = live == a.P ? v : v / head_live * head_vecs + v % head_live;
            if (v < nv) x[k] = __builtin_nontemporal_load(from + at[k]);
        }
#pragma unroll
        for (int k = 0; k < kCopyLoads; k++)
            if (v0 + 256 * k < nv) __builtin_nontemporal_store(x[k], to + at[k]);
    }
}

int ilog2i(int x) {
    int r = 0;
    while ((1 << r) < x) r++;
    return r;
}

unsigned grid_of(long long n) { return (unsigned)((n + 255) / 256); }

}  // namespace

hipError_t launch_fork(const sv_pages_desc& d, int rows_in, const int32_t* table_in, const int32_t* lens_in,
                       const int32_t* parent, int32_t* table_out, int32_t* lens_out, int32_t* ref,
                       hipStream_t stream) {
    const ForkArgs a{table_in, lens_in, parent, table_out, lens_out, ref, d.num_reqs, rows_in, d.max_pages_per_req,
                     d.num_pages, ilog2i(d.page_size)};
    const long long n = ((long long)d.num_reqs + rows_in) * d.max_pages_per_req;
    hipLaunchKernelGGL(fork_kernel, dim3(grid_of(n)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_release(const sv_pages_desc& d, int window, int sinks, int32_t* table, int32_t* ref,
                          const int32_t* lens, hipStream_t stream) {
    const ReleaseArgs a{table, ref, lens, d.num_reqs, d.max_pages_per_req, d.num_pages, ilog2i(d.page_size), window,
                        sinks};
    hipLaunchKernelGGL(release_kernel, dim3(grid_of((long long)d.num_reqs * d.max_pages_per_req)), dim3(256), 0,
                       stream, a);
    return hipGetLastError();
}

hipError_t launch_reserve(const sv_pages_desc& d, const ReservePlan& p, int32_t* table, int32_t* ref,
                          const int32_t* ctx, const int32_t* new_lens, int32_t* copy_src, int32_t* copy_dst,
                          int32_t* copy_tokens, int32_t* info, void* ws, hipStream_t stream) {
    int32_t* w = (int32_t*)ws;
    const ReserveArgs a{table, ref, ctx, new_lens, copy_src, copy_dst, copy_tokens, info, d.num_reqs,
                        d.max_pages_per_req, d.num_pages, ilog2i(d.page_size), p.chunks, w + p.writers, w + p.last,
                        w + p.demand, w + p.copy_of, w + p.upto, w + p.copies, w + p.chunk_free, ref};
    if (p.alone) {
        hipLaunchKernelGGL(reserve_alone_kernel, dim3(1), dim3(kWalkThreads), 0, stream, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(reserve_demand_kernel, dim3(1 + p.chunks), dim3(kWalkThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(reserve_assign_kernel, dim3(p.chunks), dim3(kWalkThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_compact(const sv_pages_desc& d, const CompactPlan& p, int32_t* table, int32_t* ref,
                          int32_t* move_src, int32_t* move_dst, int32_t* info, void* ws, hipStream_t stream) {
    int32_t* w = (int32_t*)ws;
    const CompactArgs a{table, ref, move_src, move_dst, info, d.num_reqs, d.max_pages_per_req, d.num_pages, p.chunks,
                        p.limit, w + p.chunk_live, w + p.move_of};
    hipLaunchKernelGGL(compact_count_kernel, dim3(p.chunks), dim3(kWalkThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(compact_pair_kernel, dim3(p.chunks), dim3(kWalkThreads), 0, stream, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(compact_entry_kernel,
                       dim3(grid_of((long long)d.num_reqs * d.max_pages_per_req + p.limit)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_copy(const sv_copy_desc& d, const int32_t* src, const int32_t* dst, const int32_t* tokens,
                       const int32_t* count, void* k_cache, void* v_cache, hipStream_t stream) {
    const size_t esz = d.dtype == SV_F32 ? 4 : 2;
    const unsigned row_vecs = (unsigned)(d.head_dim * esz / 16);
    const size_t page_vecs = (size_t)row_vecs * d.page_size * d.num_kv_heads;
    const size_t layer = d.layer_stride ? (size_t)d.layer_stride * esz : page_vecs * 16 * d.num_pages;
    const CopyArgs a{src, dst, tokens, count, (char*)k_cache, (char*)v_cache, layer, d.max_copies, d.num_layers,
                     d.num_kv_heads, d.page_size, d.num_pages, row_vecs,
                     (unsigned)((page_vecs + kPiece - 1) / kPiece)};
    const long long items = 2LL * d.max_copies * d.num_layers * a.pieces;
    hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)std::min<long long>(items, 256 * 8)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sv
