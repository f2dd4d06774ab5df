// Rotary positions on several axes, and the append of the rotated keys and the values to the
// paged cache (sv_rope_append). A row's angles are the same in all its heads: the first waves
// compute sine and cosine of each pair once per workgroup into LDS, and the threads then
// turn 16-byte chunks of the heads. The angle is taken in turns, x * (f / 2 pi) in fp64, and only its
// fraction goes to fp32, so a far position loses nothing; sine, cosine and the rotation
// are fp32, with one rounding to the storage type.
// Bound by the copy of the rows (each read and written once) and, for few rows, by the latency of the
// dependent steps: the packing, the page, the rows.
#include <algorithm>

#include "attn_tile.h"
#include "sv_internal.h"

namespace sv {
namespace {

struct RopeArgs {
    const char* q;  // rows q_stride bytes apart
    const char* k;
    const char* v;
    const int32_t* positions;  // [axes, total]
    const double* inv_freq;    // [pairs]
    const int32_t* page_table;
    const int32_t* qo;
    const int32_t* ctx;
    char* q_out;
    char* kc;
    char* vc;
    size_t q_stride, k_stride, v_stride;
    int R, total, Hq, Hkv, d, pairs, axes, cycle, log2P, maxp, num_pages;
    int section[SV_MAX_ROPE_AXES];
    float scale;
    int tasks, tasks_per_head;        // of a row; of a head of q or k
    int turn_chunks, turns, copy_chunks;  // dims of either half: chunks of pairs, with single pairs; chunks passed through
};

constexpr int kMaxPairs = 512;

// the axis of pair p
__device__ inline int pair_axis(const RopeArgs& a, int p) {
    if (a.cycle) {
        const int x = p % a.axes;
        return p / a.axes < a.section[x] ? x : 0;
    }
    int x = 0, past = a.section[0];
    while (x + 1 < a.axes && p >= past) past += a.section[++x];
    return x;
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Chunk;  // 16 bytes of a row as floats, at any element
template <> struct Chunk<float> {
    static constexpr int N = 4;
    typedef u32x4 Any __attribute__((aligned(4)));
    static __device__ void get(const u32x4& x, float* f) {
        f[0] = __uint_as_float(x.x), f[1] = __uint_as_float(x.y), f[2] = __uint_as_float(x.z),
        f[3] = __uint_as_float(x.w);
    }
    static __device__ u32x4 put(const float* f) {
        return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};
template <> struct Chunk<uint16_t> {
    static constexpr int N = 8;
    typedef u32x4 Any __attribute__((aligned(2)));
    static __device__ void get(const u32x4& x, float* f) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            f[2 * e] = __uint_as_float(w[e] << 16);
            f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    }
    static __device__ u32x4 put(const float* f) {
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; e++) b[e] = (__bf16)f[e];
        return __builtin_bit_cast(u32x4, b);
    }
};

__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ inline void store1(float* p, float f) { *p = f; }
__device__ inline void store1(uint16_t* p, float f) { *p = f2bf(f); }

// grid (row, part of the row's tasks). A task turns the pairs of one chunk (adjacent dims) or of two chunks (dims of
// either half), or copies a chunk. Halves that are no whole chunks have their second chunks at any element, and single pairs
// and elements at the end (512 rows of 80 heads with 30 pairs 8.3 us, with 32 pairs 6.6 us; a task per pair and
// element 19 us). STREAM: rows are read and written past the caches. (Two tasks per thread in flight, the first ones under the row's angles and
// page, took 3.5 us instead of 3.2 for 4 rows and 53 instead of 48 for 14996.)
template <typename T, bool ADJ, bool STREAM>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    __shared__ float2 cs[kMaxPairs];
    __shared__ long long s_slot;  // the row's slot in the cache's first kv-head, -1: none
    __shared__ int s_ok;
    constexpr int N = Chunk<T>::N;
    typedef typename Chunk<T>::Any Any;
    const int row = blockIdx.x, tid = threadIdx.x;
    if (row >= a.qo[a.R]) return;
    if (tid < 64) {
        // the request: the last one whose rows start at or before this row, 64 at a time
        int lo = 0, n = a.R;
        while (n > 1) {
            const int step = (n + 63) / 64;
            const int at = lo + tid * step;
            const bool before = tid * step < n && a.qo[min(at, a.R)] <= row;
            const int c = __popcll(__ballot(before));
            lo += max(c - 1, 0) * step;
            n = min(step, n - max(c - 1, 0) * step);
        }
        if (tid == 0) {
            const int q0 = a.qo[lo], q1 = a.qo[lo + 1];
            const bool ok = q0 >= 0 && q0 <= row && row < q1 && q1 <= a.total;
            long long slot = -1;
            const int L = a.ctx[lo];
            if (ok && L >= 0) {
                const long long s = (long long)L + (row - q0), col = s >> a.log2P;
                if (col < a.maxp) {
                    const int pg = a.page_table[(size_t)lo * a.maxp + col];
                    if (pg >= 0 && pg < a.num_pages)
                        slot = (((long long)pg * a.Hkv) << a.log2P) + (s & ((1 << a.log2P) - 1));
                }
            }
            s_ok = ok;
            s_slot = slot;
        }
    }
    for (int p = (tid + 192) & 255; p < a.pairs; p += 256) {
        const double x = a.positions[(size_t)pair_axis(a, p) * a.total + row] * (a.inv_freq[p] * 0.15915494309189535);
        float s, c;
        sincospif((float)(2.0 * (x - rint(x))), &s, &c);
        cs[p] = float2{c * a.scale, s * a.scale};
    }
    __syncthreads();
    if (!s_ok) return;
    const long long slot = s_slot;
    const int heads = a.Hq + a.Hkv, d = a.d, half = a.pairs;
    auto chunk = [](const T* p) -> u32x4 {
        if constexpr (STREAM) return __builtin_nontemporal_load((const Any*)p);
        else return *(const Any*)p;
    };
    auto store = [](T* p, u32x4 x) {
        if constexpr (STREAM) __builtin_nontemporal_store((Any)x, (Any*)p);
        else *(Any*)p = x;
    };
    for (int t = blockIdx.y * 256 + tid; t < a.tasks; t += gridDim.y * 256) {
        const bool value = t >= heads * a.tasks_per_head;
        // head and task in the head; the kinds of tasks one after the other, so that a wave has one kind (with the kinds of
        // each head together 10.5 instead of 8.3 us for 30 pairs)
        int u = value ? t - heads * a.tasks_per_head : t, per = value ? d / N : a.tasks_per_head, c0 = 0;
        if (!ADJ && !value) {
            const int ends[4] = {a.turn_chunks, a.turns, a.turns + a.copy_chunks, a.tasks_per_head};
            per = ends[0];
#pragma unroll
            for (int x = 0; x < 3; x++)
                if (u >= heads * per) {
                    u -= heads * per;
                    c0 = ends[x];
                    per = ends[x + 1] - c0;
                } else {
                    break;
                }
        }
        const int hx = u / per, c = c0 + u % per;
        const bool key = !value && hx >= a.Hq;
        if ((value || key) && slot < 0) continue;
        const int h = key ? hx - a.Hq : hx;
        const T* src = (const T*)((value ? a.v + row * a.v_stride : key ? a.k + row * a.k_stride
                                                                        : a.q + row * a.q_stride)) + (size_t)h * d;
        T* dst = value || key ? (T*)(value ? a.vc : a.kc) + ((size_t)slot + ((size_t)h << a.log2P)) * d
                              : (T*)a.q_out + ((size_t)row * a.Hq + h) * d;
        if (value) {
            store(dst + c * N, chunk(src + c * N));
        } else if constexpr (ADJ) {
            u32x4 raw = chunk(src + c * N);
            if (c * N < 2 * half) {
                float x[N];
                Chunk<T>::get(raw, x);
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const int p = (c * N + e) / 2;
                    if (p >= half) continue;
                    const float2 w = cs[p];
                    const float u0 = x[e] * w.x - x[e + 1] * w.y, u1 = x[e + 1] * w.x + x[e] * w.y;
                    x[e] = u0, x[e + 1] = u1;
                }
                raw = Chunk<T>::put(x);
            }
            store(dst + c * N, raw);
        } else if (c < a.turn_chunks) {
            float x[N], y[N];
            Chunk<T>::get(chunk(src + c * N), x);
            Chunk<T>::get(chunk(src + half + c * N), y);
#pragma unroll
            for (int e = 0; e < N; e++) {
                const float2 w = cs[c * N + e];
                const float u0 = x[e] * w.x - y[e] * w.y, u1 = y[e] * w.x + x[e] * w.y;
                x[e] = u0, y[e] = u1;
            }
            store(dst + c * N, Chunk<T>::put(x));
            store(dst + half + c * N, Chunk<T>::put(y));
        } else if (c < a.turns) {
            const int p = a.turn_chunks * N + (c - a.turn_chunks);
            const float x = load1(src + p), y = load1(src + half + p);
            const float2 w = cs[p];
            store1(dst + p, x * w.x - y * w.y);
            store1(dst + half + p, y * w.x + x * w.y);
        } else if (c < a.turns + a.copy_chunks) {
            const int at = 2 * half + (c - a.turns) * N;
            store(dst + at, chunk(src + at));
        } else {
            const int at = 2 * half + a.copy_chunks * N + (c - a.turns - a.copy_chunks);
            dst[at] = src[at];
        }
    }
}

int ilog2i(int x) {
    int r = 0;
    while ((1 << r) < x) r++;
    return r;
}

}  // namespace

hipError_t launch_rope(const sv_rope_desc& d, const void* q, const void* k_new, const void* v_new,
                       const int32_t* positions, const double* inv_freq, const int32_t* page_table,
                       const int32_t* qo_indptr, const int32_t* ctx_lens, void* q_out, void* k_cache, void* v_cache,
                       hipStream_t stream) {
    const int esz = d.dtype == SV_F32 ? 4 : 2, N = 16 / esz;
    RopeArgs a{};
    a.q = (const char*)q;
    a.k = (const char*)k_new;
    a.v = (const char*)v_new;
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.page_table = page_table;
    a.qo = qo_indptr;
    a.ctx = ctx_lens;
    a.q_out = (char*)q_out;
    a.kc = (char*)k_cache;
    a.vc = (char*)v_cache;
    a.q_stride = (size_t)(d.q_stride ? d.q_stride : d.num_q_heads * d.head_dim) * esz;
    a.k_stride = (size_t)(d.k_stride ? d.k_stride : d.num_kv_heads * d.head_dim) * esz;
    a.v_stride = (size_t)(d.v_stride ? d.v_stride : d.num_kv_heads * d.head_dim) * esz;
    a.R = d.num_reqs;
    a.total = d.total_max;
    a.Hq = d.num_q_heads;
    a.Hkv = d.num_kv_heads;
    a.d = d.head_dim;
    a.pairs = d.rot_dim / 2;
    a.axes = d.num_axes;
    a.cycle = d.order == SV_ROPE_CYCLE;
    for (int x = 0; x < d.num_axes; x++) a.section[x] = d.section[x];
    a.log2P = ilog2i(d.page_size);
    a.maxp = d.max_pages_per_req;
    a.num_pages = d.num_pages;
    a.scale = d.scale == 0.0f ? 1.0f : d.scale;
    const bool adj = d.pairing == SV_ROPE_ADJACENT;
    const int rest = d.head_dim - d.rot_dim;
    a.turn_chunks = a.pairs / N;
    a.turns = a.turn_chunks + a.pairs % N;
    a.copy_chunks = rest / N;
    a.tasks_per_head = adj ? d.head_dim / N : a.turns + a.copy_chunks + rest % N;
    a.tasks = (d.num_q_heads + d.num_kv_heads) * a.tasks_per_head + d.num_kv_heads * (d.head_dim / N);
    // a row is divided among workgroups where the rows alone are too few
    const int parts = std::max(1, std::min((a.tasks + 255) / 256, 2048 / d.total_max));
    const dim3 grid(d.total_max, parts);
    // Rows of many megabytes go past the caches both ways. 14996 rows (138 MB in, as much out): 47 us, through the caches
    // 55 us from memory and 47 us where the rows still lie in the last-level cache; 7500 rows 26 us, 32 and 23 us. Fewer rows
    // were just written and are about to be read: 512 rows 6.5 us past the caches, 5.9 us through them. Halves that are no
    // whole chunks write lines in parts, which the caches put together (14996 rows with 55 pairs 79 us, past them 121 us).
    const bool past = (adj || a.pairs % N == 0) && (size_t)d.total_max * (d.num_q_heads + 2 * d.num_kv_heads) * d.head_dim * esz > (size_t)64 << 20;
#define SV_ROPE(T, ADJ) \
    if (past) hipLaunchKernelGGL((rope_kernel<T, ADJ, true>), grid, dim3(256), 0, stream, a); \
    else hipLaunchKernelGGL((rope_kernel<T, ADJ, false>), grid, dim3(256), 0, stream, a)
#define SV_ROPE_TYPE(T) \
    if (adj) { SV_ROPE(T, true); } \
    else { SV_ROPE(T, false); }
    if (d.dtype == SV_F32) { SV_ROPE_TYPE(float) }
    else { SV_ROPE_TYPE(uint16_t) }
#undef SV_ROPE_TYPE
#undef SV_ROPE
    return hipGetLastError();
}

}  // namespace sv
