// Attention with a sliding window and visible first tokens over the paged cache (sv_window_attn).
// The row at position p sees the keys s <= p with s < S or s > p - W:
//     z_s = scale <q, K_s>,  lse = ln sum exp(z_s),  o = sum exp(z_s - lse) V_s.
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
    int R, total_q, Hq, Hkv, G, block, HD;
    int log2P, maxp, num_pages, max_kv_len;
    int window, sinks;
    float scale;  // sm_scale
};

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

// One workgroup of four waves per (query row, head); wave w takes every fourth run of 64 of the
// row's visible keys, and the waves' softmax states are merged at the end.
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
    const int q0 = a.qo[lo], k_i = a.qo[lo + 1] - q0;
    const int kv_len = min(a.kv_lens[lo], a.max_kv_len);
    if (!rows_in_batch(q0, k_i, a.block, a.total_q) || kv_len < k_i || row < q0 || row >= q0 + k_i) return;
    const int p = kv_len - k_i + (row - q0);
    const int first = max(0, p - a.window + 1), head_n = min(a.sinks, first), n = head_n + p - first + 1;
    const T* qp = (const T*)a.q + ((size_t)row * a.Hq + head) * HD;
    const int32_t* pt = a.page_table + (size_t)lo * a.maxp;
    const int P = 1 << a.log2P, h = head / a.G;
    float o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.0f;
    for (int base = 64 * wv; base < n; base += 256) {
        const int t = base + lane;
        float z = -INFINITY;
        size_t off = 0;
        bool ok = false;
        if (t < n) {
            const int s = t < head_n ? t : first + (t - head_n);
            const int col = s >> a.log2P, pg = col < a.maxp ? pt[col] : -1;
            if (pg >= 0 && pg < a.num_pages) {
                off = ((((size_t)pg * a.Hkv + h) << a.log2P) + (s & (P - 1))) * HD;
                float dot = 0.0f;
                for (int e = 0; e < HD; e += 4) {
                    const f32x4 x = Vec4<T>::get((const T*)a.kc + off + e), y = Vec4<T>::get(qp + e);
                    dot += x[0] * y[0] + x[1] * y[1] + x[2] * y[2] + x[3] * y[3];
                }
                z = dot * a.scale;
                ok = true;
            }
        }
        float mx = z;
        for (int x = 32; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x, 64));
        const float m_new = fmaxf(m, mx);
        const bool any_nan = __any(ok && z != z);
        if (m_new == -INFINITY && !any_nan) continue;
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
        const float mw = s_ml[w][0], wt = mw == -INFINITY ? 0.0f : expf(mw - M);
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

int ilog2(int x) {
    int r = 0;
    while ((1 << r) < x) r++;
    return r;
}

}  // namespace

hipError_t launch_window(const sv_window_desc& w, const void* q, const void* k_cache, const void* v_cache,
                         const int32_t* page_table, const int32_t* qo_indptr, const int32_t* kv_lens, void* out,
                         float* lse, void* ws, hipStream_t stream) {
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
    a.scale = d.sm_scale > 0.0f ? d.sm_scale : 1.0f / sqrtf((float)d.head_dim);
    const dim3 grid(d.total_q_max * d.num_q_heads);
    if (d.dtype == SV_F32) hipLaunchKernelGGL(window_rows_kernel<float>, grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(window_rows_kernel<uint16_t>, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sv
