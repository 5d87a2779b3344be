// Attention over the paged 8-bit cache.  Part of the translation unit wm_pages.cu.
#pragma once

namespace wm {

struct AttendArgs {
    wm_pages p;
    uint32_t page_shift;
    const int32_t* table;
    uint32_t table_stride;
    const int32_t* kv_len;
    const int32_t* q_start;
    uint32_t n;
    const void* q;
    void* out;
    uint64_t q_row, q_head, o_row, o_head;
    float* lse;
    uint32_t n_rows, q_heads, group;
    float scale;
    uint32_t causal, window;
    wm_pages_report* rep;
};

__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_float(__nv_bfloat16& o, float v) { o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(__half& o, float v) { o = __float2half_rn(v); }
__device__ __forceinline__ float code_value(unsigned char c)
{
    const uint32_t h = from_e4m3x2(c);
    return __half2float(*reinterpret_cast<const __half*>(&h));
}

// A block per (row, query head): the scores of 128 tokens, then their values.
template <typename T, int D>
__global__ void __launch_bounds__(128)
k_attend_rows(AttendArgs a)
{
    __shared__ float s_q[D], s_p[128], s_vs[128], s_red[8];
    __shared__ int64_t s_at[128];
    __shared__ uint32_t s_req, s_bad;
    const uint32_t tid = threadIdx.x, row = blockIdx.x, qh = blockIdx.y, h = qh / a.group;
    grid_dep_wait();
    grid_dep_launch();
    if (tid == 0) { s_req = 0xFFFFFFFFu; s_bad = 0; }
    __syncthreads();
    for (uint32_t i = tid; i < a.n; i += 128) {
        const int32_t s = a.q_start[i], e = a.q_start[i + 1], kv = a.kv_len[i];
        const bool ok = s >= 0 && e >= s && (uint32_t)e <= a.n_rows && kv >= 0 && (uint32_t)kv <= (a.table_stride << a.page_shift);
        if (!ok) { if (row == 0 && qh == 0) pages_fault(a.rep, WM_ERR_ARG, i); }
        else if ((int32_t)row >= s && (int32_t)row < e) s_req = i;
    }
    __syncthreads();
    if (s_req == 0xFFFFFFFFu) return;
    const uint32_t i = s_req;
    const int64_t kv = a.kv_len[i], pos = kv - (a.q_start[i + 1] - (int32_t)row);
    int64_t lo = 0, hi = kv;
    if (a.causal) hi = pos + 1 < hi ? pos + 1 : hi;
    if (a.window) lo = pos + 1 - (int64_t)a.window > 0 ? pos + 1 - (int64_t)a.window : 0;
    for (uint32_t d = tid; d < D; d += 128) s_q[d] = to_float(static_cast<const T*>(a.q)[row * a.q_row + qh * a.q_head + d]) * a.scale;
    float m = -INFINITY, l = 0.0f, o = 0.0f;
    for (int64_t t0 = lo; t0 < hi; t0 += 128) {
        __syncthreads();
        const int64_t t = t0 + tid;
        float s = -INFINITY, vs = 0.0f;
        int64_t at = -1;
        if (t < hi) {
            const int32_t page = a.table[(size_t)i * a.table_stride + (t >> a.page_shift)];
            if ((uint32_t)page >= a.p.n_pages) {
                s = vs = NAN;
                pages_fault(a.rep, WM_ERR_ARG, i);
            } else {
                at = (int64_t)page * a.p.page_stride + h * a.p.head_stride + (t & (a.p.page_tokens - 1u)) * a.p.token_stride;
                const unsigned char* k = static_cast<const unsigned char*>(a.p.k) + at;
                float sum = 0.0f;
                for (int d = 0; d < D; d++) sum += s_q[d] * code_value(k[d]);
                s = sum * a.p.k_scale[(size_t)page * a.p.kv_heads + h];
                vs = a.p.v_scale[(size_t)page * a.p.kv_heads + h];
            }
        }
        float top = s;
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        if (tid % 32 == 0) s_red[tid / 32] = top;
        __syncthreads();
        top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
        const float m1 = fmaxf(m, top), base = m1 == -INFINITY ? 0.0f : m1;
        const float keep = __expf(m - base), p = t < hi ? __expf(s - base) : 0.0f;
        float sum = p;
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (tid % 32 == 0) s_red[4 + tid / 32] = sum;
        s_p[tid] = p; s_vs[tid] = vs; s_at[tid] = at;
        __syncthreads();
        l = l * keep + ((s_red[4] + s_red[5]) + (s_red[6] + s_red[7]));
        m = m1;
        if (tid < D) {
            float acc = 0.0f;
            const int n = hi - t0 < 128 ? (int)(hi - t0) : 128;
            for (int j = 0; j < n; j++)
                acc += s_p[j] * s_vs[j] * (s_at[j] < 0 ? 0.0f : code_value(static_cast<const unsigned char*>(a.p.v)[s_at[j] + tid]));
            o = o * keep + acc;
        }
    }
    if (tid < D) {
        T r;
        from_float(r, hi > lo ? o / l : 0.0f);
        static_cast<T*>(a.out)[row * a.o_row + qh * a.o_head + tid] = r;
    }
    if (tid == 0 && a.lse) a.lse[(size_t)row * a.q_heads + qh] = hi > lo ? m + logf(l) : -INFINITY;
}

}  // namespace wm
