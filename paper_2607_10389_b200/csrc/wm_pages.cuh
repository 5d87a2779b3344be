// The paged 8-bit cache: block tables and slot maps from lengths (k_pages_plan), new keys and
// values into the pool (k_pages_append).  Attention over it: wm_attend.cuh.
// Part of the translation unit wm_pages.cu.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

namespace wm {

constexpr uint32_t kMaxRequests = WM_PAGES_MAX_REQUESTS;        // 3 prefix sums of them take 48 KB of shared memory

// The record of a pages call, written only where something is wrong: the lowest status and the lowest index.
__device__ __forceinline__ void pages_fault(wm_pages_report* rep, int32_t status, uint32_t index)
{
    if (!rep) return;
    atomicMin(&rep->status, status);
    uint32_t cur = *reinterpret_cast<volatile uint32_t*>(&rep->first);
    while (cur == 0u || cur > index + 1u) {
        const uint32_t seen = atomicCAS(&rep->first, cur, index + 1u);
        if (seen == cur) break;
        cur = seen;
    }
}

// ------------------------------------------------------------------ wm_pages_plan

struct PlanArgs {
    const int32_t* old_len;
    const int32_t* new_len;
    uint32_t n, page, page_shift, n_pages;
    int32_t* table;
    uint32_t stride;
    int32_t* free_pages;
    const uint32_t* free_count;
    uint32_t* free_count_out;
    int32_t* start;
    int32_t* slots;
    uint32_t n_slots;
    uint32_t slots_apart;       // the slots are k_pages_slots'
    wm_pages_report* rep;
};

constexpr uint32_t kPlanThreads = 1024;
constexpr uint32_t kPlanPer = (kMaxRequests + kPlanThreads - 1) / kPlanThreads;    // requests a thread scans
constexpr uint32_t kPlanBlocks = 8;                             // of a cluster
// Slots up to which k_pages_plan lists them itself.  Measured in a graph (us, there and in a kernel of their own): 256 requests with a
// token each 4.0 and 6.6, 4000 6.5 and 10.2; 5,800 slots of 200 requests 8.2 and 6.6, 11,600 13.2 and 6.5.
constexpr uint32_t kPlanSlots = 4096;

// The last i with s[i] <= x (s ascending, s[0] = 0, s[n] > x).
__device__ __forceinline__ uint32_t last_not_above(const uint32_t* s, uint32_t n, uint32_t x)
{
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (s[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Every block of the cluster scans all lengths (16 KB at most, from L2) and keeps the three prefix sums (tokens, pages
// taken, pages given back) in shared memory; then the blocks share the outputs.  A token's page is looked up where it
// comes from (the table's old part, or the free list), never where this call writes it, so the blocks need no order
// among themselves; the one word that is read and written by different blocks is the free count (in a graph it
// is updated in place), hence the cluster with one barrier behind the reading.
template <bool CLUSTER>
__global__ void __launch_bounds__(kPlanThreads)
k_pages_plan(PlanArgs a)
{
    extern __shared__ uint32_t plan_smem[];
    uint32_t* s_tok = plan_smem;                        // [n + 1]
    uint32_t* s_take = s_tok + a.n + 1;
    uint32_t* s_give = s_take + a.n + 1;
    __shared__ unsigned long long s_w[3][32];
    __shared__ uint32_t s_bad_arg, s_bad_cap;           // 1 + the lowest request concerned
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    grid_dep_wait();
    grid_dep_launch();
    if (tid == 0) s_bad_arg = s_bad_cap = 0xFFFFFFFFu;
    const uint32_t have = ld_volatile_u32(a.free_count);
    __syncthreads();

    unsigned long long tok[kPlanPer], mine_tok = 0;
    uint32_t take[kPlanPer], give[kPlanPer], mine_take = 0, mine_give = 0;
    const uint32_t per = (a.n + kPlanThreads - 1) / kPlanThreads;       // consecutive requests a thread
#pragma unroll
    for (uint32_t k = 0; k < kPlanPer; k++) {
        const uint32_t i = per * tid + k;
        tok[k] = 0; take[k] = 0; give[k] = 0;
        if (k < per && i < a.n) {
            const int32_t o = a.old_len[i], w = a.new_len[i];
            const uint32_t held = ((uint32_t)o + a.page - 1u) >> a.page_shift, want = ((uint32_t)w + a.page - 1u) >> a.page_shift;
            if (o < 0 || w < 0 || held > a.stride) atomicMin(&s_bad_arg, i);
            else if (want > a.stride) atomicMin(&s_bad_cap, i);
            else {
                tok[k] = w > o ? (uint32_t)(w - o) : 0u;
                take[k] = want > held ? want - held : 0u;
                give[k] = held > want ? held - want : 0u;
            }
        }
        mine_tok += tok[k]; mine_take += take[k]; mine_give += give[k];
    }
    unsigned long long it = mine_tok;
    uint32_t ia = mine_take, ig = mine_give;
#pragma unroll
    for (uint32_t d = 1; d < 32; d <<= 1) {
        const unsigned long long ot = __shfl_up_sync(0xFFFFFFFFu, it, d);
        const uint32_t oa = __shfl_up_sync(0xFFFFFFFFu, ia, d), og = __shfl_up_sync(0xFFFFFFFFu, ig, d);
        if (lane >= d) { it += ot; ia += oa; ig += og; }
    }
    if (lane == 31) { s_w[0][warp] = it; s_w[1][warp] = ia; s_w[2][warp] = ig; }
    __syncthreads();
    unsigned long long rt = it - mine_tok, total_tok = 0;
    uint32_t ra = ia - mine_take, rg = ig - mine_give, total_take = 0, total_give = 0;
    {
        unsigned long long t = s_w[0][lane];
        uint32_t x = (uint32_t)s_w[1][lane], g = (uint32_t)s_w[2][lane];
        unsigned long long bt = lane < warp ? t : 0;
        uint32_t bx = lane < warp ? x : 0, bg = lane < warp ? g : 0;
#pragma unroll
        for (uint32_t d = 16; d; d >>= 1) {
            t += __shfl_xor_sync(0xFFFFFFFFu, t, d);
            bt += __shfl_xor_sync(0xFFFFFFFFu, bt, d);
        }
        total_tok = t; rt += bt;
        total_take = __reduce_add_sync(0xFFFFFFFFu, x); total_give = __reduce_add_sync(0xFFFFFFFFu, g);
        ra += __reduce_add_sync(0xFFFFFFFFu, bx); rg += __reduce_add_sync(0xFFFFFFFFu, bg);
    }
    const bool bad_list = have > a.n_pages || (unsigned long long)have + total_give > (unsigned long long)a.n_pages + total_take;
    const bool bad_arg = s_bad_arg != 0xFFFFFFFFu || bad_list;
    const bool bad_cap = s_bad_cap != 0xFFFFFFFFu || total_tok > a.n_slots || (unsigned long long)total_take > (unsigned long long)have + total_give;
    const bool bad = bad_arg || bad_cap;
#pragma unroll
    for (uint32_t k = 0; k < kPlanPer; k++) {
        const uint32_t i = per * tid + k;
        if (k < per && i < a.n) { s_tok[i] = (uint32_t)rt; s_take[i] = ra; s_give[i] = rg; }
        rt += tok[k]; ra += take[k]; rg += give[k];
    }
    if (tid == 0) { s_tok[a.n] = (uint32_t)total_tok; s_take[a.n] = total_take; s_give[a.n] = total_give; }
    if (CLUSTER) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }

    const uint32_t gid = blockIdx.x * kPlanThreads + tid, step = gridDim.x * kPlanThreads;
    const uint32_t after = have + total_give - total_take;
    if (gid == 0) {
        *a.free_count_out = bad ? have : after;
        if (bad_arg) pages_fault(a.rep, WM_ERR_ARG, s_bad_arg != 0xFFFFFFFFu ? s_bad_arg : 0u);
        if (bad_cap) pages_fault(a.rep, WM_ERR_CAPACITY, s_bad_cap != 0xFFFFFFFFu ? s_bad_cap : 0u);
    }
    for (uint32_t i = gid; i <= a.n; i += step) a.start[i] = bad ? 0 : (int32_t)s_tok[i];
    if (bad) {
        if (a.slots_apart) return;
        for (uint32_t t = gid; t < a.n_slots; t += step) a.slots[t] = -1;
        return;
    }
    // the k-th page given back, and the page that the k-th taker gets
    auto given = [&](uint32_t k) {
        const uint32_t i = last_not_above(s_give, a.n, k);
        const uint32_t want = ((uint32_t)a.new_len[i] + a.page - 1u) >> a.page_shift;
        return a.table[(size_t)i * a.stride + want + (k - s_give[i])];
    };
    auto taken = [&](uint32_t k) {
        const uint32_t at = have + total_give - 1u - k;
        return at < have ? a.free_pages[at] : given(at - have);
    };
    for (uint32_t k = gid; k < total_take; k += step) {
        const uint32_t i = last_not_above(s_take, a.n, k);
        const uint32_t held = ((uint32_t)a.old_len[i] + a.page - 1u) >> a.page_shift;
        a.table[(size_t)i * a.stride + held + (k - s_take[i])] = taken(k);
    }
    for (uint32_t at = have + gid; at < after; at += step) a.free_pages[at] = given(at - have);
    if (a.slots_apart) return;
    for (uint32_t t = gid; t < a.n_slots; t += step) {
        int32_t slot = -1;
        if (t < (uint32_t)total_tok) {
            const uint32_t i = last_not_above(s_tok, a.n, t);
            const uint32_t old = (uint32_t)a.old_len[i], pos = old + (t - s_tok[i]);
            const uint32_t held = (old + a.page - 1u) >> a.page_shift, at = pos >> a.page_shift;
            const int32_t page = at < held ? a.table[(size_t)i * a.stride + at] : taken(s_take[i] + (at - held));
            if ((uint32_t)page < a.n_pages) slot = (int32_t)(((uint32_t)page << a.page_shift) + (pos & (a.page - 1u)));
            else pages_fault(a.rep, WM_ERR_ARG, i);
        }
        a.slots[t] = slot;
    }
}

// Many slots, behind k_pages_plan: the table is complete, and the row offsets say which request a token is (a failed plan's
// are all zero: every slot -1).  A thread has four tokens.  Measured: 1000 requests, 427,000 slots, pages of 16: 66 us with the slots in
// k_pages_plan's eight blocks, 11 us this way.
__global__ void __launch_bounds__(kPlanThreads)
k_pages_slots(PlanArgs a)
{
    extern __shared__ uint32_t slots_smem[];            // [n + 1] the row offsets
    grid_dep_wait();
    grid_dep_launch();
    for (uint32_t i = threadIdx.x; i <= a.n; i += kPlanThreads) slots_smem[i] = (uint32_t)a.start[i];
    __syncthreads();
    const uint32_t total = slots_smem[a.n];
    for (uint32_t t0 = (blockIdx.x * kPlanThreads + threadIdx.x) * 4u; t0 < a.n_slots; t0 += gridDim.x * kPlanThreads * 4u) {
        int32_t slot[4] = {-1, -1, -1, -1};
        if (t0 < total) {
            uint32_t i = last_not_above(slots_smem, a.n, t0), at_page = 0xFFFFFFFFu;
            int32_t page = -1;
#pragma unroll
            for (uint32_t k = 0; k < 4; k++) {
                const uint32_t t = t0 + k;
                if (t >= total) break;
                while (t >= slots_smem[i + 1]) { i++; at_page = 0xFFFFFFFFu; }
                const uint32_t pos = (uint32_t)a.old_len[i] + (t - slots_smem[i]), at = pos >> a.page_shift;
                if (at != at_page) { page = a.table[(size_t)i * a.stride + at]; at_page = at; }
                if ((uint32_t)page < a.n_pages) slot[k] = (int32_t)(((uint32_t)page << a.page_shift) + (pos & (a.page - 1u)));
                else pages_fault(a.rep, WM_ERR_ARG, i);
            }
        }
        if (t0 + 4u <= a.n_slots && (reinterpret_cast<uintptr_t>(a.slots) & 15u) == 0) {
            *reinterpret_cast<int4*>(a.slots + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
        } else {
#pragma unroll
            for (uint32_t k = 0; k < 4; k++)
                if (t0 + k < a.n_slots) a.slots[t0 + k] = slot[k];
        }
    }
}

// ------------------------------------------------------------------ wm_pages_append

struct AppendArgs {
    wm_pages p;
    uint32_t page_shift;
    const void* src[2];             // keys, values
    uint64_t row_stride[2], head_stride[2];
    const int32_t* slots;
    uint32_t n_rows, per_warp;
    wm_pages_report* rep;
};

__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t w, __half)
{
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

// N consecutive elements as floats.
template <typename T, int N> __device__ __forceinline__ void load_row(const T* p, float (&x)[N])
{
    constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    if constexpr (kWords == 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (kWords == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; i++) {
            const float2 f = unpack2(w[i], T());
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    }
}

// Two values to two e4m3 codes (lo in the low byte), to nearest even; finite overflow and infinities become +-448, NaN stays.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two codes to two halves (exact: e4m3 is a subset of half).
__device__ __forceinline__ uint32_t from_e4m3x2(uint32_t codes)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
    return r;
}

// The smallest power of two s with amax <= 448 s = 1.75 * 2^8 s, not below 2^-126 (bit arithmetic, so exact).
__device__ __forceinline__ float scale_for(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(e < 1 ? 1 : e) << 23);
}
// The power of two that is not below s (s >= 0 and finite; not below 2^-126).
__device__ __forceinline__ float power_not_below(float s)
{
    const uint32_t u = __float_as_uint(s);
    const uint32_t e = (u >> 23) + ((u & 0x7FFFFFu) ? 1u : 0u);
    return __uint_as_float((e < 1u ? 1u : e > 254u ? 254u : e) << 23);
}

// a * b with what does not fit in 32 bits kept as an odd last bit: rounded to fewer bits afterwards, it goes where the exact
// product would (a product rounded to nearest can come to lie on the middle of two codes).  Below the normal floats it is too small for
// any code.
__device__ __forceinline__ float product_to_odd(float a, float b)
{
    const float p = __fmul_rz(a, b);
    return __uint_as_float(__float_as_uint(p) | (fmaf(a, b, -p) != 0.0f ? 1u : 0u));
}

// Eight elements a lane, LPR lanes a row.
template <typename T> __device__ __forceinline__ void load8(const T* p, uint32_t (&w)[2 * sizeof(T)])
{
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    if constexpr (sizeof(T) == 4) {
        const uint4 u = *reinterpret_cast<const uint4*>(p + 4);
        w[4] = u.x; w[5] = u.y; w[6] = u.z; w[7] = u.w;
    }
}
template <typename T> __device__ __forceinline__ void unpack8(const uint32_t (&w)[2 * sizeof(T)], float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 f = unpack2(w[i], T());
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    }
}

// A warp takes one run of rows that go into one page, for one head, keys or values: its largest value first, then the codes of
// what the page keeps (only if the scale has grown), then the new rows'.  Bound by memory where runs are long (rows in once, codes
// out once: 103 MB of prompts in 20 us, 0.78 of the copy rate), by the chain slot, row, scale, code where they are short (3.5 us).  A warp looks at `a.per_warp` rows for the firsts of runs,
// with a lane for each (one row a warp, prompts spent most of the call on starting warps that had nothing to do); a run of up to
// kRows rows stays in registers between the two looks at it, of a longer one the last kRows do.
// KL: loads in registers; few where a warp looks at one row and most runs are short (so that all warps fit at once), else as many as pay.
template <typename T, int D, int KL>
__global__ void __launch_bounds__(128)
k_pages_append(AppendArgs a)
{
    constexpr uint32_t LPR = D / 8, RPL = 32 / LPR, kRows = KL * RPL;      // lanes a row, rows a load
    const uint32_t lane = threadIdx.x % 32, part = lane % LPR, sub = lane / LPR;
    const uint32_t units = 2u * a.p.kv_heads, job = blockIdx.x * 4u + threadIdx.x / 32, unit = job % units, row0 = job / units * a.per_warp;
    grid_dep_wait();
    grid_dep_launch();
    if (row0 >= a.n_rows) return;
    const uint32_t head = unit >> 1, side = unit & 1u;
    const uint32_t n_slots = a.p.n_pages << a.page_shift, mask = a.p.page_tokens - 1u;
    // the next 32 slots, and the one before: runs that end among them need no further look
    const uint32_t r = row0 + lane;
    const int32_t slot = r < a.n_rows ? a.slots[r] : -1;
    int32_t before = lane == 0 && r > 0 ? a.slots[r - 1] : -1;
    {
        const int32_t up = __shfl_up_sync(0xFFFFFFFFu, slot, 1);
        if (lane > 0) before = up;
    }
    bool leads = false;
    if (lane < a.per_warp && r < a.n_rows) {
        if (slot != -1) {
            bool wrong = (uint32_t)slot >= n_slots;
            if (!wrong) {
                const bool same = (uint32_t)before < n_slots && (uint32_t)before >> a.page_shift == (uint32_t)slot >> a.page_shift;
                wrong = same && before + 1 != slot;
                leads = !same;
            }
            if (wrong && unit == 0u) pages_fault(a.rep, WM_ERR_ARG, r);
        }
    }
    for (uint32_t todo = __ballot_sync(0xFFFFFFFFu, leads); todo; todo &= todo - 1u) {
        const uint32_t at = __ffs((int)todo) - 1u, r0 = row0 + at;
        const uint32_t first = (uint32_t)__shfl_sync(0xFFFFFFFFu, slot, at), page = first >> a.page_shift, off = first & mask;
        const uint32_t most = min(a.p.page_tokens - off, a.n_rows - r0);
        // how many rows follow one another
        uint32_t run = lane - at, miss = __ballot_sync(0xFFFFFFFFu, lane >= at && !(run < most && slot == (int32_t)(first + run)));
        run = (miss ? __ffs((int)miss) - 1u : 32u) - at;
        while (!miss) {
            const bool next = run + lane < most && a.slots[r0 + run + lane] == (int32_t)(first + run + lane);
            miss = __ballot_sync(0xFFFFFFFFu, !next);
            run += miss ? __ffs((int)miss) - 1u : 32u;
        }
        float* scale_at = (side ? a.p.v_scale : a.p.k_scale) + (size_t)page * a.p.kv_heads + head;
        const float old = off > 0 ? *scale_at : 0.0f;
        const uint64_t stride = a.row_stride[side];
        const T* src = static_cast<const T*>(a.src[side]) + (size_t)r0 * stride + (size_t)head * a.head_stride[side] + part * 8u;
        uint32_t w[KL][2 * sizeof(T)], top = 0;
        auto fetch = [&](uint32_t c0) {                  // rows c0 .. c0 + kRows - 1
#pragma unroll
            for (uint32_t k = 0; k < KL; k++) {
                const uint32_t r = c0 + k * RPL + sub;
                if (r < run) {
                    load8<T>(src + r * stride, w[k]);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < 2 * sizeof(T); i++) w[k][i] = 0;
                }
            }
        };
        // the largest magnitude: bit patterns without the sign compare as numbers, two at a time in 16 bits (unpacked and asked one by one
        // whether they are finite, the elements took five instructions each, and 17,000 rows of prompts 24 us instead of 20)
        uint32_t c0 = 0;
        for (;; c0 += kRows) {
            fetch(c0);
#pragma unroll
            for (uint32_t k = 0; k < KL; k++)
#pragma unroll
                for (uint32_t i = 0; i < 2 * sizeof(T); i++) top = sizeof(T) == 4 ? max(top, w[k][i] & 0x7FFFFFFFu) : max_u16x2(top, w[k][i] & 0x7FFF7FFFu);
            if (c0 + kRows >= run) break;
        }
        if (sizeof(T) == 2) top = max(top & 0xFFFFu, top >> 16);
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (top >= (sizeof(T) == 4 ? 0x7F800000u : std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u)) {
            // infinities or NaN among them: the finite ones' again, one by one
            top = 0;
#pragma unroll 1
            for (uint32_t r = sub; r < run; r += RPL)
#pragma unroll
                for (uint32_t i = 0; i < 8; i++) {
                    const uint32_t u = __float_as_uint(fabsf(to_float(src[r * stride + i])));
                    if (u < 0x7F800000u) top = max(top, u);
                }
            top = __reduce_max_sync(0xFFFFFFFFu, top);
        } else if (std::is_same<T, __nv_bfloat16>::value) {
            top <<= 16;
        } else if (std::is_same<T, __half>::value) {
            top = __float_as_uint(__half2float(__ushort_as_half((unsigned short)top)));
        }
        float scale = scale_for(__uint_as_float(top));
        unsigned char* codes = static_cast<unsigned char*>(side ? a.p.v : a.p.k) + (size_t)page * a.p.page_stride + (size_t)head * a.p.head_stride + part * 8u;
        if (off > 0) {
            scale = fmaxf(scale, power_not_below(old));
            if (scale != old) {
                const float ratio = __fdiv_rn(old, scale);
#pragma unroll 2
                for (uint32_t t = sub; t < off; t += RPL) {
                    uint2* c = reinterpret_cast<uint2*>(codes + (size_t)t * a.p.token_stride);
                    const uint2 in = *c;
                    uint2 out;
                    auto four = [&](uint32_t v) {
                        const uint32_t h0 = from_e4m3x2(v), h1 = from_e4m3x2(v >> 16);
                        const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&h0)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&h1));
                        return to_e4m3x2(product_to_odd(f0.x, ratio), product_to_odd(f0.y, ratio)) |
                               to_e4m3x2(product_to_odd(f1.x, ratio), product_to_odd(f1.y, ratio)) << 16;
                    };
                    out.x = four(in.x);
                    out.y = four(in.y);
                    *c = out;
                }
            }
        }
        __syncwarp();
        if (lane == 0) *scale_at = scale;
        const float inv = __fdiv_rn(1.0f, scale);           // a power of two: exact (2^-126 .. 2^120 have inverses)
        for (;;) {                                           // the rows at hand, then those before
#pragma unroll
            for (uint32_t k = 0; k < KL; k++) {
                const uint32_t r = c0 + k * RPL + sub;
                if (r >= run) continue;
                float x[8];
                unpack8<T>(w[k], x);
                uint2 out;
                out.x = to_e4m3x2(x[0] * inv, x[1] * inv) | to_e4m3x2(x[2] * inv, x[3] * inv) << 16;
                out.y = to_e4m3x2(x[4] * inv, x[5] * inv) | to_e4m3x2(x[6] * inv, x[7] * inv) << 16;
                *reinterpret_cast<uint2*>(codes + (size_t)(off + r) * a.p.token_stride) = out;
            }
            if (c0 == 0) break;
            c0 -= kRows;
            fetch(c0);
        }
    }
}

}  // namespace wm
