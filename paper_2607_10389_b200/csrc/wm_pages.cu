// The paged 8-bit cache: kernels (sm_100a) and C ABI.
//   wm_pages_plan    : k_pages_plan, and behind it k_pages_slots where there are many
//   wm_pages_append  : k_pages_append
//   wm_pages_attend  : k_attend_few -> k_attend_join; in front of them, or in their place, where requests have many rows,
//                      k_attend_groups -> k_attend_many -> k_attend_many_join
#include <cstdint>
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <mutex>
#include <type_traits>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/wm.h"
#include "wm_device.cuh"
#include "wm_host.h"
#include "wm_launch.h"
#include "wm_units.h"
#include "wm_pages.cuh"
#include "wm_mma.cuh"
#include "wm_attend.cuh"
#include "wm_prompt.cuh"

namespace wm {

// Whether words may be read and written at all of these (NULL included).
static bool words_ok(std::initializer_list<const void*> at)
{
    for (const void* p : at)
        if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) return false;
    return true;
}

// The pool's geometry: what every call checks before anything is launched.
static bool pages_ok(const wm_pages* p, uint32_t& shift)
{
    if (!p || !p->k || !p->v || !p->k_scale || !p->v_scale) return false;
    if (!aligned16(p->k) || !aligned16(p->v) || !words_ok({p->k_scale, p->v_scale})) return false;
    if (((p->page_stride | p->head_stride | p->token_stride) & 15u) != 0) return false;
    shift = p->page_tokens == 16 ? 4 : p->page_tokens == 32 ? 5 : p->page_tokens == 64 ? 6 : p->page_tokens == 128 ? 7 : 0;
    if (!shift || (p->head_dim != 64 && p->head_dim != 128)) return false;
    if (((p->page_stride | p->head_stride | p->token_stride) >> 40) != 0) return false;
    if ((p->kv_heads > 1 && p->head_stride < p->head_dim) || (p->n_pages > 1 && p->page_stride < p->head_dim)) return false;    // shared bytes
    if (p->token_stride < p->head_dim || p->kv_heads == 0 || p->kv_heads > 1024) return false;
    if (p->n_pages == 0 || (uint64_t)p->n_pages * p->page_tokens >= (1ull << 31)) return false;
    return true;
}

// Rows whose bytes every 16-byte access may touch; `size`: bytes of an element.
static bool rows_ok(const wm_rows* r, uint32_t size)
{
    return r && r->ptr && aligned16(r->ptr) && (r->row_stride * size) % 16 == 0 && (r->head_stride * size) % 16 == 0;
}

constexpr uint64_t kAppendWarps = 148 * 64;             // (of a whole B200: a full load of warps for its 148 SMs)
// Rows a warp looks at: one while that many warps still fit the GPU a few times over, up to 32 beyond.  Measured in a graph (us, with a
// quarter of kAppendWarps, with it, with four times as many; 8 key heads of 128, pages of 64): 256 rows of tokens 4.8, 3.4 and 3.4, 1000
// 14.0, 9.2 and 8.0, 3,700 rows of prompts 8.5, 9.5 and 13.1, 17,000 19.6, 19.6 and 24.1.  17,000 rows with up to 16 rows a warp 22, with
// one (and more work a row) 73.  Loads of 16 bytes a lane that stay in registers: 8 there (20 us; 4: 21.4, 16: 20.5), 4 where a warp looks
// at one row (256 rows: 3.5 us, with 16 7.7).
template <typename T>
static void append_launch(AppendArgs a, cudaStream_t s)
{
    const uint64_t units = 2ull * a.p.kv_heads;
    a.per_warp = 1;
    while (a.per_warp < 32u && units * ((a.n_rows + a.per_warp - 1u) / a.per_warp) > kAppendWarps) a.per_warp *= 2u;
    const uint64_t jobs = units * ((a.n_rows + a.per_warp - 1u) / a.per_warp);
    constexpr int kMany = sizeof(T) == 4 ? 4 : 8, kFew = sizeof(T) == 4 ? 2 : 4;
    const bool few = a.per_warp == 1u;
    launch_after(a.p.head_dim == 64 ? (few ? k_pages_append<T, 64, kFew> : k_pages_append<T, 64, kMany>)
                                    : (few ? k_pages_append<T, 128, kFew> : k_pages_append<T, 128, kMany>), (uint32_t)((jobs + 3u) / 4u), 128, 0, s, a);
}

// ---- what a device is asked once: its SMs, the kernels' shared memory
struct PagesDevice {
    uint32_t sms = 0;
    bool ready = false;
};
static PagesDevice g_pages_dev[64];
static std::mutex g_pages_mutex;
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled g_encode_tiled = nullptr;

template <typename T, int D, int RT> static bool few_ready()
{
    return cudaFuncSetAttribute((const void*)k_attend_few<T, D, RT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Few<T, D, RT>::kSmem) == cudaSuccess;
}
template <typename T, int D> static bool few_ready_all() { return few_ready<T, D, 8>() && few_ready<T, D, 16>() && few_ready<T, D, 32>(); }

template <typename T, int D> static bool many_ready()
{
    for (const void* f : {(const void*)k_attend_many<T, D, 16>, (const void*)k_attend_many<T, D, 64>}) {
        // its warpgroups deal the registers that a block starts with out anew: with fewer than they count on they would wait for ever
        cudaFuncAttributes attr;
        if (cudaFuncGetAttributes(&attr, f) != cudaSuccess || attr.numRegs < (int)kManyRegs) return false;
        if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Many<T, D>::kSmem) != cudaSuccess) return false;
    }
    return true;
}

static const PagesDevice* pages_device()
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    std::lock_guard<std::mutex> lock(g_pages_mutex);
    PagesDevice& d = g_pages_dev[dev];
    if (d.ready) return &d;
    if (!g_encode_tiled) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
        g_encode_tiled = (EncodeTiled)f;
    }
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return nullptr;
    if (!few_ready_all<__nv_bfloat16, 64>() || !few_ready_all<__nv_bfloat16, 128>() || !few_ready_all<__half, 64>() || !few_ready_all<__half, 128>()) return nullptr;
    if (!many_ready<__nv_bfloat16, 64>() || !many_ready<__nv_bfloat16, 128>() || !many_ready<__half, 64>() || !many_ready<__half, 128>()) return nullptr;
    d.sms = (uint32_t)n;
    d.ready = true;
    return &d;
}

// The codes as a tensor of (page, head, token, channel); a box is one page of one head, its rows swizzled as the MMAs read them.
static bool page_map(CUtensorMap* map, const wm_pages& p, void* codes)
{
    const cuuint64_t dims[4] = {p.head_dim, p.page_tokens, p.kv_heads, p.n_pages};
    const cuuint64_t strides[3] = {p.token_stride, p.kv_heads > 1 ? p.head_stride : p.token_stride, p.n_pages > 1 ? p.page_stride : p.token_stride};
    const cuuint32_t box[4] = {p.head_dim, p.page_tokens, 1, 1}, step[4] = {1, 1, 1, 1};
    return g_encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, codes, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          p.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, int RT>
static void few_launch(const AttendArgs& a, const CUtensorMap& k, const CUtensorMap& v, uint32_t workers, cudaStream_t s)
{
    launch_after(k_attend_few<T, D, RT>, workers, 192, Few<T, D, RT>::kSmem, s, a, k, v);
    launch_after(k_attend_join<T, D, RT>, dim3(workers, RT / 8), 2 * D, 0, s, a);
}
// Rows of a request and key head up to which the kernel for few rows has them: what it can do in one pass over the cache.  Measured (us, the
// kernel for few rows and the one for many; 8 key heads of 128): 16 requests of 8192 tokens 32 rows 94 and 134, 64 rows 164 and 136; 2
// requests of 60000 tokens 91 and 125, 155 and 130; 2 of 1000 tokens 64 rows 20 and 30.
constexpr uint32_t kFewRows = 32;
template <typename T, int D>
static void attend_launch(AttendArgs a, const CUtensorMap& k, const CUtensorMap& v, uint32_t sms, uint32_t rows, bool alike, cudaStream_t s)
{
    g_launches = 2;
    a.few_rows = 0xFFFFFFFFu;
    if (rows > kFewRows) {
        a.few_rows = alike ? 0u : kFewRows;
        const uint32_t workers = std::min(sms, kMaxManyWorkers);
        launch_after(k_attend_groups, 1, 1024, 0, s, a);
        launch_after(a.p.page_tokens >= 64 ? k_attend_many<T, D, 64> : k_attend_many<T, D, 16>, workers, 640, Many<T, D>::kSmem, s, a, k, v);
        launch_after(k_attend_many_join<T, D>, dim3(workers, kManyRows / 32), 2 * D, 0, s, a);
        g_launches = alike ? 3 : 5;
        if (alike) return;
    }
    // the smallest tile of rows that has them all in one.  Measured (us, tiles of 8, 16 and 32 rows; 8 key heads of 128): 64 requests of
    // 4096 to 8192 tokens, 8 rows a key head 138, 180 and 270, 16 rows 189 (16) and 276 (32); one request of 1000 tokens, 4 rows 9.8,
    // 10.6 and 11.7
    const uint32_t workers = std::min(2u * sms, kMaxWorkers);
    if (rows <= 8) few_launch<T, D, 8>(a, k, v, workers, s);
    else if (rows <= 16) few_launch<T, D, 16>(a, k, v, workers, s);
    else few_launch<T, D, 32>(a, k, v, workers, s);
}

}  // namespace wm

using namespace wm;

extern "C" {

wm_status wm_pages_plan(const int32_t* old_len, const int32_t* new_len, uint32_t n_requests, uint32_t page_tokens, uint32_t n_pages,
                        int32_t* table, uint32_t table_stride, int32_t* free_pages, const uint32_t* free_count,
                        uint32_t* free_count_out, int32_t* start, int32_t* slots, uint32_t n_slots,
                        wm_pages_report* report, void* stream)
{
    const uint32_t shift = page_tokens == 16 ? 4 : page_tokens == 32 ? 5 : page_tokens == 64 ? 6 : page_tokens == 128 ? 7 : 0;
    if (!old_len || !new_len || !table || !free_pages || !free_count || !free_count_out || !start || (!slots && n_slots)) return WM_ERR_ARG;
    if (!words_ok({old_len, new_len, table, free_pages, free_count, free_count_out, start, slots, report})) return WM_ERR_ARG;
    if (!shift || n_requests == 0 || n_requests > kMaxRequests || table_stride == 0 || n_slots >= (1u << 31)) return WM_ERR_ARG;
    if (n_pages == 0 || ((uint64_t)n_pages << shift) >= (1ull << 31) || (uint64_t)n_requests * table_stride >= (1ull << 31)) return WM_ERR_ARG;
    const PlanArgs a = {old_len, new_len, n_requests, page_tokens, shift, n_pages, table, table_stride, free_pages, free_count,
                        free_count_out, start, slots, n_slots, n_slots > kPlanSlots, report};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // one block, or a cluster of eight with a barrier among them.  Measured in a graph (us, one and eight): 64 requests 3.7 and 4.2, 1000
    // 4.8 and 5.2, 2000 6.3 and 5.6, 4000 9.3 and 6.5 (a token each; 1024 requests with four each 6.8 and 5.0)
    const bool small = n_requests <= 1024u && n_slots <= kPlanSlots;
    launch_after_clustered(small ? k_pages_plan<false> : k_pages_plan<true>, small ? 1 : kPlanBlocks, kPlanThreads,
                           3u * (n_requests + 1u) * 4u, small ? 1 : kPlanBlocks, s, a);
    if (a.slots_apart) {
        const uint32_t blocks = std::min((n_slots + 4u * kPlanThreads - 1u) / (4u * kPlanThreads), 1024u);
        launch_after(k_pages_slots, blocks, kPlanThreads, (n_requests + 1u) * 4u, s, a);
    }
    g_launches = a.slots_apart ? 2 : 1;
    return launch_status();
}

wm_status wm_pages_append(const wm_pages* pages, const wm_rows* k, const wm_rows* v, int type, const int32_t* slots, uint32_t n_rows,
                          wm_pages_report* report, void* stream)
{
    uint32_t shift = 0;
    if (type < WM_TYPE_BF16 || type > WM_TYPE_F32) return WM_ERR_ARG;
    const uint32_t size = type == WM_TYPE_F32 ? 4 : 2;
    if (!pages_ok(pages, shift) || !k || !v || n_rows >= (1u << 24) || !words_ok({slots, report})) return WM_ERR_ARG;
    g_launches = 0;
    if (n_rows == 0) return WM_OK;
    if (!rows_ok(k, size) || !rows_ok(v, size) || !slots) return WM_ERR_ARG;
    const AppendArgs a = {*pages, shift, {k->ptr, v->ptr}, {k->row_stride, v->row_stride}, {k->head_stride, v->head_stride}, slots, n_rows, 1, report};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == WM_TYPE_BF16) append_launch<__nv_bfloat16>(a, s);
    else if (type == WM_TYPE_F16) append_launch<__half>(a, s);
    else append_launch<float>(a, s);
    g_launches = 1;
    return launch_status();
}

uint64_t wm_pages_workspace_bytes(uint32_t head_dim)
{
    return head_dim == 64 || head_dim == 128 ? attend_workspace() + many_workspace() : 0;
}

wm_status wm_pages_attend(const wm_pages* pages, const int32_t* table, uint32_t table_stride, const int32_t* kv_len,
                          const int32_t* q_start, uint32_t n_requests, const wm_rows* q, const wm_rows* out, int type, float* lse,
                          uint32_t n_rows, uint32_t q_heads, uint32_t max_q, float scale, uint32_t options, uint32_t window,
                          void* workspace, uint64_t workspace_bytes, wm_pages_report* report, void* stream)
{
    uint32_t shift = 0;
    if (!pages_ok(pages, shift) || !q || !out || !table || !kv_len || !q_start) return WM_ERR_ARG;
    if (!words_ok({table, kv_len, q_start, lse, report})) return WM_ERR_ARG;
    if ((type != WM_TYPE_BF16 && type != WM_TYPE_F16) || (options & ~WM_ATTEND_CAUSAL) || (window && !(options & WM_ATTEND_CAUSAL))) return WM_ERR_ARG;
    if (n_requests == 0 || n_requests > kMaxRequests || table_stride == 0 || (uint64_t)n_requests * table_stride >= (1ull << 31)) return WM_ERR_ARG;
    if ((uint64_t)table_stride << shift > (1ull << 30) || n_rows >= (1u << 24) || !std::isfinite(scale)) return WM_ERR_ARG;
    if (q_heads == 0 || q_heads % pages->kv_heads || q_heads / pages->kv_heads > 64u) return WM_ERR_ARG;
    if ((uint64_t)n_rows * (q_heads / pages->kv_heads) > (1ull << 24)) return WM_ERR_ARG;
    if (!workspace || !aligned16(workspace) || workspace_bytes < wm_pages_workspace_bytes(pages->head_dim)) return WM_ERR_ARG;
    g_launches = 0;
    if (n_rows == 0) return WM_OK;
    if (!rows_ok(q, 2) || !rows_ok(out, 2) || max_q == 0) return WM_ERR_ARG;
    if ((n_rows > 1 && out->row_stride < pages->head_dim) || (q_heads > 1 && out->head_stride < pages->head_dim)) return WM_ERR_ARG;
    if (window >= (1u << 30)) window = 0;             // (no request is longer: such a window hides nothing)
    const AttendArgs a = {*pages, shift, table, table_stride, kv_len, q_start, n_requests, q->ptr, out->ptr, q->row_stride, q->head_stride,
                          out->row_stride, out->head_stride, lse, n_rows, q_heads, q_heads / pages->kv_heads, scale,
                          options & WM_ATTEND_CAUSAL, window, 0u, static_cast<unsigned char*>(workspace), wait_budget_ns(), inject_bits(), report};
    const PagesDevice* dev = pages_device();
    if (!dev) return WM_ERR_CUDA;
    CUtensorMap k, v;
    if (!page_map(&k, *pages, pages->k) || !page_map(&v, *pages, pages->v)) return WM_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uint32_t rows = (uint32_t)std::min((uint64_t)std::min(max_q, n_rows) * a.group, (uint64_t)0xFFFFFFFFu);
    // where there are rows enough for every request to have max_q of them, the kernel for many rows takes all there are (8 us less)
    const bool alike = (uint64_t)n_requests * max_q <= n_rows;
    if (type == WM_TYPE_BF16) {
        if (pages->head_dim == 64) attend_launch<__nv_bfloat16, 64>(a, k, v, dev->sms, rows, alike, s);
        else attend_launch<__nv_bfloat16, 128>(a, k, v, dev->sms, rows, alike, s);
    } else {
        if (pages->head_dim == 64) attend_launch<__half, 64>(a, k, v, dev->sms, rows, alike, s);
        else attend_launch<__half, 128>(a, k, v, dev->sms, rows, alike, s);
    }
    return launch_status();
}

}  // extern "C"
