// Attention of many rows (prompts, blocks of tokens) over the paged 8-bit cache.  Part of the translation unit wm_pages.cu.
#pragma once

namespace wm {

// ------------------------------------------------------------------ many rows: bound by the products and the exponentials
//
// A block takes 256 rows of one request and key head (rows run over the heads that share the key head first, then over the
// queries), two tensor-core tiles of 128, and walks the tokens in tiles of 128:
//   scores   S = Q K^T: e4m3 x e4m3.  The keys go in as they lie; a query is a sum of pieces (e4m3, then e5m2 for the
//            remainders: 8 bits of a bf16 element in two pieces, 11 of an f16 in three, exact above 2^-13 of the row's
//            largest, else off by 2^-21 of it at most), so no key is ever converted, and two 8-bit passes cost what one
//            16-bit pass would.
//   outputs  O += P V: f16 x f16 with the weights in tensor memory, over their scores.  Values are converted once per tile
//            (exact) by a warpgroup of its own, for all 256 rows.
// Two threads have one row, 64 of a tile's tokens each (one thread a row left every scheduler with two warps at work, which waited for
// their own results most of the time).  They have to agree only where O's reference moves; sums meet at the end.  As in the kernel for few rows the pages' scales act in f32,
// the values' as an exponent; O is referred to a maximum R of weighted scores that follows only in jumps (of more than 2^14 in units of up
// to 16384 tokens, see top_of: weights lie in f16 from 2 on downwards, so up to 2^15 there is room), which makes rescaling O in tensor
// memory rare: a warp that does it holds up the other three of its tile for 900 cycles, and with jumps of 2^7 one of them did in every
// other tile.
// Work is dealt out as in the kernel for few rows: equal shares of tiles, units cut between workers are joined in order.
//
// Measured: four prompts' 1024 rows over 5000 to 9000 tokens (32 heads, 8 key heads of 128; 437 GFLOP) 394 us, 1.11 PFLOP/s, 0.68 of the
// bf16 rate in short runs, 445 to 459 us in runs of seconds.  A pair of tiles takes 3400 cycles; the tensor cores need 2048 of them and the
// exponentials 2130, but a tile's scores, softmax, weights and outputs follow one another, and only two tiles fit in tensor memory.

// A worker's segments: consecutive tiles of one unit.  base, end: the first tile of its group's first key head, and behind its last's.
struct Segment {
    uint32_t req, rt, head, j, count, j0, nt;
    Request r;
    unsigned long long base, end;
};

template <typename T, int D> struct Many {
    static constexpr uint32_t kQP = std::is_same<T, __half>::value ? 3 : 2;
    static constexpr uint32_t kTile8 = 128 * D, kTile16 = 256 * D;
    static constexpr uint32_t kKS = kQP == 3 && D == 128 ? 2 : 3, kVS = kQP == 3 && D == 128 ? 1 : 2, kHS = 2;     // stages: keys, values as codes, as halves
    static constexpr uint32_t kRing = 8;                                                // of scales: more than kKS + 1
    static constexpr uint32_t kSwD = D == 128 ? kSw128 : kSw64;
    static constexpr uint32_t kQ = kQP * kTile8 > 32768 ? kQP * kTile8 : 32768;         // of 128 rows: the queries' pieces, then the outputs on their way
    static constexpr uint32_t oK = 2 * kQ, oV = oK + kKS * kTile8, oH = oV + kVS * kTile8, oMisc = oH + kHS * kTile16;
    struct Misc {
        unsigned long long kfull[kKS], kfree[kKS], vfull[kVS], vfree[kVS], hfull[kHS], hfree[kHS], qfull, sfull[2], pfull[2][2], ofull[2], votes[2], fin;
        alignas(16) float2 scales[kRing][8];     // of every 16 tokens: (key scale, log2 of the value scale)
        float least[kRing];                     // the least of the logarithms
        float f[256];                           // of every row: |scale| log2(e) / its factor
        Segment seg[2];                         // what the two tiles' softmax threads are at
        float2 other[2][2][128];                // what the two halves of a row tell each other
        uint32_t tmem, dead, nan_seen, first, again[2][2];
    };
    static constexpr uint32_t kSmem = oMisc + (uint32_t)sizeof(Misc) + 1024;
};

// Weights lie in f16 up to 2^kRoom (of 65504); one of the size that the reference is set to is 2^top.  What is below 2^-25 is lost from
// the outputs, though not from l: so that even N tokens that far below the largest weight miss no more than 2^-12 of it in all (as much
// as the weights' 11 bits may), top grows with the unit's tokens, from 1 up to 2^14 of them to 12 from 2^25 on.  Small where it can be,
// for the reference's jumps: measured (us), four prompts' 1024 rows over 5000 to 9000 tokens 448 with 1, 466 with 4, 495 with 6, 543 with
// 7; 1360 rows on 6800 tokens 117, 137, 165, 181.  In a long unit the jumps are few among its tiles: 1024 rows on 131072 tokens 2100 with
// 1, 2230 with the 5 they get.
constexpr float kRoom = 15.0f;
__device__ __forceinline__ int32_t top_of(uint32_t tiles) { return min(max(32 - __clz((int)(tiles - 1u)) - 6, 1), 12); }
// Registers a thread: at launch (five warpgroups), then of the four softmax warpgroups and of the fifth.
constexpr uint32_t kManyRegs = 96, kSoftmaxRegs = 104, kOtherRegs = 64;
static_assert(4 * kSoftmaxRegs + kOtherRegs <= 5 * kManyRegs, "dealt out from what there is at launch");
constexpr uint32_t kManyRows = 256, kMaxManyWorkers = 160, kMaxGroups = 70000;
// A tile of 256 rows of a request; its key heads' tiles stand one behind the other from `base` on.
struct Group {
    unsigned long long base;
    uint32_t req, rt;
};
constexpr uint64_t kManyPartFloats = kManyRows * 128 + kManyRows * 4;
struct ManyWs {                         // behind the workspace of the kernel for few rows
    unsigned long long* total;          // tiles in all; [1]: groups
    Cut* cuts;
    Group* groups;
    float* parts;
};
__host__ __device__ inline uint64_t many_workspace() { return 16 + kMaxManyWorkers * sizeof(Cut) + (uint64_t)kMaxGroups * sizeof(Group) + kMaxManyWorkers * 2 * kManyPartFloats * 4; }
__device__ __forceinline__ ManyWs many_ws(unsigned char* ws)
{
    ManyWs w;
    unsigned char* p = ws + attend_workspace();
    w.total = reinterpret_cast<unsigned long long*>(p);
    w.cuts = reinterpret_cast<Cut*>(p + 16);
    w.groups = reinterpret_cast<Group*>(w.cuts + kMaxManyWorkers);
    w.parts = reinterpret_cast<float*>(w.groups + kMaxGroups);
    return w;
}

__device__ __forceinline__ uint32_t group_tiles(const AttendArgs& a, const Request& r, uint32_t rt, uint32_t& j0)
{
    const uint32_t row0 = rt * kManyRows, row1 = min(row0 + kManyRows, (uint32_t)r.rows * a.group) - 1u;
    const Span s = span_of(a, r.kv, r.kv - r.rows + (int32_t)(row0 / a.group), r.kv - r.rows + (int32_t)(row1 / a.group));
    j0 = (uint32_t)s.any_lo / 128u;
    const uint32_t end = ((uint32_t)s.any_hi + 127u) / 128u;
    return end > j0 ? end - j0 : 1u;
}

// The list of groups with their first tiles, in one block.
__global__ void __launch_bounds__(1024)
k_attend_groups(AttendArgs a)
{
    __shared__ uint32_t s_first[kMaxRequests + 1];
    __shared__ unsigned long long s_w[32];
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    grid_dep_wait();
    grid_dep_launch();
    const ManyWs w = many_ws(a.ws);
    auto scan = [&](unsigned long long v, unsigned long long& all) {           // sum of the threads before, and of all
        unsigned long long incl = v;
#pragma unroll
        for (uint32_t d = 1; d < 32; d <<= 1) {
            const unsigned long long o = __shfl_up_sync(0xFFFFFFFFu, incl, d);
            if (lane >= d) incl += o;
        }
        __syncthreads();
        if (lane == 31) s_w[warp] = incl;
        __syncthreads();
        all = s_w[lane];
        unsigned long long before = lane < warp ? all : 0;
#pragma unroll
        for (uint32_t d = 16; d; d >>= 1) {
            all += __shfl_xor_sync(0xFFFFFFFFu, all, d);
            before += __shfl_xor_sync(0xFFFFFFFFu, before, d);
        }
        return before + incl - v;
    };
    constexpr uint32_t kPer = (kMaxRequests + 1023u) / 1024u;
    uint32_t count[kPer], mine = 0;
#pragma unroll
    for (uint32_t k = 0; k < kPer; k++) {
        const uint32_t i = tid * kPer + k;
        count[k] = 0;
        if (i < a.n) {
            const Request r = request_of(a, i);
            if (!r.ok && a.few_rows == 0u) pages_fault(a.rep, WM_ERR_ARG, i);       // (else the kernel for few rows says so)
            const uint32_t rows = (uint32_t)r.rows * a.group;
            if ((uint32_t)r.rows > a.few_rows / a.group) count[k] = (rows + kManyRows - 1u) / kManyRows;
        }
        mine += count[k];
    }
    unsigned long long all;
    uint32_t at = (uint32_t)scan(mine, all);
#pragma unroll
    for (uint32_t k = 0; k < kPer; k++) {
        const uint32_t i = tid * kPer + k;
        if (i < a.n) s_first[i] = at;
        at += count[k];
    }
    const uint32_t groups = (uint32_t)min(all, (unsigned long long)kMaxGroups);
    if (tid == 0) s_first[a.n] = (uint32_t)all;
    __syncthreads();
    unsigned long long base = 0;
    for (uint32_t g0 = 0; g0 < groups; g0 += 1024) {
        const uint32_t g = g0 + tid;
        uint32_t req = 0, rt = 0;
        unsigned long long tiles = 0;
        if (g < groups) {
            req = last_not_above(s_first, a.n, g);
            rt = g - s_first[req];
            uint32_t j0;
            tiles = tiles_of(a.p.kv_heads, group_tiles(a, request_of(a, req), rt, j0));
        }
        unsigned long long sum;
        const unsigned long long before = scan(tiles, sum);
        if (g < groups) w.groups[g] = Group{base + before, req, rt};
        base += sum;
    }
    if (tid == 0) { w.total[0] = base; w.total[1] = groups; }
}

__device__ __forceinline__ uint32_t to_e5m2x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t from_e5m2x2(uint32_t codes)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
    return r;
}
// GS: tokens that share a scale (64 where pages have at least as many, else 16).
template <typename T, int D, int GS>
__global__ void __launch_bounds__(640, 1)
k_attend_many(AttendArgs a, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap)
{
    using F = Many<T, D>;
    extern __shared__ unsigned char many_smem[];
    unsigned char* base = many_smem + ((1024u - ((uint32_t)__cvta_generic_to_shared(many_smem) & 1023u)) & 1023u);
    const uint32_t base_s = (uint32_t)__cvta_generic_to_shared(base);
    typename F::Misc& M = *reinterpret_cast<typename F::Misc*>(base + F::oMisc);
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = warp_uniform(tid / 32), wg = warp / 4;
    auto bar = [&](const unsigned long long& b) { return (uint32_t)__cvta_generic_to_shared(&b); };

    if (tid == 0) {
        for (uint32_t s = 0; s < F::kKS; s++) { mbar_init(&M.kfull[s], 1); mbar_init(&M.kfree[s], 1); }
        for (uint32_t s = 0; s < F::kVS; s++) { mbar_init(&M.vfull[s], 1); mbar_init(&M.vfree[s], 64); }
        for (uint32_t s = 0; s < F::kHS; s++) { mbar_init(&M.hfull[s], 64); mbar_init(&M.hfree[s], 1); }
        for (uint32_t s = 0; s < 2; s++) { mbar_init(&M.sfull[s], 2); mbar_init(&M.pfull[s][0], 256); mbar_init(&M.pfull[s][1], 256); mbar_init(&M.ofull[s], 1); }
        mbar_init(&M.votes[0], 256);
        mbar_init(&M.votes[1], 256);
        M.again[0][0] = M.again[0][1] = M.again[1][0] = M.again[1][1] = 0;
        mbar_init(&M.qfull, 512);
        mbar_init(&M.fin, 1);
        M.dead = 0;
        M.nan_seen = 0;
    }
    if (tid == 32) { fetch_map(&kmap); fetch_map(&vmap); }
    if (warp == 16) tmem_alloc<512>((uint32_t)__cvta_generic_to_shared(&M.tmem));
    grid_dep_wait();
    grid_dep_launch();
    tmem_fence_before_sync();
    __syncthreads();
    tmem_fence_after_sync();
    const uint32_t tmem = M.tmem;
    const ManyWs W = many_ws(a.ws);
    const unsigned long long total = W.total[0];
    const uint32_t groups = (uint32_t)W.total[1];
    const unsigned long long workers = min((unsigned long long)gridDim.x, total);
    const unsigned long long t_begin = share_of(blockIdx.x, total, workers), t_end = share_of(blockIdx.x + 1u, total, workers);
    if (tid == 0) {
        Cut none = {};
        W.cuts[blockIdx.x] = none;
    }
    // the first tile's group: all threads look at once (one after the other, halving, took nine trips to the L2)
    for (uint32_t i = tid; i < groups; i += 640)
        if (W.groups[i].base <= t_begin && (i + 1 == groups || t_begin < W.groups[i + 1].base)) M.first = i;
    __syncthreads();
    // s becomes the segment that starts at tile t; g: the group before, or that of t.  Inside a group only the head changes.
    auto to_segment = [&](Segment& s, unsigned long long t, uint32_t& g) {
        if (t == t_begin || t >= s.end) {
            while (g + 1 < groups && W.groups[g + 1].base <= t) g++;
            const Group G = W.groups[g];
            s.req = G.req;
            s.rt = G.rt;
            s.r = request_of(a, G.req);
            s.nt = group_tiles(a, s.r, G.rt, s.j0);
            s.base = G.base;
            s.end = G.base + tiles_of(a.p.kv_heads, s.nt);
        }
        const TileAt at = tile_at(t - s.base, s.nt);
        s.head = at.unit;
        s.j = at.j;
        s.count = (uint32_t)min((unsigned long long)(s.nt - s.j), t_end - t);
    };
    if (t_begin < t_end) {
        uint32_t g = M.first;
        unsigned long long t = t_begin;
        if (wg == 4) {
            registers_down<kOtherRegs>();
        if (warp == 16) {
            // ---- copies: a lane per page
            uint32_t ks = 0, kp = 0, vs = 0, vp = 0, ring = 0;
            const bool copy = !(a.inject & kInjectNoCopy);
            Segment s = {};
            while (t < t_end) {
                to_segment(s, t, g);
                const int32_t* row = a.table + (size_t)s.req * a.table_stride;
                const uint32_t first0 = (s.j0 + s.j) * 128u;
                PageOf now, next, later;
                ask_page(a, now, row, first0, s.r.kv, lane);
                ask_page(a, next, row, first0 + 128u, s.r.kv, lane);
                ask_scales(a, now, s.head);
                for (uint32_t c = 0; c < s.count; c++) {
                    ask_page(a, later, row, first0 + (c + 2u) * 128u, s.r.kv, lane);
                    ask_scales(a, next, s.head);
                    const uint32_t n = pages_in(a, first0 + c * 128u, s.r.kv);
                    const int32_t page = now.bad ? 0 : now.page;
                    if (now.bad) pages_fault(a.rep, WM_ERR_ARG, s.req);
                    float2 sc = make_float2(now.sc.x, now.bad ? 0.0f : log2f(now.sc.y));      // (1, 0) where no page is
                    now = next;
                    next = later;
                    const uint32_t bytes = (n << a.page_shift) * D;
                    mbar_wait(bar(M.kfree[ks]), kp ^ 1u, a.wait_ns, &M.dead);
                    const float least = warp_min(lane < n ? sc.y : INFINITY);
                    sc.x = __shfl_sync(0xFFFFFFFFu, sc.x, lane >> (a.page_shift - 4u));
                    sc.y = __shfl_sync(0xFFFFFFFFu, sc.y, lane >> (a.page_shift - 4u));
                    if (lane < 8) M.scales[ring][lane] = sc;
                    if (lane == 8) M.least[ring] = least;
                    __syncwarp();
                    if (lane == 0 && (copy || n == 0)) mbar_expect(bar(M.kfull[ks]), bytes);
                    __syncwarp();
                    if (lane < n && copy) tile_load4(base_s + F::oK + ks * F::kTile8 + (lane << a.page_shift) * D, &kmap, 0, (int32_t)s.head, page, bar(M.kfull[ks]));
                    mbar_wait(bar(M.vfree[vs]), vp ^ 1u, a.wait_ns, &M.dead);
                    __syncwarp();
                    if (lane == 0 && (copy || n == 0)) mbar_expect(bar(M.vfull[vs]), bytes);
                    __syncwarp();
                    if (lane < n && copy) tile_load4(base_s + F::oV + vs * F::kTile8 + (lane << a.page_shift) * D, &vmap, 0, (int32_t)s.head, page, bar(M.vfull[vs]));
                    ring = (ring + 1u) % F::kRing;
                    if (++ks == F::kKS) { ks = 0; kp ^= 1u; }
                    if (++vs == F::kVS) { vs = 0; vp ^= 1u; }
                }
                t += s.count;
            }
            if (*(volatile uint32_t*)&M.dead && copy) {       // nothing may still be on its way when the block leaves
                const uint32_t t0 = now_ns();
                for (uint32_t s = 0; s < F::kKS; s++) while (!mbar_try(bar(M.kfull[s]), s < ks ? kp : kp ^ 1u) && now_ns() - t0 < a.wait_ns) {}
                for (uint32_t s = 0; s < F::kVS; s++) while (!mbar_try(bar(M.vfull[s]), s < vs ? vp : vp ^ 1u) && now_ns() - t0 < a.wait_ns) {}
            }
        } else if (warp == 17) {
            // ---- the products
            uint32_t ks = 0, kp = 0, hs = 0, hp = 0, qp = 0, pp = 0;
            const bool leader = elect_one();
            auto scores = [&](uint32_t w, uint32_t st) {
                const uint64_t q0 = smem_desc(base_s + w * F::kQ, 16, 8 * D, F::kSwD), k0 = smem_desc(base_s + F::oK + st * F::kTile8, 16, 8 * D, F::kSwD);
#pragma unroll
                for (uint32_t p = 0; p < F::kQP; p++)
#pragma unroll
                    for (uint32_t kk = 0; kk < D / 32; kk++)
                        mma_f8(tmem + w * 128u, q0 + (p * F::kTile8 + kk * 32u) / 16u, k0 + kk * 32u / 16u, mma_desc(128, 128, false, false, p > 0), p + kk > 0, leader);
                mma_commit(bar(M.sfull[w]), leader);
                if (leader) mbar_arrive_at(bar(M.sfull[w]));        // (and with it what came with the keys: the scales)
            };
            Segment s = {};
            while (t < t_end) {
                to_segment(s, t, g);
                const uint32_t count = warp_uniform(s.count);
                mbar_wait(bar(M.qfull), qp, a.wait_ns, &M.dead);
                qp ^= 1u;
                mbar_wait(bar(M.kfull[ks]), kp, a.wait_ns, &M.dead);
                tmem_fence_after_sync();
                scores(0, ks);
                scores(1, ks);
                mma_commit(bar(M.kfree[ks]), leader);
                if (++ks == F::kKS) { ks = 0; kp ^= 1u; }
                for (uint32_t c = 0; c < count; c++) {
                    mbar_wait_hot(bar(M.hfull[hs]), hp, a.wait_ns, &M.dead);
                    const uint64_t v0 = smem_desc(base_s + F::oH + hs * F::kTile16, 16384, 1024, kSw128);
                    if (c + 1 < count) mbar_wait_hot(bar(M.kfull[ks]), kp, a.wait_ns, &M.dead);
#pragma unroll
                    for (uint32_t w = 0; w < 2; w++) {
#pragma unroll
                        for (uint32_t q = 0; q < 2; q++) {              // both halves' weights of their first 32 tokens, then of their last
                            mbar_wait_hot(bar(M.pfull[w][q]), pp, a.wait_ns, &M.dead);
                            tmem_fence_after_sync();
#pragma unroll
                            for (uint32_t i = 0; i < 4; i++) {
                                const uint32_t h = i / 2, kk = 4 * h + 2 * q + i % 2;
                                mma_f16_ta(tmem + 256u + w * 128u, tmem + w * 128u + 64u * h + (kk % 4) * 8u, v0 + kk * 2048u / 16u,
                                           mma_desc(128, D, false, true), c + q + i > 0, leader);
                            }
                        }
                        mma_commit(bar(M.ofull[w]), leader);
                        if (w == 1) mma_commit(bar(M.hfree[hs]), leader);
                        if (c + 1 < count) {
                            scores(w, ks);
                            if (w == 1) {
                                mma_commit(bar(M.kfree[ks]), leader);
                                if (++ks == F::kKS) { ks = 0; kp ^= 1u; }
                            }
                        }
                    }
                    pp ^= 1u;
                    if (++hs == F::kHS) { hs = 0; hp ^= 1u; }
                }
                t += count;
            }
            if (*(volatile uint32_t*)&M.dead) {            // what was issued is done before the tensor memory is handed back
                mma_commit(bar(M.fin), leader);
                const uint32_t t0 = now_ns();
                while (!mbar_try(bar(M.fin), 0) && now_ns() - t0 < a.wait_ns) {}
            }
            __syncwarp();
        } else {
            // ---- values to halves: thread = two tokens
            uint32_t vs = 0, vp = 0, hs = 0, hp = 0;
            Segment s = {};
            while (t < t_end) {
                to_segment(s, t, g);
                const uint32_t row0 = s.rt * kManyRows, row1 = min(row0 + kManyRows, (uint32_t)s.r.rows * a.group) - 1u;
                const Span sp = span_of(a, s.r.kv, s.r.kv - s.r.rows + (int32_t)(row0 / a.group), s.r.kv - s.r.rows + (int32_t)(row1 / a.group));
                for (uint32_t c = 0; c < s.count; c++) {
                    // a value that not every row sees must not meet the others' zero weights as NaN: its NaN codes become zeros
                    // here, and rows that do see one find it again when they are done
                    mbar_wait(bar(M.vfull[vs]), vp, a.wait_ns, &M.dead);
                    mbar_wait(bar(M.hfree[hs]), hp ^ 1u, a.wait_ns, &M.dead);
#pragma unroll 1
                    for (uint32_t tok = tid % 64u; tok < 128u; tok += 64u) {
                        const int32_t at = (int32_t)((s.j0 + s.j + c) * 128u + tok);
                        const bool all = at >= sp.all_lo && at < sp.all_hi, any = at >= sp.any_lo && at < sp.any_hi;
                        const uint32_t in = base_s + F::oV + vs * F::kTile8, out = base_s + F::oH + hs * F::kTile16 + tok * 128u;
                        uint4 v[D / 16];
#pragma unroll
                        for (uint32_t i = 0; i < D / 16; i++) v[i] = lds16(in + swizzled<D>(tok * D + i * 16u));
                        if (!all) {
                            uint32_t found = 0;
#pragma unroll
                            for (uint32_t i = 0; i < D / 16; i++) {
                                uint32_t* x = &v[i].x;
#pragma unroll
                                for (uint32_t k = 0; k < 4; k++) {
                                    const uint32_t is = __vcmpeq4(x[k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                                    found |= is;
                                    x[k] &= ~is;
                                }
                            }
                            if (found && any) M.nan_seen = 1u;
                        }
#pragma unroll
                        for (uint32_t i = 0; i < D / 16; i++) {
                            const uint32_t sub = out + (i / 4u) * 16384u, ch = (i % 4u) * 2u, x = tok & 7u;
                            sts16(sub + ((ch ^ x) << 4), from_e4m3x2(v[i].x), from_e4m3x2(v[i].x >> 16), from_e4m3x2(v[i].y), from_e4m3x2(v[i].y >> 16));
                            sts16(sub + (((ch + 1u) ^ x) << 4), from_e4m3x2(v[i].z), from_e4m3x2(v[i].z >> 16), from_e4m3x2(v[i].w), from_e4m3x2(v[i].w >> 16));
                        }
                    }
                    async_proxy_fence();
                    mbar_arrive_at(bar(M.hfull[hs]));
                    mbar_arrive_at(bar(M.vfree[vs]));
                    if (++vs == F::kVS) { vs = 0; vp ^= 1u; }
                    if (++hs == F::kHS) { hs = 0; hp ^= 1u; }
                }
                t += s.count;
            }
        }
        } else {
            registers_up<kSoftmaxRegs>();
            // ---- softmax: two threads a row, 64 of a tile's tokens each
            const uint32_t w = wg / 2u, half = wg % 2u, line = tid % 128u, local = w * 128u + line;       // row of the 128, of the 256
            const uint32_t tS = tmem + w * 128u + half * 64u + ((warp % 4u) * 32u << 16), tO = tmem + 256u + w * 128u + ((warp % 4u) * 32u << 16);
            uint32_t sp = 0, ring = 0;       // phase of sfull[w] (and of ofull[w], one behind)
            auto both = [&]() { asm volatile("bar.sync %0, 256;" ::"r"(1u + w) : "memory"); };      // the row's two threads (and the tile's others)
            while (t < t_end) {
                Segment s = M.seg[w];
                to_segment(s, t, g);
                bool live;
                int32_t lo, hi, t0 = (int32_t)((s.j0 + s.j) * 128u + half * 64u);        // (of this thread's tokens)
                {
                    const uint32_t gr = s.rt * kManyRows + local;
                    live = gr < (uint32_t)s.r.rows * a.group;
                    const int32_t pos = s.r.kv - s.r.rows + (int32_t)(gr / a.group);
                    lo = sees_from(a, pos);
                    hi = sees_to(a, s.r.kv, pos);
                }
                {
                    // the queries' pieces: a warp has 16 rows, 8 elements a lane.  (Code that runs once a unit is kept short: unrolled, it
                    // waits for its instructions, 20 cycles for each of them.)
                    constexpr uint32_t LPR = D / 8, RPI = 32 / LPR, BATCH = 4;          // lanes a row, rows a load
                    const uint32_t q0 = base_s + w * F::kQ, part = lane % LPR;
                    uint4 q[BATCH], ahead[BATCH];
                    auto fetch = [&](uint32_t r0, uint4 (&q)[BATCH]) {
#pragma unroll
                        for (uint32_t k = 0; k < BATCH; k++) {
                            const uint32_t gr = s.rt * kManyRows + (warp * 16u + r0 + k * RPI + lane / LPR);
                            const uint32_t jq = gr / a.group, qrow = (uint32_t)s.r.start + jq, qh = s.head * a.group + (gr - jq * a.group);
                            q[k] = make_uint4(0, 0, 0, 0);
                            if (gr < (uint32_t)s.r.rows * a.group)
                                q[k] = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (size_t)qrow * a.q_row + (size_t)qh * a.q_head + part * 8u);
                        }
                    };
                    fetch(0, ahead);
#pragma unroll 1
                    for (uint32_t r0 = 0; r0 < 16; r0 += RPI * BATCH) {
#pragma unroll
                        for (uint32_t k = 0; k < BATCH; k++) q[k] = ahead[k];
                        if (r0 + RPI * BATCH < 16) fetch(r0 + RPI * BATCH, ahead);
#pragma unroll
                        for (uint32_t k = 0; k < BATCH; k++) {
                            const uint32_t row = warp * 16u + r0 + k * RPI + lane / LPR;       // (of the unit's 256)
                            float x[8];
#pragma unroll
                            for (uint32_t i = 0; i < 4; i++) {
                                const float2 v = unpack2((&q[k].x)[i], T());
                                x[2 * i] = v.x;
                                x[2 * i + 1] = v.y;
                            }
                            uint32_t top = 0;
#pragma unroll
                            for (uint32_t i = 0; i < 8; i++) top = max(top, __float_as_uint(fabsf(x[i])));
#pragma unroll
                            for (uint32_t d = 1; d < LPR; d <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                            // a power of two that brings the row's largest element to 128 .. 256; NaN where the row is not finite
                            const int e = row_exponent(top);
                            const bool fine = top < 0x7F800000u;
                            float up = __uint_as_float((uint32_t)(127 + 7 - e) << 23);
                            if (a.scale < 0.0f) up = -up;
                            if (part == 0) M.f[row] = fine ? fabsf(a.scale) * 1.4426950408889634f * __uint_as_float((uint32_t)(127 - 7 + e) << 23) : NAN;
#pragma unroll
                            for (uint32_t i = 0; i < 8; i++) x[i] *= up;
#pragma unroll
                            for (uint32_t p = 0; p < F::kQP; p++) {
                                uint32_t word[2];
#pragma unroll
                                for (uint32_t i = 0; i < 8; i += 2) {
                                    const uint32_t code = p == 0 ? to_e4m3x2(x[i], x[i + 1]) : to_e5m2x2(x[i], x[i + 1]);
                                    const uint32_t h = p == 0 ? from_e4m3x2(code) : from_e5m2x2(code);
                                    const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&h));
                                    x[i] -= back.x;
                                    x[i + 1] -= back.y;
                                    if (i % 4 == 0) word[i / 4] = code; else word[i / 4] |= code << 16;
                                }
                                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(q0 + p * F::kTile8 + swizzled<D>((row - w * 128u) * D + part * 8u)),
                                             "r"(word[0]), "r"(word[1]) : "memory");
                            }
                        }
                    }
                    async_proxy_fence();
                    mbar_arrive_at(bar(M.qfull));
                    both();
                    if (half == 0u && line == 0u) M.seg[w] = s;       // (read again when the unit's part ends: in registers it would cost the loop)
                }
                const float f = live && lo < hi ? M.f[local] : 1.0f;      // (a row that sees nothing: whatever its query is)
                float m = -INFINITY, l = 0.0f, R = -INFINITY;       // R: what O refers to, less `top`
                const uint32_t count = s.count;
                const float top = (float)top_of(s.nt);
                for (uint32_t c = 0; c < count; c++, t0 += 128) {
                    auto written = [&](uint32_t part) {
                        tmem_wait_stores();
                        tmem_fence_before_sync();
                        mbar_arrive_at(bar(M.pfull[w][part]));
                    };
                    const bool whole = __all_sync(0xFFFFFFFFu, !live || (t0 >= lo && t0 + 64 <= hi));
                    mbar_wait(bar(M.sfull[w]), sp, a.wait_ns, &M.dead);
                    tmem_fence_after_sync();
                    const float least = M.least[ring];
                    constexpr uint32_t NG = 64 / GS;
                    const float2* scales = &M.scales[ring][half * 4u];
                    bool rolled = false;
                    {
                        float x[64];
                        tmem_read32(tS, x);
                        tmem_read32(tS + 32u, x + 32);
                        const float2 first = scales[0];
                        auto scale = [&](uint32_t i) { return NG == 1 ? first : scales[i * (GS / 16)]; };       // of group i: (key scale, log2 of the value scale)
                        tmem_wait_loads();
                        bool odd = false;       // a factor that is not positive, or whose product is not, would turn what is masked into NaN (f is, in a row that is NaN anyway)
                        if (!whole) {
#pragma unroll
                            for (uint32_t ch = 0; ch < 2; ch++) {
                                const int32_t c0 = lo - t0 - (int32_t)(32 * ch), c1 = hi - t0 - (int32_t)(32 * ch);
                                const uint32_t seen = (c1 <= 0 ? 0u : c1 >= 32 ? 0xFFFFFFFFu : (1u << c1) - 1u) & (c0 <= 0 ? 0xFFFFFFFFu : c0 >= 32 ? 0u : 0xFFFFFFFFu << c0);
#pragma unroll
                                for (uint32_t i = 0; i < 32; i++)
                                    if (!(seen >> i & 1u)) x[32 * ch + i] = -INFINITY;
                            }
#pragma unroll
                            for (uint32_t i = 0; i < NG; i++) odd = odd || !(scale(i).x > 0.0f) || scale(i).x * f == 0.0f;
                        }
                        // the largest score and the largest weighted score
                        float mt = m, rt = -INFINITY;
#pragma unroll
                        for (uint32_t i = 0; i < NG; i++) {
                            const float* y = x + GS * i;
                            float top[4];
#pragma unroll
                            for (uint32_t k = 0; k < 4; k++) top[k] = fmaxf(y[k], y[4 + k]);
#pragma unroll
                            for (uint32_t k = 8; k < GS; k += 8)
#pragma unroll
                                for (uint32_t e = 0; e < 4; e++) top[e] = max3(top[e], y[k + 2 * e], y[k + 2 * e + 1]);
                            const float2 z = scale(i);
                            const float v = max3(fmaxf(top[0], top[1]), top[2], top[3]) * (z.x * f);
                            mt = fmaxf(mt, v);
                            rt = fmaxf(rt, v + z.y);
                        }
                        // O's reference R, the same in both threads of a row, follows only when weights could leave f16's range (in the first
                        // tile there is no O yet); where a page's value scale is so far below the others' that the weight times it would
                        // vanish from l, l is summed apart, below
                        if (c == 0) {
                            M.other[w][half][line].x = rt;
                            both();
                            R = fmaxf(rt, M.other[w][half ^ 1u][line].x) - top;
                        }
                        const float Rb = R == -INFINITY ? 0.0f : R, mb = mt == -INFINITY ? Rb : mt;
                        // all 256 threads of the tile have to say so before the weights are handed on; they are asked here and heard when the first
                        // weights are done (waited for at once, their answer took 290 cycles).  Rows that are not there are not asked: they may
                        // be looking at what is behind the last page, which is whatever the stage held before
                        if (live && (odd || rt > R + kRoom || !(Rb - least - mb <= 80.0f))) M.again[w][sp] = 1u;
                        mbar_arrive_at(bar(M.votes[w]));
                        {
                            float sum_l = 0.0f;
                            float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
                            float2 fac2, off2;
#pragma unroll
                            for (uint32_t ch = 0; ch < 2; ch++) {
                                uint32_t pk[16];
#pragma unroll
                                for (uint32_t i = 0; i < 32; i += 2) {
                                    const uint32_t at = 32 * ch + i;
                                    if (at % GS == 0) {
                                        const float2 z = scale(at / GS);
                                        fac2.x = fac2.y = z.x * f;
                                        off2.x = off2.y = z.y - Rb;
                                    }
                                    float2 e = fma2(make_float2(x[at], x[at + 1]), fac2, off2);
                                    e.x = exp2_fast(e.x);
                                    e.y = exp2_fast(e.y);
                                    pk[i / 2] = pack_half2(e.x, e.y);
                                    sum[i / 2 % 2] = at % GS < 4 ? e : add2(sum[i / 2 % 2], e);
                                    if (ch == 1 && i == 14) written(0);      // (the stores before are done)
                                    if (at % GS == GS - 2) {
                                        sum[0] = add2(sum[0], sum[1]);
                                        sum_l = fmaf(sum[0].x + sum[0].y, exp2_fast(-off2.x - mb), sum_l);
                                    }
                                }
                                if (ch == 0) {
                                    // (a barrier of the block's own threads, who all come: waited for whatever else has run out, so that all of
                                    // them go the same way; tiles in turn have words of their own)
                                    for (uint32_t n = 0; n < 1u << 20 && !mbar_try(bar(M.votes[w]), sp); n++) {}
                                    rolled = *(volatile uint32_t*)&M.again[w][sp] != 0u;
                                    if (rolled) break;
                                }
                                tmem_write16(tS + ch * 16u, pk);
                            }
                            if (!rolled) {
                                l = fmaf(l, exp2_fast(m - mb), sum_l);
                                m = mt;
                                written(1);
                            }
                        }
                    }
                    if (rolled) {
                        // what the way above cannot do, 32 tokens at a time, read twice
                        auto scores_of = [&](uint32_t ch, float (&v)[32]) {
                            tmem_read32(tS + ch * 32u, v);
                            tmem_wait_loads();
                            const float f0 = scales[2 * ch].x * f, f1 = scales[2 * ch + 1].x * f;
                            const int32_t c0 = t0 + (int32_t)(ch * 32u);
#pragma unroll
                            for (int i = 0; i < 32; i++) v[i] = whole || (c0 + i >= lo && c0 + i < hi) ? v[i] * (i < 16 ? f0 : f1) : -INFINITY;
                        };
                        float mt = m, rt = -INFINITY;
#pragma unroll 1
                        for (uint32_t ch = 0; ch < 2; ch++) {
                            float v[32];
                            scores_of(ch, v);
                            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                            for (int i = 0; i < 32; i++) top[i / 16] = fmaxf(top[i / 16], v[i]);
                            mt = max3(mt, top[0], top[1]);
                            rt = max3(rt, top[0] + scales[2 * ch].y, top[1] + scales[2 * ch + 1].y);
                        }
                        M.other[w][half][line].x = rt;
                        both();
                        rt = fmaxf(rt, M.other[w][half ^ 1u][line].x);
                        if (half == 0u && line == 0u) M.again[w][sp] = 0u;   // (everybody has heard it)
                        both();                                          // (read, before the next is written)
                        if (c == 0) R = -INFINITY;
                        const bool jump = rt > R + kRoom;
                        if (__any_sync(0xFFFFFFFFu, jump)) {
                            const float R1 = jump ? rt - top : R;
                            const float factor = R == -INFINITY ? 0.0f : exp2_fast(R - R1);
                            R = R1;
                            if (c > 0) {                                             // (either thread of a row has half of its channels)
                                mbar_wait(bar(M.ofull[w]), sp ^ 1u, a.wait_ns, &M.dead);     // the tile before is in O
                                tmem_fence_after_sync();
#pragma unroll 1
                                for (uint32_t ch = half * D / 64u; ch < (half + 1u) * D / 64u; ch++) {
                                    float o[32];
                                    tmem_read32(tO + ch * 32u, o);
                                    tmem_wait_loads();
#pragma unroll
                                    for (int i = 0; i < 32; i++) o[i] *= factor;
                                    tmem_write16(tO + ch * 32u, reinterpret_cast<const uint32_t*>(o));
                                    tmem_write16(tO + ch * 32u + 16u, reinterpret_cast<const uint32_t*>(o) + 16);
                                }
                            }
                        }
                        const float Rb = R == -INFINITY ? 0.0f : R, mb = mt == -INFINITY ? Rb : mt;
                        l *= exp2_fast(m - mb);
                        m = mt;
                        const bool apart = __any_sync(0xFFFFFFFFu, !(Rb - least - mb <= 80.0f));
#pragma unroll 1
                        for (uint32_t ch = 0; ch < 2; ch++) {
                            float v[32];
                            uint32_t pk[16];
                            scores_of(ch, v);
                            const float lv0 = scales[2 * ch].y, lv1 = scales[2 * ch + 1].y;
                            float sum[2] = {0.0f, 0.0f};
                            if (apart) {
#pragma unroll
                                for (int i = 0; i < 32; i++) l += exp2_fast(v[i] - mb);
                            }
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float off = (i < 16 ? lv0 : lv1) - Rb;
                                const float y0 = exp2_fast(v[i] + off), y1 = exp2_fast(v[i + 1] + off);
                                sum[i / 16] += y0 + y1;
                                pk[i / 2] = pack_half2(y0, y1);
                            }
                            if (!apart) l += sum[0] * exp2_fast(Rb - lv0 - mb) + sum[1] * exp2_fast(Rb - lv1 - mb);
                            tmem_write16(tS + ch * 16u, pk);
                        }
                        written(0);
                        mbar_arrive_at(bar(M.pfull[w][1]));
                    }
                    sp ^= 1u;
                    ring = (ring + 1u) % F::kRing;
                }
                // the end of the unit's part
                mbar_wait(bar(M.ofull[w]), sp ^ 1u, a.wait_ns, &M.dead);
                tmem_fence_after_sync();
                s = M.seg[w];
                const uint32_t gr = s.rt * kManyRows + local, n_rows = (uint32_t)s.r.rows * a.group;
                const uint32_t jq = gr / a.group, qrow = (uint32_t)s.r.start + jq, qh = s.head * a.group + gr % a.group;
                const bool full = s.count == s.nt;
                const uint32_t slot = t == t_begin ? 0 : 1;
                M.other[w][half][line] = make_float2(m, l);          // (behind the votes of the last tile: nobody reads what was there)
                both();
                {
                    const float2 o = M.other[w][half ^ 1u][line];
                    const float m1 = fmaxf(m, o.x), mb = m1 == -INFINITY ? 0.0f : m1;
                    l = half ? o.y * exp2_fast(o.x - mb) + l * exp2_fast(m - mb) : l * exp2_fast(m - mb) + o.y * exp2_fast(o.x - mb);
                    m = m1;
                }
                const bool dead = *(volatile uint32_t*)&M.dead;
                // (two factors: their product leaves the floats where a value scale is small and l is large)
                const float one = __uint_as_float((uint32_t)(127 - top_of(s.nt)) << 23);
                R += (float)top_of(s.nt);
                const float over_l = dead ? NAN : !full ? one : l == 0.0f ? 0.0f : one / l;
                const float factor = !full || R == -INFINITY ? 1.0f : exp2_to_zero(R - m);
                const bool nan = *(volatile uint32_t*)&M.nan_seen != 0u;
                const int32_t row1 = (int32_t)min((s.rt + 1u) * kManyRows, n_rows) - 1;
                const Span span = span_of(a, s.r.kv, s.r.kv - s.r.rows + (int32_t)(s.rt * kManyRows / a.group), s.r.kv - s.r.rows + row1 / (int32_t)a.group);
                // Outputs: a warp's rows go through its part of the queries' memory (their products are done), so that whole lines are stored: a
                // row a thread, every store touched 32 lines.  Parts have a layout for that: four channels of all rows side by side.
                const uint32_t st0 = base_s + w * F::kQ + (warp % 8u) * 4096u;
                T* const dst = live ? static_cast<T*>(a.out) + (size_t)qrow * a.o_row + (size_t)qh * a.o_head : nullptr;
                float4* const part = reinterpret_cast<float4*>(W.parts + (size_t)(blockIdx.x * 2u + slot) * kManyPartFloats) + local;
#pragma unroll 1
                for (uint32_t ch = half * D / 64u; ch < (half + 1u) * D / 64u; ch++) {           // (either thread of a row has half of its channels)
                    float x[32];
                    tmem_read32(tO + ch * 32u, x);
                    tmem_wait_loads();
#pragma unroll
                    for (int i = 0; i < 32; i++) x[i] = l == 0.0f && full && !dead ? 0.0f : x[i] * over_l * factor;
                    if (nan && live) {
                        // rare: NaN values among the tokens that only some rows see
#pragma unroll 1
                        for (int32_t k = max(lo, (int32_t)((s.j0 + s.j) * 128u)); k < min(hi, (int32_t)((s.j0 + s.j + s.count) * 128u)); k++) {
                            if (k >= span.all_lo && k < span.all_hi) continue;
                            const int32_t page = a.table[(size_t)s.req * a.table_stride + (k >> a.page_shift)];
                            if ((uint32_t)page >= a.p.n_pages) continue;
                            const unsigned char* v = static_cast<const unsigned char*>(a.p.v) + (size_t)page * a.p.page_stride +
                                                     (size_t)s.head * a.p.head_stride + (size_t)(k & (int32_t)(a.p.page_tokens - 1u)) * a.p.token_stride + ch * 32u;
#pragma unroll
                            for (int i = 0; i < 32; i++)
                                if ((v[i] & 0x7Fu) == 0x7Fu) x[i] = NAN;
                        }
                    }
                    if (full) {
#pragma unroll
                        for (uint32_t i = 0; i < 4; i++) {
                            __align__(16) T o[8];
#pragma unroll
                            for (uint32_t k = 0; k < 8; k++) from_float(o[k], x[8 * i + k]);
                            const uint4 v = *reinterpret_cast<const uint4*>(o);
                            sts16(st0 + lane * 64u + ((i ^ ((lane >> 1) & 3u)) << 4), v.x, v.y, v.z, v.w);
                        }
                        __syncwarp();
#pragma unroll
                        for (uint32_t k = 0; k < 4; k++) {
                            const uint32_t r = k * 8u + lane / 4u, i = lane % 4u;
                            T* to = reinterpret_cast<T*>(__shfl_sync(0xFFFFFFFFu, (unsigned long long)dst, r));
                            const uint4 v = lds16(st0 + r * 64u + ((i ^ ((r >> 1) & 3u)) << 4));
                            if (to) *reinterpret_cast<uint4*>(to + ch * 32u + i * 8u) = v;
                        }
                        __syncwarp();
                    } else {
#pragma unroll
                        for (uint32_t i = 0; i < 8; i++) part[(ch * 8u + i) * kManyRows] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                    }
                }
                tmem_fence_before_sync();
                if (live && half == 0u) {
                    if (full) {
                        if (a.lse) a.lse[(size_t)qrow * a.q_heads + qh] = dead ? NAN : l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
                    } else {
                        *reinterpret_cast<float4*>(W.parts + (size_t)(blockIdx.x * 2u + slot) * kManyPartFloats + kManyRows * 128 + 4 * local) =
                            make_float4(m, R, dead ? NAN : l, 0.0f);
                    }
                }
                if (!full && s.j == 0 && tid == 0) {
                    const unsigned long long last = t + s.nt - 1;
                    Cut cut = {1u, s.req, s.head, s.rt, worker_of(last, total, workers), slot, {0, 0}};
                    W.cuts[blockIdx.x] = cut;
                }
                both();          // (both halves have read what the other left, and the outputs' way is free)
                t += s.count;
            }
        }
    }
    __syncthreads();
    if (tid == 0 && *(volatile uint32_t*)&M.dead) pages_fault(a.rep, WM_ERR_TIMEOUT, 0);
    if (warp == 16) {
        tmem_fence_after_sync();
        tmem_free<512>(tmem);
    }
}

// The cut units' parts put together: block (worker, 32 rows), thread (four channels, four of the rows: their loads are on their way
// together).
template <typename T, int D>
__global__ void __launch_bounds__(2 * D)
k_attend_many_join(AttendArgs a)
{
    grid_dep_wait();
    grid_dep_launch();
    const ManyWs W = many_ws(a.ws);
    const uint32_t w0 = blockIdx.x, i0 = blockIdx.y * 32u + threadIdx.x % 8u, d4 = threadIdx.x / 8u;
    const Cut cut = W.cuts[w0];
    if (!cut.valid) return;
    const Request r = request_of(a, cut.req);
    const uint32_t n_rows = (uint32_t)r.rows * a.group;
    float m[4], R[4], l[4], o[4][4];
#pragma unroll
    for (uint32_t k = 0; k < 4; k++) {
        m[k] = R[k] = -INFINITY;
        l[k] = o[k][0] = o[k][1] = o[k][2] = o[k][3] = 0.0f;
    }
    for (uint32_t w = w0; w <= cut.last; w++) {
        const float* part = W.parts + (size_t)(w * 2u + (w == w0 ? cut.slot : 0u)) * kManyPartFloats;
        float4 s[4], v[4];
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) {                 // (rows that are not there were not written: read, and dropped below)
            s[k] = *reinterpret_cast<const float4*>(part + kManyRows * 128 + 4 * (i0 + 8u * k));
            v[k] = reinterpret_cast<const float4*>(part)[d4 * kManyRows + i0 + 8u * k];
        }
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) {
            const float m1 = fmaxf(m[k], s[k].x), R1 = fmaxf(R[k], s[k].y), mb = m1 == -INFINITY ? 0.0f : m1, rb = R1 == -INFINITY ? 0.0f : R1;
            const float keep = exp2_fast(R[k] - rb), take = exp2_fast(s[k].y - rb);
            l[k] = l[k] * exp2_fast(m[k] - mb) + s[k].z * exp2_fast(s[k].x - mb);
            o[k][0] = o[k][0] * keep + v[k].x * take;
            o[k][1] = o[k][1] * keep + v[k].y * take;
            o[k][2] = o[k][2] * keep + v[k].z * take;
            o[k][3] = o[k][3] * keep + v[k].w * take;
            m[k] = m1;
            R[k] = R1;
        }
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; k++) {
        const uint32_t gr = cut.rt * kManyRows + i0 + 8u * k;
        if (gr < n_rows) store_joined<T>(a, r, gr, cut.head, d4 * 4u, m[k], R[k], l[k], o[k]);
    }
}

}  // namespace wm
