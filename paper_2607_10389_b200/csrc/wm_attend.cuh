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
    uint32_t causal, window;    // window: below 2^30, 0 for none
    uint32_t few_rows;          // requests with more rows (times heads that share a key head) are the kernel's for many
    unsigned char* ws;
    uint32_t wait_ns, inject;
    wm_pages_report* rep;
};

__device__ __forceinline__ void from_float(__nv_bfloat16& o, float v) { o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(__half& o, float v) { o = __float2half_rn(v); }

// A request as the kernels see it: `rows` is 0 where there is nothing to do (or the request cannot be answered).
struct Request {
    int32_t start, rows, kv;
    bool ok;
};
__device__ __forceinline__ Request request_of(const AttendArgs& a, uint32_t i)
{
    Request r;
    r.start = a.q_start[i];
    const int32_t end = a.q_start[i + 1];
    r.kv = a.kv_len[i];
    r.ok = r.start >= 0 && end >= r.start && (uint32_t)end <= a.n_rows && r.kv >= 0 && (uint32_t)r.kv <= (a.table_stride << a.page_shift);
    r.rows = r.ok ? end - r.start : 0;
    return r;
}

// (as k_attend_few sees it)
__device__ __forceinline__ Request few_request_of(const AttendArgs& a, uint32_t i)
{
    Request r = request_of(a, i);
    if ((uint32_t)r.rows > a.few_rows / a.group) r.rows = 0;
    return r;
}

// ------------------------------------------------------------------ few rows: the cache is read once, split over all SMs
//
// For one key head the rows of a request (its queries times the heads that share the key head) are few, and every byte of
// the cache is used for few products: reading it is what the time goes to.  So codes go from memory into the tensor cores as they
// are, without passing a register: the tile of 128 tokens is the MMA's 128-row operand, and the few queries its columns.
//   scores   S[token][column] = K[token][:] . Q[column][:]           (K as it lies: K-major)
//   outputs  O[channel][column] = sum_token V[token][channel] P[token][column]   (V as it lies: MN-major)
// Both are e4m3 x e4m3 with f32 sums.  Queries and weights have more than e4m3's four bits, so each is held as a sum of pieces
// in columns of their own, every piece the rounded remainder of the one before times 16: 4 bits a piece, two for a bf16 query
// (8 bits: exact for elements above 2^-13 of the row's largest, else off by 2^-21 of it at most), three for f16's 11 bits and for the
// weights.  The columns are
// there anyway: an MMA of 128 rows costs as much for 16 columns as for 8.
// A page's scales are applied in f32: the key's to the score, the value's to the weight (as an addition of its logarithm in the
// exponent, so that weights keep their bits however far apart the scales are): p' = 2^(x + log2 vs - R) <= 1 with a running
// maximum R of its own beside the softmax's m, and out = O 2^(R - m) / l.
//
// Work is dealt out in tiles: all units (request, key head, tile of rows) one behind the other give T tiles of 128 tokens, worker
// w (a block; two on an SM) takes tiles w T / W .. (w + 1) T / W.  A unit that ends inside a worker's share is finished there; one that is cut
// leaves (o, m, R, l) in the workspace, and k_attend_join puts the pieces together in the workers' order (no atomics: the
// result does not depend on timing).
//
// Measured: 64 single rows over 705 MB of codes (8 key heads of 128, groups of 8) 123 us, 5.7 TB/s, 0.88 of the copy rate in short
// runs, 131 us, 0.83, in runs of seconds; one row over
// 2 MB 9.5 us, of which 5 are the first tile's way (4000 cycles until a block knows its share, the copy, one tile's chain).

template <typename T, int D, int RT> struct Few {
    static constexpr uint32_t kQP = sizeof(T) == 2 && std::is_same<T, __half>::value ? 3 : 2;     // pieces of a query
    static constexpr uint32_t kNQ = (RT * kQP + 15) / 16 * 16, kNP = (RT * 3 + 15) / 16 * 16;     // columns of S and of O
    static constexpr uint32_t kWP = kNP <= 32 ? 32 : kNP <= 64 ? 64 : 128;                       // bytes of a token's row of P
    static constexpr uint32_t kSwP = kWP == 32 ? kSw32 : kWP == 64 ? kSw64 : kSw128, kSwD = D == 128 ? kSw128 : kSw64;
    static constexpr uint32_t kHalf = 128 * D, kStage = 2 * kHalf;                                 // a tile's keys; with its values
    // three tiles of keys and values in flight, two where three would not leave room for a second block on the SM
    static constexpr uint32_t kRest = kNQ * D + 128 * kWP + 140 * RT + 2048;
    static constexpr uint32_t kStages = (3 * 32768 + kRest <= 115712 ? 3 : 2) * (128 / D);
    // tensor memory: S, O of a tile, and for more than one group of eight rows the sums so far (l by token, o by channel)
    static constexpr uint32_t cO = kNQ, cL = kNQ + kNP, cA = cL + (RT > 8 ? RT : 0), kUsed = cA + (RT > 8 ? RT : 0);
    static constexpr uint32_t kCols = kUsed <= 64 ? 64 : kUsed <= 128 ? 128 : 256;
    static_assert(kUsed <= 256, "two blocks share an SM's tensor memory");
    // shared memory, from a 1024-byte boundary on
    static constexpr uint32_t oQ = kStages * kStage, oP = oQ + (kNQ * D + 1023) / 1024 * 1024, oMisc = oP + 128 * kWP;
    struct Misc {
        unsigned long long kfull[kStages], vfull[kStages], empty[kStages], sbar, obar, qbar, pbar, fin;
        float2 scales[kStages][8];        // (key scale, value scale) of the tile's pages
        float top[4][RT][2];              // a warp's largest score and largest weighted score
        alignas(16) float state[4][RT][4];            // per warp: m, R, factors of l and of o
        alignas(16) float f[RT];          // scale log2(e) / the query row's factor
        float sum[4][RT];
        unsigned long long scan[4], total;
        unsigned long long first_prefix;
        int2 span[RT];                    // the tokens a row sees: from, to
        Request first;
        uint32_t first_req, tmem, dead;
    };
    static constexpr uint32_t kSmem = oMisc + (uint32_t)sizeof(Misc) + 1024;
};

constexpr uint32_t kMaxWorkers = 320, kPartRows = 32;
// A cut unit's description, left by the worker that has its first tile.
struct Cut {
    uint32_t valid, req, head, rt, last, slot, pad[2];
};
constexpr uint32_t kPartFloats = kPartRows * 128 + kPartRows * 4;
__host__ __device__ constexpr uint64_t attend_workspace() { return kMaxWorkers * sizeof(Cut) + (uint64_t)kMaxWorkers * 2 * kPartFloats * 4; }
__device__ __forceinline__ float* part_of(unsigned char* ws, uint32_t worker, uint32_t slot)
{
    return reinterpret_cast<float*>(ws + kMaxWorkers * sizeof(Cut)) + (size_t)(worker * 2 + slot) * kPartFloats;
}

struct UnitShape {
    uint32_t row_tiles, j0, nt;
    unsigned long long tiles;
};
template <int RT> __device__ __forceinline__ UnitShape shape_of(const AttendArgs& a, const Request& r)
{
    UnitShape u;
    u.row_tiles = ((uint32_t)r.rows * a.group + RT - 1u) / RT;
    const int32_t lo = a.window ? max(0, r.kv - r.rows + 1 - (int32_t)a.window) : 0;
    u.j0 = (uint32_t)lo / 128u;
    const uint32_t end = ((uint32_t)r.kv + 127u) / 128u;
    u.nt = end > u.j0 ? end - u.j0 : 1u;
    u.tiles = tiles_of(a.p.kv_heads * u.row_tiles, u.nt);
    return u;
}

// Where byte `at` of a tile of D-byte rows lies (the copies' and descriptors' swizzle).
template <int D> __device__ __forceinline__ uint32_t swizzled(uint32_t at) { return at ^ (((at >> 7) & (D == 128 ? 7u : 3u)) << 4); }

// What the rows at positions pos0 (first) .. pos1 (last) see.
struct Span {
    int32_t any_lo, any_hi, all_lo, all_hi;
};
__device__ __forceinline__ int32_t sees_from(const AttendArgs& a, int32_t pos) { return a.window ? max(0, pos + 1 - (int32_t)a.window) : 0; }
__device__ __forceinline__ int32_t sees_to(const AttendArgs& a, int32_t kv, int32_t pos) { return a.causal ? min(kv, max(0, pos + 1)) : kv; }
__device__ __forceinline__ Span span_of(const AttendArgs& a, int32_t kv, int32_t pos0, int32_t pos1)
{
    return {sees_from(a, pos0), sees_to(a, kv, pos1), sees_from(a, pos1), sees_to(a, kv, pos0)};
}

// Four channels of a joined row: o in units of 2^R, l of 2^m.
template <typename T>
__device__ __forceinline__ void store_joined(const AttendArgs& a, const Request& r, uint32_t gr, uint32_t head, uint32_t d, float m, float R, float l, const float (&o)[4])
{
    const uint32_t qrow = (uint32_t)r.start + gr / a.group, qh = head * a.group + gr % a.group;
    const float factor = exp2_to_zero(R == -INFINITY ? 0.0f : R - m);
    __align__(8) T out[4];
#pragma unroll
    for (int k = 0; k < 4; k++) from_float(out[k], l == 0.0f ? 0.0f : o[k] / l * factor);        // (the other way round a large or small scale leaves the floats)
    *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + (size_t)qrow * a.o_row + (size_t)qh * a.o_head + d) = *reinterpret_cast<const uint2*>(out);
    if (d == 0 && a.lse) a.lse[(size_t)qrow * a.q_heads + qh] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// Whether `p` holds in any of the 128 threads that have the softmax.
__device__ __forceinline__ bool any_of_128(bool p)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)p) : "memory");
    return r != 0u;
}

// What a lane of the copying warp needs of a tile: its page (lane = page of the tile) and that page's scales.  They are asked for
// ahead, the page two tiles and the scales one: one after the other in front of every copy they took longer than the tile.
struct PageOf {
    int32_t page;          // -1: none in this lane
    bool bad;
    float2 sc;
};
__device__ __forceinline__ uint32_t pages_in(const AttendArgs& a, uint32_t first, int32_t kv)
{
    const uint32_t tokens = first < (uint32_t)kv ? min(128u, (uint32_t)kv - first) : 0u;
    return (tokens + a.p.page_tokens - 1u) >> a.page_shift;
}
__device__ __forceinline__ void ask_page(const AttendArgs& a, PageOf& p, const int32_t* row, uint32_t first, int32_t kv, uint32_t lane)
{
    p.page = lane < pages_in(a, first, kv) ? row[(first >> a.page_shift) + lane] : -1;
    p.bad = lane < pages_in(a, first, kv) && (uint32_t)p.page >= a.p.n_pages;
}
__device__ __forceinline__ void ask_scales(const AttendArgs& a, PageOf& p, uint32_t head)
{
    p.sc = make_float2(p.bad ? NAN : 1.0f, p.bad ? 0.0f : 1.0f);       // NaN where a row sees a page that there is not; what it loads does not matter
    if (p.page >= 0 && !p.bad) {
        const size_t at = (size_t)p.page * a.p.kv_heads + head;
        p.sc = make_float2(a.p.k_scale[at], a.p.v_scale[at]);
    }
}

// The exponent that a query row is scaled by, of its largest element's bits: down to 2^-119, so that both powers of two that
// come from it, 2^(7 - e) and 2^(e - 7), are floats.  A row of zeros takes any factor.
__device__ __forceinline__ int row_exponent(uint32_t top) { return top == 0u ? 7 : min(max((int)(top >> 23) - 127, -119), 127); }

template <typename T> __device__ __forceinline__ void store_out(const AttendArgs& a, uint32_t row, uint32_t qh, uint32_t d, float v)
{
    T r;
    from_float(r, v);
    static_cast<T*>(a.out)[row * a.o_row + qh * a.o_head + d] = r;
}

template <typename T, int D, int RT>
__global__ void __launch_bounds__(192, 2)
k_attend_few(AttendArgs a, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap)
{
    using F = Few<T, D, RT>;
    extern __shared__ unsigned char few_smem[];
    unsigned char* base = few_smem + ((1024u - ((uint32_t)__cvta_generic_to_shared(few_smem) & 1023u)) & 1023u);
    const uint32_t base_s = (uint32_t)__cvta_generic_to_shared(base);
    typename F::Misc& M = *reinterpret_cast<typename F::Misc*>(base + F::oMisc);
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = warp_uniform(tid / 32);
    auto bar = [&](const unsigned long long& b) { return (uint32_t)__cvta_generic_to_shared(&b); };

    if (tid == 0) {
        for (uint32_t s = 0; s < F::kStages; s++) { mbar_init(&M.kfull[s], 1); mbar_init(&M.vfull[s], 1); mbar_init(&M.empty[s], 1); }
        mbar_init(&M.sbar, 1);
        mbar_init(&M.obar, 1);
        mbar_init(&M.qbar, 128);
        mbar_init(&M.pbar, 128);
        mbar_init(&M.fin, 1);
        M.dead = 0;
    }
    if (tid == 32) { fetch_map(&kmap); fetch_map(&vmap); }
    if (warp == 4) tmem_alloc<F::kCols>((uint32_t)__cvta_generic_to_shared(&M.tmem));
    grid_dep_wait();
    grid_dep_launch();

    // this worker's share: each of 128 threads sums the tiles of some consecutive requests
    const uint32_t per = (a.n + 127u) / 128u;
    unsigned long long mine = 0, incl = 0;
    Request mine_r = {};
    if (warp < 4) {
        for (uint32_t i = tid * per; i < min((tid + 1) * per, a.n); i++) {
            mine_r = few_request_of(a, i);
            if (!mine_r.ok && blockIdx.x == 0) pages_fault(a.rep, WM_ERR_ARG, i);
            if (mine_r.rows) mine += shape_of<RT>(a, mine_r).tiles;
        }
        incl = mine;
#pragma unroll
        for (uint32_t d = 1; d < 32; d <<= 1) {
            const unsigned long long o = __shfl_up_sync(0xFFFFFFFFu, incl, d);
            if (lane >= d) incl += o;
        }
        if (lane == 31) M.scan[warp] = incl;
    }
    tmem_fence_before_sync();
    __syncthreads();
    tmem_fence_after_sync();
    const uint32_t tmem = M.tmem;
    const unsigned long long total = M.scan[0] + M.scan[1] + M.scan[2] + M.scan[3];
    const unsigned long long workers = min((unsigned long long)gridDim.x, total);       // so that every share has a tile
    const unsigned long long t_begin = share_of(blockIdx.x, total, workers), t_end = share_of(blockIdx.x + 1u, total, workers);
    if (warp < 4) {
        for (uint32_t w = 0; w < warp; w++) incl += M.scan[w];
        unsigned long long at = incl - mine;
        if (at <= t_begin && t_begin < incl) {
            uint32_t i = tid * per;
            if (per > 1)
                for (;; i++) {
                    mine_r = few_request_of(a, i);
                    const unsigned long long t = mine_r.rows ? shape_of<RT>(a, mine_r).tiles : 0;
                    if (t_begin < at + t) break;
                    at += t;
                }
            M.first_req = i;
            M.first = mine_r;
            M.first_prefix = at;
        }
    }
    if (tid == 0) {
        Cut none = {};
        reinterpret_cast<Cut*>(a.ws)[blockIdx.x] = none;
    }
    __syncthreads();

    if (t_begin < t_end) {
        uint32_t req = M.first_req;
        Request r = M.first;
        UnitShape u = shape_of<RT>(a, r);
        unsigned long long prefix = M.first_prefix, t = t_begin;
        auto to_request = [&]() {                        // r, u: of the request that has tile t
            while (t >= prefix + u.tiles) {
                prefix += u.tiles;
                req++;
                r = few_request_of(a, req);
                u = r.rows ? shape_of<RT>(a, r) : UnitShape{0, 0, 1, 0};
            }
        };
        if (warp == 4) {
            // ---- the copies: a lane per page of the tile
            const uint32_t pages = 128u >> a.page_shift;
            uint32_t stage = 0, phase = 0;
            while (t < t_end) {
                to_request();
                const TileAt at = tile_at(t - prefix, u.nt);
                const uint32_t j = at.j, head = at.unit / u.row_tiles;
                const uint32_t count = (uint32_t)min((unsigned long long)(u.nt - j), t_end - t);
                const int32_t* row = a.table + (size_t)req * a.table_stride;
                const uint32_t first0 = (u.j0 + j) * 128u;
                PageOf now, next, later;
                ask_page(a, now, row, first0, r.kv, lane);
                ask_page(a, next, row, first0 + 128u, r.kv, lane);
                ask_scales(a, now, head);
                for (uint32_t c = 0; c < count; c++) {
                    ask_page(a, later, row, first0 + (c + 2u) * 128u, r.kv, lane);
                    ask_scales(a, next, head);
                    const uint32_t n = pages_in(a, first0 + c * 128u, r.kv);
                    const int32_t page = now.bad ? 0 : now.page;
                    if (now.bad) pages_fault(a.rep, WM_ERR_ARG, req);
                    const float2 sc = now.sc;
                    now = next;
                    next = later;
                    mbar_wait(bar(M.empty[stage]), phase ^ 1u, a.wait_ns, &M.dead);
                    if (lane < pages) M.scales[stage][lane] = sc;
                    __syncwarp();
                    const uint32_t bytes = (n << a.page_shift) * D;
                    const bool copy = !(a.inject & kInjectNoCopy);
                    if (lane == 0) {
                        if (copy || n == 0) { mbar_expect(bar(M.kfull[stage]), bytes); mbar_expect(bar(M.vfull[stage]), bytes); }
                    }
                    __syncwarp();
                    if (lane < n && copy) {
                        const uint32_t dst = base_s + stage * F::kStage + (lane << a.page_shift) * D;
                        tile_load4(dst, &kmap, 0, (int32_t)head, page, bar(M.kfull[stage]));
                        tile_load4(dst + F::kHalf, &vmap, 0, (int32_t)head, page, bar(M.vfull[stage]));
                    }
                    if (++stage == F::kStages) { stage = 0; phase ^= 1u; }
                }
                t += count;
            }
            // nothing may still be on its way into this block's shared memory when it leaves
            if (*(volatile uint32_t*)&M.dead && !(a.inject & kInjectNoCopy)) {
                for (uint32_t s = 0; s < F::kStages; s++) {
                    const uint32_t t0 = now_ns();
                    const uint32_t parity = s < stage ? phase : phase ^ 1u;
                    while (!(mbar_try(bar(M.kfull[s]), parity) && mbar_try(bar(M.vfull[s]), parity)) && now_ns() - t0 < a.wait_ns) {}
                }
            }
        } else if (warp == 5) {
            // ---- the products
            uint32_t stage = 0, phase = 0, qphase = 0, pphase = 0;
            const bool leader = elect_one();
            auto scores = [&](uint32_t st) {
                const uint64_t k0 = smem_desc(base_s + st * F::kStage, 16, 8 * D, F::kSwD), q0 = smem_desc(base_s + F::oQ, 16, 8 * D, F::kSwD);
#pragma unroll
                for (uint32_t kk = 0; kk < D / 32; kk++) mma_f8(tmem, k0 + kk * 2u, q0 + kk * 2u, mma_desc(128, F::kNQ, false, false), kk > 0, leader);
                mma_commit(bar(M.sbar), leader);
            };
            while (t < t_end) {
                to_request();
                const uint32_t j = tile_at(t - prefix, u.nt).j, count = warp_uniform((uint32_t)min((unsigned long long)(u.nt - j), t_end - t));
                mbar_wait_hot(bar(M.kfull[stage]), phase, a.wait_ns, &M.dead);
                mbar_wait_hot(bar(M.qbar), qphase, a.wait_ns, &M.dead);
                qphase ^= 1u;
                tmem_fence_after_sync();
                scores(stage);
                for (uint32_t c = 0; c < count; c++) {
                    const uint32_t next = stage + 1 == F::kStages ? 0 : stage + 1, next_phase = next ? phase : phase ^ 1u;
                    mbar_wait_hot(bar(M.vfull[stage]), phase, a.wait_ns, &M.dead);
                    mbar_wait_hot(bar(M.pbar), pphase, a.wait_ns, &M.dead);
                    pphase ^= 1u;
                    tmem_fence_after_sync();
                    const uint64_t v0 = smem_desc(base_s + stage * F::kStage + F::kHalf, 0, 8 * D, F::kSwD), p0 = smem_desc(base_s + F::oP, 0, 8 * F::kWP, F::kSwP);
#pragma unroll
                    for (uint32_t kk = 0; kk < 4; kk++)
                        mma_f8(tmem + F::cO, v0 + kk * 2u * D, p0 + kk * 2u * F::kWP, mma_desc(128, F::kNP, true, true), kk > 0, leader);
                    mma_commit(bar(M.obar), leader);
                    mma_commit(bar(M.empty[stage]), leader);
                    if (c + 1 < count) {
                        mbar_wait_hot(bar(M.kfull[next]), next_phase, a.wait_ns, &M.dead);
                        scores(next);
                    }
                    stage = next;
                    phase = next_phase;
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
            // ---- scores, softmax, outputs: thread = token of the tile, then channel.  Rows in groups of eight, one after the other in the same
            // code (unrolled over 32 rows it was so long that a block that runs it two or three times waited for its instructions: 26 us
            // for three tiles)
            constexpr uint32_t G8 = RT / 8;
            uint32_t stage = 0, kphase = 0, sphase = 0, ophase = 0;
            const uint32_t lane_t = tmem + ((warp * 32u) << 16);
            const uint32_t qs = base_s + F::oQ, ps = base_s + F::oP;
            while (t < t_end) {
                to_request();
                const TileAt at = tile_at(t - prefix, u.nt);
                const uint32_t j = at.j, head = at.unit / u.row_tiles, rt = at.unit % u.row_tiles;
                const uint32_t count = (uint32_t)min((unsigned long long)(u.nt - j), t_end - t);
                const uint32_t row0 = rt * RT, rows = min((uint32_t)RT, (uint32_t)r.rows * a.group - row0);
                // what the unit's first and last row see: [lo, hi)
                const int32_t pos0 = r.kv - r.rows + (int32_t)(row0 / a.group), pos1 = r.kv - r.rows + (int32_t)((row0 + rows - 1u) / a.group);
                const Span sp = span_of(a, r.kv, pos0, pos1);

                // the queries' pieces: TPR threads a row
                {
                    constexpr uint32_t TPR = 128 / RT, EPT = D / TPR;
                    const uint32_t rr = tid / TPR, part = tid % TPR;
                    float x[EPT];
                    if (rr < rows) {
                        const uint32_t gr = row0 + rr, qrow = (uint32_t)r.start + gr / a.group, qh = head * a.group + gr % a.group;
                        const T* src = static_cast<const T*>(a.q) + (size_t)qrow * a.q_row + (size_t)qh * a.q_head + part * EPT;
#pragma unroll
                        for (uint32_t e = 0; e < EPT; e += 4) load_row<T, 4>(src + e, *reinterpret_cast<float (*)[4]>(&x[e]));
                    } else {
#pragma unroll
                        for (uint32_t e = 0; e < EPT; e++) x[e] = 0.0f;
                    }
                    uint32_t top = 0;
#pragma unroll
                    for (uint32_t e = 0; e < EPT; e++) top = max(top, __float_as_uint(fabsf(x[e])));
#pragma unroll
                    for (uint32_t d = 1; d < TPR; d <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                    // a power of two that brings the row's largest element to 128 .. 256 (NaN where the row is not finite)
                    const int e = row_exponent(top);
                    const float up = top >= 0x7F800000u ? NAN : __uint_as_float((uint32_t)(127 + 7 - e) << 23);
                    const float down = __uint_as_float((uint32_t)(127 - 7 + e) << 23);
                    if (part == 0) M.f[rr] = a.scale * 1.4426950408889634f * (top >= 0x7F800000u ? NAN : down);
#pragma unroll
                    for (uint32_t p = 0; p < F::kQP; p++) {
                        const uint32_t n = p * RT + rr;
#pragma unroll
                        for (uint32_t e4 = 0; e4 < EPT; e4 += 4) {
                            uint32_t w = 0;
#pragma unroll
                            for (uint32_t k = 0; k < 4; k += 2) {
                                float& x0 = x[e4 + k];
                                float& x1 = x[e4 + k + 1];
                                if (p == 0) { x0 *= up; x1 *= up; }
                                const uint32_t c = to_e4m3x2(x0, x1), h = from_e4m3x2(c);
                                const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&h));
                                x0 = (x0 - back.x) * 16.0f;
                                x1 = (x1 - back.y) * 16.0f;
                                w |= c << (8 * k);
                            }
                            const uint32_t byte = n * D + part * EPT + e4;
                            sts_now(qs + (byte ^ (((byte >> 7) & (D == 128 ? 7u : 3u)) << 4)), w);
                        }
                    }
                }
                async_proxy_fence();
                mbar_arrive_at(bar(M.qbar));
                if (tid < RT) {
                    const int32_t pos = r.kv - r.rows + (int32_t)((row0 + tid) / a.group);
                    M.span[tid] = make_int2(sees_from(a, pos), sees_to(a, r.kv, pos));
                }
                if (G8 > 1) {                             // the sums so far, in tensor memory
                    const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 1
                    for (uint32_t g = 0; g < 2 * G8; g++) tmem_write8(lane_t + F::cL + 8u * g, zero);
                    tmem_wait_stores();
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");

                float o[8], l[8];                          // (of the one group, where there is one)
#pragma unroll
                for (uint32_t i = 0; i < 8; i++) { o[i] = 0.0f; l[i] = 0.0f; }
                float m_run = -INFINITY, r_run = -INFINITY;       // of row `lane`, the same in every warp
                for (uint32_t c = 0; c < count; c++) {
                    const int32_t t0 = (int32_t)((u.j0 + j + c) * 128u), tok = t0 + (int32_t)tid;
                    const bool whole = t0 >= sp.all_lo && t0 + 128 <= sp.all_hi;      // every row sees every token
                    mbar_wait(bar(M.sbar), sphase, a.wait_ns, &M.dead);
                    sphase ^= 1u;
                    tmem_fence_after_sync();
                    mbar_wait(bar(M.kfull[stage]), kphase, a.wait_ns, &M.dead);   // (long since done: for the scales behind it)
                    const float2 sc = M.scales[stage][tid >> a.page_shift];
                    const float lv = log2f(sc.y);
                    uint32_t seen = 0xFFFFFFFFu;          // by which rows
                    if (!whole) {
                        seen = 0;
#pragma unroll 8
                        for (uint32_t i = 0; i < RT; i++) {
                            const int2 s = M.span[i];
                            seen |= (tok >= s.x && tok < s.y ? 1u : 0u) << i;
                        }
                    }
                    auto scores_of = [&](uint32_t g, float (&x)[8]) {
                        float s[F::kQP][8];
#pragma unroll
                        for (uint32_t p = 0; p < F::kQP; p++) tmem_read8(lane_t + p * RT + 8u * g, s[p]);
                        float f[8];
                        *reinterpret_cast<float4*>(f) = *reinterpret_cast<const float4*>(&M.f[8u * g]);
                        *reinterpret_cast<float4*>(f + 4) = *reinterpret_cast<const float4*>(&M.f[8u * g + 4u]);
                        tmem_wait_loads();
#pragma unroll
                        for (uint32_t i = 0; i < 8; i++) {
                            float v = s[1][i];
                            if (F::kQP == 3) v = fmaf(s[F::kQP - 1][i], 0.0625f, v);
                            x[i] = fmaf(v, 0.0625f, s[0][i]) * (f[i] * sc.x);
                        }
                        if (!whole) {
#pragma unroll
                            for (uint32_t i = 0; i < 8; i++)
                                if (!(seen >> (8u * g + i) & 1u)) x[i] = -INFINITY;
                        }
                    };
                    float x[8];
                    {
                        float mt = -INFINITY, mr = -INFINITY;
#pragma unroll 1
                        for (uint32_t g = 0; g < G8; g++) {
                            scores_of(g, x);
#pragma unroll
                            for (uint32_t i = 0; i < 8; i++) {
                                const float v = warp_max(x[i]), w = warp_max(x[i] + lv);
                                if (lane == 8u * g + i) { mt = v; mr = w; }
                            }
                        }
                        if (lane < RT) *reinterpret_cast<float2*>(M.top[warp][lane]) = make_float2(mt, mr);
                    }
                    asm volatile("bar.sync 1, 128;" ::: "memory");
                    if (lane < RT) {
                        float mt = m_run, mo = -INFINITY;
#pragma unroll
                        for (uint32_t w = 0; w < 4; w++) {
                            const float2 v = *reinterpret_cast<const float2*>(M.top[w][lane]);
                            mt = fmaxf(mt, v.x);
                            mo = fmaxf(mo, v.y);
                        }
                        const float mr = fmaxf(r_run, mo);
                        const float mb = mt == -INFINITY ? 0.0f : mt, rb = mr == -INFINITY ? 0.0f : mr, ob = mo == -INFINITY ? 0.0f : mo;
                        // what exponents refer to, and the factors of l, of o and of this tile's outputs
                        *reinterpret_cast<float4*>(M.state[warp][lane]) = make_float4(mb, ob - 8.0f, exp2_fast(m_run - mb), exp2_fast(r_run - rb));
                        // (no outputs from a tile of which the row sees nothing: its ob stands for nothing, and 2^(ob - rb) may be infinite)
                        M.sum[warp][lane] = mo == -INFINITY ? 0.0f : exp2_fast(ob - 8.0f - rb);
                        m_run = mt;
                        r_run = mr;
                    }
                    __syncwarp();
                    // weights: l in f32, pieces of p' 2^8 into P
#pragma unroll 1
                    for (uint32_t g = 0; g < G8; g++) {
                        if (G8 > 1) {
                            tmem_read8(lane_t + F::cL + 8u * g, l);
                            scores_of(g, x);
                        }
                        uint32_t piece[3][2];
#pragma unroll
                        for (uint32_t i = 0; i < 8; i += 2) {
                            const float4 s0 = *reinterpret_cast<const float4*>(M.state[warp][8u * g + i]), s1 = *reinterpret_cast<const float4*>(M.state[warp][8u * g + i + 1]);
                            l[i] = fmaf(l[i], s0.z, exp2_fast(x[i] - s0.x));
                            l[i + 1] = fmaf(l[i + 1], s1.z, exp2_fast(x[i + 1] - s1.x));
                            float y0 = exp2_fast(x[i] + lv - s0.y), y1 = exp2_fast(x[i + 1] + lv - s1.y);
                            if (G8 == 1) { o[i] *= s0.w; o[i + 1] *= s1.w; }
#pragma unroll
                            for (uint32_t p = 0; p < 3; p++) {
                                const uint32_t cc = to_e4m3x2(y0, y1), h = from_e4m3x2(cc);
                                const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&h));
                                y0 = (y0 - back.x) * 16.0f;
                                y1 = (y1 - back.y) * 16.0f;
                                if (i % 4 == 0) piece[p][i / 4] = cc; else piece[p][i / 4] |= cc << 16;
                            }
                        }
                        if (G8 > 1) tmem_write8(lane_t + F::cL + 8u * g, l);
                        const uint32_t swz = F::kWP == 128 ? tid & 7u : F::kWP == 64 ? (tid >> 1) & 3u : (tid >> 2) & 1u;
#pragma unroll
                        for (uint32_t p = 0; p < 3; p++) {
                            const uint32_t byte = p * RT + 8u * g;
                            asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(ps + tid * F::kWP + (((byte >> 4) ^ swz) << 4) + (byte & 8u)), "r"(piece[p][0]), "r"(piece[p][1]) : "memory");
                        }
                    }
                    // values that not every row sees must not meet the others' zero weights as NaN: tokens that no row sees are cleared,
                    // NaN codes of tokens that some rows see are taken out and put into those rows' outputs below
                    uint32_t nan_at[D / 32], found = 0;
                    if (!whole) {
                        mbar_wait(bar(M.vfull[stage]), kphase, a.wait_ns, &M.dead);
                        const uint32_t v0 = base_s + stage * F::kStage + F::kHalf;
                        const bool any = tok >= sp.any_lo && tok < sp.any_hi, all = tok >= sp.all_lo && tok < sp.all_hi;
#pragma unroll
                        for (uint32_t i = 0; i < D / 32; i++) nan_at[i] = 0;
                        if (!any) {
#pragma unroll
                            for (uint32_t i = 0; i < D; i += 16)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v0 + tid * D + i), "r"(0u) : "memory");
                        } else if (!all) {
                            // a byte of 0x7F without its sign carries into bit 7 when one is added
#pragma unroll
                            for (uint32_t i = 0; i < D; i += 16) {
                                const uint4 v = lds16(v0 + swizzled<D>(tid * D + i));
                                found |= ((v.x & 0x7F7F7F7Fu) + 0x01010101u) | ((v.y & 0x7F7F7F7Fu) + 0x01010101u) | ((v.z & 0x7F7F7F7Fu) + 0x01010101u) |
                                         ((v.w & 0x7F7F7F7Fu) + 0x01010101u);
                            }
                            found &= 0x80808080u;
                            if (found) {
#pragma unroll
                                for (uint32_t k = 0; k < D / 32; k++)
#pragma unroll 1
                                    for (uint32_t i = 0; i < 32; i += 4) {
                                        const uint32_t at = v0 + swizzled<D>(tid * D + 32u * k + i), v = lds_now<0>(at);
                                        const uint32_t is = __vcmpeq4(v & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                                        sts_now(at, v & ~is);
                                        nan_at[k] |= ((is & 1u) | (is >> 7 & 2u) | (is >> 14 & 4u) | (is >> 21 & 8u)) << i;
                                    }
                            }
                        }
                    }
                    async_proxy_fence();
                    if (G8 > 1) tmem_wait_stores();
                    tmem_fence_before_sync();
                    mbar_arrive_at(bar(M.pbar));
                    mbar_wait(bar(M.obar), ophase, a.wait_ns, &M.dead);
                    ophase ^= 1u;
                    tmem_fence_after_sync();
                    // (asked of all threads at one barrier: they have to agree even where a wait ran out and some are ahead)
                    const bool poison = !whole && any_of_128(found != 0u);
                    if (poison) {                          // rare: the marks through P's memory (its MMAs are done)
#pragma unroll
                        for (uint32_t i = 0; i < D / 32; i++) sts_now(ps + tid * 16u + 4u * i, nan_at[i]);
                        asm volatile("bar.sync 1, 128;" ::: "memory");
                    }
#pragma unroll 1
                    for (uint32_t g = 0; g < G8; g++) {
                        float s[3][8];
#pragma unroll
                        for (uint32_t p = 0; p < 3; p++) tmem_read8(lane_t + F::cO + p * RT + 8u * g, s[p]);
                        if (G8 > 1) tmem_read8(lane_t + F::cA + 8u * g, o);
                        tmem_wait_loads();
#pragma unroll
                        for (uint32_t i = 0; i < 8; i++) {
                            if (G8 > 1) o[i] *= M.state[warp][8u * g + i][3];
                            o[i] = fmaf(fmaf(fmaf(s[2][i], 0.0625f, s[1][i]), 0.0625f, s[0][i]), M.sum[warp][8u * g + i], o[i]);
                        }
                        if (poison) {
                            const uint32_t d = tid % D;
#pragma unroll 1
                            for (uint32_t k = 0; k < 128; k++) {
                                if (!(lds_now<0>(ps + k * 16u + 4u * (d / 32u)) >> (d % 32u) & 1u)) continue;
#pragma unroll
                                for (uint32_t i = 0; i < 8; i++) {
                                    const int2 s = M.span[8u * g + i];
                                    if (t0 + (int32_t)k >= s.x && t0 + (int32_t)k < s.y) o[i] = NAN;
                                }
                            }
                        }
                        if (G8 > 1) tmem_write8(lane_t + F::cA + 8u * g, o);
                    }
                    if (G8 > 1) tmem_wait_stores();
                    if (++stage == F::kStages) { stage = 0; kphase ^= 1u; }
                }

                // the end of the unit's part: l over the threads, then the outputs or the workspace
                asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll 1
                for (uint32_t g = 0; g < G8; g++) {
                    if (G8 > 1) {
                        tmem_read8(lane_t + F::cL + 8u * g, l);
                        tmem_wait_loads();
                    }
                    // eight sums over 32 lanes: halves of the rows change hands with the lanes, so that nine exchanges do instead of forty
                    float v[8];
#pragma unroll
                    for (uint32_t i = 0; i < 8; i++) v[i] = l[i];
#pragma unroll
                    for (uint32_t n = 4; n; n >>= 1) {
                        const bool upper = lane & (4u * n);
#pragma unroll
                        for (uint32_t i = 0; i < n; i++) {
                            const float give = upper ? v[i] : v[n + i], keep = upper ? v[n + i] : v[i];
                            v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, 4 * n);
                        }
                    }
                    v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], 2);
                    v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], 1);
                    if (lane % 4u == 0u) M.sum[warp][8u * g + lane / 4u] = v[0];
                }
                if (lane < RT) *reinterpret_cast<float2*>(M.state[warp][lane]) = make_float2(m_run, r_run);
                asm volatile("bar.sync 1, 128;" ::: "memory");
                const bool dead = *(volatile uint32_t*)&M.dead;
                const bool full = count == u.nt;
                const uint32_t slot = t == t_begin ? 0 : 1;
                float* part = part_of(a.ws, blockIdx.x, slot);
#pragma unroll 1
                for (uint32_t g = 0; 8u * g < rows; g++) {
                    if (G8 > 1) {
                        tmem_read8(lane_t + F::cA + 8u * g, o);
                        tmem_wait_loads();
                    }
#pragma unroll
                    for (uint32_t k = 0; k < 8; k++) {
                        const uint32_t i = 8u * g + k;
                        if (i >= rows) break;
                        const float2 mr = *reinterpret_cast<const float2*>(M.state[warp][i]);
                        float sum = (M.sum[0][i] + M.sum[1][i]) + (M.sum[2][i] + M.sum[3][i]);
                        if (dead) sum = NAN;
                        if (full) {
                            const uint32_t gr = row0 + i, qrow = (uint32_t)r.start + gr / a.group, qh = head * a.group + gr % a.group;
                            const float v = sum == 0.0f ? 0.0f : o[k] / sum * exp2_to_zero(mr.y == -INFINITY ? 0.0f : mr.y - mr.x);
                            if (tid < D) store_out<T>(a, qrow, qh, tid, v);
                            if (tid == 0 && a.lse) a.lse[(size_t)qrow * a.q_heads + qh] = sum == 0.0f ? -INFINITY : (mr.x + log2f(sum)) * 0.6931471805599453f;
                        } else {
                            if (tid < D) part[i * D + tid] = o[k];
                            if (tid == 0) *reinterpret_cast<float4*>(part + kPartRows * 128 + 4 * i) = make_float4(mr.x, mr.y, sum, 0.0f);
                        }
                    }
                }
                if (!full && j == 0 && tid == 0) {
                    // the worker that has the unit's last tile
                    const unsigned long long last = t + u.nt - 1;
                    Cut cut = {1u, req, head, rt, worker_of(last, total, workers), slot, {0, 0}};
                    reinterpret_cast<Cut*>(a.ws)[blockIdx.x] = cut;
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");
                t += count;
            }
        }
    }
    tmem_fence_before_sync();
    __syncthreads();
    if (tid == 0 && *(volatile uint32_t*)&M.dead) pages_fault(a.rep, WM_ERR_TIMEOUT, 0);
    if (warp == 4) {
        tmem_fence_after_sync();
        tmem_free<F::kCols>(tmem);
    }
}

// The cut units' parts put together: block (worker, eight rows), thread (row, four channels).
template <typename T, int D, int RT>
__global__ void __launch_bounds__(2 * D)
k_attend_join(AttendArgs a)
{
    grid_dep_wait();
    grid_dep_launch();
    const uint32_t w0 = blockIdx.x, i = blockIdx.y * 8u + threadIdx.x / (D / 4), d = threadIdx.x % (D / 4) * 4u;
    const Cut cut = reinterpret_cast<const Cut*>(a.ws)[w0];
    if (!cut.valid) return;
    const Request r = request_of(a, cut.req);
    const uint32_t gr = cut.rt * RT + i;
    if (gr >= (uint32_t)r.rows * a.group) return;
    float m = -INFINITY, R = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (uint32_t w = w0; w <= cut.last; w++) {
        const float* part = part_of(a.ws, w, w == w0 ? cut.slot : 0u);
        const float4 s = *reinterpret_cast<const float4*>(part + kPartRows * 128 + 4 * i), v = *reinterpret_cast<const float4*>(part + i * D + d);
        const float m1 = fmaxf(m, s.x), R1 = fmaxf(R, s.y), mb = m1 == -INFINITY ? 0.0f : m1, rb = R1 == -INFINITY ? 0.0f : R1;
        const float keep = exp2_fast(R - rb), take = exp2_fast(s.y - rb);
        l = l * exp2_fast(m - mb) + s.z * exp2_fast(s.x - mb);
        o[0] = o[0] * keep + v.x * take;
        o[1] = o[1] * keep + v.y * take;
        o[2] = o[2] * keep + v.z * take;
        o[3] = o[3] * keep + v.w * take;
        m = m1;
        R = R1;
    }
    store_joined<T>(a, r, gr, cut.head, d, m, R, l, o);
}

}  // namespace wm
