// Tensor-core building blocks: matrix descriptors, tcgen05.mma and its completion, tensor-memory reads,
// tiled (tensor-map) copies, and waits bounded by time.  Part of the translation unit wm_pages.cu.
#pragma once

namespace wm {

// Shared-memory operand descriptor: start, the two strides (bytes) and the swizzle of its rows (2: 128 bytes, 4: 64, 6: 32).
// K-major tiles (rows of the operand along the swizzled bytes): `stride` is the distance of groups of eight rows.
// MN-major tiles (the operand's rows run along the swizzled bytes): `stride` is the distance of groups of eight k, `lead` that
// of blocks of one swizzle width along the rows.
constexpr uint32_t kSw128 = 2, kSw64 = 4, kSw32 = 6;
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead, uint32_t stride, uint32_t swizzle)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 | (uint64_t)swizzle << 61;
}
// Instruction descriptors: f32 sums of e4m3 x e4m3 (kind f8f6f4) or f16 x f16 (kind f16); mn_a / mn_b: the operand is MN-major.
// (e5m2_a: A's elements are e5m2 instead).
__host__ __device__ constexpr uint32_t mma_desc(uint32_t m, uint32_t n, bool mn_a, bool mn_b, bool e5m2_a = false)
{
    return 1u << 4 | (e5m2_a ? 1u << 7 : 0u) | (mn_a ? 1u << 15 : 0u) | (mn_b ? 1u << 16 : 0u) | (n >> 3) << 17 | (m >> 4) << 24;
}
// The issuing instructions are executed by a whole warp and take effect in the one lane for which `leader` holds: the code around
// them stays uniform, so that descriptors live in uniform registers (issued from inside a branch of one lane, every operand is moved
// there by itself; eight MMAs then took 840 cycles to issue).
__device__ __forceinline__ void mma_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add, bool leader = true)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add), "r"((uint32_t)leader) : "memory");
}
// f16 x f16 with A in tensor memory (a row per lane, two elements a column).
__device__ __forceinline__ void mma_f16_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, bool add, bool leader = true)
{
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(desc), "r"((uint32_t)add), "r"((uint32_t)leader) : "memory");
}
// An arrival on the barrier when everything this thread has issued so far is done.
__device__ __forceinline__ void mma_commit(uint32_t bar_s, bool leader = true)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                 ::"r"(bar_s), "r"((uint32_t)leader) : "memory");
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
template <uint32_t N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <uint32_t N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <uint32_t COLS> __device__ __forceinline__ void tmem_alloc(uint32_t smem_result)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_result), "n"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <uint32_t COLS> __device__ __forceinline__ void tmem_free(uint32_t taddr)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "n"(COLS) : "memory");
}
// 8 columns of this thread's lane (no wait: tmem_wait_loads before the values are used).
__device__ __forceinline__ void tmem_read8(uint32_t taddr, float* v)
{
    uint32_t* w = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "r"(taddr) : "memory");
}
#define WM_R8(w, i) "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]), "=r"(w[i + 6]), "=r"(w[i + 7])
#define WM_I8(w, i) "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7])
__device__ __forceinline__ void tmem_read32(uint32_t taddr, float* v)
{
    uint32_t* w = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : WM_R8(w, 0), WM_R8(w, 8), WM_R8(w, 16), WM_R8(w, 24) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_write8(uint32_t taddr, const float* v)
{
    const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), WM_I8(w, 0) : "memory");
}
__device__ __forceinline__ void tmem_write16(uint32_t taddr, const uint32_t* w)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), WM_I8(w, 0), WM_I8(w, 8) : "memory");
}
#undef WM_R8
#undef WM_I8
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// One box of a 4-d tensor map into shared memory; rows that lie outside the tensor arrive as zeros.
__device__ __forceinline__ void tile_load4(uint32_t dst, const void* map, int32_t c1, int32_t c2, int32_t c3, uint32_t bar_s)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(c1), "r"(c2), "r"(c3), "r"(bar_s) : "memory");
}
// The map itself, ahead of its first use.
__device__ __forceinline__ void fetch_map(const void* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t bar_s, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar_s), "r"(bytes) : "memory");
}

// A wait that gives up after budget_ns.  `dead` is the block's flag in shared memory: once it is up, every wait of the block
// returns at once, the block runs through to its end on whatever is there and reports the failure.
__device__ __forceinline__ void mbar_wait(uint32_t bar_s, uint32_t parity, uint32_t budget_ns, volatile uint32_t* dead)
{
    if (mbar_try(bar_s, parity)) return;
    const uint32_t t0 = now_ns();
    while (!*dead) {
        if (mbar_try(bar_s, parity)) return;
        if (now_ns() - t0 > budget_ns) { *dead = 1u; return; }
    }
}

// The same where what is waited for is usually there: asked without going to sleep (a wait that does not have to wait took 130
// cycles more through try_wait).
__device__ __forceinline__ void mbar_wait_hot(uint32_t bar_s, uint32_t parity, uint32_t budget_ns, volatile uint32_t* dead)
{
    for (uint32_t i = 0; i < 64u; i++)
        if (mbar_test(bar_s, parity)) return;
    mbar_wait(bar_s, parity, budget_ns, dead);
}

// 16 bytes of shared memory.
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The same down to the smallest floats: for the outputs' last factor.
__device__ __forceinline__ float exp2_to_zero(float x)
{
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_min(float x)
{
    float r;
    asm volatile("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
// Two at a time: a * b + c and a + b.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
        "l"(*reinterpret_cast<unsigned long long*>(&c)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
    return *reinterpret_cast<float2*>(&r);
}
// The largest of the warp's values (NaN only if all are).
__device__ __forceinline__ float warp_max(float x)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace wm
