// kvx_umma.cuh -- device helpers of the attention kernels on the tensor cores (library-internal): thread copies
// that announce themselves, MMAs with an operand in TMEM, packed fp32 arithmetic.
#pragma once

#include <cuda.h>

#include "kvx_tc_common.cuh"

namespace kvx {
namespace {

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
// An arrival on the barrier once the thread's copies so far are complete (counted by the barrier as any other).
__device__ __forceinline__ void cp_async_arrive(uint32_t mbar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(mbar) : "memory");
}

// D[tmem] (+)= A[tmem] . B[smem], bf16 inputs, fp32 accumulate
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// MN-major 128-byte-swizzled operand: lbo between 64-channel blocks, 1024 bytes between 8-row groups.
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr, uint32_t lbo)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)((lbo >> 4) & 0x3FFFu) << 16 | (uint64_t)(1024u >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// 32 columns of the warp's lanes into 32 consecutive values of an array
__device__ __forceinline__ void tmem_ld32_to(uint32_t* r, uint32_t taddr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]),"=r"(r[1]),"=r"(r[2]),"=r"(r[3]),"=r"(r[4]),"=r"(r[5]),"=r"(r[6]),"=r"(r[7]),
          "=r"(r[8]),"=r"(r[9]),"=r"(r[10]),"=r"(r[11]),"=r"(r[12]),"=r"(r[13]),"=r"(r[14]),"=r"(r[15]),
          "=r"(r[16]),"=r"(r[17]),"=r"(r[18]),"=r"(r[19]),"=r"(r[20]),"=r"(r[21]),"=r"(r[22]),"=r"(r[23]),
          "=r"(r[24]),"=r"(r[25]),"=r"(r[26]),"=r"(r[27]),"=r"(r[28]),"=r"(r[29]),"=r"(r[30]),"=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Waiter whose bound (~1 s) starts again while another warp of the CTA reports progress in *beat.
struct BeatWaiter {
    volatile int* abort;
    volatile int* beat;
    unsigned* status;
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) const
    {
        if (mbar_try_wait(bar, parity)) return true;
        unsigned long long t0 = globaltimer();
        int seen = *beat;
        while (true) {
            if (mbar_try_wait_sleep(bar, parity, 100000u)) return true;
            if (*abort) return false;
            if (globaltimer() - t0 > kWaitNs) {
                if (*beat == seen) {
                    *abort = 1;
                    set_status(status, KVX_DEV_WAIT_TIMEOUT);
                    return false;
                }
                seen = *beat;
                t0 = globaltimer();
            }
        }
    }
};
// After a wait has run out: a copy still on its way must not land in shared memory that is no longer this CTA's.
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity)
{
    const unsigned long long t0 = globaltimer();
    while (!mbar_try_wait(bar, parity) && globaltimer() - t0 < kWaitNs) {}
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
// Values a completed load has written: what uses them stays behind this point.
__device__ __forceinline__ void pin32(uint32_t* r)
{
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
          "l"(reinterpret_cast<unsigned long long&>(c)));
    return reinterpret_cast<float2&>(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return reinterpret_cast<float2&>(r);
}
// Barriers (8 bytes each) in the control block.
template <int STAGES> struct Bars {
    static constexpr int full = 0, empty = STAGES, sfull = 2 * STAGES, pfull = sfull + 2, ofull = pfull + 2, qfull = ofull + 2,
                         qempty = qfull + 1, done = qempty + 1, mlfull = done + 1, mlempty = mlfull + 1, added = mlempty + 1;
};
// Tensor copy of a box, completing on an mbarrier.
__device__ __forceinline__ void tma_box3(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t mbar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
                 "l"(map), "r"(mbar), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
// Lane j of four holds row j's chunks 0 .. 3 of four words; afterwards chunk j of rows 0 .. 3.
__device__ __forceinline__ void transpose_quad(uint32_t (&v)[16])
{
    const uint32_t lane = threadIdx.x;
#pragma unroll
    for (int s = 1; s <= 2; s <<= 1) {
        const bool up = lane & s;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (c & s) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t& a = v[c * 4 + e];
                uint32_t& b = v[(c + s) * 4 + e];
                const uint32_t t = __shfl_xor_sync(0xffffffffu, up ? a : b, s);
                if (up) a = t;
                else b = t;
            }
        }
    }
}
// N (16 or 32) columns of the warp's lanes written
template <int N> __device__ __forceinline__ void store_p(uint32_t taddr, const uint32_t* r)
{
    if constexpr (N == 32) tmem_st32(taddr, r);
    else tmem_st16(taddr, *reinterpret_cast<const uint32_t(*)[16]>(r));
}
// Threads of a group (whole warps) wait for one another, and learn whether any of them says so.
__device__ __forceinline__ bool group_any(int id, int threads, bool mine)
{
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(any)
        : "r"((uint32_t)mine), "r"(id), "r"(threads)
        : "memory");
    return any != 0;
}
// Threads of a group (whole warps) wait for one another.
__device__ __forceinline__ void group_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled tiled_encoder()
{
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

}  // namespace
}  // namespace kvx
