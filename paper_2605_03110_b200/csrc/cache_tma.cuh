// TMA access to the pages of a cache and to the new tokens' queries: maps, loads, warp-level matrix instructions.
#pragma once

#include "cache_dev.cuh"
#include "gram_tc_dev.cuh"

namespace ada {
namespace tc {

static __device__ __forceinline__ void tma_load_4d(const CUtensorMap* map, unsigned long long* bar, void* dst, int c0,
                                                   int c1, int c2, int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<unsigned long long>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1),
          "r"(c2), "r"(c3)
        : "memory");
}

// One lane of a converged warp, the same one every time.  The compiler knows that it is one: operands of MMAs and TMA loads,
// which are uniform registers, are then moved there once, and not lane by lane as behind a comparison with the lane's
// number.
static __device__ __forceinline__ bool elect_one() {
    unsigned p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0u;
}
// MMAs of a converged warp, executed by the lane whose `lead` is not 0 (elect_one): without a branch around them, and with
// descriptors as their low words (address and leading offset; the high word, SBO 1024, version 1, 128-byte swizzle, is a
// constant), an instruction takes 68 cycles to issue beside two busy warps on its scheduler, where the tensor core takes 64;
// behind `if (elect_one())` 78, behind `if (lane == 0)` 168.
static constexpr unsigned DESC_HI = 0x40004040u;
static __device__ __forceinline__ void umma_ss(unsigned tmem_d, unsigned a_lo, unsigned b_lo, unsigned idesc,
                                               unsigned accumulate, unsigned lead) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 x, y;\n\t"
        "mov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %6, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(DESC_HI), "r"(lead)
        : "memory");
}
// left operand in TMEM
static __device__ __forceinline__ void umma_ts(unsigned tmem_d, unsigned tmem_a, unsigned b_lo, unsigned idesc,
                                               unsigned accumulate, unsigned lead) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 y;\n\t"
        "mov.b64 y, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %6, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(DESC_HI), "r"(lead)
        : "memory");
}
static __device__ __forceinline__ void umma_commit_lead(unsigned long long* bar, unsigned lead) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %1, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
        ::"r"(smem_u32(bar)), "r"(lead)
        : "memory");
}
// low descriptor words of a K-major tile (rows of 128 bytes) and of an MN-major one (128-byte rows of 64 elements, the
// next 64 elements `next` bytes further on)
static __device__ __forceinline__ unsigned desc_lo(unsigned addr) { return (addr >> 4) | 0x10000u; }
static __device__ __forceinline__ unsigned desc_lo_mn(unsigned addr, unsigned next) { return (addr >> 4) | ((next >> 4) << 16); }

static __device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

static __device__ __forceinline__ void ldsm4(unsigned addr, unsigned (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
static __device__ __forceinline__ void ldsm4t(unsigned addr, unsigned (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
static __device__ __forceinline__ void mma16816(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// one of eight bf16 is NaN or infinite (an exponent of all ones: 0 times it is NaN)
static __device__ __forceinline__ bool nonfinite8(const uint4& w) {
    const __nv_bfloat162 zero = __float2bfloat162_rn(0.f);
    __nv_bfloat162 x = zero;
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&u[i]), zero, x);
    const unsigned y = *reinterpret_cast<const unsigned*>(&x);
    return (y & 0x7fff7fffu) != 0u;
}

// Takes the elements that are not finite out of eight bf16 in shared memory: put(element, as +inf, as -inf), a NaN as both
// (what is added to a sum in their stead later: +inf and -inf make NaN).
template <typename F>
static __device__ __forceinline__ void take_nonfinite(uint4* at, F put) {
    unsigned* u = reinterpret_cast<unsigned*>(at);
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {
        const unsigned h = u[e >> 1] >> (16 * (e & 1)) & 0xffffu;
        if ((h & 0x7f80u) != 0x7f80u) continue;
        const bool nan = (h & 0x7fu) != 0u;
        put(e, nan || h == 0x7f80u, nan || h != 0x7f80u);
        u[e >> 1] &= (e & 1) ? 0x0000ffffu : 0xffff0000u;
    }
}

// transposes an 8 x 8 matrix of 16-bit elements held as a matrix fragment (two elements of a row per lane)
static __device__ __forceinline__ unsigned transposed(unsigned x) {
    unsigned y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// (element, slot, head, page): boxes of 64 elements x `box_rows` slots of one head and page, 128-byte swizzle
static inline bool encode_pages(CUtensorMap* map, const CacheView& c, const void* base, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    const int ps = 1 << c.shift;
    const cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)ps, (cuuint64_t)c.h_kv, (cuuint64_t)c.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)c.d * 2, (cuuint64_t)ps * c.d * 2, (cuuint64_t)c.page_stride * 2};
    const cuuint32_t box[4] = {(cuuint32_t)BK, (cuuint32_t)box_rows, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace tc
}  // namespace ada
