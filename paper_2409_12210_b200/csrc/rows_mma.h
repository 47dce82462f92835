// Products of rows of a weight matrix with a few token rows, fragments straight from global memory: shared by the kernels
// that stream weights once (linear_rows.cu, decode.cu).
//
// Fragments without shared memory: a sum over k may be taken in any order as long as both operands agree on it.  Thread
// t of a group of four loads 16 contiguous bytes of its row of w and the same 16 bytes of its row of x; the k-th pair of
// 16-bit numbers in them plays the part of the fragment's columns 2t, 2t+1 (+8).  Four such loads of neighbouring threads
// cover 64 contiguous bytes of a row.  8-bit operands are widened to fp16 on the way (exact) and use the fp16 form.
#pragma once

#include "modse_internal.h"

namespace modse {

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool f16)
{
    if (f16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16 bytes, or zeros where there are none.  volatile: the loads of a step stay ahead of its products.  Not the read-only
// path: the kernel ahead may still be writing x when this one starts, and that path promises nothing for such data, even
// where it is read after wait_for_earlier_kernels.
__device__ __forceinline__ uint4 load_stream(const unsigned char *p, bool in)
{
    uint4 v;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\t"
                 "mov.b32 %3, 0;\n\t@q ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((int)in));
    return v;
}
__device__ __forceinline__ uint4 load_shared_rows(const unsigned char *p, bool in)      // x: every block reads it, L1 may keep it
{
    uint4 v;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\t"
                 "mov.b32 %3, 0;\n\t@q ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((int)in));
    return v;
}

__device__ __forceinline__ uint32_t word_at(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

}  // namespace modse
