// What the bf16 kernels on the legacy matrix instructions share: asynchronous 16-byte copies, fragments, products, and
// where a 16-byte chunk of a row stands in shared memory.
#pragma once
#include "ptx.cuh"

namespace skipffn {

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool on)
{
    // `on` false: 16 zero bytes, nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// all but the last N groups of this thread have landed
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// four 8x8 matrices: thread t holds row t/4, columns 2(t%4), +1 of each; shared-memory rows at the threads' addresses
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// D[16 x 8] += A[16 x 16] B[16 x 8]
__device__ __forceinline__ void mma_16x8(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// byte of 16-byte chunk ch of row r in a tile of DP columns: chunks of eight neighbouring rows fall on different banks
template <int DP> __device__ __forceinline__ uint32_t chunk_at(int r, int ch) { return r * DP * 2 + ((ch & ~7) | ((ch ^ r) & 7)) * 16; }

}  // namespace skipffn
