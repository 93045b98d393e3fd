// tc_tiles.cuh -- tiles of 16-bit values for the 5th generation tensor cores:
// TMA copies of boxes of 64 columns (128 bytes a row, 128-byte swizzle), shared
// memory descriptors that read such a tile along either axis, and
// multiplications with both operands in shared memory.
//
// A box holds `rows` rows of 128 bytes; 16-byte chunk c of row r sits at
// r * 128 + ((c ^ (r & 7)) << 4) (boxes start on 1024 bytes).  Read as an operand
// it is either
//   K-major:  rows are M or N, the 64 columns are K; 16 of K are 32 bytes on;
//   MN-major: the 64 columns are M or N, rows are K; 16 of K are 16 rows on, the
//             next 64 of M or N another box, `lbo` bytes on.
#pragma once
#include <stdint.h>

#include "async.cuh"
#include "tc_signed.cuh"

namespace tiles {

constexpr uint32_t kBoxCols = 64;
constexpr uint32_t kRowBytes = 128;

__device__ __forceinline__ uint32_t chunk_at(uint32_t row, uint32_t chunk)
{
    return row * kRowBytes + ((chunk ^ (row & 7)) << 4);
}

__device__ __forceinline__ uint64_t desc(uint32_t addr, uint32_t lbo)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) |
           ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
constexpr uint32_t kStepK = 32 >> 4;               // descriptor step of 16 of K, K-major
constexpr uint32_t kStepMN = 16 * kRowBytes >> 4;  // the same, MN-major

// kind::f16: D fp32; A and B bf16 or f16, each K-major or MN-major; M = 128
__host__ __device__ constexpr uint32_t idesc(bool bf16, bool a_mn, bool b_mn, uint32_t n)
{
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) |
           ((b_mn ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t id, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(id), "r"((uint32_t)accumulate)
        : "memory");
}

// sixteen 32-bit columns of this warp's lanes (complete after wait_ld)
__device__ __forceinline__ void ld16(uint32_t taddr, float (&v)[16])
{
    uint32_t *u = reinterpret_cast<uint32_t *>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15}, [%16];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
          "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
        : "r"(taddr)
        : "memory");
}

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *tm, uint32_t x, uint32_t y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap *tm, uint32_t x, uint32_t y, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                     reinterpret_cast<uint64_t>(tm)),
                 "r"(x), "r"(y), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// until the stores committed have read their shared memory
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

__device__ __forceinline__ void prefetch_map(const CUtensorMap *tm)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory");
}

__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(p));
    return p != 0;
}

// Bounded waits of one CTA.  The first that gives up sets the CTA's flag and the
// context's error flag; from then on no wait waits and `going` is false, and every
// loop runs to its end on whatever the buffers hold (no address depends on them).
struct Waits {
    int *abort;  // shared memory
    int *err;
    uint64_t limit_ns;

    __device__ __noinline__ void slow(uint32_t bar, uint32_t parity) const
    {
        volatile int *flag = abort;
        if (*flag || async::mbar_wait_bounded(bar, parity, flag, limit_ns) || *flag) return;
        *flag = 1;
        atomicOr(err, 1);
    }
    __device__ __forceinline__ void pass(uint32_t bar, uint32_t parity) const
    {
        if (!async::mbar_try_wait(bar, parity)) slow(bar, parity);
    }
    __device__ __forceinline__ bool going() const { return *(volatile int *)abort == 0; }
};

// waits for something already under way, whoever gave up before
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity)
{
    const int never = 0;
    async::mbar_wait_bounded(bar, parity, &never, 20000000);
}

}  // namespace tiles
