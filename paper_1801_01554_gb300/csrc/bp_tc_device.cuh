// Device helpers of the tcgen05 kernels: barriers with bounded waits, TMA, tensor-core and TMEM
// instructions, and the turn between rows and 16-byte pieces in an epilogue.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <utility>

#include "bp_internal.h"

namespace bp {
namespace {

using bf16 = __nv_bfloat16;

constexpr int BM = 128;   // rows of a tile (TMEM lanes)
constexpr int BK = 64;    // K per stage: 64 bf16 = one 128-byte swizzle row
constexpr int UMMA_K = 16;

constexpr unsigned long long kWaitNs = 2000000000ull;
constexpr unsigned kWaitIters = 1u << 28;

// ------------------------------------------------------------ PTX helpers
__device__ __forceinline__ uint32_t smem_u32(const void* p) {
    return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ unsigned long long global_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void mbar_init(uint64_t* bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count)
                 : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)),
                 "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, unsigned parity) {
    unsigned done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
// Whether the phase is complete, without waiting.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, unsigned parity) {
    unsigned done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
// Bounded wait.  Returns false if it ran out or another role aborted.
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, unsigned parity, volatile int* abort_flag,
                                          int* flags) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    for (unsigned it = 1; it < kWaitIters; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 255u) == 0) {
            if (*abort_flag) return false;
            if (global_ns() - t0 > kWaitNs) break;
        }
    }
    *abort_flag = 1;
    atomicOr(flags, kFlagTimeout);
    return false;
}

__device__ __forceinline__ void tma_load_2d(void* smem_dst, const CUtensorMap* map, int c0, int c1,
                                            uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(smem_dst)),
        "l"((unsigned long long)map), "r"(c0), "r"(c1), "r"(smem_u32(bar))
        : "memory");
}

// True in one lane of the (converged) warp.  Unlike a test of the lane number it tells
// the compiler that a single thread follows, so that the operands of the TMA and MMA
// instructions can stay in uniform registers.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// Programmatic dependent launch: wait for the kernels this one depends on (their
// writes are then visible), and let the next kernel of the stream start its setup.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Shared-memory matrix descriptor, 128-byte swizzle (tcgen05 descriptor version 1).
//   K-major:  the operand's rows are 128 bytes (64 of K); 8-row groups 1024 bytes
//             apart (stride offset); the leading offset is unused.
//   MN-major: blocks of 64 K rows x 64 of M or N (128 bytes); 8 K rows are 1024
//             bytes apart (stride offset), the next 64 of M or N one block, 8 KB
//             (leading offset).
// The upper word is constant; the lower one holds the address (in 16-byte units, below
// 2^14) and the leading offset, so that stages and K steps are plain additions to it.
constexpr uint32_t kMnBlockBytes = BK * 64 * 2;
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);   // stride offset, version 1, 128-byte swizzle
template <bool MN>
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr) {
    return (addr >> 4) | (((MN ? kMnBlockBytes : 16u) >> 4) << 16);
}
// From one K step of UMMA_K to the next inside a stage, in 16-byte units.
template <bool MN>
__device__ __forceinline__ constexpr uint32_t k_step_units() { return (MN ? UMMA_K * 128 : UMMA_K * 2) >> 4; }

// Instruction descriptor of tcgen05.mma kind::f16: bf16 A and B, fp32 D, M x N
// tile, each operand K-major or MN-major.
__host__ __device__ constexpr uint32_t idesc_bf16(int M, int N, bool a_mn, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// One tcgen05.mma: operands by the lower words of their descriptors; the first one of
// a tile overwrites the accumulator.
template <uint32_t IDESC>
__device__ __forceinline__ void umma_bf16(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(tmem_d),
        "r"(a_lo), "r"(b_lo), "n"(kDescHi), "n"(IDESC), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void umma_commit(uint64_t* bar) {
    asm volatile(
        "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
            smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tc_fence_before() {
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after() {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// 32 lanes x 32 consecutive fp32 columns from TMEM.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
          "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// Logistic for bf16 outputs: hardware exp2 and reciprocal (1 ulp each; an IEEE divide
// here cost a quarter of a training step in the epilogues).  For 1 + e^-x beyond the
// largest float the quotient is 0, the logistic's value there.
__device__ __forceinline__ float sigmoid_fast(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + __expf(-x)));
    return r;
}

// 32 lanes x 16 consecutive fp32 columns from TMEM.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// And back.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&v)[16]) {
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]),
        "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A warp's 32 x 32 block of bf16 as 16-byte pieces (8 columns).  Global memory is read
// and written with lane (row 8 j + lane / 4, piece lane % 4), four lanes to a 64-byte
// row segment; the arithmetic wants lane = row.  The warp's 2 KB of shared memory turns
// one into the other (pieces permuted by row so that both sides spread over the banks).
// Loading a row per lane instead costs 32 cache-line lookups an instruction (the output
// layer's epilogue took 17,200 clocks a 128 x 256 tile, 14,600 with whole segments; a
// 1024-2048-2048-512 step of 1,001 patterns 81.8 us, 79.8), but no turn through shared
// memory: it is kept for 64-column tiles, one chunk per warp, where the latency of that
// counts for more (208-1024-32 at 512 patterns: 20.6 us against 20.9).
struct Row32 {
    uint4 u[4];
};
__device__ __forceinline__ uint4* piece_at(uint4* sS4, int row, int piece) {
    return sS4 + row * 4 + (piece ^ ((row >> 1) & 3));
}
// rows past `rows` and pieces past `pieces` are zero
__device__ __forceinline__ void load_block(Row32& r, const bf16* p, int ld, int rows, int pieces) {
    const int lane = threadIdx.x & 31, piece = lane & 3;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = 8 * j + (lane >> 2);
        r.u[j] = (row < rows && piece < pieces) ? *reinterpret_cast<const uint4*>(p + (size_t)row * ld + piece * 8)
                                                : make_uint4(0u, 0u, 0u, 0u);
    }
}
__device__ __forceinline__ void load_own_row(Row32& r, const bf16* p, int ld, int rows, int pieces) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        r.u[k] = (lane < rows && k < pieces) ? reinterpret_cast<const uint4*>(p + (size_t)lane * ld)[k]
                                             : make_uint4(0u, 0u, 0u, 0u);
}
__device__ __forceinline__ void block_to_rows(Row32& r, uint4* sS4) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < 4; ++j) *piece_at(sS4, 8 * j + (lane >> 2), lane & 3) = r.u[j];
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) r.u[k] = *piece_at(sS4, lane, k);
    __syncwarp();   // the block is rewritten
}
__device__ __forceinline__ float row_value(const Row32& r, int c) {   // c is a compile-time constant
    const uint4& u = r.u[c >> 3];
    const uint32_t w = ((c >> 1) & 3) == 0 ? u.x : ((c >> 1) & 3) == 1 ? u.y : ((c >> 1) & 3) == 2 ? u.z : u.w;
    return __uint_as_float((c & 1) ? (w & 0xffff0000u) : (w << 16));
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
    asm volatile("prefetch.tensormap [%0];" ::"l"((unsigned long long)m) : "memory");
}

// Launch whose setup may overlap the previous kernel's tail (the kernel calls pdl_wait).
template <class... P, class... A>
cudaError_t launch_pdl_grid(void (*k)(P...), dim3 grid, dim3 threads, size_t smem, cudaStream_t s, A&&... args) {
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = grid;
    c.blockDim = threads;
    c.dynamicSmemBytes = smem;
    c.stream = s;
    c.attrs = at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, k, std::forward<A>(args)...);
}
template <class... P, class... A>
cudaError_t launch_pdl(void (*k)(P...), int grid_x, int grid_y, int threads, size_t smem, cudaStream_t s, A&&... args) {
    return launch_pdl_grid(k, dim3(grid_x, grid_y), dim3(threads), smem, s, std::forward<A>(args)...);
}

}  // namespace
}  // namespace bp
