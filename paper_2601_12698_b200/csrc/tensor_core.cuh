// The fifth-generation tensor cores (sm_100a): tensor memory, matrix products, descriptors.
#pragma once

#include "attend_common.cuh"

namespace rt {

// ---- tensor memory and matrix instructions -----------------------------------------------------------------

__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
        "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
// Waits for this thread's loads.  The registers are named, so that nothing that uses them is moved ahead of the wait.
__device__ __forceinline__ void tmem_wait_load(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                   "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27])
                 :
                 : "memory");
    asm volatile("" : "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void tmem_wait_load(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :
                 : "memory");
}
// The registers of a load that an earlier statement has waited for.
__device__ __forceinline__ void tmem_loaded(uint32_t (&r)[32])
{
    asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                      "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
    asm volatile("" : "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                      "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]),
        "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tc_commit(uint64_t* bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// One lane of a converged warp.  The warp that issues products runs converged and elects a lane only around the instructions
// themselves: addresses and descriptors then live in uniform registers, which is where the instruction wants them.  (With the
// warp's number taken by shuffle as well, so that the compiler sees the role as one of whole warps, the prefix kernel went from
// 201 to 194 us at 256 sequences x 4 heads x 8 key/value heads of 128, prefix 32768; with constant slots, to 188.)
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// D (128 x N, binary32, tensor memory) (+)= A B with A and B described in shared memory.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// The same with A (128 x 16 of 16-bit elements, two to a column) in tensor memory.
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
                 "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Shared memory matrix descriptor.  The operand's rows are ROW_BYTES long (32, 64 or 128: the swizzle), strides in bytes:
// `stride` between groups of eight rows; `leading`, for an operand whose rows run along the product's inner axis, between
// blocks of ROW_BYTES columns.
// The parts that do not depend on the address are constants; addresses are added in units of 16 bytes.
template <int ROW_BYTES = 128>
__host__ __device__ __forceinline__ constexpr uint64_t tc_layout(uint32_t leading, uint32_t stride)
{
    return ((uint64_t)((leading >> 4) & 0x3FFFu) << 16) | ((uint64_t)((stride >> 4) & 0x3FFFu) << 32) | (1ull << 46) |
           ((ROW_BYTES == 128 ? 2ull : ROW_BYTES == 64 ? 4ull : 6ull) << 61);
}
__device__ __forceinline__ uint64_t tc_descriptor(uint64_t layout, uint32_t addr16)  // addr16: shared memory address / 16
{
    return layout | addr16;
}
// Instruction descriptor: binary32 accumulator, A and B both bf16 or both fp16, M = 128.  a_rows / b_rows: the operand's
// rows in shared memory run along the inner axis of the product.
template <typename M>
__device__ __forceinline__ constexpr uint32_t tc_instruction(int n, bool a_rows, bool b_rows)
{
    const uint32_t type = std::is_same<M, __nv_bfloat16>::value ? 1u : 0u;
    return (1u << 4) | (type << 7) | (type << 10) | ((a_rows ? 1u : 0u) << 15) | ((b_rows ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
           ((128u >> 4) << 24);
}

// Bounded wait whose polls sleep in hardware for up to kWaitSleepNs each: many roles wait most of the time.  Gives up after
// poll_limit polls or about a second, as mbarrier_wait_bounded.
constexpr uint32_t kWaitSleepNs = 20000;
__device__ __forceinline__ bool mbarrier_wait_sleeping(uint64_t* bar, uint32_t parity, unsigned poll_limit = kMbarrierPollLimit)
{
    const uint32_t addr = smem_u32(bar);
    long long t0 = 0;
    for (unsigned it = 0;; ++it) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done) : "r"(addr), "r"(parity), "r"(kWaitSleepNs) : "memory");
        if (done) return true;
        if (it == 0) t0 = clock64();
        if (it >= poll_limit || clock64() - t0 > kMbarrierCycleLimit) return false;
    }
}

__device__ __forceinline__ void mbarrier_arrive(uint64_t* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// The paged tiles that both tensor-core kernels read: 128 rows (keys) of COLS elements of 16 bits, in blocks of 64 columns,
// a block's rows 128 bytes long with their 16-byte pieces exchanged by the row number (the 128-byte swizzle).
constexpr int kTileBlockBytes = 128 * 128;

// Fetches this thread's pieces of one tile (128 rows x COLS elements of 16 bits from a plain cache) into shared memory with
// cp.async: piece u of rows r0, r0 + STEP, ...  The places are read ahead of the copies, eight at a time (a copy is a
// volatile statement that no load moves across: one at a time, each copy waited for its place, 125 cycles apiece), and since
// STEP is a multiple of eight the swizzle is the same for all of them.  `off`: byte offsets, negative = zeros.
template <int COLS>
__device__ __forceinline__ void fetch_plain_tile(unsigned char* dst, const unsigned char* side, const long long* off, int p, bool dims_there, int dim_bytes)
{
    constexpr int UNITS = COLS / 8, STEP = 128 / UNITS, N = 128 / STEP;
    static_assert(STEP % 8 == 0, "rows of a thread share the swizzle");
    const int u = p % UNITS, r0 = p / UNITS;
    const uint32_t to = smem_u32(dst) + (u >> 3) * kTileBlockBytes + r0 * 128 + (((u & 7) ^ (r0 & 7)) << 4);
    const unsigned char* from = side + dim_bytes + u * 16;
#pragma unroll
    for (int h = 0; h < N; h += 8) {
        long long o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = off[r0 + (h + i) * STEP];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool there = o[i] >= 0 && dims_there;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (h + i) * STEP * 128), "l"(there ? from + o[i] : side),
                         "r"(there ? 16 : 0) : "memory");
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}

// The same for codes: 16 a piece, turned into fp16 (two 16-byte pieces) on the way through registers.  N pieces per thread and
// tile; piece i of the next tile is asked for as soon as piece i of this one has been stored, so the loads never stop.
template <int COLS>
struct CodePieces {
    static constexpr int UNITS = COLS / 16, STEP = 128 / UNITS, N = 128 / STEP;
    static_assert(STEP % 8 == 0, "rows of a thread share the swizzle");
};
template <int FMT>
__device__ __forceinline__ void store_codes(unsigned char* lo, unsigned char* hi, const uint4& x)
{
    uint4 a, b;
    codes_to_half4<FMT>(x.x, a.x, a.y);
    codes_to_half4<FMT>(x.y, a.z, a.w);
    codes_to_half4<FMT>(x.z, b.x, b.y);
    codes_to_half4<FMT>(x.w, b.z, b.w);
    *reinterpret_cast<uint4*>(lo) = a;
    *reinterpret_cast<uint4*>(hi) = b;
}

}  // namespace rt
