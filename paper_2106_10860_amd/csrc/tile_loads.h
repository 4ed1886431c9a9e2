// What the products on 8-bit matrices share: the way of a tile of rows from memory to LDS, and the order of the tiles.
#pragma once

#include "block_common.h"

namespace maddness {

// The first `keep` of 16 bytes, 0 for the others.
__device__ __forceinline__ i32x4 first_bytes(i32x4 v, int64_t keep)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int b = (int)min(max(keep - 4 * i, (int64_t)0), (int64_t)4);
        v[i] = b == 4 ? v[i] : v[i] & (int)((1u << (8 * b)) - 1);
    }
    return v;
}

// Buffers of plain bytes, and the longest row of 8-bit values that 256 of stay below 2^32 bytes.
constexpr int kBufferFlags = 0x00027000;
constexpr int64_t kMostStride = (int64_t)1 << 23;
constexpr int kReads = 0x100, kProducts = 0x8;      // kinds of instructions to __builtin_amdgcn_sched_group_barrier

__device__ __forceinline__ i32x4 buffer_of(const uint8_t *base, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)at), __builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)),
                 __builtin_amdgcn_readfirstlane((int)bytes), kBufferFlags};
}

// 16 bytes for each lane from `at` in the buffer to lds + 16 lane, past the registers; zeros from beyond its end.  As text, because the compiler
// waits for all such loads before any read of LDS, the next block's too: wait_for_loads is called where they are needed.
__device__ __forceinline__ void load_to_lds(i32x4 buffer, uint32_t at, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(at), "s"(buffer) : "memory", "m0");
}

// The same where `wanted` is not 0: a branch that the compiler does not see, and so does not gather other instructions around.
__device__ __forceinline__ void load_to_lds_if(uint32_t wanted, i32x4 buffer, uint32_t at, uint32_t lds)
{
    asm volatile("s_cmp_eq_u32 %3, 0\n\ts_cbranch_scc1 .Lno_load%=\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds\n.Lno_load%=:" ::"s"(lds),
                 "v"(at), "s"(buffer), "s"(wanted)
                 : "memory", "m0", "scc");
}

// Waits until this wavefront's loads have come and its reads of LDS are done.
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// Waits until all but the last N loads of this wavefront have come and its reads of LDS are done.
template <int N>
__device__ __forceinline__ void wait_for_loads_but() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }

__device__ __forceinline__ void wait_for_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Waits for the workgroup's other wavefronts.
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }

// The index among a launch's workgroups that work, such that each of the 8 dies (workgroups go to them in turn) gets neighbours.
__device__ __forceinline__ uint32_t by_die(uint32_t id, uint32_t total)
{
    const uint32_t die = id % 8, each = total / 8, more = total % 8;
    return die * each + min(die, more) + id / 8;
}

}  // namespace maddness
