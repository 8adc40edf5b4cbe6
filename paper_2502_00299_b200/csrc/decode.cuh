// Device helpers shared by the kernels that work on the decode cache (rotate.cu, attend.cu, evict.cu): rows of a paged cache
// [num_pages, page_size, Hkv, d] found through a sequence's block table, bf16 pairs, vector loads, and the ordering against the
// kernel ahead.
//
// These kernels are on the SMs while the kernel ahead, which may be one of them, still writes what they read: queries, lengths, sums, rows, and, from a
// program's own kernels, tables, positions and angles. All of that is therefore read with coherent loads (plain ones, asynchronous copies,
// load_once), which stay behind the wait. The read-only path (the intrinsic and the .nc loads) is for data that nothing writes as long as a kernel
// lives: the compiler may move such a load in front of the wait, and no wait makes it see what was written meanwhile.
#pragma once
#include "decode.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace chunkkv {

// Row `row` (below cap) of the sequence with table `table` as a row of the cache, page * page_size + slot; -1: its page is outside the cache.
__device__ __forceinline__ int paged_row(const PagedCache& c, const int32_t* table, int row) {
    const int p = static_cast<int>((__umulhi(c.magic, static_cast<uint32_t>(row)) + static_cast<uint32_t>(row)) >> c.shift);
    const int page = table[p];
    return static_cast<unsigned>(page) < static_cast<unsigned>(c.num_pages) ? page * c.page_size + (row - p * c.page_size) : -1;
}

__device__ __forceinline__ float2 bf16_pair(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 16 bytes that are read once: no line of the L1 is kept for them.
__device__ __forceinline__ uint4 load_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Launched as a programmatic dependent: everything that the kernel ahead (and those before it) wrote is there after this; only then may
// the kernel behind be set up. A kernel that is always launched behind one that begins so may therefore read what that one's predecessors wrote
// before its own wait: attend_join_kernel does (lengths), behind attend_kernel. No other may: attend_join_kernel itself and the prefill's kernels
// let the kernel behind be set up before they have waited.
__device__ __forceinline__ void begin_dependent() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

}  // namespace chunkkv
