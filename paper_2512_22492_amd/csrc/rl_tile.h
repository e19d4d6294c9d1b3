// rl_tile.h -- key and value tiles in LDS as the matrix-core kernels read them
// (gfx950): the swizzled row layout, direct global-to-LDS loads, transposed
// reads, and lane exchanges between the scores of one query row.  Internal header.
#pragma once

#include "rl_common.h"

namespace rl_da {

// K and V stage tiles are [key][dim] rows of 256 bytes whose sixteen 16-byte
// chunks are stored at position chunk ^ chunk_swizzle(row); every four rows
// stay one contiguous kilobyte (what a wavefront's direct global-to-LDS load
// fills).  The swizzle keeps both operand reads free of bank conflicts, as
// measured with the LDS counters on gfx950 (64 banks of 4 bytes):
// ds_read_b128 serves its 64 lanes sixteen at a time, lanes l and l ^ 1,
// l ^ 2, l ^ 20, l ^ 24 (and their combinations) together, so the K operand
// reads (lane 16g + i: row i, chunk (4ks + g) ^ swizzle(i)) need swizzle(r ^
// d) != swizzle(r) ^ (the g difference) for those lane pairs -- rows r and
// r ^ 8 in particular, which the XOR with (row & 8) separates (without it
// the reads were 2-way conflicted); ds_read_b64_tr_b16 serves 32 lanes at a
// time, so the transposed V reads (eight consecutive rows, two adjacent
// chunks each) need swizzle(row) >> 1 distinct over eight consecutive rows.
__device__ __forceinline__ int chunk_swizzle(int row)
{
    return (((row & 7) << 1) | ((row >> 3) & 1)) ^ (row & 8);
}

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_short4_t;

// Four bf16 of one dim from four consecutive key rows of a [key][dim] LDS
// tile (ds_read_b64_tr_b16).  Within each 16-lane group, lane j receives
// element j % 4 of the 8-byte chunks addressed by lanes j / 4 + 4e, e = 0..3:
// when lane s addresses row (base + s / 4), dims (d0 + 4 (s % 4)) .. +3, lane
// j gets rows base .. base + 3 of dim d0 + j.
__device__ __forceinline__ uint2 lds_read_transposed(const uint16_t* p)
{
    const short4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)p);
    return __builtin_bit_cast(uint2, v);
}

// A lane's value and that of lane l ^ 16 (permlane16_swap exchanges 16-lane
// rows 1 <-> 0 and 3 <-> 2 between its two operands: with both equal to v,
// lane l receives v of lanes l & ~16 and l | 16), or of lane l ^ 32
// (permlane32_swap, the two halves).  Vector-ALU operations, no LDS round
// trip.  The maxima are IEEE `maximum` (no canonicalising copies of the
// operands); the row maxima they combine are finite or -inf.
__device__ __forceinline__ float max_lanes_xor16(float v)
{
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v),
                                                    false, false);
    return __builtin_elementwise_maximum(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float max_lanes_xor32(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v),
                                                    false, false);
    return __builtin_elementwise_maximum(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_lanes_xor16(float v)
{
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v),
                                                    false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float sum_lanes_xor32(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v),
                                                    false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// A direct global-to-LDS load of 16 bytes per lane, from a per-lane global
// address to LDS address lds + 16 * lane (lds uniform, in M0), written as
// inline assembly so that the compiler neither tracks these loads nor waits
// for them: the kernel waits for its own loads before each stage barrier,
// and the compiler, not knowing which LDS buffer a load fills, would
// otherwise wait for it before every read of the other buffer.  (The nop is
// the wait state between the M0 write and the load that reads it.)
__device__ __forceinline__ void dma16(const uint8_t* gaddr, uint32_t lds)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 :
                 : "v"(gaddr), "{m0}"(lds)
                 : "memory");
}

}  // namespace rl_da
