// Values that move between the lanes of a wave by instruction modifiers, without LDS, and sums over lanes made of them.  Every lane has to
// take part.
#pragma once

#include "basq_internal.h"

namespace basq {
namespace {

// the value of another lane: CTRL, ROWS and BANKS as in the instruction's modifier; lanes that it leaves out give `old`
template <int CTRL, int ROWS = 0xF, int BANKS = 0xF>
__device__ __forceinline__ uint64_t moved(uint64_t old, uint64_t v) {
    const unsigned lo = __builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, ROWS, BANKS, false);
    const unsigned hi = __builtin_amdgcn_update_dpp((int)(old >> 32), (int)(v >> 32), CTRL, ROWS, BANKS, false);
    return (uint64_t)hi << 32 | lo;
}
template <int CTRL, int ROWS = 0xF, int BANKS = 0xF>
__device__ __forceinline__ unsigned moved(unsigned old, unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, ROWS, BANKS, false);
}
// sums of the lanes of half a wave up to this one, within rows of 16, then over two; then of the wave
template <class T>
__device__ __forceinline__ T half_scan(T v) {
    const T none = 0;
    v += moved<0x111>(none, v);                            // (row_shr 1, 2, 4, 8)
    v += moved<0x112>(none, v);
    v += moved<0x114>(none, v);
    v += moved<0x118>(none, v);
    v += moved<0x142, 0xA>(none, v);                       // (the last lane of rows 0 and 2, to rows 1 and 3)
    return v;
}
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
    v = half_scan(v);
    v += moved<0x143, 0xC>((T)0, v);                       // (lane 31, to rows 2 and 3)
    return v;
}
}  // namespace
}  // namespace basq
