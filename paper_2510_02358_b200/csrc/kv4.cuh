// The 4-bit form of keys and values in the paged cache, shared by the kernels that write, read and
// attend over it.  Layout: dsp.h.  The order within a run of 16 tokens is that of the operand
// fragments of a 16x8x16 matrix instruction whose 16 rows are keys (channels inside a lane are
// contracted, so their order is free) or value channels (tokens inside a lane are contracted):
// a lane's codes of a run are whole 16-byte vectors and a warp's load is 512 contiguous bytes.
#pragma once

#include "dsp_common.cuh"

namespace dsp {

template <int D> struct Kv4 {
    static_assert(D == 64 || D == 128, "head sizes of the 4-bit cache");
    static constexpr int kRun = 16;                      // tokens of a run
    static constexpr int kRunBytes = kRun * (D + 8);
    static constexpr int kValueOff = kRun * D / 2;       // value codes behind the key codes
    static constexpr int kParamOff = kRun * D;           // the tokens' scales and offsets behind both
    // byte of the 32-bit word `w` (channels 8w .. 8w+7) of token t (0..15) within the key codes
    static __host__ __device__ __forceinline__ int key_word(int t, int w) {
        return D == 128 ? t * 64 + w * 4 : (t & 7) * 64 + (w >> 1) * 16 + (t >> 3) * 8 + (w & 1) * 4;
    }
    // and within the value codes
    static __host__ __device__ __forceinline__ int value_word(int t, int w) {
        const int c = (t & 7) >> 1;
        return D == 128 ? (t >> 3) * 512 + (w >> 1) * 64 + c * 16 + (t & 1) * 8 + (w & 1) * 4
                        : w * 64 + c * 16 + (t >> 3) * 8 + (t & 1) * 4;
    }
};

// Run of 16 tokens that holds slot `s` of head h: its number, for the cache's address.
__device__ __forceinline__ long long run_index(long long block, int place, int h, int Hkv, int page) {
    return (block * Hkv + h) * (page >> 4) + (place >> 4);
}

// Block of a slot (>= 0): a 64-bit division only where the slot needs it.
__device__ __forceinline__ long long block_of(long long slot, int page) {
    return (slot >> 32) ? slot / page : (long long)((uint32_t)slot / (uint32_t)page);
}

}  // namespace dsp
