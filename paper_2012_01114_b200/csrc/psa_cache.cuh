// Layout of the cache held in 4 bits, and the pieces that its kernels share.
//
// A page holds `page_size` tokens (a multiple of 16) of all key/value heads of a layer: [kv_heads][page_size / 16] blocks of
// 20 d bytes, a block being 16 tokens of one head.  A group of 32 channels of a token has two fp16 numbers S and M, and a code c
// stands for M + S (1 + c / 16).  In a block, with G = d / 32 groups:
//     0      K codes   [16 tokens][4 t][G] words: bits 4j hold channel 32 w + 8 t + 2 j, bits 16 + 4j the channel after it
//     8 d    K scales  [16 tokens][G] pairs (S, M)
//     10 d   V codes   [8 pairs of tokens][8 g][G] words: bits 4j hold channel 32 w + 4 g + j of the even token, bits 16 + 4j of the odd one
//     18 d   V scales  [8 pairs of tokens][G] (S even, S odd, M even, M odd)
// The words are those that a lane (g = lane / 4, t = lane % 4) of mma.m16n8k16 needs for its A operand, K with a token per row and V with a
// channel per row, so that a lane reads its words in one piece and nothing is transposed.  Bytes still belong to one token each: appending a token
// touches no other.  K's words give four operand registers with a mask each (a code at the low end of a half is the subnormal fp16 number c 2^-24) and one
// shift, V's with a shift, a three-way logic operation and an fma each: a code shifted to bits 6-9 and joined with 0x3c00 is the fp16 number 1 + c / 16,
// hence the form of the grid.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace psa {

constexpr int CACHE_BLOCK = 16;                 // tokens of a block
constexpr float CACHE_MAX = 20000.f;            // |x| beyond this is held as this: M = x - S reaches 3.2 times it, the most that fp16 takes

template <int D>
struct CacheBlock {
    static constexpr int G = D / 32;
    static constexpr int K_CODES = 0, K_SCALES = 8 * D, V_CODES = 10 * D, V_SCALES = 18 * D, BYTES = 20 * D;
};

// The numbers 1 + c / 16 of four pairs of codes in a word.  The two constants are kept in registers (opaque to the compiler, which would put them into
// instructions of their own each time): a shift and one three-way operation a pair.
struct CacheOnes {
    uint32_t mask, one;
    __device__ __forceinline__ CacheOnes() {
        asm volatile("mov.b32 %0, 0x03C003C0;" : "=r"(mask));
        asm volatile("mov.b32 %0, 0x3C003C00;" : "=r"(one));
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t w, int j) const {
        const uint32_t s = j == 0 ? w << 6 : j == 1 ? w << 2 : j == 2 ? w >> 2 : w >> 6;
        uint32_t r;
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(s), "r"(mask), "r"(one));      // (s & mask) | one
        return r;
    }
};

}  // namespace psa
