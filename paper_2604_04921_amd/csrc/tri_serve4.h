// Caches held in 4 bits: what their kernels share.
#pragma once

#include "tri_serve.h"

namespace tri {

constexpr int kScaleNaN = 255, kScaleLeast = 3, kScaleMost = 252;   // scale bytes: not numbers, 2^-124, 2^125

// A slot's word of scale bytes lies where its position does: element offset of both.
__device__ __forceinline__ int64_t word_of(const CacheView &c, int64_t base, int64_t block, int n) { return base + block * c.pos_stride_sb + n; }

// The scale byte of 32 elements whose largest magnitude has these bits: the least power of two of which it is at most 7, 7 being 1.75 * 2^2.
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits)
{
    if (bits >= 0x7f800000u) return kScaleNaN;
    const int b = (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x600000u);
    return (uint32_t)min(max(b, kScaleLeast), kScaleMost);
}
__device__ __forceinline__ uint32_t scale_byte(uint64_t bits)   // (a double's; NaN is beyond 2^128, too)
{
    if (bits >= (uint64_t)(1023 + 128) << 52) return kScaleNaN;
    const int b = (int)(bits >> 52) - 1023 + 127 - 2 + ((bits & 0xfffffffffffffull) > 0xc000000000000ull);
    return (uint32_t)min(max(b, kScaleLeast), kScaleMost);
}

// Eight numbers of a word as bf16.  The conversion takes the scale from bits 30 to 23 of its operand, whatever the others hold.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint4 read8(uint32_t word, float scale)
{
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3));
    return r;
}
// The operand of a conversion from byte g of a word of scales: turned so that it lies in bits 30 to 23.
__device__ __forceinline__ float scale_at(uint32_t word, uint32_t g) { return __uint_as_float(__builtin_amdgcn_alignbit(word, word, (8 * g + 9) & 31)); }

struct Append4Args {
    AppendArgs a;   // a.cache: the 4-bit numbers'
    uint32_t *k_scale, *v_scale;
};
tri_status launch_append4(const Append4Args &a, int32_t rows, hipStream_t st);
int64_t append4_groups(int64_t n_tokens, int64_t n_kv_heads);

// Slots from one cache to another, one of them in 4 bits.
struct Pack4Args {
    CacheView src, dst;
    BandTurns turns;
    const int32_t *kept_idx, *kept_cnt;   // kept_idx NULL: 0, 1, ...; kept_cnt NULL: the lengths of src
    int32_t *new_seq_len;
    uint32_t *k_scale, *v_scale;          // of the cache in 4 bits
    int32_t budget, slots;                // entries of kept_idx per head-instance; most slots of one
    int32_t src_blocks, dst_blocks;       // n_blocks
    int32_t row_blocks;                   // workgroups per head-instance
};
int32_t pack4_row_blocks(int32_t slots);
int32_t unpack4_row_blocks(int32_t slots);
tri_status launch_pack4(const Pack4Args &a, int64_t groups, int32_t dtype, bool turn, bool half, hipStream_t st);   // (dtype: of the cache in full precision)
tri_status launch_unpack4(const Pack4Args &a, int64_t groups, int32_t dtype, hipStream_t st);

AttendSplit attend4_split(const tri_model &m, const tri_cache &c, int32_t max_tokens, int32_t n_tokens, int32_t rows);
tri_status launch_attend4(AttendArgs a, int32_t rows, hipStream_t st);   // (a.src.cache: the 4-bit numbers')

}  // namespace tri
