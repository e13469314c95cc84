// What the attention kernels share.
#pragma once

#include "tri_serve.h"

namespace tri {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kNoScore = -__builtin_inff();
constexpr int kNonTemporal = 2;   // the cache policy operand of buffer loads

__device__ __forceinline__ void store8(float *p, const float *x)
{
    *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(__bf16 *p, const float *x)
{
    bf16x8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (__bf16)x[e];
    *reinterpret_cast<bf16x8 *>(p) = b;
}
template <typename U>
__device__ __forceinline__ uint4 as_uint4(const U &u) { return __builtin_bit_cast(uint4, u); }
__device__ __forceinline__ void widen8(const uint4 &u, float *x)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}

// The keys of a part: split's share of the sequence's keys, at least what attend_split says where there are so many, in whole groups of 128 (pages of sixteen and more are not cut by a
// tile of 32 or 16).
struct KeyRange {
    int lo, hi;
};
__device__ __forceinline__ KeyRange keys_of_split(const AttendArgs &a, const AttendSource &src, int s, int h, int split)
{
    const int n = keys_of(a, src, s, h);
    const auto nth = [&](int parts) { return ((uint32_t)n + parts - 1) / (uint32_t)parts; };
    uint32_t share = max(nth(src.n_split), (uint32_t)src.least_keys);
    if (src.fill_keys) share = max(share, min(nth(src.fill), (uint32_t)src.fill_keys));
    const int64_t per = (share + 127) & ~127u;
    const int lo = (int)min(split * per, (int64_t)n);
    return KeyRange{lo, (int)min(lo + per, (int64_t)n)};
}

// Which part of which sequence's head workgroup (or group of row tiles) w has.  Parts come last: the first of all heads are spread over the eight XCDs, which workgroups go to in turn, and those
// that turn out to have no keys end together.  (Two chunks of 1024 tokens over 8192 keys, cut into eight parts of which one had keys: 2013 us with a head's parts next to each other, all work on one XCD then, 365 so.)
struct Unit {
    int split, h, s;
};
__device__ __forceinline__ Unit unit_of(const AttendSource &src, uint32_t w)
{
    const uint32_t H = src.cache.n_kv_heads, S = src.cache.n_seqs;
    return Unit{(int)(w / H / S), (int)(w % H), (int)(w / H % S)};
}

// A part without a key says so; its sums are not read.
__device__ __forceinline__ void no_keys(const AttendArgs &a, const AttendSource &src, int split, int t0, int r0, int rows, int h, int Hq)
{
    for (int i = threadIdx.x; i < rows; i += blockDim.x) {
        const int r = r0 + i;
        a.part_ml[((int64_t)(src.part0 + split) * a.n_tokens + t0 + r / a.group_size) * Hq + h * a.group_size + r % a.group_size] = make_float2(kNoScore, 0.f);
    }
}

// The same value, as the compiler cannot tell: what follows from it is worked out where it is used instead of being kept in registers from tile to tile.
__device__ __forceinline__ void fresh(uint32_t &x) { asm volatile("" : "+v"(x)); }

// The lane's number worked out on the spot, in no register before or after.
__device__ __forceinline__ uint32_t lane_again()
{
    uint32_t none = 0;
    fresh(none);
    return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}

// lane ^ 8 of each sixteen
__device__ __forceinline__ float across_8(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, false)); }
// the maximum over the four lanes that share lane & 15
__device__ __forceinline__ float max_over_kq(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Element e of eight rows' pieces: v[i][j] is the piece of key 4 i + j of the lane's eight.
__device__ __forceinline__ bf16x8 column(const uint4 (&v)[2][4], int e)
{
    const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;
    auto word = [&](const uint4 &u) { return e < 4 ? (e < 2 ? u.x : u.y) : (e < 6 ? u.z : u.w); };
    uint4 r;
    r.x = __builtin_amdgcn_perm(word(v[0][1]), word(v[0][0]), pick);
    r.y = __builtin_amdgcn_perm(word(v[0][3]), word(v[0][2]), pick);
    r.z = __builtin_amdgcn_perm(word(v[1][1]), word(v[1][0]), pick);
    r.w = __builtin_amdgcn_perm(word(v[1][3]), word(v[1][2]), pick);
    return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ bool not_finite(const uint4 &u)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    return odd;
}
__device__ __forceinline__ uint4 finite_only(const uint4 &u)
{
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
        if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// 1 where an element is the infinity `which` (0x7f80 or 0xff80) or NaN, else 0
__device__ __forceinline__ bf16x8 where_not_below(const bf16x8 &x, uint32_t which)
{
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = __builtin_bit_cast(uint16_t, (__bf16)x[e]);
        r[e] = b == which || (b & 0x7fffu) > 0x7f80u ? (__bf16)1.f : (__bf16)0.f;
    }
    return r;
}

// Eight dimensions of a row whose keys are all seen to: to the output, or as a part.
template <typename T>
__device__ __forceinline__ void finish_row(const AttendArgs &a, const AttendSource &src, int split, int t, int hq, int Hq, int d0, float best, float total, float *x)
{
    if (a.part_o) {
        const int64_t at = ((int64_t)(src.part0 + split) * a.n_tokens + t) * Hq + hq;
        if (d0 == 0) a.part_ml[at] = make_float2(best, total);
        store8(a.part_o + at * kHeadDim + d0, x);
        return;
    }
    const float inv = 1.f / total;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = total != 0.f ? x[e] * inv : 0.f;   // (no key: zeros; scores that are no number: NaN)
    store8(reinterpret_cast<T *>(a.out) + (int64_t)t * a.out_stride_token + (int64_t)hq * a.out_stride_head + d0, x);
}

constexpr int kTileRows = 128;   // rows of a workgroup of the tile kernel
tri_status launch_attend_tile(const AttendArgs &a, int64_t groups, hipStream_t st);
tri_status launch_attend4_tile(const AttendArgs &a, int64_t groups, hipStream_t st);   // (a.src is held in 4 bits)
tri_status launch_attend_rows(AttendArgs a, int32_t rows, hipStream_t st);   // a.src, and a.other where it has sequences

}  // namespace tri
