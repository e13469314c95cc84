// What tri_append and the attention kernels share: the step's tokens, a slot's place in a cache, and the rotation by a position.
#pragma once

#include "tri_internal.h"

namespace tri {

// omega_f / 2 pi of the 64 bands in 64-bit fixed point (fractions of a revolution, < 0.16 for theta > 1).
struct BandTurns {
    uint64_t w[kBands];
};
BandTurns band_turns(double theta);

// Phase of band w at a position, in 2^-32 revolutions: the position times w modulo one revolution is the low 64 bits of their product,
// whose upper half is kept.  Off by less than 2^-32 revolutions (what is not kept) and |pos| 2^-62 (w is off by less than that): 1.5 * 2^-31, 5e-9 rad, for
// every int32 position, at the price of two integer multiplications; in double precision the product alone has 2^-32 only up to positions of 2^20.
__device__ __forceinline__ uint32_t phase_of(int32_t pos, uint32_t w_lo, uint32_t w_hi)
{
    const uint32_t p = (uint32_t)pos;
    return p * w_hi + __umulhi(p, w_lo) - (pos < 0 ? w_lo : 0u);
}

// cos and sin of a phase.  bf16: the hardware's, whose argument is in revolutions (absolute error about 2^-20, a rounding to
// bf16 being 2^-9).  fp32: the nearest quarter turn is taken off in integers, which leaves |x| <= pi/4 with a relative error of 2^-24, and the
// Taylor polynomials of degree 9 and 10 are off by less than 2e-9 there.
__device__ __forceinline__ void turn_fast(uint32_t phase, float *c, float *s)
{
    const float r = (float)(int32_t)phase * 0x1p-32f;
    *c = __builtin_amdgcn_cosf(r);
    *s = __builtin_amdgcn_sinf(r);
}
__device__ __forceinline__ void turn_exact(uint32_t phase, float *c, float *s)
{
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(phase - (quarter << 30)) * (float)(6.283185307179586476925 * 0x1p-32);
    const float z = x * x;
    const float sn = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), x);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const float a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;
    *c = (quarter + 1) & 2 ? -a : a;
    *s = quarter & 2 ? -b : b;
}

// The tokens of a sequence: [t0, t0 + n), inside [0, n_tokens] whatever the device arrays hold.
struct TokenRange {
    int t0, n;
};
__device__ __forceinline__ int clamp_to(int x, int hi) { return min(max(x, 0), hi); }

// Element offset of slot n inside layer and head (whose offsets are in `base`), or -1 where its block is not there.
__device__ __forceinline__ int block_of(const CacheView &c, int n_blocks, int s, int n)
{
    const int b = c.block_table[(int64_t)s * c.max_blocks + (n >> c.block_shift)];
    return n_blocks > 0 && b >= n_blocks ? -1 : b;
}
__device__ __forceinline__ int64_t row_of(const CacheView &c, int64_t base, int b, int n)
{
    return base + (int64_t)b * c.stride_sb + slot_offset(c, n);
}

struct AppendArgs {
    CacheView cache;
    BandTurns turns;
    const int32_t *start, *pos, *head_len;   // start NULL: one token per sequence
    const char *k_new, *v_new;
    int32_t *new_seq_len;
    int64_t stride_token, stride_head;
    int32_t layer, n_tokens, n_blocks, rotate, half;
};

tri_status launch_append(const AppendArgs &a, int32_t dtype, hipStream_t st);

// One cache that a step's queries attend to.
struct AttendSource {
    CacheView cache;
    const int32_t *group;      // [n_seqs + 1] sequences of the step behind each of this cache's (a prefix's), NULL: one each
    const int32_t *head_len;
    int32_t n_blocks;
    int32_t all;               // one prefix for all the step's sequences (group is NULL then)
    int32_t max_tokens;        // tokens that attend to one sequence of this cache, at most
    int32_t n_split, part0;    // its keys are cut into n_split ranges; the results are entries part0 and on of the partial results
    int32_t least_keys;        // of a range that is not the last
    int32_t fill, fill_keys;   // a range is no shorter than the smaller of a fill-th of the keys and fill_keys
    int32_t scan;              // keys behind the tokens' positions are likely at its end (a chunk's own tokens)
};
struct AttendArgs {
    AttendSource src;
    AttendSource other;        // attend_rows_kernel: workgroups from first_groups on work on this one
    uint32_t first_groups;
    BandTurns turns;
    const int32_t *start, *pos;
    const char *q;
    char *out;
    int64_t q_stride_token, q_stride_head, out_stride_token, out_stride_head;
    float *part_o;             // [parts][n_tokens][Hq][128], NULL: results go to out at once
    float2 *part_ml;           // [parts][n_tokens][Hq]: highest product q . k and sum of exponentials
    float scale_log2;          // scale * log2(e)
    int32_t n_steps_seqs;      // the step's sequences
    int32_t layer, n_tokens, group_size, causal, rotate_q, half;
    int32_t row_tiles;
};

// Tokens that attend to sequence s of the source.
__device__ __forceinline__ TokenRange tokens_of(const AttendArgs &a, const AttendSource &src, int s)
{
    int lo = s, hi = s + 1;
    if (src.all) lo = 0, hi = a.n_steps_seqs;
    if (src.group) lo = clamp_to(src.group[s], a.n_steps_seqs), hi = clamp_to(src.group[s + 1], a.n_steps_seqs);
    if (a.start) lo = a.start[lo], hi = a.start[hi];
    lo = clamp_to(lo, a.n_tokens), hi = clamp_to(hi, a.n_tokens);
    return TokenRange{lo, min(max(hi - lo, 0), src.max_tokens)};
}
__device__ __forceinline__ int keys_of(const AttendArgs &a, const AttendSource &src, int s, int h)
{
    const CacheView &c = src.cache;
    const int n = src.head_len ? src.head_len[((int64_t)a.layer * c.n_seqs + s) * c.n_kv_heads + h] : c.seq_len[s];
    return clamp_len(n, c.max_seq_len);
}

constexpr int64_t kMostGroups = 0xffffffffu / 256;   // workgroups of a launch, which are of 256 threads: HIP takes fewer than 2^32 threads on an axis

// How the keys of a cache are cut: ranges per head, and their least keys (a function of bounds alone, for the workspace's size); the workgroups of its launch.
struct AttendSplit {
    int32_t n_split, least_keys, fill, fill_keys;
    int64_t groups;
};
AttendSplit attend_split(const tri_model &m, const tri_cache &c, int32_t max_tokens, int32_t n_tokens);
int64_t join_groups(int64_t rows, int32_t parts);
int64_t append_threads(int64_t rows, int32_t dtype);
tri_status launch_attend(AttendArgs a, const tri_cache &c, hipStream_t st);   // (c: a.src's)
// a.src and a.other, in one launch where that is worth it
tri_status launch_attend_both(AttendArgs a, const tri_cache &c, const tri_cache &other, hipStream_t st);
tri_status launch_join(const AttendArgs &a, int32_t parts, int32_t n_q_heads, int32_t dtype, hipStream_t st);

}  // namespace tri
