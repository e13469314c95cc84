// Rows into 4 bits and back: a step's keys and values (tri_append4), slots of a cache in full precision (tri_pack4), and reading them back (tri_unpack4).
#include <algorithm>

#include "tri_serve4.h"

namespace tri {

namespace {

constexpr int kPackThreads = 256, kLanes = 8, kPackRows = kPackThreads / kLanes;   // threads to a row, rows of a workgroup
// Rows of a thread that reads back (sixteen ragged sequences: in bf16 158 us with one, 151 with two, 148 with four; in fp32 256 with two, 325 with four), and of its workgroup.
constexpr int kReadPasses = 2, kReadRows = kReadPasses * kPackThreads / 16;

// Eight elements of a row as they come.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const float *p)
    {
        // (not non-temporal: a lane's two pieces are halves of one line with its neighbour's; three fp32 caches packed and read back 21 us, 25 with that hint)
        const uint4 a = *reinterpret_cast<const uint4 *>(p), b = *reinterpret_cast<const uint4 *>(p + 4);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
    __device__ __forceinline__ void widen(float *x) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    }
    __device__ __forceinline__ uint32_t most() const   // bits of the largest magnitude, that of what is no number being the largest
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const
    {
        uint32_t r = 0;
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[4]), __uint_as_float(w[5]), scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(w[6]), __uint_as_float(w[7]), scale, 3);
    }
};
template <>
struct Eight<__bf16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __bf16 *p)
    {
        const uint4 a = load_stream16((const char *)p);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    }
    __device__ __forceinline__ void widen(float *x) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    __device__ __forceinline__ uint32_t most() const
    {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 m{0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
        return (uint32_t)max(m[0], m[1]) << 16;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const
    {
        uint32_t r = 0;
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
    }
};

// The four lanes of 32 elements.
__device__ __forceinline__ uint32_t most_of_4(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true));          // lane ^ 1
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true));       // lane ^ 2
}
__device__ __forceinline__ uint64_t most_of_4(uint64_t x)
{
    x = max(x, (uint64_t)__shfl_xor((unsigned long long)x, 1));
    return max(x, (uint64_t)__shfl_xor((unsigned long long)x, 2));
}

__device__ __forceinline__ uint32_t codes8(const float *x, float scale)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

// Element d of a row rotated in double precision: the angle is the position's product with the band's frequency modulo one revolution, off by |pos| 2^-62 revolutions at most; less the nearest quarter turn it is
// at most pi / 4, where the Taylor polynomials of degree 17 and 16 are off by less than 2^-58.
template <typename T, bool HALF>
__device__ double rotated(const T *row, int d, int32_t pos, const BandTurns &turns)
{
    const int f = HALF ? d & 63 : d >> 1;
    const double re = (double)row[HALF ? f : 2 * f], im = (double)row[HALF ? f + 64 : 2 * f + 1];
    const uint64_t phase = (uint64_t)(int64_t)pos * turns.w[f], quarter = (phase + (1ull << 61)) >> 62;
    const double x = (double)(int64_t)(phase - (quarter << 62)) * (6.283185307179586476925 * 0x1p-64), z = x * x;
    double sn = 1.0 / 355687428096000.0, cs = 1.0 / 20922789888000.0;   // 1 / 17!, 1 / 16!
    sn = fma(sn, z, -1.0 / 1307674368000.0), cs = fma(cs, z, -1.0 / 87178291200.0);
    sn = fma(sn, z, 1.0 / 6227020800.0), cs = fma(cs, z, 1.0 / 479001600.0);
    sn = fma(sn, z, -1.0 / 39916800.0), cs = fma(cs, z, -1.0 / 3628800.0);
    sn = fma(sn, z, 1.0 / 362880.0), cs = fma(cs, z, 1.0 / 40320.0);
    sn = fma(sn, z, -1.0 / 5040.0), cs = fma(cs, z, -1.0 / 720.0);
    sn = fma(sn, z, 1.0 / 120.0), cs = fma(cs, z, 1.0 / 24.0);
    sn = fma(sn, z, -1.0 / 6.0), cs = fma(cs, z, -0.5);
    sn = fma(sn * z, x, x), cs = fma(cs, z, 1.0);
    const double a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;
    const double c = (quarter + 1) & 2 ? -a : a, s = quarter & 2 ? -b : b;
    return (HALF ? d < 64 : !(d & 1)) ? fma(re, c, -(im * s)) : fma(re, s, im * c);
}
__device__ __forceinline__ uint32_t code_of(double v, uint32_t byte)
{
    const double t = ldexp(fabs(v), 127 - (int)byte);
    return (t > 0.25) + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5.0) + (signbit(v) ? 8u : 0u);
}

struct Codes {
    uint32_t word[2];    // dimensions 8 part to 8 part + 7, and those 64 further on
    uint32_t byte[2];    // their scales
};

// A lane's sixteen elements, as they are, to 4 bits.
template <typename T>
__device__ __forceinline__ Codes to_codes(const Eight<T> (&x)[2])
{
    Codes got;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        got.byte[p] = scale_byte(most_of_4(x[p].most()));
        got.word[p] = got.byte[p] == kScaleNaN ? 0 : x[p].codes(__uint_as_float(got.byte[p] << 23));
    }
    return got;
}

// Cosine and sine of a lane's eight bands at a position.
struct Angles {
    float c[8], s[8];
};
template <bool HALF>
__device__ __forceinline__ Angles angles_of(int32_t pos, const BandTurns &turns, int part)
{
    Angles a;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint64_t w = turns.w[HALF ? 8 * part + e : 32 * (e / 4) + 4 * part + (e & 3)];
        turn_fast(phase_of(pos, (uint32_t)w, (uint32_t)(w >> 32)), &a.c[e], &a.s[e]);
    }
    return a;
}

// A lane's sixteen elements to 4 bits, rotated first.  In fp32 a rotated element is off by less than (|re| + |im|) 2^-21: the hardware's cosine and sine by 1.9e-7 (measured over all 2^32 phases, as a test does again), the angle by 5e-9, the
// products' roundings by 2^-23.  |re| + |im| is at most twice the larger of the pair's rotated elements, of which `apart` below has the largest, its own error being far below the bound's slack.  Where what lies within
// `apart` of an element does not all have one code, or the group's largest not one scale (or, next to 2^128, is not on one side of it), the element is worked out in double precision: one or two waves in a hundred of
// Gaussian rows.
template <typename T, bool HALF>
__device__ __forceinline__ Codes to_codes(const Eight<T> (&raw)[2], const Angles &angles, const T *row, int32_t pos, const BandTurns &turns, int part)
{
    float x[2][8];
    raw[0].widen(x[0]);
    raw[1].widen(x[1]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float &r = HALF ? x[0][e] : x[e / 4][2 * (e & 3)], &i = HALF ? x[1][e] : x[e / 4][2 * (e & 3) + 1];
        const float re = r, im = i;
        r = fmaf(re, angles.c[e], -(im * angles.s[e]));
        i = fmaf(re, angles.s[e], im * angles.c[e]);
    }
    uint32_t bits_of[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        bits_of[p] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) bits_of[p] = max(bits_of[p], __float_as_uint(x[p][e]) & 0x7fffffffu);   // (what is no number is the largest)
        bits_of[p] = most_of_4(bits_of[p]);
    }
    Codes got;
    constexpr uint32_t kLargest = 0x7f7fffffu;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        // (half-split pairs lie in both of the lanes' groups; infinities may be roundings of numbers: as the largest number)
        const float most = __uint_as_float(min(bits_of[p], kLargest)), apart = 0x1p-20f * (HALF ? __uint_as_float(min(max(bits_of[0], bits_of[1]), kLargest)) : most);
        uint32_t byte = kScaleNaN;
        if (bits_of[p] <= 0x7f800000u) {   // (beyond: what came was no number)
            byte = scale_byte(__float_as_uint(most + apart));
            if (scale_byte(__float_as_uint(fmaxf(most - apart, 0.f))) != byte) {   // (all four lanes)
                uint64_t exact = 0;   // (the bits: what is no number is the largest)
#pragma unroll 1
                for (int e = 0; e < 8; ++e) exact = max(exact, (uint64_t)__double_as_longlong(fabs(rotated<T, HALF>(row, 64 * p + 8 * part + e, pos, turns))));
                byte = scale_byte(most_of_4(exact));
            }
        }
        const float scale = __uint_as_float(byte << 23);
        float below[8], above[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) below[e] = x[p][e] - apart, above[e] = x[p][e] + apart;
        uint32_t word = codes8(below, scale), open = byte == kScaleNaN ? 0 : word ^ codes8(above, scale);
#pragma unroll 1
        while (open) {
            const int at = (__ffs(open) - 1) & ~3;
            const uint32_t code = code_of(rotated<T, HALF>(row, 64 * p + 8 * part + at / 4, pos, turns), byte);
            word = (word & ~(15u << at)) | code << at;
            open &= ~(15u << at);
        }
        got.word[p] = byte == kScaleNaN ? 0 : word;
        got.byte[p] = byte;
    }
    return got;
}

// A row's codes and its word of scales to a slot.  All eight lanes of the row take part (the ones without a place have `there` unset).
__device__ __forceinline__ void put_row(void *rows, uint32_t *scales, const Codes &x, int part, bool there, int64_t at_bytes, int64_t at_word)
{
    const uint32_t mine = x.byte[0] | x.byte[1] << 16;
    const uint32_t word = mine | (uint32_t)__shfl_xor((int)mine, 4) << 8;   // (lanes 0 to 3: groups 0 and 2, the others 1 and 3)
    if (!there) return;
    char *p = (char *)rows + at_bytes + 4 * part;
    *reinterpret_cast<uint32_t *>(p) = x.word[0];
    *reinterpret_cast<uint32_t *>(p + 32) = x.word[1];
    if (part == 0) scales[at_word] = word;
}

// A workgroup takes 32 neighbouring tokens of HEADS KV heads, eight threads to a row of K and of V, each with two pieces of eight elements half a row apart: both parts of its bands lie in them in either pair layout, and
// four lanes hold the 32 elements of a scale.  Neighbouring rows are neighbouring slots: 64 bytes each, a wave writes 512 side by side.  The heads of a token have its angles in common.
// Bound by bytes and, nearly as much, by vector instructions (rotation, scales, codes and the test of what rounding might have changed are some 200 to a lane's 32 elements): the prompts of four requests, 20 thousand
// tokens of 8 heads, 105 MB, take 27 us (3.9 TB/s); by latency for a token, 4.0 us.
template <typename T, bool TURN, bool HALF, int HEADS>
__global__ __launch_bounds__(kPackThreads) void append4_kernel(Append4Args args)
{
    const AppendArgs &a = args.a;
    const CacheView &c = a.cache;
    const int S = c.n_seqs, H = c.n_kv_heads;
    // All that is needed of the arguments is asked for at once, not where it is needed, one wait after the other: a token 4.4 -> 4.0 us.  (Not so below: sixteen ragged sequences are read back in 154 us, 172 so.)
    asm volatile("" ::"s"(a.new_seq_len), "s"(a.head_len), "s"(a.start), "s"(a.k_new), "s"(a.v_new), "s"(a.pos), "s"(a.stride_token), "s"(a.stride_head), "s"(a.n_tokens), "s"(a.layer), "s"(a.n_blocks), "s"(c.seq_len),
                 "s"(c.max_seq_len), "s"(c.n_seqs), "s"(c.n_kv_heads), "s"(c.block_shift), "s"(c.block_table), "s"(c.max_blocks), "s"(c.stride_layer), "s"(c.stride_head));
    asm volatile("" ::"s"(c.stride_sb), "s"(c.stride_slot), "s"(c.pos_stride_layer), "s"(c.pos_stride_head), "s"(c.pos_stride_sb), "s"(c.k), "s"(c.v), "s"(c.pos), "s"(args.k_scale), "s"(args.v_scale));
    const int64_t i = (int64_t)blockIdx.x * kPackThreads + threadIdx.x;
    if (a.new_seq_len && i < S) {
        const int s = (int)i;
        const int n = clamp_len(a.head_len ? a.head_len[((int64_t)a.layer * S + s) * H] : c.seq_len[s], c.max_seq_len);
        int got = 1;
        if (a.start) got = max(clamp_to(a.start[s + 1], a.n_tokens) - clamp_to(a.start[s], a.n_tokens), 0);
        a.new_seq_len[s] = (int)min((int64_t)n + got, (int64_t)c.max_seq_len);
    }
    const uint32_t groups = (uint32_t)(H + HEADS - 1) / HEADS;
    const int h0 = (int)(blockIdx.x % groups) * HEADS, part = threadIdx.x % kLanes;
    const int64_t t0 = (int64_t)(blockIdx.x / groups) * kPackRows;
    const int64_t t_wave = t0 + (threadIdx.x & ~63) / kLanes;
    if (t_wave >= a.n_tokens) return;   // (the whole wave)
    const int64_t t_mine = t0 + threadIdx.x / kLanes;
    const int t = (int)min(t_mine, (int64_t)a.n_tokens - 1);
    // the rows are asked for before their place is known
    const T *k_row = reinterpret_cast<const T *>(a.k_new) + (int64_t)t * a.stride_token + (int64_t)h0 * a.stride_head;
    const T *v_row = reinterpret_cast<const T *>(a.v_new) + (int64_t)t * a.stride_token + (int64_t)h0 * a.stride_head;
    Eight<T> k[2], v[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) k[p].load(k_row + 64 * p + 8 * part), v[p].load(v_row + 64 * p + 8 * part);
    const int32_t pos = a.pos[t];
    Angles angles;
    if (TURN) angles = angles_of<HALF>(pos, a.turns, part);
    bool mine = t_mine < a.n_tokens;
    int s = t, first = t;
    if (a.start) {
        s = 0;
        for (int j = 0; j < S; j += 64) {
            const int e = j + (int)(threadIdx.x & 63);
            s += __popcll(__ballot(e < S && a.start[min(e, S - 1) + 1] <= (int)t_wave));
        }
        while (s < S && a.start[s + 1] <= t) ++s;
        mine &= s < S;
        s = min(s, S - 1);
        first = a.start[s];
        mine &= t >= first;
    }
    bool there = false;
    int n = 0;
    int64_t block = 0;
    const auto find = [&](int length) {   // the token's slot behind a length
        const int64_t slot = (int64_t)clamp_len(length, c.max_seq_len) + (t - first);
        there = mine & (slot < c.max_seq_len);
        n = there ? (int)slot : 0;
        block = s;
        if (c.block_shift >= 0) {
            block = there ? block_of(c, a.n_blocks, s, n) : -1;
            there &= block >= 0;
            n &= (1 << c.block_shift) - 1;
        }
    };
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        const int h = h0 + j;
        if (h >= H) break;
        if (j == 0 || a.head_len) find(a.head_len ? a.head_len[((int64_t)a.layer * S + s) * H + h] : c.seq_len[s]);
        const int64_t to = ((int64_t)a.layer * c.stride_layer + (int64_t)h * c.stride_head + block * c.stride_sb + slot_offset(c, n)) / 2;
        const int64_t word = word_of(c, (int64_t)a.layer * c.pos_stride_layer + (int64_t)h * c.pos_stride_head, block, n);
        Eight<T> k_here[2] = {k[0], k[1]}, v_here[2] = {v[0], v[1]};
        const T *row = k_row;
        if (j + 1 < HEADS && h + 1 < H) {   // the next head's
            k_row += a.stride_head, v_row += a.stride_head;
#pragma unroll
            for (int p = 0; p < 2; ++p) k[p].load(k_row + 64 * p + 8 * part), v[p].load(v_row + 64 * p + 8 * part);
        }
        Codes kc;
        if constexpr (TURN) kc = to_codes<T, HALF>(k_here, angles, row, pos, a.turns, part);
        else kc = to_codes<T>(k_here);
        const Codes vc = to_codes<T>(v_here);
        put_row(const_cast<void *>(c.k), args.k_scale, kc, part, there, to, word);
        put_row(const_cast<void *>(c.v), args.v_scale, vc, part, there, to, word);
        if (there && part == 0) const_cast<int32_t *>(c.pos)[word] = pos;
    }
}

// Which slots a workgroup of tri_pack4 / tri_unpack4 moves, and where from.
struct Instance {
    int l, s, h, count;
    uint32_t inst;
};
__device__ __forceinline__ Instance instance_of(const Pack4Args &a, uint32_t inst)
{
    Instance x;
    x.inst = inst;
    const uint32_t H = a.src.n_kv_heads, S = a.src.n_seqs, ls = inst / H;
    x.h = (int)(inst - ls * H);
    x.l = (int)(ls / S);
    x.s = (int)(ls - x.l * S);
    x.count = clamp_to(a.kept_cnt ? a.kept_cnt[inst] : a.src.seq_len[x.s], a.slots);
    return x;
}
struct Place {
    int64_t row, word;   // elements of k and v; of pos and the scales
    bool there;
};
__device__ __forceinline__ Place place_of(const CacheView &c, int n_blocks, const Instance &x, int n)
{
    int64_t block = x.s;
    int in = n;
    if (c.block_shift >= 0) {
        block = block_of(c, n_blocks, x.s, n);
        in = n & ((1 << c.block_shift) - 1);
    }
    return Place{(int64_t)x.l * c.stride_layer + (int64_t)x.h * c.stride_head + block * c.stride_sb + slot_offset(c, in),
                 word_of(c, (int64_t)x.l * c.pos_stride_layer + (int64_t)x.h * c.pos_stride_head, block, in), block >= 0};
}
__device__ __forceinline__ int slot_to_read(const Pack4Args &a, const Instance &x, int j)
{
    return a.kept_idx ? min(max(a.kept_idx[(int64_t)x.inst * a.budget + j], 0), a.src.max_seq_len - 1) : j;
}

// As append4_kernel, from slots to slots; a slot's row and its place are each found by the lane (slots kept are in any order).  Bound by bytes: 2048 kept slots in four layers of eight sequences, 344 MB, take 76 us (4.5 TB/s; a large copy 4.8),
// pre-RoPE and scattered.  (The bound on registers, six workgroups to a CU, which three registers are spilled for: interleaved pairs of sixteen sequences 240 us, 244 without; half-split pairs and fp32 would spill more.)
template <typename T, bool TURN, bool HALF>
__global__ __launch_bounds__(kPackThreads, sizeof(T) == 2 && !HALF ? 6 : 1) void pack4_kernel(Pack4Args a)
{
    const uint32_t inst = blockIdx.x / (uint32_t)a.row_blocks;
    const int rb = (int)(blockIdx.x - inst * (uint32_t)a.row_blocks), part = threadIdx.x % kLanes;
    const Instance x = instance_of(a, inst);
    if (a.new_seq_len && x.l == 0 && x.h == 0 && rb == 0 && threadIdx.x == 0) a.new_seq_len[x.s] = x.count;
    const int j = rb * kPackRows + (int)threadIdx.x / kLanes;
    if (rb * kPackRows + (int)(threadIdx.x & ~63) / kLanes >= x.count) return;   // (the whole wave)
    const int last = min(j, x.count - 1);
    const Place from = place_of(a.src, a.src_blocks, x, slot_to_read(a, x, last)), to = place_of(a.dst, a.dst_blocks, x, last);
    const bool there = j < x.count && from.there && to.there;
    const int64_t at = from.there ? from.row : 0, at_word = from.there ? from.word : 0;
    const T *row = reinterpret_cast<const T *>(a.src.k) + at, *v_row = reinterpret_cast<const T *>(a.src.v) + at;
    Eight<T> k[2], v[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) k[p].load(row + 64 * p + 8 * part), v[p].load(v_row + 64 * p + 8 * part);
    const int32_t pos = a.src.pos[at_word];
    Codes kc;
    if constexpr (TURN) kc = to_codes<T, HALF>(k, angles_of<HALF>(pos, a.turns, part), row, pos, a.turns, part);
    else kc = to_codes<T>(k);
    const Codes vc = to_codes<T>(v);
    put_row(const_cast<void *>(a.dst.k), a.k_scale, kc, part, there, to.row / 2, to.word);
    put_row(const_cast<void *>(a.dst.v), a.v_scale, vc, part, there, to.row / 2, to.word);
    if (there && part == 0) const_cast<int32_t *>(a.dst.pos)[to.word] = pos;
}

// A thread's eight numbers of a row: neighbours in bf16, two times four half a row apart in fp32, so that sixteen threads' stores of 16 bytes lie side by side in either (with 32 bytes of its own each, sixteen ragged sequences in two layers took 504 us to read back in fp32, 256 so).
template <typename T>
struct Numbers;
template <>
struct Numbers<__bf16> {
    static __device__ __forceinline__ uint32_t load(const char *row, int part) { return reinterpret_cast<const uint32_t *>(row)[part]; }
    static __device__ __forceinline__ void store(__bf16 *row, int part, uint32_t word, uint32_t scales) { store_stream16((char *)(row + 8 * part), read8(word, scale_at(scales, part / 4))); }
};
template <>
struct Numbers<float> {
    static __device__ __forceinline__ uint32_t load(const char *row, int part)
    {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row);
        return (uint32_t)p[part] | (uint32_t)p[16 + part] << 16;
    }
    static __device__ __forceinline__ void store(float *row, int part, uint32_t word, uint32_t scales)
    {
        const uint4 a = read8(word, scale_at(scales, part / 8)), b = read8(word, scale_at(scales, 2 + part / 8));
        store_stream16((char *)(row + 4 * part), make_uint4(a.x << 16, a.x & 0xffff0000u, a.y << 16, a.y & 0xffff0000u));
        store_stream16((char *)(row + 64 + 4 * part), make_uint4(b.z << 16, b.z & 0xffff0000u, b.w << 16, b.w & 0xffff0000u));
    }
};

// Sixteen threads to a row, eight numbers each; every bf16 number is exact.  Bound by the bytes it writes: sixteen ragged sequences in two layers, 164 MB read and 603 written, 150 us, 5.1 TB/s, where a large copy has 4.8;
// one layer of one sequence 4.6 us.
template <typename T>
__global__ __launch_bounds__(kPackThreads) void unpack4_kernel(Pack4Args a)
{
    const uint32_t inst = blockIdx.x / (uint32_t)a.row_blocks;
    const int rb = (int)(blockIdx.x - inst * (uint32_t)a.row_blocks), part = threadIdx.x % 16;
    const Instance x = instance_of(a, inst);
    if (a.new_seq_len && x.l == 0 && x.h == 0 && rb == 0 && threadIdx.x == 0) a.new_seq_len[x.s] = x.count;
    // all rows are asked for before the first is written
    Place from[kReadPasses], to[kReadPasses];
    uint32_t k[kReadPasses], v[kReadPasses], k_scale[kReadPasses], v_scale[kReadPasses];
    int32_t pos[kReadPasses];
    bool there[kReadPasses];
    if (rb * kReadRows >= x.count) return;
#pragma unroll
    for (int i = 0; i < kReadPasses; ++i) {
        const int j = rb * kReadRows + i * (kPackThreads / 16) + (int)threadIdx.x / 16, at = min(j, x.count - 1);
        from[i] = place_of(a.src, a.src_blocks, x, slot_to_read(a, x, at));
        to[i] = place_of(a.dst, a.dst_blocks, x, at);
        there[i] = (j < x.count) & from[i].there & to[i].there;
    }
#pragma unroll
    for (int i = 0; i < kReadPasses; ++i) {
        const int64_t row = from[i].there ? from[i].row / 2 : 0, word = from[i].there ? from[i].word : 0;
        k[i] = Numbers<T>::load((const char *)a.src.k + row, part);
        v[i] = Numbers<T>::load((const char *)a.src.v + row, part);
        k_scale[i] = a.k_scale[word];
        v_scale[i] = a.v_scale[word];
        pos[i] = a.src.pos[word];
    }
#pragma unroll
    for (int i = 0; i < kReadPasses; ++i) {
        if (!there[i]) continue;
        Numbers<T>::store((T *)a.dst.k + to[i].row, part, k[i], k_scale[i]);
        Numbers<T>::store((T *)a.dst.v + to[i].row, part, v[i], v_scale[i]);
        if (part == 0) const_cast<int32_t *>(a.dst.pos)[to[i].word] = pos[i];
    }
}

}  // namespace

// Heads of a workgroup: four share their tokens' angles where there are workgroups enough all the same (8192 tokens of 8 heads 14.2 us, 15.4 with one; 4096 tokens, the border, 10.5 and 10.0, 2048 9.6 and 6.9, one 6.6 and 4.1).
// Measured with 8 heads alone; with one or two there is little to share, and the rule does not ask for that.
static int append4_heads(int64_t n_tokens, int64_t n_kv_heads) { return n_tokens * n_kv_heads >= 32768 ? 4 : 1; }
int64_t append4_groups(int64_t n_tokens, int64_t n_kv_heads)
{
    const int64_t heads = append4_heads(n_tokens, n_kv_heads);
    return (n_tokens + kPackRows - 1) / kPackRows * ((n_kv_heads + heads - 1) / heads);
}
int32_t pack4_row_blocks(int32_t slots) { return std::max(1, (int32_t)(((int64_t)slots + kPackRows - 1) / kPackRows)); }
int32_t unpack4_row_blocks(int32_t slots) { return std::max(1, (int32_t)(((int64_t)slots + kReadRows - 1) / kReadRows)); }

tri_status launch_append4(const Append4Args &a, int32_t rows, hipStream_t st)
{
    const int64_t lengths = a.a.new_seq_len ? (a.a.cache.n_seqs + kPackThreads - 1) / kPackThreads : 0;
    const uint32_t blocks = (uint32_t)std::max(append4_groups(a.a.n_tokens, a.a.cache.n_kv_heads), lengths);
    if (blocks == 0) return TRI_OK;
    const auto launch = [&](auto kernel) { kernel<<<blocks, kPackThreads, 0, st>>>(a); };
    const auto of = [&](auto plain, auto half, auto interleaved) { !a.a.rotate ? launch(plain) : a.a.half ? launch(half) : launch(interleaved); };
    const bool one = append4_heads(a.a.n_tokens, a.a.cache.n_kv_heads) == 1;
    if (rows == TRI_BF16 && one) of(append4_kernel<__bf16, false, false, 1>, append4_kernel<__bf16, true, true, 1>, append4_kernel<__bf16, true, false, 1>);
    else if (rows == TRI_BF16) of(append4_kernel<__bf16, false, false, 4>, append4_kernel<__bf16, true, true, 4>, append4_kernel<__bf16, true, false, 4>);
    else if (one) of(append4_kernel<float, false, false, 1>, append4_kernel<float, true, true, 1>, append4_kernel<float, true, false, 1>);
    else of(append4_kernel<float, false, false, 4>, append4_kernel<float, true, true, 4>, append4_kernel<float, true, false, 4>);
    return hip_status("append4_kernel");
}

tri_status launch_pack4(const Pack4Args &a, int64_t groups, int32_t dtype, bool turn, bool half, hipStream_t st)
{
    const auto launch = [&](auto kernel) { kernel<<<(uint32_t)groups, kPackThreads, 0, st>>>(a); };
    const auto of = [&](auto plain, auto with_half, auto interleaved) { !turn ? launch(plain) : half ? launch(with_half) : launch(interleaved); };
    if (dtype == TRI_BF16) of(pack4_kernel<__bf16, false, false>, pack4_kernel<__bf16, true, true>, pack4_kernel<__bf16, true, false>);
    else of(pack4_kernel<float, false, false>, pack4_kernel<float, true, true>, pack4_kernel<float, true, false>);
    return hip_status("pack4_kernel");
}

tri_status launch_unpack4(const Pack4Args &a, int64_t groups, int32_t dtype, hipStream_t st)
{
    if (dtype == TRI_BF16) unpack4_kernel<__bf16><<<(uint32_t)groups, kPackThreads, 0, st>>>(a);
    else unpack4_kernel<float><<<(uint32_t)groups, kPackThreads, 0, st>>>(a);
    return hip_status("unpack4_kernel");
}

}  // namespace tri
