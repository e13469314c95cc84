// Rows into 4 bits and back: a step's keys and values (tri_append4), slots of a cache in full precision (tri_pack4), and reading them back (tri_unpack4).
#include <algorithm>

#include "tri_serve4.h"

namespace tri {

namespace {

constexpr int kPackThreads = 256, kLanes = 8, kPackRows = kPackThreads / kLanes;   // threads to a row, rows of a workgroup
constexpr int kReadPasses = 4, kReadRows = kReadPasses * kPackThreads / 16;

template <typename T>
__device__ __forceinline__ void load8(const char *p, float *x);
template <>
__device__ __forceinline__ void load8<float>(const char *p, float *x)
{
    const uint4 a = load_stream16(p), b = load_stream16(p + 16);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
}
template <>
__device__ __forceinline__ void load8<__bf16>(const char *p, float *x)
{
    const uint4 a = load_stream16(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}

// The four lanes of 32 elements.
__device__ __forceinline__ uint32_t most_of_4(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));          // lane ^ 1
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));       // lane ^ 2
}
__device__ __forceinline__ double most_of_4(double x)
{
    x = fmax(x, __shfl_xor(x, 1));
    return fmax(x, __shfl_xor(x, 2));
}

__device__ __forceinline__ uint32_t codes8(const float *x, float scale)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

// Element d of a row rotated in double precision: the angle is the position's product with the band's frequency modulo one revolution, off by |pos| 2^-62 revolutions at most.
template <typename T, bool HALF>
__device__ double rotated(const T *row, int d, int32_t pos, const BandTurns &turns)
{
    const int f = HALF ? d & 63 : d >> 1;
    const double re = (double)row[HALF ? f : 2 * f], im = (double)row[HALF ? f + 64 : 2 * f + 1];
    const int64_t phase = (int64_t)((uint64_t)(int64_t)pos * turns.w[f]);
    double s, c;
    sincospi((double)phase * 0x1p-63, &s, &c);
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

// A lane's sixteen elements x, unrotated, to 4 bits.  TURN: rotated first.  In fp32 a rotated element is off by at most (|re| + |im|) 2^-20 (sine and cosine by 2.2e-7, the products' roundings); where what lies within
// that of it does not all have one code, or the group's largest not one scale, the element is worked out in double precision: one wave in thirty of Gaussian rows.
template <typename T, bool TURN, bool HALF>
__device__ __forceinline__ Codes to_codes(float (*x)[8], const T *row, int32_t pos, const BandTurns &turns, int part)
{
    float off[2][8];
    if (TURN) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {   // eight bands
            float &r = HALF ? x[0][e] : x[e / 4][2 * (e & 3)], &i = HALF ? x[1][e] : x[e / 4][2 * (e & 3) + 1];
            const uint64_t w = turns.w[HALF ? 8 * part + e : 32 * (e / 4) + 4 * part + (e & 3)];
            float cs, sn;
            turn_exact(phase_of(pos, (uint32_t)w, (uint32_t)(w >> 32)), &cs, &sn);
            const float re = r, im = i;
            (HALF ? off[0][e] : off[e / 4][2 * (e & 3)]) = (HALF ? off[1][e] : off[e / 4][2 * (e & 3) + 1]) = (fabsf(re) + fabsf(im)) * 0x1p-20f;
            r = fmaf(re, cs, -(im * sn));
            i = fmaf(re, sn, im * cs);
        }
    }
    Codes got;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        uint32_t hi = 0, lo = 0;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t a = __float_as_uint(x[p][e]) & 0x7fffffffu;
            if (TURN) {
                odd |= a >= 0x7f800000u;
                hi = max(hi, min(__float_as_uint(fabsf(x[p][e]) + off[p][e]), 0x7f7fffffu));
                lo = max(lo, __float_as_uint(fmaxf(fabsf(x[p][e]) - off[p][e], 0.f)));
            } else {
                hi = max(hi, a);
            }
        }
        if (TURN && odd) hi = lo = 0xffffffffu;
        hi = most_of_4(hi);
        uint32_t byte = scale_byte(hi);
        if (TURN) {
            lo = most_of_4(lo);
            if (hi < 0x7f800000u && scale_byte(lo) != byte) {   // (all four lanes)
                double most = 0.0;
                for (int e = 0; e < 8; ++e) most = fmax(most, fabs(rotated<T, HALF>(row, 64 * p + 8 * part + e, pos, turns)));
                byte = scale_byte(most_of_4(most));
            }
        }
        const float scale = __uint_as_float(byte << 23);
        uint32_t word;
        if (TURN) {
            float below[8], above[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) below[e] = x[p][e] - off[p][e], above[e] = x[p][e] + off[p][e];
            word = codes8(below, scale);
            uint32_t open = byte == kScaleNaN ? 0 : word ^ codes8(above, scale);
            while (open) {
                const int at = (__ffs(open) - 1) & ~3;
                const uint32_t code = code_of(rotated<T, HALF>(row, 64 * p + 8 * part + at / 4, pos, turns), byte);
                word = (word & ~(15u << at)) | code << at;
                open &= ~(15u << at);
            }
        } else {
            word = codes8(x[p], scale);
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

// A workgroup takes 32 neighbouring tokens of a KV head, eight threads to a row of K and of V, each with two pieces of eight elements half a row apart: both parts of its bands lie in them in either pair layout, and
// four lanes hold the 32 elements of a scale.  Neighbouring rows are neighbouring slots: 64 bytes each, a wave writes 512 side by side.
template <typename T, bool TURN, bool HALF>
__global__ __launch_bounds__(kPackThreads) void append4_kernel(Append4Args args)
{
    const AppendArgs &a = args.a;
    const CacheView &c = a.cache;
    const int S = c.n_seqs, H = c.n_kv_heads;
    const int64_t i = (int64_t)blockIdx.x * kPackThreads + threadIdx.x;
    if (a.new_seq_len && i < S) {
        const int s = (int)i;
        const int n = clamp_len(a.head_len ? a.head_len[((int64_t)a.layer * S + s) * H] : c.seq_len[s], c.max_seq_len);
        int got = 1;
        if (a.start) got = max(clamp_to(a.start[s + 1], a.n_tokens) - clamp_to(a.start[s], a.n_tokens), 0);
        a.new_seq_len[s] = (int)min((int64_t)n + got, (int64_t)c.max_seq_len);
    }
    const int h = blockIdx.x % H, part = threadIdx.x % kLanes;
    const int64_t t0 = (int64_t)(blockIdx.x / H) * kPackRows;
    const int64_t t_wave = t0 + (threadIdx.x & ~63) / kLanes;
    if (t_wave >= a.n_tokens) return;   // (the whole wave)
    const int64_t t_mine = t0 + threadIdx.x / kLanes;
    const int t = (int)min(t_mine, (int64_t)a.n_tokens - 1);
    // the rows are asked for before their place is known
    const int64_t from = ((int64_t)t * a.stride_token + (int64_t)h * a.stride_head) * (int64_t)sizeof(T);
    float k[2][8], v[2][8];
#pragma unroll
    for (int p = 0; p < 2; ++p) load8<T>(a.k_new + from + (64 * p + 8 * part) * sizeof(T), k[p]), load8<T>(a.v_new + from + (64 * p + 8 * part) * sizeof(T), v[p]);
    const int32_t pos = a.pos[t];
    bool there = t_mine < a.n_tokens;
    int s = t, first = t;
    if (a.start) {
        s = 0;
        for (int j = 0; j < S; j += 64) {
            const int e = j + (int)(threadIdx.x & 63);
            s += __popcll(__ballot(e < S && a.start[min(e, S - 1) + 1] <= (int)t_wave));
        }
        while (s < S && a.start[s + 1] <= t) ++s;
        there &= s < S;
        s = min(s, S - 1);
        first = a.start[s];
        there &= t >= first;
    }
    const int len = clamp_len(a.head_len ? a.head_len[((int64_t)a.layer * S + s) * H + h] : c.seq_len[s], c.max_seq_len);
    const int64_t slot = (int64_t)len + (t - first);
    there &= slot < c.max_seq_len;
    int n = there ? (int)slot : 0;
    int64_t block = s;
    if (c.block_shift >= 0) {
        block = there ? block_of(c, a.n_blocks, s, n) : -1;
        there &= block >= 0;
        n &= (1 << c.block_shift) - 1;
    }
    const int64_t to = ((int64_t)a.layer * c.stride_layer + (int64_t)h * c.stride_head + block * c.stride_sb + slot_offset(c, n)) / 2;
    const int64_t word = word_of(c, (int64_t)a.layer * c.pos_stride_layer + (int64_t)h * c.pos_stride_head, block, n);
    const Codes kc = to_codes<T, TURN, HALF>(k, reinterpret_cast<const T *>(a.k_new + from), pos, a.turns, part);
    const Codes vc = to_codes<T, false, false>(v, nullptr, 0, a.turns, part);
    put_row(const_cast<void *>(c.k), args.k_scale, kc, part, there, to, word);
    put_row(const_cast<void *>(c.v), args.v_scale, vc, part, there, to, word);
    if (there && part == 0) const_cast<int32_t *>(c.pos)[word] = pos;
}

// Which slots a workgroup of tri_pack4 / tri_unpack4 moves, and where from.
struct Instance {
    int l, s, h, count;
    int64_t inst;
};
__device__ __forceinline__ Instance instance_of(const Pack4Args &a, int64_t inst)
{
    Instance x;
    x.inst = inst;
    x.h = (int)(inst % a.src.n_kv_heads);
    const int64_t ls = inst / a.src.n_kv_heads;
    x.s = (int)(ls % a.src.n_seqs);
    x.l = (int)(ls / a.src.n_seqs);
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
    return a.kept_idx ? min(max(a.kept_idx[x.inst * a.budget + j], 0), a.src.max_seq_len - 1) : j;
}

// As append4_kernel, from slots to slots.
template <typename T, bool TURN, bool HALF>
__global__ __launch_bounds__(kPackThreads) void pack4_kernel(Pack4Args a)
{
    const int64_t inst = blockIdx.x / (uint32_t)a.row_blocks;
    const int rb = (int)(blockIdx.x - inst * a.row_blocks), part = threadIdx.x % kLanes;
    const Instance x = instance_of(a, inst);
    if (a.new_seq_len && x.l == 0 && x.h == 0 && rb == 0 && threadIdx.x == 0) a.new_seq_len[x.s] = x.count;
    const int j = rb * kPackRows + (int)threadIdx.x / kLanes;
    if (rb * kPackRows + (int)(threadIdx.x & ~63) / kLanes >= x.count) return;   // (the whole wave)
    const int last = min(j, x.count - 1);
    const Place from = place_of(a.src, a.src_blocks, x, slot_to_read(a, x, last)), to = place_of(a.dst, a.dst_blocks, x, last);
    const bool there = j < x.count && from.there && to.there;
    const int64_t at = from.there ? from.row : 0, at_word = from.there ? from.word : 0;
    const T *row = reinterpret_cast<const T *>(a.src.k) + at;
    float k[2][8], v[2][8];
#pragma unroll
    for (int p = 0; p < 2; ++p) load8<T>((const char *)(row + 64 * p + 8 * part), k[p]), load8<T>((const char *)(reinterpret_cast<const T *>(a.src.v) + at + 64 * p + 8 * part), v[p]);
    const int32_t pos = a.src.pos[at_word];
    const Codes kc = to_codes<T, TURN, HALF>(k, row, pos, a.turns, part);
    const Codes vc = to_codes<T, false, false>(v, nullptr, 0, a.turns, part);
    put_row(const_cast<void *>(a.dst.k), a.k_scale, kc, part, there, to.row / 2, to.word);
    put_row(const_cast<void *>(a.dst.v), a.v_scale, vc, part, there, to.row / 2, to.word);
    if (there && part == 0) const_cast<int32_t *>(a.dst.pos)[to.word] = pos;
}

template <typename T>
__device__ __forceinline__ void store_read8(T *p, uint32_t word, float scale);
template <>
__device__ __forceinline__ void store_read8<__bf16>(__bf16 *p, uint32_t word, float scale) { store_stream16((char *)p, read8(word, scale)); }
template <>
__device__ __forceinline__ void store_read8<float>(float *p, uint32_t word, float scale)
{
    const uint4 b = read8(word, scale);
    store_stream16((char *)p, make_uint4(b.x << 16, b.x & 0xffff0000u, b.y << 16, b.y & 0xffff0000u));
    store_stream16((char *)(p + 4), make_uint4(b.z << 16, b.z & 0xffff0000u, b.w << 16, b.w & 0xffff0000u));
}

// Sixteen threads to a row, eight numbers each; every bf16 number is exact.
template <typename T>
__global__ __launch_bounds__(kPackThreads) void unpack4_kernel(Pack4Args a)
{
    const int64_t inst = blockIdx.x / (uint32_t)a.row_blocks;
    const int rb = (int)(blockIdx.x - inst * a.row_blocks), part = threadIdx.x % 16;
    const Instance x = instance_of(a, inst);
    if (a.new_seq_len && x.l == 0 && x.h == 0 && rb == 0 && threadIdx.x == 0) a.new_seq_len[x.s] = x.count;
#pragma unroll
    for (int i = 0; i < kReadPasses; ++i) {
        const int j = rb * kReadRows + i * (kPackThreads / 16) + (int)threadIdx.x / 16;
        if (j >= x.count) continue;
        const Place from = place_of(a.src, a.src_blocks, x, slot_to_read(a, x, j)), to = place_of(a.dst, a.dst_blocks, x, j);
        if (!from.there || !to.there) continue;
        const uint32_t kw = reinterpret_cast<const uint32_t *>((const char *)a.src.k + from.row / 2)[part], vw = reinterpret_cast<const uint32_t *>((const char *)a.src.v + from.row / 2)[part];
        store_read8<T>((T *)a.dst.k + to.row + 8 * part, kw, scale_at(a.k_scale[from.word], part / 4));
        store_read8<T>((T *)a.dst.v + to.row + 8 * part, vw, scale_at(a.v_scale[from.word], part / 4));
        if (part == 0) const_cast<int32_t *>(a.dst.pos)[to.word] = a.src.pos[from.word];
    }
}

}  // namespace

int64_t append4_groups(int64_t n_tokens, int64_t n_kv_heads) { return (n_tokens + kPackRows - 1) / kPackRows * n_kv_heads; }
int32_t pack4_row_blocks(int32_t slots) { return std::max(1, (int32_t)(((int64_t)slots + kPackRows - 1) / kPackRows)); }
int32_t unpack4_row_blocks(int32_t slots) { return std::max(1, (int32_t)(((int64_t)slots + kReadRows - 1) / kReadRows)); }

tri_status launch_append4(const Append4Args &a, int32_t rows, hipStream_t st)
{
    const int64_t lengths = a.a.new_seq_len ? (a.a.cache.n_seqs + kPackThreads - 1) / kPackThreads : 0;
    const uint32_t blocks = (uint32_t)std::max(append4_groups(a.a.n_tokens, a.a.cache.n_kv_heads), lengths);
    if (blocks == 0) return TRI_OK;
    const auto launch = [&](auto kernel) { kernel<<<blocks, kPackThreads, 0, st>>>(a); };
    const auto of = [&](auto plain, auto half, auto interleaved) { !a.a.rotate ? launch(plain) : a.a.half ? launch(half) : launch(interleaved); };
    if (rows == TRI_BF16) of(append4_kernel<__bf16, false, false>, append4_kernel<__bf16, true, true>, append4_kernel<__bf16, true, false>);
    else of(append4_kernel<float, false, false>, append4_kernel<float, true, true>, append4_kernel<float, true, false>);
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
