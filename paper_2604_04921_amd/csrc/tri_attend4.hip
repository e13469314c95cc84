// Attention over caches held in 4 bits.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "tri_attend_common.h"
#include "tri_serve4.h"

namespace tri {

namespace {

constexpr int kThreads = 256, kTile = 64;   // keys that a wave takes at a time
constexpr float kStaleBits = 8.f;   // powers of two by which a score may pass the maximum that weights are relative to
constexpr int kWaves = kThreads / 64;

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Both parts of a band of a row of q.
template <typename T>
__device__ __forceinline__ void load_band(const T *row, int f, bool half, float *re, float *im)
{
    if (half) {
        *re = (float)row[f], *im = (float)row[f + 64];
    } else {
        typedef T pair __attribute__((ext_vector_type(2)));
        const pair x = *reinterpret_cast<const pair *>(row + 2 * f);
        *re = (float)x[0], *im = (float)x[1];
    }
}

// lanes ^ 1, ^ 2, and the halves and the whole of each sixteen turned round: each lane of a sixteen has the result
template <typename F>
__device__ __forceinline__ int over_16(int x, F f)
{
    x = f(x, __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true));
    x = f(x, __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true));
    x = f(x, __builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true));
    return f(x, __builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true));
}
__device__ __forceinline__ float most_of_wave(float x)
{
    return max_over_kq(__int_as_float(over_16(__float_as_int(x), [](int a, int b) { return __float_as_int(fmaxf(__int_as_float(a), __int_as_float(b))); })));
}

// x of lanes FIRST + 0, 1, ... of each sixteen
template <int FIRST, int... N>
__device__ __forceinline__ void spread(uint32_t x, uint32_t *out, std::integer_sequence<int, N...>)
{
    ((out[N] = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x150 + FIRST + N, 0xf, 0xf, true)), ...);
}
// x + that of lane ^ 8 of each sixteen
__device__ __forceinline__ float add_across_8(float x) { return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xf, 0xf, true)); }
// x + that of lane ^ 4
__device__ __forceinline__ float add_across_4(float x) { return x + __shfl_xor(x, 4); }

// finish_row for N neighbouring dimensions.
template <typename T, int N>
__device__ __forceinline__ void finish(const AttendArgs &a, int split, int t, int hq, int Hq, int d0, float best, float total, float (&x)[N])
{
    if constexpr (N == 8) {
        finish_row<T>(a, a.src, split, t, hq, Hq, d0, best, total, x);
    } else {
        typedef float Sums __attribute__((ext_vector_type(N)));
        typedef T Out __attribute__((ext_vector_type(N)));
        if (a.part_o) {
            const int64_t at = ((int64_t)(a.src.part0 + split) * a.n_tokens + t) * Hq + hq;
            if (d0 == 0) a.part_ml[at] = make_float2(best, total);
            Sums y;
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = x[e];
            *reinterpret_cast<Sums *>(a.part_o + at * kHeadDim + d0) = y;
            return;
        }
        const float inv = 1.f / total;
        Out y;
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = (T)(total != 0.f ? x[e] * inv : 0.f);   // (no key: zeros; scores that are no number: NaN)
        *reinterpret_cast<Out *>(reinterpret_cast<T *>(a.out) + (int64_t)t * a.out_stride_token + (int64_t)hq * a.out_stride_head + d0) = y;
    }
}

// NT column tiles of sixteen rows against 64 keys at a time.  S^T[key][row] = K Q^T runs on v_mfma_scale_f32_16x16x128_f8f6f4, which takes the keys as they lie in memory -- a lane (m = lane & 15, kq = lane >> 4) has the
// 32 dimensions from 32 kq on of its key, and their scale -- and queries as e4m3 numbers: QPARTS of them to an element, each of what rounding left of the one before, four bits each (a part's scale is 2^-4 of the last
// one's, the first's brings the row's largest to [128, 256)).  O^T[dim][row] = V^T P^T runs on v_mfma_f32_16x16x32_bf16: values become bf16 numbers in registers, exactly (a conversion for two of them, scale and all),
// weights are WPARTS bf16 numbers each.  A lane's key is 4 (m & 3) + m / 4 of each sixteen, so that the first product leaves with it scores of keys 4 d + kq, and the rows of V that a load takes for them (dimensions
// 8 m to 8 m + 7 of four keys) are four neighbouring slots.  A lane has the words (position, scales, block) of one of the tile's 64 keys.
// COLS rows to a column tile.  8: columns 8 to 15 hold every second part of the rows, and one product does for two parts.  4: so do they for the first product; in the second, columns 4 to 7 and 12 to 15 hold second parts, and
// of each pair of dimensions that a conversion leaves in a register columns 0 to 7 have weights for the even one and zeros for the other, columns 8 to 15 the other way round, so that values need not be brought into the
// order of keys.
// What is held: the four parts have a bf16 q with 16 bits, weights of two parts have 16, as in attend_rows_kernel.  The instruction adds the products of eight neighbouring dimensions as multiples of 2^-13 of the largest
// one's power of two and the sixteen sums in fp32: rows at random come out 2^-16.4 of their largest product off (root mean square; 2^-12.4 at most), a thirtieth of what rounding a turned q to bf16 costs.  For fp32 rows that
// would be too much (22 standard deviations of fp32's roundings): they take three bf16 parts of q and of the weights against keys turned into bf16 numbers, with three times the matrix work.
// Bound by the cache's bytes where there are many keys: 32 ragged sequences of 1000 to 32768 keys in pages of 16, 622 MB, 116 us (5.3 TB/s; a plain read of as much 6.97 TB/s, 89 us), a sixth of that the prologue and
// the joining of waves of the last workgroups to begin; by latency where there are few: a token over 2176 keys 6.7 us, half of it the chain of arguments, lengths, rows and keys, then some 1500 instructions of one tile and
// the joining; by instructions with 9 to 64 rows: 32 sequences of 16000 keys take 145, 147, 301 and 300 us with 20, 32, 36 and 64 rows (96 with 4, the bytes alone 82), vector instructions being 55 to 61 % of the SIMDs'
// cycles and the matrix pipe 39 to 43 %.  Four e4m3 parts of a query are multiplied however many it needs, each wave decodes all values for its own rows, and from 33 rows on keys are read and weighed twice.  32 rows spill one
// register in pages of 16 and more, four in smaller ones.  Steps on the way (32 ragged sequences, us): as bf16 numbers in the first product too 159, keys as they are 135, four rows by zeros among the weights 126, a row of q turned once per workgroup 115; turned by
// every wave for itself, eight tokens' rows took 31 us of 26.  A third wave per SIMD by launch bounds (4) spills: 124 -> 170.
template <typename T, int NT, int COLS, int PAGES>
__global__ __launch_bounds__(kThreads, 2) void attend4_rows_kernel(AttendArgs a)
{
    constexpr bool DIRECT = sizeof(T) == 2, LO = COLS < 16, QUAD = COLS == 4;
    static_assert(!QUAD || (DIRECT && NT == 1), "");
    constexpr int QPARTS = DIRECT ? 4 : 3, WPARTS = DIRECT ? 2 : 3;
    constexpr int kQ = LO ? (QPARTS + 1) / 2 : QPARTS, kW = LO ? (WPARTS + 1) / 2 : WPARTS;   // products
    typedef std::conditional_t<DIRECT, i32x8, uint4[4]> Row;
    constexpr int kRows = COLS * NT, kSums = QUAD ? 4 : 8;
    typedef std::conditional_t<DIRECT, uint8_t, __bf16> Part;
    __shared__ int32_t q_unit[kRows], q_pos[kRows];
    __shared__ float wave_m[kWaves][kRows], wave_l[kWaves][kRows];
    __shared__ __align__(16) float wave_o[kWaves][kRows][kHeadDim + 4];
    Part(*q_parts)[kRows][kHeadDim] = reinterpret_cast<Part(*)[kRows][kHeadDim]>(wave_o);   // (which is written behind the loop, the parts being read before it and a barrier between)
    static_assert(sizeof(Part[QPARTS][kRows][kHeadDim]) <= sizeof(wave_o), "");
    const AttendSource &src = a.src;
    const CacheView &c = src.cache;
    const int H = c.n_kv_heads, G = a.group_size, Hq = H * G;
    // All that a workgroup needs of the arguments is asked for at once.  Asked for where it is needed, one wait came after the other: one sequence of 64 keys 6.8 us, 6.3 so, and 0.4 of any call.
    asm volatile("" ::"s"(c.k), "s"(c.v), "s"(c.pos), "s"(c.stride_sb), "s"(c.stride_layer), "s"(c.stride_head), "s"(c.stride_slot), "s"(c.pos_stride_sb), "s"(c.pos_stride_layer), "s"(c.pos_stride_head), "s"(c.n_seqs),
                 "s"(c.block_table), "s"(src.head_len), "s"(src.max_tokens), "s"(src.n_split), "s"(src.least_keys), "s"(a.k_scale), "s"(a.v_scale), "s"(a.q), "s"(a.q_stride_token), "s"(a.q_stride_head), "s"(a.pos));
    asm volatile("" ::"s"(a.layer), "s"(a.causal), "s"(a.rotate_q), "s"(a.half), "s"(a.group_size), "s"(a.part_o), "s"(a.start), "s"(a.row_tiles));
    // Row tiles of the same keys run next to each other on one XCD; a head's parts next to each other, which part comes first going round the heads (see attend_rows_kernel).
    const uint32_t x8 = blockIdx.x & 7, y8 = blockIdx.x >> 3;
    uint32_t in_eight = y8, row_tile = 0;
    if (a.row_tiles > 1) in_eight = y8 / (uint32_t)a.row_tiles, row_tile = y8 - in_eight * (uint32_t)a.row_tiles;
    const uint32_t w = in_eight * 8 + x8;
    const uint32_t n = src.n_split, head = w / n, even = min(n & -n, 32u);
    if (head >= (uint32_t)(H * c.n_seqs)) return;
    const uint32_t turned = w - head * n + ((head * even / 32) & (even - 1));
    const int split = turned < n ? turned : turned - n, h = head % H, s = head / H;
    const TokenRange tr = tokens_of(a, src, s);
    const KeyRange range = keys_of_split(a, src, s, h, split);   // (both are asked for at once)
    const int r0 = (int)row_tile * kRows, all_rows = tr.n * G, rows = min(all_rows - r0, kRows);
    if (rows <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, kq = lane >> 4;
    if (range.lo >= range.hi && a.part_o) {
        no_keys(a, src, split, tr.t0, r0, rows, h, Hq);
        return;
    }
    const int k_hi = __builtin_amdgcn_readfirstlane(range.hi);
    const int64_t base = ((int64_t)a.layer * c.stride_layer + (int64_t)h * c.stride_head) / 2;   // bytes
    const int64_t pbase = (int64_t)a.layer * c.pos_stride_layer + (int64_t)h * c.pos_stride_head;
    const uint32_t sb = (uint32_t)c.stride_slot / 2u;                       // bytes, too
    const uint64_t block_bytes = (uint64_t)c.stride_sb / 2u;
    const int in_block = PAGES ? (1 << c.block_shift) - 1 : 0;
    const int my_key = 4 * (m & 3) + (m >> 2);   // of each sixteen, whose row this lane loads
    // A lane has the words of the tile's key 4 m + kq, so that those of keys 16 i + 4 d + kq lie with lane 4 i + d of each sixteen.
    auto of_my_key = [&](uint32_t x, int i) { return (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (16 * (m >> 2) + (m & 3) + 4 * i), (int)x); };   // of key 16 i + my_key
    const uint32_t blocks = src.n_blocks ? (uint32_t)src.n_blocks : 0x80000000u;
    auto is_block = [&](int b) { return (uint32_t)b < blocks; };
    // the block of the lane's key of the 64 from k0 on
    auto block_at = [&](int k0) { return PAGES ? c.block_table[(int64_t)s * c.max_blocks + (min(k0 + 4 * m + kq, max(k_hi - 1, 0)) >> c.block_shift)] : 0; };
    auto there_of = [&](int k0, int block) { return __ballot((k0 + 4 * m + kq < k_hi) & (!PAGES || is_block(block))); };

    struct Words {
        int32_t pos;
        uint32_t k, v;
    };
    auto load_words = [&](int k0, int block, uint64_t there) {
        Words r{0, 0, 0};
        if ((there >> lane) & 1) {
            const int key = k0 + 4 * m + kq;
            const int64_t at = pbase + (PAGES ? (int64_t)block * c.pos_stride_sb + (key & in_block) : (int64_t)s * c.pos_stride_sb + key);
            r.pos = a.causal ? c.pos[at] : 0;
            r.k = a.k_scale[at];
            r.v = a.v_scale[at];
        }
        return r;
    };
    auto rsrc = [&](const void *p, int64_t at, int keys) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((const char *)p) + at, 0, __builtin_amdgcn_readfirstlane(keys > 0 ? (keys - 1) * sb + kHeadDim / 2 : 0), 0x00027000);
    };
    // where sixteen keys lie, and how many of them there are
    auto place = [&](int k0, int i, int block, int *keys) {
        const int first = k0 + 16 * i;
        int left = min(k_hi - first, 16);   // (what is below one makes no descriptor)
        int64_t at = base;
        if (PAGES) {
            const int b = __builtin_amdgcn_readlane(block, 4 * i);
            left = is_block(b) ? left : 0;
            at += (int64_t)((uint32_t)(left > 0 ? b : 0) * block_bytes + (uint64_t)(uint32_t)(first & in_block) * sb);
        } else {
            at += (int64_t)((uint32_t)s * block_bytes + (uint64_t)(uint32_t)first * sb);
        }
        *keys = left;
        return at;
    };
    // (PAGES 2: below sixteen slots) the row of the key that the lane has the words of; keys that are not there bring the pool's first row, with scales of zero.  (Worked out
    // once and handed round.  By every lane for the rows that it loads, twenty products in 64 bits, it left too few registers: 8 sequences of 4000 keys in pages of 4, eight tokens 92 us, 25 so; four 58 and 20; one 21 and 18.)
    auto slot_of = [&](int k0, int block, uint64_t there) {
        return (there >> lane) & 1 ? base + (int64_t)((uint32_t)block * block_bytes + (uint64_t)(uint32_t)((k0 + 4 * m + kq) & in_block) * sb) : base;
    };
    int64_t my_row = 0;
    uint4 k[4];
    uint32_t v[4][4];
    int64_t at[4];
    int keys[4];
    auto load_k = [&](int k0, int block, uint64_t there) {
        if (PAGES == 2) my_row = slot_of(k0, block, there);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
            if (PAGES == 2) {
                const char *p = (const char *)c.k + (int64_t)((uint64_t)of_my_key((uint32_t)(my_row >> 32), i) << 32 | of_my_key((uint32_t)my_row, i));
                if (DIRECT) {
                    k[i] = load_stream16(p + 16 * kq);
                } else {
                    const uint2v x = *reinterpret_cast<const uint2v *>(p + 8 * kq), y = *reinterpret_cast<const uint2v *>(p + 32 + 8 * kq);
                    k[i] = make_uint4(x.x, x.y, y.x, y.y);
                }
                continue;
            }
            at[i] = place(k0, i, block, &keys[i]);
            const auto b = rsrc(c.k, at[i], keys[i]);
            if (DIRECT) {
                k[i] = as_uint4(__builtin_amdgcn_raw_buffer_load_b128(b, my_key * sb + 16 * kq, 0, kNonTemporal));
            } else {
                const uint2v x = __builtin_bit_cast(uint2v, __builtin_amdgcn_raw_buffer_load_b64(b, my_key * sb + 8 * kq, 0, 0)), y = __builtin_bit_cast(uint2v, __builtin_amdgcn_raw_buffer_load_b64(b, my_key * sb + 32 + 8 * kq, 0, 0));
                k[i] = make_uint4(x.x, x.y, y.x, y.y);
            }
        }
    };
    auto load_v = [&] {
        if (PAGES == 2) {
            const auto some = [&](auto first) {   // (eight at a time: the compiler would have all addresses before the first load)
                uint32_t low[8], high[8];
                spread<first.value>((uint32_t)my_row, low, std::make_integer_sequence<int, 8>());
                spread<first.value>((uint32_t)(my_row >> 32), high, std::make_integer_sequence<int, 8>());
#pragma unroll
                for (int n = 0; n < 8; ++n)
                    v[(first.value + n) / 4][n % 4] = *reinterpret_cast<const uint32_t *>((const char *)c.v + (int64_t)((uint64_t)high[n] << 32 | low[n]) + 4 * m);
                __builtin_amdgcn_sched_barrier(0);
            };
            some(std::integral_constant<int, 0>()), some(std::integral_constant<int, 8>());
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto b = rsrc(c.v, at[i], keys[i]);
#pragma unroll
            for (int d = 0; d < 4; ++d) v[i][d] = __builtin_amdgcn_raw_buffer_load_b32(b, (kq + 4 * d) * sb + 4 * m, 0, kNonTemporal);   // (the scalar offset would not be checked against the size)
        }
    };
    constexpr int kStep = kWaves * kTile;
    int k0 = __builtin_amdgcn_readfirstlane(range.lo) + kTile * wave;
    // A wave turns the rows wave, wave + 4, ..., a band to a lane.  They are asked for ahead of the first tile (loads come in their order), which is on its way while they are turned.
    constexpr int kTurns = (kRows + kWaves - 1) / kWaves;
    const uint64_t turn = a.rotate_q ? a.turns.w[lane] : 0;
    float re[kTurns], im[kTurns];
    int32_t pos[kTurns];
    // (the last rows' places are whole rows, too: they hold the last row again, and nobody reads them)
    const int t_first = r0 / G, r_first = r0 - t_first * G;
    const float of_group = __builtin_amdgcn_rcpf((float)G);
    const T *q_row[kTurns];
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int r = r_first + min(wave + kWaves * i, rows - 1);   // (below G + 32)
        int t = (int)((r + 0.5f) * of_group);                       // r / G, or, in groups of tens of thousands, one off
        t += (r >= (t + 1) * G) - (r < t * G);
        const int token = tr.t0 + t_first + t, hq = h * G + r - t * G;
        q_row[i] = reinterpret_cast<const T *>(a.q) + (int64_t)token * a.q_stride_token + (int64_t)hq * a.q_stride_head;
        pos[i] = a.causal || a.rotate_q ? a.pos[token] : 0;
    }
    if (a.half) {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) load_band(q_row[i], lane, true, &re[i], &im[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) load_band(q_row[i], lane, false, &re[i], &im[i]);
    }
    int block = block_at(k0);
    uint64_t there = there_of(k0, block);
    Words words = load_words(k0, block, there);
    load_k(k0, block, there);
    load_v();
    int ahead = block_at(k0 + kStep);
    const int first = a.half ? lane : 2 * lane, second_at = a.half ? lane + 64 : 2 * lane + 1;   // the dimensions of the band
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int row = wave + kWaves * i;
        float c, s;
        const uint32_t phase = phase_of(pos[i], (uint32_t)turn, (uint32_t)(turn >> 32));
        if (DIRECT) turn_fast(phase, &c, &s);
        else turn_exact(phase, &c, &s);
        float x = a.rotate_q ? fmaf(re[i], c, -(im[i] * s)) : re[i], y = a.rotate_q ? fmaf(re[i], s, im[i] * c) : im[i];
        if constexpr (DIRECT) {
            // the power of two of the row's largest, at least what leaves the last part a scale
            const int unit = max((int)(__float_as_uint(most_of_wave(fmaxf(fabsf(x), fabsf(y)))) >> 23), 127 - 99);
            const float by = __uint_as_float((uint32_t)(261 - unit) << 23);
            x *= by, y *= by;
#pragma unroll
            for (int p = 0; p < QPARTS; ++p) {
                const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false);
                q_parts[p][row][first] = (uint8_t)w, q_parts[p][row][second_at] = (uint8_t)(w >> 8);
                x = (x - __builtin_amdgcn_cvt_f32_fp8(w, 0)) * 16.f;
                y = (y - __builtin_amdgcn_cvt_f32_fp8(w, 1)) * 16.f;
            }
            if (lane == 0) q_unit[row] = unit;
        } else {
#pragma unroll
            for (int p = 0; p < QPARTS; ++p) {
                const __bf16 u = (__bf16)x, w = (__bf16)y;
                q_parts[p][row][first] = u;
                q_parts[p][row][second_at] = w;
                x -= (float)u, y -= (float)w;
            }
        }
        if (lane == 0) q_pos[row] = pos[i];
    }
    __syncthreads();

    // this lane's rows: columns m of the column tiles
    Row q[NT][kQ];
    uint32_t q_scale[NT];   // a byte for every part
    int32_t t_pos[NT], first_pos = 0x7fffffff;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = min(t * COLS + (m & (COLS - 1)), rows - 1);
        t_pos[t] = a.causal ? q_pos[row] : 0x7fffffff;
        first_pos = min(first_pos, t_pos[t]);
        q_scale[t] = 0;
#pragma unroll
        for (int p = 0; p < kQ; ++p) {
            const int part = LO ? min(2 * p + (m >= 8), QPARTS - 1) : p;
            const uint4 *from = reinterpret_cast<const uint4 *>(q_parts[part][row]);
            if constexpr (DIRECT) {
                const uint4 x = from[kq], y = from[4 + kq];
                q[t][p] = i32x8{(int)x.x, (int)x.y, (int)x.z, (int)x.w, (int)y.x, (int)y.y, (int)y.z, (int)y.w};
                q_scale[t] |= (uint32_t)(q_unit[row] - 7 - 4 * part) << (8 * p);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    q[t][p][j] = from[8 * (j / 2) + 2 * kq + j % 2];
                    if (LO && 2 * p + 1 >= QPARTS && m >= 8) q[t][p][j] = make_uint4(0, 0, 0, 0);   // (three parts: the last has its product to itself)
                }
            }
        }
    }
    first_pos = __builtin_amdgcn_readfirstlane(over_16(first_pos, [](int x, int y) { return min(x, y); }));
    __syncthreads();

    // (QUAD) bytes 1, 0 below zeros or above them; of the upper half
    const uint32_t pick = m < 8 ? 0x0c0c0100u : 0x01000c0cu, pick_next = m < 8 ? 0x0202u : 0x02020000u;
    const float second = m & (QUAD ? 4 : 8) ? 1.f : 0.f;   // whether this column has second parts of weights
    f32x4 o[NT][kSums];
    float top[NT], sum[NT];
    uint32_t not_numbers[NT];   // bit 8 g + 7: dimensions 32 g and on of a value that the row attends to are none
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        not_numbers[t] = 0;
        top[t] = kNoScore;
        sum[t] = 0.f;
#pragma unroll
        for (int e = 0; e < kSums; ++e) o[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (; k0 < k_hi; k0 += kStep) {
        const int block_next = ahead;
        const uint64_t there_next = there_of(k0 + kStep, block_next);
        ahead = block_at(k0 + 2 * kStep);
        const Words words_next = load_words(k0 + kStep, block_next, there_next);
        f32x4 sc[4][NT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t word = of_my_key(words.k, i);
#pragma unroll
            for (int t = 0; t < NT; ++t) sc[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (DIRECT) {
                const uint32_t scale = word >> (8 * kq);
                const i32x8 x{(int)k[i].x, (int)k[i].y, (int)k[i].z, (int)k[i].w, 0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const auto product = [&](auto part) {   // (e2m1 times e4m3)
                        constexpr int p = decltype(part)::value;
                        if constexpr (p < kQ) sc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, q[t][p], sc[i][t], 4, 0, 0, scale, p, q_scale[t]);
                    };
                    product(std::integral_constant<int, 3>()), product(std::integral_constant<int, 2>()), product(std::integral_constant<int, 1>()), product(std::integral_constant<int, 0>());
                }
            } else {
                const uint32_t kw[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8 x = __builtin_bit_cast(bf16x8, read8(kw[j], scale_at(word, j / 2 * 2 + kq / 2)));
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int p = kQ - 1; p >= 0; --p) sc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8, q[t][p][j]), sc[i][t], 0, 0, 0);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);   // (phases are kept apart: the compiler would have all of a tile's conversions under way at once)
        Words here = words;
        words = words_next;
        load_k(k0 + kStep, block_next, there_next);
        if (LO) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int d = 0; d < 4; ++d) sc[i][t][d] = add_across_8(sc[i][t][d]);
        }
        // keys that are not there, or behind the position of one of the rows
        const bool late = __ballot(((there >> lane) & 1) & (here.pos > first_pos));   // (not causal: nothing is)
        if (late || there != ~0ull) {
            const uint32_t is = (uint32_t)(there >> (16 * kq));   // bit 4 i + d
            int32_t p[16];
            spread<0>((uint32_t)here.pos, reinterpret_cast<uint32_t *>(p), std::make_integer_sequence<int, 16>());
#pragma unroll
            for (int n = 0; n < 16; ++n)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (!((is >> n) & 1) | (p[n] > t_pos[t])) sc[n / 4][t][n % 4] = kNoScore;
        }
        float best[NT];
        bool higher = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            best[t] = kNoScore;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < 4; ++d) best[t] = fmaxf(best[t], sc[i][t][d]);
            best[t] = max_over_kq(best[t]);
            higher |= best[t] > top[t] && !((best[t] - top[t]) * a.scale_log2 <= kStaleBits);
        }
        if (__ballot(higher)) {   // (rare after the first tile: weights are relative to a maximum that scores may pass by a factor of 2^8)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float next_top = fmaxf(top[t], best[t]);
                const float shrink = next_top == kNoScore ? 1.f : __builtin_amdgcn_exp2f((top[t] - next_top) * a.scale_log2);
                top[t] = next_top;
                sum[t] *= shrink;
#pragma unroll
                for (int e = 0; e < kSums; ++e) o[t][e] *= shrink;
            }
        }
        // Values that are not numbers (a scale byte of 255) make the sums of their 32 dimensions no numbers in the rows that attend to their key: that is written down, and they are left out of the product.
        const uint32_t ff = here.v & ((here.v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
        for (uint64_t odd = __ballot(ff != 0); odd; odd &= odd - 1) {
            const int key = __builtin_ctzll(odd);
            const uint32_t which = __builtin_amdgcn_readlane(ff, key);
            const int32_t p = __builtin_amdgcn_readlane(here.pos, key);
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (!a.causal || p <= t_pos[t]) not_numbers[t] |= which;
        }
        here.v &= ~((ff << 1) - (ff >> 7));
#pragma unroll
        for (int U = 0; U < 2; ++U) {   // 32 keys
            __builtin_amdgcn_sched_barrier(0);
            bf16x8 weight[NT][kW];
            uint32_t pair[8];   // QUAD: a key's weight and zero, or zero and the weight
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float ref = top[t] == kNoScore ? 0.f : top[t], off = ref * a.scale_log2;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int d = 0; d < 4; d += 2) {
                        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                        float p[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            // (in fp32 a difference before the product: its rounding is not the product's)
                            p[e] = __builtin_amdgcn_exp2f(DIRECT ? fmaf(sc[2 * U + i][t][d + e], a.scale_log2, -off) : (sc[2 * U + i][t][d + e] - ref) * a.scale_log2);
                            sum[t] += p[e];
                        }
#pragma unroll
                        for (int u = 0; u < kW; ++u) {
                            bf16x2 part{(__bf16)p[0], (__bf16)p[1]};
                            if (LO) {   // lanes of the second eight columns have the part behind this one
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const float rest = fmaf(-(float)part[e], second, p[e]);
                                    p[e] -= (float)part[e];
                                    part[e] = (__bf16)rest;
                                    if (u + 1 < kW) p[e] -= (float)(__bf16)p[e];
                                }
                            } else if (u + 1 < kW) {
#pragma unroll
                                for (int e = 0; e < 2; ++e) p[e] -= (float)part[e];
                            }
                            if (QUAD) {
                                const uint32_t both = __builtin_bit_cast(uint32_t, part);
                                pair[4 * i + d] = __builtin_amdgcn_perm(0, both, pick);
                                pair[4 * i + d + 1] = __builtin_amdgcn_perm(0, both, pick + pick_next);
                            } else {
                                weight[t][u][4 * i + d] = part[0];
                                weight[t][u][4 * i + d + 1] = part[1];
                            }
                        }
                    }
            }
            uint32_t scales[8];
            if (U == 0) spread<0>(here.v, scales, std::make_integer_sequence<int, 8>());
            else spread<8>(here.v, scales, std::make_integer_sequence<int, 8>());
            uint4 values[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < 4; ++d) values[i][d] = read8(v[2 * U + i][d], scale_at(scales[4 * i + d], m >> 2));
            if (QUAD) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const bf16x8 w = __builtin_bit_cast(bf16x8, make_uint4(pair[4 * i], pair[4 * i + 1], pair[4 * i + 2], pair[4 * i + 3]));
                    const auto word = [](const uint4 &x, int e) { return e == 0 ? x.x : e == 1 ? x.y : e == 2 ? x.z : x.w; };
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint4 x = make_uint4(word(values[i][0], e), word(values[i][1], e), word(values[i][2], e), word(values[i][3], e));
                        o[0][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), w, o[0][e], 0, 0, 0);
                    }
                }
                continue;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bf16x8 x = column(values, e);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int p = kW - 1; p >= 0; --p) o[t][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, weight[t][p], o[t][e], 0, 0, 0);
            }
        }
        load_v();
        block = block_next;
        there = there_next;
    }
    // Join the waves: O's lane has dimensions 32 kq + 8 d + e of its row (QUAD: 32 kq + 8 d + 2 e, and those after them in the lanes of m >= 8).  Where lanes hold the same sums, each writes half of them.
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int at = t * COLS + (m & (COLS - 1));
        sum[t] += __shfl_xor(sum[t], 16);
        sum[t] += __shfl_xor(sum[t], 32);
        if (kq == 0 && m < COLS) wave_m[wave][at] = top[t], wave_l[wave][at] = sum[t];
        const bool other = LO && (m & (QUAD ? 4 : 8));
#pragma unroll
        for (int i = 0; i < (LO ? 2 : 4); ++i) {
            const int d = LO ? 2 * other + i : i;
#pragma unroll
            for (int e = 0; e < kSums; e += 4) {
                f32x4 y;
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const float first = o[t][e + n][i], later = o[t][e + n][LO ? 2 + i : i];
                    const float here = QUAD ? add_across_4(first) : LO ? add_across_8(first) : first, there = QUAD ? add_across_4(later) : LO ? add_across_8(later) : later;
                    y[n] = other ? there : here;
                }
                if (__ballot(not_numbers[t] != 0) && (not_numbers[t] >> (8 * kq + 7)) & 1) y = __builtin_nanf("");
                *reinterpret_cast<f32x4 *>(&wave_o[wave][at][32 * kq + 8 * d + (QUAD ? 4 * (m >> 3) : e)]) = y;
            }
        }
    }
    __syncthreads();
    constexpr int kOut = std::min(8, kRows * kHeadDim / kThreads), kLanesOut = kHeadDim / kOut;   // dimensions of a thread, threads of a row
#pragma unroll
    for (int i = 0; i < kRows * kLanesOut / kThreads; ++i) {
        const int row = (i * kThreads + tid) / kLanesOut, d0 = kOut * (tid % kLanesOut);
        if (row >= rows) break;
        float best = kNoScore, total = 0.f, x[kOut] = {};
#pragma unroll
        for (int j = 0; j < kWaves; ++j) best = fmaxf(best, wave_m[j][row]);
        const float ref = best == kNoScore ? 0.f : best;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) {
            const float by = __builtin_amdgcn_exp2f((wave_m[j][row] - ref) * a.scale_log2);
            total = fmaf(wave_l[j][row], by, total);
            const float *y = wave_o[j][row];
            if (QUAD) {
                const int lie = (d0 & ~7) + (d0 & 7) / 2;
                x[0] = fmaf(y[lie], by, x[0]), x[1] = fmaf(y[lie + 4], by, x[1]);
            } else {
#pragma unroll
                for (int e = 0; e < kOut; ++e) x[e] = fmaf(y[d0 + e], by, x[e]);
            }
        }
        const int r = r0 + row;
        finish<T, kOut>(a, split, tr.t0 + r / G, h * G + r % G, Hq, d0, best, total, x);
    }
}

// Rows that a workgroup takes.  More than 64 in bf16 are attend_tile_kernel's, which takes 128 of them over its tiles of keys where rows kernels take 32: 32 sequences of 16000 keys with 20, 32, 36 and 64 rows per KV head take
// 145, 147, 301 and 300 us here, 309, 306, 350 and 351 there; a third pass over the keys would not pay.
// A prefix counts as if all of the step's tokens were behind it, as for prefixes in full precision.  Where many prefixes have few tokens each, that is the wrong one of the two: 16 sequences with prefixes of 16000 keys of their
// own (64 rows in all) take 132 us, 32 take 304, and 256 with 1000 each 722, tri_attend4 over as many caches of that length 96 (32) and 52 (256).
bool is_tile(int32_t type, int64_t rows) { return type == TRI_BF16 && rows > 64; }
int64_t tile_rows(int32_t type, int64_t rows) { return is_tile(type, rows) ? kTileRows : rows <= 8 ? 8 : type == TRI_F32 || rows <= 16 ? 16 : 32; }

int64_t row_tiles_of(int32_t type, int64_t rows)
{
    const int64_t per = tile_rows(type, rows);
    return (rows + per - 1) / per;
}

}  // namespace

// As attend_split.  For rows: parts of about 3500 keys (32 ragged sequences, 32 of 16900 keys, the first in groups of eight take 141, 119 and 147 us in parts of 1024, 122, 110 and 131 of 2048, 120, 106 and 126 of 4096, 123, 103
// and 133 of 6144), or shorter ones, as many as give a CU three workgroups (32 sequences of 16900 and four of 30000: 101 and 30 us, with two 107 and 31, with four 107 and 33), but no shorter than 256 keys, a tile for each
// wave.  Partial results are kept below 64 MiB.
AttendSplit attend4_split(const tri_model &m, const tri_cache &c, int32_t max_tokens, int32_t n_tokens, int32_t type)
{
    const int64_t G = m.n_q_heads / m.n_kv_heads, rows = max_tokens * G, per = tile_rows(type, rows);
    const bool tile = is_tile(type, rows);
    const int64_t part = tile ? 8192 : 3500;
    const int64_t tiles = std::max<int64_t>(c.n_seqs, (n_tokens * G + per - 1) / per + c.n_seqs / 2);
    const int64_t units = m.n_kv_heads * tiles;
    const int64_t least = tile ? 256 : std::min<int64_t>(part, std::max<int64_t>(256, part * units / 256));
    const int64_t fill = std::max<int64_t>(1, ((tile ? 512 : 768) + units / 2) / units);
    const int64_t room = ((int64_t)64 << 20) / (std::max<int64_t>(n_tokens, 1) * m.n_q_heads * kHeadDim * (int64_t)sizeof(float));
    int64_t want = std::max<int64_t>(fill, std::min<int64_t>(c.max_seq_len / part, room));
    if (want * units < 2048) want = want / fill * fill;
    AttendSplit s{};
    s.least_keys = (int32_t)least;
    s.fill = tile ? (int32_t)fill : 1;
    s.fill_keys = tile ? (int32_t)part : 0;
    s.n_split = (int32_t)std::max<int64_t>(1, std::min<int64_t>({want, (c.max_seq_len + least - 1) / least, 256}));
    s.groups = ((int64_t)s.n_split * m.n_kv_heads * c.n_seqs + 7) / 8 * 8 * row_tiles_of(type, rows);
    return s;
}

tri_status launch_attend4(AttendArgs a, int32_t type, hipStream_t st)
{
    const int64_t rows = (int64_t)a.src.max_tokens * a.group_size;
    a.row_tiles = (int32_t)row_tiles_of(type, rows);
    const uint32_t blocks = (uint32_t)(((int64_t)a.src.n_split * a.src.cache.n_kv_heads * a.src.cache.n_seqs + 7) / 8 * 8 * a.row_tiles);
    const int shift = a.src.cache.block_shift;
    const auto launch = [&](auto kernel) { kernel<<<blocks, kThreads, 0, st>>>(a); };
    const auto of = [&](auto direct, auto paged, auto small) { shift < 0 ? launch(direct) : shift >= 4 ? launch(paged) : launch(small); };
    if (is_tile(type, rows)) return launch_attend4_tile(a, blocks, st);
    if (type == TRI_F32 && rows <= 8) of(attend4_rows_kernel<float, 1, 8, 0>, attend4_rows_kernel<float, 1, 8, 1>, attend4_rows_kernel<float, 1, 8, 2>);
    else if (type == TRI_F32) of(attend4_rows_kernel<float, 1, 16, 0>, attend4_rows_kernel<float, 1, 16, 1>, attend4_rows_kernel<float, 1, 16, 2>);
    else if (rows <= 4) of(attend4_rows_kernel<__bf16, 1, 4, 0>, attend4_rows_kernel<__bf16, 1, 4, 1>, attend4_rows_kernel<__bf16, 1, 4, 2>);
    else if (rows <= 8) of(attend4_rows_kernel<__bf16, 1, 8, 0>, attend4_rows_kernel<__bf16, 1, 8, 1>, attend4_rows_kernel<__bf16, 1, 8, 2>);
    else if (rows <= 16) of(attend4_rows_kernel<__bf16, 2, 8, 0>, attend4_rows_kernel<__bf16, 2, 8, 1>, attend4_rows_kernel<__bf16, 2, 8, 2>);
    else of(attend4_rows_kernel<__bf16, 2, 16, 0>, attend4_rows_kernel<__bf16, 2, 16, 1>, attend4_rows_kernel<__bf16, 2, 16, 2>);
    return hip_status("attend4_rows_kernel");
}

}  // namespace tri
