// Attention of a step's tokens over a cache (tri_attend, tri_attend_shared): the general kernel (fp32 matrix instructions, any type, any number of rows) and the
// joining of partial results.
#include <algorithm>

#include "tri_attend_common.h"

namespace tri {

namespace {

constexpr int kAttendThreads = 256;
constexpr int64_t kPartKeys = 2800;

template <typename T>
__device__ __forceinline__ void load4(const char *p, float *x);
template <>
__device__ __forceinline__ void load4<float>(const char *p, float *x)
{
    const f32x4 u = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = u[e];
}
template <>
__device__ __forceinline__ void load4<__bf16>(const char *p, float *x)
{
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    x[0] = __uint_as_float(u.x << 16), x[1] = __uint_as_float(u.x & 0xffff0000u);
    x[2] = __uint_as_float(u.y << 16), x[3] = __uint_as_float(u.y & 0xffff0000u);
}
// Rotates a lane's 32 elements of a row: x[c][e] is dimension 16 c + 4 kq + e, so both parts of a band lie in one lane in either pair layout.
template <bool HALF>
__device__ __forceinline__ void rotate32(float (*x)[4], int32_t pos, int kq, const uint64_t *turns)
{
#pragma unroll
    for (int c = 0; c < (HALF ? 4 : 8); ++c)
#pragma unroll
        for (int e = 0; e < (HALF ? 4 : 2); ++e) {
            const uint64_t w = turns[HALF ? 16 * c + 4 * kq + e : 8 * c + 2 * kq + e];
            float cs, sn;
            turn_exact(phase_of(pos, (uint32_t)w, (uint32_t)(w >> 32)), &cs, &sn);
            float &r = HALF ? x[c][e] : x[c][2 * e], &i = HALF ? x[(c + 4) & 7][e] : x[c][(2 * e + 1) & 3];
            const float re = r, im = i;
            r = fmaf(re, cs, -(im * sn));
            i = fmaf(re, sn, im * cs);
        }
}

// One wave takes 16 keys at a time against NT times 16 rows.  S^T[key][row] = K Q^T and O^T[dim][row] = V^T P^T run on v_mfma_f32_16x16x4_f32, whose lane (m = lane & 15,
// kq = lane >> 4) holds one element of either operand: contractions may take their terms in any order, so a lane feeds the four dimensions (QK) of a 16-byte piece of
// its key's row in turn, and O's rows are numbered so that the V rows it loads whole are operands as they are (dimension 64 b + 4 m + e is row m of tile (b, e)).
// S^T leaves key 4 kq + i of row (lane & 15) in register i, which is where the second product wants it: no data crosses lanes but the
// maximum and, at the end, the sum over kq.  The maximum is that of the products before the scale, which their differences are multiplied
// by (a score of 30 powers of two rounded as such is off by 2^-20).  The workgroup's four waves take every fourth tile of the range and join in LDS.
// Takes fp32 caches, and bf16 ones whose slots lie 2^24 elements apart or more.  fp32, 8 KV heads, G = 4: four sequences of 30238 keys 175 us (5.7 TB/s), pre-RoPE 184; chunks of 256 tokens over 4352 keys, two
// sequences, 295 us, 83 TFLOP/s of the 153 that a library product reaches (317 with the row tiles of a head on all XCDs).
template <typename T, int NT, bool TURN, bool HALF>
__global__ __launch_bounds__(kAttendThreads, NT == 1 ? 2 : 1) void attend_general_kernel(AttendArgs a)
{
    constexpr int kRows = 16 * NT;
    __shared__ uint64_t turns[kBands];
    __shared__ float wave_m[4][kRows], wave_l[4][kRows];
    __shared__ __align__(16) float wave_o[4][kRows][kHeadDim + 4];
    const CacheView &c = a.src.cache;
    const int H = c.n_kv_heads, G = a.group_size, Hq = H * G;
    // row tiles of the same keys next to each other on one XCD, as in attend_tile_kernel
    const uint32_t y = blockIdx.x >> 3;
    const int rt = y % a.row_tiles;
    const Unit unit = unit_of(a.src, (y / a.row_tiles) * 8 + (blockIdx.x & 7));
    const int split = unit.split, h = unit.h, s = unit.s;
    if (split >= a.src.n_split) return;
    const TokenRange tr = tokens_of(a, a.src, s);
    const int rows = tr.n * G, r0 = rt * kRows;
    if (r0 >= rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, kq = lane >> 4;
    if (tid < kBands) turns[tid] = a.turns.w[tid];
    __syncthreads();
    const KeyRange range = keys_of_split(a, a.src, s, h, split);
    const int k_lo = range.lo, k_hi = range.hi;
    if (k_lo >= k_hi && a.part_o) {
        no_keys(a, a.src, split, tr.t0, r0, min(rows - r0, kRows), h, Hq);
        return;
    }

    // this lane's rows: columns m of the column tiles of S^T and O^T
    float q[NT][8][4];
    int32_t t_pos[NT], first_pos = 0x7fffffff;
    bool real[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = r0 + 16 * n + m, r = min(at, rows - 1), t = tr.t0 + r / G, hq = h * G + r % G;
        real[n] = at < rows;
        t_pos[n] = a.pos ? a.pos[t] : 0;
        first_pos = min(first_pos, t_pos[n]);
        const char *p = a.q + ((int64_t)t * a.q_stride_token + (int64_t)hq * a.q_stride_head) * (int64_t)sizeof(T);
#pragma unroll
        for (int j = 0; j < 8; ++j) load4<T>(p + (16 * j + 4 * kq) * sizeof(T), q[n][j]);
        if (a.rotate_q) {
            if (TURN ? HALF : (bool)a.half) rotate32<true>(q[n], t_pos[n], kq, turns);
            else rotate32<false>(q[n], t_pos[n], kq, turns);
        }
    }
#pragma unroll
    for (int i = 1; i < 16; i *= 2) first_pos = min(first_pos, __shfl_xor(first_pos, i));
    f32x4 o[NT][8];
    float top[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = kNoScore;
        sum[n] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int64_t base = (int64_t)a.layer * c.stride_layer + (int64_t)h * c.stride_head;
    const int64_t pbase = (int64_t)a.layer * c.pos_stride_layer + (int64_t)h * c.pos_stride_head;
    const int in_block = c.block_shift < 0 ? 0x7fffffff : (1 << c.block_shift) - 1;
    // A lane's key of a tile is k0 + m.  Its block, or -1 where it is not there (keys of which the pool's first block is read instead).
    auto block_at = [&](int k0) { return c.block_shift < 0 || k_hi == 0 ? s : block_of(c, a.src.n_blocks, s, min(k0 + m, k_hi - 1)); };
    auto there_at = [&](int k0, int block) { return (k0 + m < k_hi) & (block >= 0); };
    auto slot_at = [&](int key) { return min(key, max(k_hi - 1, 0)) & in_block; };
    float k[8][4], v[4][2][4];
    int32_t k_pos = 0;
    auto load_k = [&](int k0, int block) {
        const int at = slot_at(k0 + m);
        const char *p = (const char *)c.k + row_of(c, base, max(block, 0), at) * (int64_t)sizeof(T);
#pragma unroll
        for (int j = 0; j < 8; ++j) load4<T>(p + (16 * j + 4 * kq) * sizeof(T), k[j]);
        k_pos = a.causal || TURN ? c.pos[pbase + (int64_t)max(block, 0) * c.pos_stride_sb + at] : 0;
    };
    auto load_v = [&](int k0, int block) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int from = 4 * kq + i;
            const char *p = (const char *)c.v + row_of(c, base, max(__shfl(block, from), 0), slot_at(k0 + from)) * (int64_t)sizeof(T);
            load4<T>(p + 4 * m * sizeof(T), v[i][0]);
            load4<T>(p + (64 + 4 * m) * sizeof(T), v[i][1]);
        }
    };
    int k0 = k_lo + 16 * wave, block = block_at(k0), ahead = block_at(k0 + 64);
    if (k0 < k_hi) {
        load_k(k0, block);
        __builtin_amdgcn_sched_barrier(0);
        load_v(k0, block);
    }
    for (; k0 < k_hi; k0 += 64) {
        if (TURN) rotate32<HALF>(k, k_pos, kq, turns);
        f32x4 sc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) sc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int n = 0; n < NT; ++n) sc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j][e], q[n][j][e], sc[n], 0, 0, 0);
        // the keys this lane has scores of (and whose V rows it has): 4 kq + i
        const bool there = there_at(k0, block);
        const int32_t pos_here = k_pos;
        const uint32_t there_bits = (uint32_t)__ballot(there) & 0xffffu;
        const int block_next = ahead;
        load_k(k0 + 64, block_next);   // (beyond the last tile: its last key again)
        ahead = block_at(k0 + 128);
        uint32_t keep[NT];   // bit i
        bool hole = false, odd = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) keep[n] = 0xfu;
        if (there_bits != 0xffffu || (a.causal && __ballot(pos_here > first_pos))) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool on = (there_bits >> (4 * kq + i)) & 1;
                const int32_t vp = __shfl(pos_here, 4 * kq + i);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const bool attends = on & (!a.causal | (vp <= t_pos[n]));
                    if (!attends) keep[n] &= ~(1u << i), sc[n][i] = kNoScore;
                    hole |= real[n] & on & !attends;
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[i][j][e] = on ? v[i][j][e] : 0.f;
            }
        }
        float p[NT][4], best[NT];
        bool higher = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            best[n] = max_over_kq(fmaxf(fmaxf(sc[n][0], sc[n][1]), fmaxf(sc[n][2], sc[n][3])));
            higher |= best[n] > top[n];
        }
        if (__ballot(higher)) {   // (rare after the first tiles)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float next = fmaxf(top[n], best[n]);
                const float shrink = next == kNoScore ? 1.f : __builtin_amdgcn_exp2f((top[n] - next) * a.scale_log2);   // (no score yet: 2^-inf = 0)
                top[n] = next;
                sum[n] *= shrink;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[n][j] *= shrink;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float ref = top[n] == kNoScore ? 0.f : top[n];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[n][i] = __builtin_amdgcn_exp2f((sc[n][i] - ref) * a.scale_log2);   // (left out: 2^-inf = 0)
                sum[n] += p[n][i];
            }
        }
        // A value that is not finite must not reach rows that do not attend to its key (0 times it is no 0).  Where a row of the tile leaves a key out, such values
        // are taken out of the product and added as what they are, by products of "attends" with "is +inf or NaN" and "is -inf or NaN".
        if (__ballot(hole)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd |= !(fabsf(v[i][j][e]) < __builtin_inff());
            if (__ballot(odd)) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            f32x4 up = f32x4{0.f, 0.f, 0.f, 0.f}, down = up;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float x = v[i][j][e], on = (keep[n] >> i) & 1 ? 1.f : 0.f;
                                up = __builtin_amdgcn_mfma_f32_16x16x4f32(x < __builtin_inff() ? 0.f : 1.f, on, up, 0, 0, 0);
                                down = __builtin_amdgcn_mfma_f32_16x16x4f32(x > -__builtin_inff() ? 0.f : 1.f, on, down, 0, 0, 0);
                            }
#pragma unroll
                            for (int d = 0; d < 4; ++d) o[n][4 * j + e][d] += (up[d] > 0.f ? __builtin_inff() : 0.f) + (down[d] > 0.f ? -__builtin_inff() : 0.f);
                            __builtin_amdgcn_sched_barrier(0);   // (one after the other: few registers, and time does not matter here)
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!(fabsf(v[i][j][e]) < __builtin_inff())) v[i][j][e] = 0.f;
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][4 * j + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i][j][e], p[n][i], o[n][4 * j + e], 0, 0, 0);
        load_v(k0 + 64, block_next);
        block = block_next;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        sum[n] += __shfl_xor(sum[n], 16);
        sum[n] += __shfl_xor(sum[n], 32);
        if (kq == 0) wave_m[wave][16 * n + m] = top[n], wave_l[wave][16 * n + m] = sum[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float all = kNoScore;
#pragma unroll
        for (int j = 0; j < 4; ++j) all = fmaxf(all, wave_m[j][16 * n + m]);
        const float mine = __builtin_amdgcn_exp2f((top[n] - (all == kNoScore ? 0.f : all)) * a.scale_log2);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int d = 0; d < 4; ++d)   // dimensions 64 j + 16 kq + 4 d + e
                *reinterpret_cast<f32x4 *>(&wave_o[wave][16 * n + m][64 * j + 16 * kq + 4 * d]) =
                    f32x4{o[n][4 * j][d], o[n][4 * j + 1][d], o[n][4 * j + 2][d], o[n][4 * j + 3][d]} * mine;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = 16 * n + (tid >> 4), d0 = 8 * (tid & 15);
        if (r0 + row >= rows) return;
        float best = kNoScore, total = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) best = fmaxf(best, wave_m[j][row]);
        const float ref = best == kNoScore ? 0.f : best;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            total += wave_l[j][row] * __builtin_amdgcn_exp2f((wave_m[j][row] - ref) * a.scale_log2);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += wave_o[j][row][d0 + e];
        }
        finish_row<T>(a, a.src, split, tr.t0 + (r0 + row) / G, h * G + (r0 + row) % G, Hq, d0, best, total, x);
    }
}

// Joins the parts of a row: sixteen threads have 8 dimensions each, and SPREAD such groups of a workgroup's sixteen share a row's parts, each going through its own in one pass
// with a running maximum; the groups are joined in LDS.  Sixteen where parts are many: one group alone walks 256 parts of a long cache one memory latency after the other.  A thread's first two parts are read with
// their maxima, the others only where those say that there is a key (lengths far below max_seq_len leave most parts empty).
// Bound by latency, then by the parts' bytes: 33 parts of 2048 rows, 35 MB, 9.5 us (13.3 with the maxima looked for first and 147 registers), 64 parts of 64 rows 4.7.
template <typename T, int SPREAD>
__global__ __launch_bounds__(kAttendThreads, 6) void join_kernel(const float *part_o, const float2 *part_ml, char *out, int64_t out_stride_token,
                                                                 int64_t out_stride_head, int32_t n_q_heads, int64_t n_rows, int32_t parts, float scale_log2)
{
    __shared__ float tops[SPREAD], totals[SPREAD];
    __shared__ __align__(16) float sums[SPREAD > 1 ? SPREAD : 1][kHeadDim];
    const int tid = threadIdx.x, group = tid >> 4, d0 = 8 * (tid & 15), first = SPREAD > 1 ? group : 0;
    const int64_t row = SPREAD > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (kAttendThreads / 16) + group;
    if (row >= n_rows) return;   // (SPREAD: never)
    float top = kNoScore, total = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const auto at = [&](int p) { return min(p, parts - 1) * n_rows + row; };
    float2 ahead[2] = {part_ml[at(first)], part_ml[at(first + SPREAD)]};
    for (int p0 = first; p0 < parts; p0 += 2 * SPREAD) {
        const float2 ml[2] = {ahead[0], ahead[1]};
        f32x4 o[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // (whatever the sums of a part without a key hold, they are not used)
            if (p0 == first || ml[i].y != 0.f) {
                const f32x4 *po = reinterpret_cast<const f32x4 *>(part_o + at(p0 + i * SPREAD) * kHeadDim + d0);
                o[i][0] = po[0], o[i][1] = po[1];
            }
            ahead[i] = part_ml[at(p0 + (2 + i) * SPREAD)];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (p0 + i * SPREAD >= parts || ml[i].y == 0.f) continue;   // (no key: nothing to bring)
            const float next = fmaxf(top, ml[i].x), ref = next == kNoScore ? 0.f : next;
            const float old = __builtin_amdgcn_exp2f((top - ref) * scale_log2), f = __builtin_amdgcn_exp2f((ml[i].x - ref) * scale_log2);
            top = next;
            total = total * old + f * ml[i].y;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] * old + f * o[i][e / 4][e % 4];
        }
    }
    if (SPREAD > 1) {
        store8(&sums[group][d0], x);
        if (d0 == 0) tops[group] = top, totals[group] = total;
        __syncthreads();
        if (group > 0) return;
        float best = kNoScore;
#pragma unroll
        for (int j = 0; j < SPREAD; ++j) best = fmaxf(best, tops[j]);
        const float ref = best == kNoScore ? 0.f : best;
        total = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
#pragma unroll 4
        for (int j = 0; j < SPREAD; ++j) {
            const float f = __builtin_amdgcn_exp2f((tops[j] - ref) * scale_log2);
            total += f * totals[j];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += f * sums[j][d0 + e];
        }
    }
    const float inv = 1.f / total;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = total != 0.f ? x[e] * inv : 0.f;
    const int64_t t = row / n_q_heads, h = row - t * n_q_heads;
    store8(reinterpret_cast<T *>(out) + t * out_stride_token + h * out_stride_head + d0, x);
}

}  // namespace

// Which kernel takes a call: the bf16 ones need sixteen rows' addresses within 32 bits.
enum class Kernel { general, rows, tile };
static Kernel kernel_of(const tri_cache &c, int64_t rows)
{
    if (c.dtype != TRI_BF16 || c.stride_slot >= (1 << 24)) return Kernel::general;
    return rows <= 32 ? Kernel::rows : Kernel::tile;
}

// Rows of a workgroup of the general kernel.  32 where that spares a second pass over the keys (fp32, eight sequences of 4096 keys, 28 rows: 89 / 83 us); with more rows two waves to a SIMD, which 16
// rows leave room for, are worth more (two chunks of 256 tokens over 4352 keys 295 us with 16, 371 with 32).
static int64_t general_rows(const tri_cache &c, int64_t rows) { return c.dtype == TRI_F32 && rows > 16 && rows <= 32 ? 32 : 16; }

// Row tiles of a sequence, and workgroups of a cache's launch: those of row tiles in whole rounds over the eight XCDs.
static int64_t row_tiles_of(Kernel kernel, const tri_cache &c, int64_t rows)
{
    const int64_t per_tile = kernel == Kernel::general ? general_rows(c, rows) : kernel == Kernel::tile ? kTileRows : rows;
    return (rows + per_tile - 1) / per_tile;
}
static int64_t groups_of(Kernel kernel, int64_t heads, int64_t row_tiles) { return kernel == Kernel::rows ? heads : (heads + 7) / 8 * 8 * row_tiles; }

// Parts.  Two workgroups of either bf16 kernel share a CU, so 512 of them fill the GPU; more even out ragged batches, and each costs what 100 to 200 keys do, and the joining of its
// results.  Measured, us by parts per head, 8 KV heads, G = 4, bf16 single tokens: 16 x 65536 keys 1023 / 630 / 642 / 637 / 661 / 850 at 1, 2, 8, 16, 48, 128 parts; 16 sequences between
// 1000 and 65536 keys 938 / 526 / 438 / 399 / 418 / 523 at the same; 16 x 4096 69 / 49 / 61 / 71 at 1, 2, 8, 16; 64 x 2176 90 / 98 / 143 at 1, 2, 8; one of 131072 at G = 8 201 / 114 / 96 /
// 107 at 16, 32, 64, 128.  fp32: 4 x 30238 1025 / 287 / 178 / 184 at 1, 4, 16, 64; 16 between 300 and 2176 92 / 57 / 51 / 47 / 55 at 1, 2, 3, 4, 8.  The tile kernel: 64 sequences behind 32768 keys
// 1253 / 351 / 133 / 111 at 1, 4, 16, 32; two chunks of 1024 tokens over 8192 keys, 480 row tiles, 321 / 364 / 387 at 1, 2, 4; one of 512 over 16384 400 / 201 / 169 / 182 at 1, 3, 4, 8.
// So: 512 workgroups (`fill` parts), or parts of 2800 keys (1400 in fp32, 8192 for row tiles) where that makes more; none below the keys that `least` gives, which the device goes by where the lengths
// turn out shorter than max_seq_len, nor, for row tiles, below what the same rule gives for the length there is: max_seq_len is a capacity, and with parts by it two chunks of 1024 tokens over 8192 keys in caches of
// 131072 were cut into sixteen, the sums of which are 0.5 GB (now 319 us; 303 where the capacity is the length).
// More than `fill` parts hold kMostPartBytes of sums together at most, a workspace being a user's memory (one fp32 chunk of 8192 tokens in a cache of 131072: 12.7 GB in 93 parts; one part, and no workspace, now).
// us at 256 / 64 / 16 MiB: two chunks of 1024 tokens over 131072 keys 4851 / 4913 / 4983, over 131072 and 8192 2604 / 2636 / 3173; fp32, two of 256 over 30000 2580 / 2424 / 2362, over 4352 in caches of 131072
// 512 / 403 / 375.
constexpr int64_t kMostPartBytes = 64 << 20;
AttendSplit attend_split(const tri_model &m, const tri_cache &c, int32_t max_tokens, int32_t n_tokens)
{
    const int64_t G = m.n_q_heads / m.n_kv_heads, rows = max_tokens * G;
    const Kernel kernel = kernel_of(c, rows);
    const int64_t per_tile = kernel == Kernel::general ? general_rows(c, rows) : kernel == Kernel::rows ? 32 : kTileRows;
    // row tiles that there are: all tokens' rows, and half a tile more per sequence, whose last one is not full
    const int64_t tiles = kernel == Kernel::rows ? c.n_seqs : std::max<int64_t>(c.n_seqs, (n_tokens * G + per_tile - 1) / per_tile + c.n_seqs / 2);
    const int64_t units = m.n_kv_heads * tiles;
    const int64_t part = kernel == Kernel::tile ? 8192 : c.dtype == TRI_F32 ? kPartKeys / 2 : kPartKeys;
    const int64_t least = kernel == Kernel::tile ? 256 : std::min<int64_t>(part, std::max<int64_t>(128, part * units / 256));
    const int64_t fill = std::max<int64_t>(1, (512 + units / 2) / units);
    const int64_t room = kMostPartBytes / (std::max<int64_t>(n_tokens, 1) * m.n_q_heads * kHeadDim * (int64_t)sizeof(float));
    int64_t want = std::max<int64_t>(fill, std::min<int64_t>(c.max_seq_len / part, room));
    if (want * units < 2048) want = want / fill * fill;   // (few rounds: whole ones; 4 x 30238 keys in fp32 178 us with 16 parts, 210 with 21)
    AttendSplit s;
    s.least_keys = (int32_t)least;
    s.fill = kernel == Kernel::tile ? (int32_t)fill : 1;
    s.fill_keys = kernel == Kernel::tile ? (int32_t)part : 0;
    s.n_split = (int32_t)std::max<int64_t>(1, std::min<int64_t>({want, (c.max_seq_len + least - 1) / least, 256}));
    s.groups = groups_of(kernel, (int64_t)s.n_split * m.n_kv_heads * c.n_seqs, row_tiles_of(kernel, c, rows));
    return s;
}

tri_status launch_attend(AttendArgs a, const tri_cache &c, hipStream_t st)
{
    const int64_t rows = (int64_t)a.src.max_tokens * a.group_size;
    const Kernel kernel = kernel_of(c, rows);
    if (kernel == Kernel::rows) return launch_attend_rows(a, (int32_t)rows, st);
    a.row_tiles = (int32_t)row_tiles_of(kernel, c, rows);
    const uint32_t blocks = (uint32_t)groups_of(kernel, (int64_t)a.src.n_split * a.src.cache.n_kv_heads * a.src.cache.n_seqs, a.row_tiles);
    if (kernel == Kernel::tile) return launch_attend_tile(a, blocks, st);
    const auto launch = [&](auto variant) { variant<<<blocks, kAttendThreads, 0, st>>>(a); };
    if (c.dtype == TRI_BF16) launch(c.k_rotated ? attend_general_kernel<__bf16, 1, false, false> : a.half ? attend_general_kernel<__bf16, 1, true, true> : attend_general_kernel<__bf16, 1, true, false>);
    else if (general_rows(c, rows) == 16) launch(c.k_rotated ? attend_general_kernel<float, 1, false, false> : a.half ? attend_general_kernel<float, 1, true, true> : attend_general_kernel<float, 1, true, false>);
    else launch(c.k_rotated ? attend_general_kernel<float, 2, false, false> : a.half ? attend_general_kernel<float, 2, true, true> : attend_general_kernel<float, 2, true, false>);
    return hip_status("attend_general_kernel");
}

// Small batches behind a prefix spend their time in one chain of memory latencies per launch: both caches go in one launch of attend_rows_kernel where both are its, of the same layout, and either take the same
// variant of it or are so few workgroups that all run at once (eight sequences of up to 130 keys behind 2048: 28 us with a launch each and the joining, 20 with one).
tri_status launch_attend_both(AttendArgs a, const tri_cache &c, const tri_cache &other, hipStream_t st)
{
    const auto rows_of = [&](const AttendSource &s) { return (int64_t)s.max_tokens * a.group_size; };
    const auto variant = [](int64_t rows) { return rows <= 8 ? 0 : rows <= 16 ? 1 : 2; };
    const auto pages = [](const AttendSource &s) { return s.cache.block_shift < 0 ? 0 : s.cache.block_shift >= 4 ? 1 : 2; };
    const auto groups = [](const AttendSource &s) { return (int64_t)s.n_split * s.cache.n_kv_heads * s.cache.n_seqs; };
    const int64_t rows = rows_of(a.src), more = rows_of(a.other);
    if (kernel_of(c, rows) == Kernel::rows && kernel_of(other, more) == Kernel::rows && pages(a.src) == pages(a.other) && a.src.cache.k_rotated == a.other.cache.k_rotated &&
        (variant(rows) == variant(more) || groups(a.src) + groups(a.other) <= 512))
        return launch_attend_rows(a, (int32_t)std::max(rows, more), st);
    const AttendSource second = a.other;
    a.other = AttendSource{};
    const tri_status rc = launch_attend(a, c, st);
    if (rc != TRI_OK) return rc;
    a.src = second;
    return launch_attend(a, other, st);
}

static bool join_spread(int32_t parts) { return parts > 8; }
int64_t join_groups(int64_t rows, int32_t parts) { return join_spread(parts) ? rows : (rows + kAttendThreads / 16 - 1) / (kAttendThreads / 16); }

tri_status launch_join(const AttendArgs &a, int32_t parts, int32_t n_q_heads, int32_t dtype, hipStream_t st)
{
    const int64_t rows = (int64_t)a.n_tokens * n_q_heads;
    const bool spread = join_spread(parts);
    const uint32_t blocks = (uint32_t)join_groups(rows, parts);
    const auto launch = [&](auto kernel) {
        kernel<<<blocks, kAttendThreads, 0, st>>>(a.part_o, a.part_ml, a.out, a.out_stride_token, a.out_stride_head, n_q_heads, rows, parts, a.scale_log2);
    };
    if (dtype == TRI_BF16) launch(spread ? join_kernel<__bf16, 16> : join_kernel<__bf16, 1>);
    else launch(spread ? join_kernel<float, 16> : join_kernel<float, 1>);
    return hip_status("join_kernel");
}

}  // namespace tri
