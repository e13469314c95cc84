// Attention with few rows per KV head (decoding): bf16, contiguous caches and pages of any size, up to 32 rows (token, query head of the group).
#include <algorithm>

#include "tri_attend_common.h"

namespace tri {

namespace {

constexpr int kRowsThreads = 256;
constexpr int kRowsTile = 32;   // keys a wave takes at a time

// Both halves of a wave's 64-byte pieces of a K row lie with one lane: x[c][e] is dimension 32 c + 8 kq + e.
template <bool HALF>
__device__ __forceinline__ void rotate_row(float (*x)[8], int32_t pos, int kq, const uint64_t *turns)
{
#pragma unroll
    for (int c = 0; c < (HALF ? 2 : 4); ++c)
#pragma unroll
        for (int e = 0; e < (HALF ? 8 : 4); ++e) {
            const uint64_t w = turns[HALF ? 32 * c + 8 * kq + e : 16 * c + 4 * kq + e];
            float cs, sn;
            turn_fast(phase_of(pos, (uint32_t)w, (uint32_t)(w >> 32)), &cs, &sn);
            float &r = HALF ? x[c][e] : x[c][2 * e], &i = HALF ? x[(c + 2) & 3][e] : x[c][(2 * e + 1) & 7];
            const float re = r, im = i;
            r = fmaf(re, cs, -(im * sn));
            i = fmaf(re, sn, im * cs);
        }
}

// NT column tiles of sixteen rows against 32 keys at a time.  S^T[key][row] = K Q^T and O^T[dim][row] = V^T P^T run on v_mfma_f32_16x16x32_bf16; a lane (m = lane & 15,
// kq = lane >> 4) holds eight terms of either operand, and since a contraction may take its terms in any order, it loads what is whole in memory: K operands are 16-byte
// pieces of the key's row; of V it loads pieces m of the rows of the eight keys whose weights it holds (4 kq + r of both halves of the tile: where the first product
// leaves them), and 32 byte permutations turn the 8 x 8 block in registers, row m of the product's tile e then being dimension 8 m + e.  Nothing passes through LDS
// or between lanes until the end but the maximum, so waves run on their own, 16 KB of loads under way each, and what bounds the kernel is the cache's bytes.
// LO: columns 8 to 15 of a tile hold what the rounding to bf16 takes off the rows 0 to 7 (of q turned by its position, and of the weights): the matrix
// instructions have that room where rows are at most eight to a tile, and both products are as good as in 16 bits of fraction.  Keys turned on the way (TURN)
// are multiplied as two bf16 numbers for the same reason.  Without LO both products are made twice: what is taken off q lies in LDS, what is taken off the weights in registers.  (The matrix pipe has the time: weights
// rounded to bf16 once, four sequences of 8192 keys and 32 rows take 35.8 us, 35.4 so; and a call's sequences keep their 16 bits when they go in one launch with a prefix of more rows.)
// Measured (8 KV heads): 32 ragged sequences up to 32768 keys in pages of 16, G = 4, 378 us, 2.29 GB at 6.1 TB/s (read once: 1.14 GB by the counter of fetches, which shows half of what is
// known to be read; a pure read stream reaches 7.0); the matrix pipe is busy for 4 % of that.  One of 131072 pre-RoPE keys at G = 8 96 us, 5.6 TB/s: 48 % of the time the vector pipe is busy turning keys.  One sequence
// of 2176 keys: 10 us, nearly all of it one chain of memory latencies.  Two workgroups to a CU: with three (168 registers, what does not fit spilled) the ragged batch takes 490.  Of the variants for
// more than eight rows, those that turn keys spill: 2 to 16 registers with LO, 40 to 45 without it in the half-split layout (both halves of a row are under way), none in the interleaved one; four sequences of
// 8192 keys and 32 rows take 35 us as they are, 45 turned interleaved, 59 turned half-split.  Operands of pages
// below sixteen slots have addresses of their own, 64 bits each: 452 us for that batch in pages of one slot.
template <int NT, bool LO, int PAGES, bool TURN, bool HALF>
__global__ __launch_bounds__(kRowsThreads, 2) void attend_rows_kernel(AttendArgs a)
{
    constexpr int kCols = LO ? 8 : 16, kRows = kCols * NT;
    __shared__ __align__(16) uint64_t turns[kBands];
    __shared__ float wave_m[4][kRows], wave_l[4][kRows];
    __shared__ __align__(16) float wave_o[4][kRows][kHeadDim + 4];
    __shared__ __align__(16) bf16x8 q_low[LO ? 1 : NT][4][64];   // what rounding takes off the rows, as operands
    const bool second = blockIdx.x >= a.first_groups;
    const AttendSource &src = second ? a.other : a.src;
    const CacheView &c = src.cache;
    const int H = c.n_kv_heads, G = a.group_size, Hq = H * G;
    // A head's parts run next to each other (with the parts of all heads one after the other, as in unit_of, the ragged batch above takes 404 us, with 382).  Workgroups go to the eight XCDs in turn, and
    // inside an XCD to its four shader engines, so the same part of all heads would meet few of them where the number of parts has a power of two in it: caches far below their capacity have only the first parts.
    // Which part comes first therefore goes round the heads: 32 of them meet all 32 engines.  64 sequences of 2000 keys in caches of 90000, 32 parts: 1710 us without, 150 with (84 at a capacity of 2000).
    const uint32_t w = blockIdx.x - (second ? a.first_groups : 0), n = src.n_split, head = w / n, even = min(n & -n, 32u);
    const uint32_t turned = w - head * n + ((head * even / 32) & (even - 1));
    const int split = turned < n ? turned : turned - n, h = head % H, s = head / H;
    const TokenRange tr = tokens_of(a, src, s);
    const int rows = min(tr.n * G, kRows);
    if (rows == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, kq = lane >> 4;
    const KeyRange range = keys_of_split(a, src, s, h, split);
    if (range.lo >= range.hi && a.part_o) {
        no_keys(a, src, split, tr.t0, 0, rows, h, Hq);
        return;
    }
    const int k_hi = __builtin_amdgcn_readfirstlane(range.hi);   // (what buffer descriptors are made of stays in scalar registers)

    const int64_t base = (int64_t)a.layer * c.stride_layer + (int64_t)h * c.stride_head;
    const int64_t pbase = (int64_t)a.layer * c.pos_stride_layer + (int64_t)h * c.pos_stride_head;
    const uint32_t sb = (uint32_t)c.stride_slot * 2u;
    const bool need_pos = a.causal || TURN;

    // Sixteen keys: which of them are there (in a block that is), and where their rows begin.  Lanes beyond the last row lie beyond the buffer and load zeros.  Pages below sixteen
    // slots have rows of their own addresses: keys that are not there load the pool's first row, and their values are cleared when they have come.
    struct Rows {
        int64_t kv, pos;
        int n;
        uint32_t there;
    };
    const int in_block = PAGES ? (1 << c.block_shift) - 1 : 0;
    auto is_block = [&](int b) { return (b >= 0) & ((src.n_blocks == 0) | (b < src.n_blocks)); };
    auto find = [&](int k0, int block_loaded) {
        Rows r;
        const int left = __builtin_amdgcn_readfirstlane(min(max(k_hi - k0, 0), 16));
        r.n = left;
        r.kv = r.pos = 0;
        if (PAGES == 2) {
            const uint32_t l = lane_again();
            r.there = (uint32_t)(__ballot(((int)(l & 15) < left) & is_block(block_loaded)) >> (k0 & 16)) & 0xffffu;
            return r;
        }
        if (PAGES == 1) {
            const int block = __builtin_amdgcn_readfirstlane(block_loaded);   // (here and not where it is asked for: that is a step ago)
            const int in = k0 & in_block;
            if (!is_block(block)) r.n = 0;
            const int b = r.n ? block : 0;
            r.kv = base + (int64_t)b * c.stride_sb + (int64_t)in * c.stride_slot;
            r.pos = pbase + (int64_t)b * c.pos_stride_sb + in;
        } else {
            r.kv = base + (int64_t)s * c.stride_sb + (int64_t)k0 * c.stride_slot;
            r.pos = pbase + (int64_t)s * c.pos_stride_sb + k0;
        }
        r.there = (1u << r.n) - 1;
        return r;
    };
    // the block of key k0, or (PAGES 2) of the lane's key of the 32 from k0 on
    auto block_at = [&](int k0) {
        if (PAGES == 2) k0 += lane_again() & 31;
        return PAGES ? c.block_table[(int64_t)s * c.max_blocks + (min(k0, max(k_hi - 1, 0)) >> c.block_shift)] : 0;
    };
    auto rsrc = [&](const void *p, int64_t at, int n) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((const char *)p) + at * 2, 0, __builtin_amdgcn_readfirstlane(n > 0 ? (n - 1) * sb + kHeadDim * 2 : 0), 0x00027000);
    };
    uint4 k[2][4], v[2][4];
    int32_t k_pos[2];
    // key `key` (0 to 31) of the tile from k0 on, its block being with lane `key`: the offset of its row
    auto slot_of = [&](int k0, int key, int block) {
        const int b = __shfl(block, key);
        return (is_block(b) & (k0 + key < k_hi)) ? base + (int64_t)b * c.stride_sb + slot_offset(c, (k0 + key) & in_block) : base;
    };
    auto load_k = [&](const Rows (&r)[2], int k0, int block) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t l = lane_again(), at = (l & 15) * sb + (l >> 4) * 16, at_pos = (l & 15) * 4;
            if (PAGES == 2) {
                const int key = 16 * i + (l & 15), b = __shfl(block, key);
                const char *p = (const char *)c.k + slot_of(k0, key, block) * 2 + (l >> 4) * 16;
#pragma unroll
                for (int j = 0; j < 4; ++j) k[i][j] = load_stream16(p + 64 * j);
                k_pos[i] = need_pos ? c.pos[pbase + ((is_block(b) & (k0 + key < k_hi)) ? (int64_t)b * c.pos_stride_sb + ((k0 + key) & in_block) : 0)] : 0;
                continue;
            }
            const auto b = rsrc(c.k, r[i].kv, r[i].n);
#pragma unroll
            for (int j = 0; j < 4; ++j) k[i][j] = as_uint4(__builtin_amdgcn_raw_buffer_load_b128(b, at + 64 * j, 0, kNonTemporal));
            const auto p = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t *>(c.pos) + r[i].pos, 0, __builtin_amdgcn_readfirstlane(need_pos ? r[i].n * 4 : 0), 0x00027000);
            k_pos[i] = __builtin_amdgcn_raw_buffer_load_b32(p, at_pos, 0, 0);
        }
    };
    auto load_v = [&](const Rows (&r)[2], int k0, int block) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t l = lane_again(), at = (l >> 4) * 4 * sb + (l & 15) * 16;
            if (PAGES == 2) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] = load_stream16((const char *)c.v + slot_of(k0, 16 * i + 4 * (l >> 4) + j, block) * 2 + (l & 15) * 16);
                continue;
            }
            const auto b = rsrc(c.v, r[i].kv, r[i].n);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = as_uint4(__builtin_amdgcn_raw_buffer_load_b128(b, at + j * sb, 0, kNonTemporal));
        }
    };
    constexpr int kStep = 4 * kRowsTile;
    int k0 = __builtin_amdgcn_readfirstlane(range.lo) + kRowsTile * wave;
    int block_here = block_at(k0), block_here2 = PAGES == 1 ? block_at(k0 + 16) : block_here;
    Rows here[2] = {find(k0, block_here), find(k0 + 16, block_here2)};
    int ahead = block_at(k0 + kStep), ahead2 = PAGES == 1 ? block_at(k0 + kStep + 16) : ahead;
    // The first tile is asked for before anything is known of the queries: in short rows most of the time is latency.
    load_k(here, k0, block_here);
    __builtin_amdgcn_sched_barrier(0);   // (in this order, as in the loop: waiting for K's loads must not wait for V's)
    load_v(here, k0, block_here);
    if (tid < kBands) turns[tid] = a.turns.w[tid];
    __syncthreads();

    // this lane's rows: columns m of the column tiles
    bf16x8 q[NT][4];
    int32_t t_pos[NT], first_pos = 0x7fffffff;
    bool real[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = n * kCols + (LO ? m & 7 : m), r = min(at, rows - 1), t = tr.t0 + r / G, hq = h * G + r % G;
        real[n] = at < rows;
        t_pos[n] = a.causal ? a.pos[t] : 0x7fffffff;
        first_pos = min(first_pos, t_pos[n]);
        const char *p = a.q + ((int64_t)t * a.q_stride_token + (int64_t)hq * a.q_stride_head) * 2;
        float x[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) widen8(*reinterpret_cast<const uint4 *>(p + 64 * j + 16 * kq), x[j]);
        if (a.rotate_q) {
            if (TURN ? HALF : (bool)a.half) rotate_row<true>(x, a.pos[t], kq, turns);
            else rotate_row<false>(x, a.pos[t], kq, turns);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const __bf16 hi = (__bf16)x[j][e];
                q[n][j][e] = LO && m >= 8 ? (__bf16)(x[j][e] - (float)hi) : hi;
                x[j][e] -= (float)hi;
            }
        if (!LO && a.rotate_q && wave == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8 low;
#pragma unroll
                for (int e = 0; e < 8; ++e) low[e] = (__bf16)x[j][e];
                q_low[n][j][lane] = low;
            }
        }
    }
    if (!LO) __syncthreads();
#pragma unroll
    for (int x = 1; x < 16; x *= 2) first_pos = min(first_pos, __shfl_xor(first_pos, x));
    first_pos = __builtin_amdgcn_readfirstlane(first_pos);

    f32x4 o[NT][8];
    float top[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = kNoScore;
        sum[n] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[n][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (; k0 < k_hi; k0 += kStep) {
        const Rows next[2] = {find(k0 + kStep, ahead), find(k0 + kStep + 16, PAGES == 1 ? ahead2 : ahead)};
        const int block_next = ahead;
        ahead = block_at(k0 + 2 * kStep);
        if (PAGES == 1) ahead2 = block_at(k0 + 2 * kStep + 16);
        f32x4 sc[2][NT];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int n = 0; n < NT; ++n) sc[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (TURN) {
                float x[4][8];
#pragma unroll
                for (int j = 0; j < 4; ++j) widen8(k[i][j], x[j]);
                rotate_row<HALF>(x, k_pos[i], kq, turns);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    bf16x8 hi, lo;
#pragma unroll
                    for (int e = 0; e < 8; ++e) hi[e] = (__bf16)x[j][e], lo[e] = (__bf16)(x[j][e] - (float)hi[e]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        sc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q[n][j], sc[i][n], 0, 0, 0);
                        sc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, q[n][j], sc[i][n], 0, 0, 0);
                        if (!LO && a.rotate_q) sc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q_low[n][j][lane], sc[i][n], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        sc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[i][j]), q[n][j], sc[i][n], 0, 0, 0);
            }
        }
        if (!LO && !TURN && a.rotate_q) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const bf16x8 low = q_low[n][j][lane];
#pragma unroll
                    for (int i = 0; i < 2; ++i) sc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[i][j]), low, sc[i][n], 0, 0, 0);
                }
        }
        const int32_t pos_here[2] = {k_pos[0], k_pos[1]};
        load_k(next, k0 + kStep, block_next);
        if (LO) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int d = 0; d < 4; ++d) sc[i][n][d] += across_8(sc[i][n][d]);
        }
        // keys that are not there, or behind the position of one of the rows
        const bool late = a.causal && __ballot(pos_here[0] > first_pos || pos_here[1] > first_pos);
        uint32_t keep[NT];   // bit 4 i + d: key 16 i + 4 kq + d is attended to
        bool hole = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) keep[n] = 0xffu;
        if (late || (here[0].there & here[1].there) != 0xffffu) {
            const uint32_t key = (lane_again() >> 4) * 4;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const bool there = (here[i].there >> (key + d)) & 1;
                    if (PAGES == 2) v[i][d] = there ? v[i][d] : make_uint4(0, 0, 0, 0);
                    const int32_t p = __shfl(pos_here[i], (int)key + d);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const bool on = there && (!a.causal || p <= t_pos[n]);
                        if (!on) keep[n] &= ~(1u << (4 * i + d)), sc[i][n][d] = kNoScore;
                        hole |= there && !on && real[n];
                    }
                }
        }
        bf16x8 weight[NT], weight_low[LO ? 1 : NT];
        float best[NT];
        bool higher = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            best[n] = kNoScore;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < 4; ++d) best[n] = fmaxf(best[n], sc[i][n][d]);
            best[n] = max_over_kq(best[n]);
            higher |= best[n] > top[n];
        }
        if (__ballot(higher)) {   // (rare after the first tiles)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float next_top = fmaxf(top[n], best[n]);
                const float shrink = next_top == kNoScore ? 1.f : __builtin_amdgcn_exp2f((top[n] - next_top) * a.scale_log2);
                top[n] = next_top;
                sum[n] *= shrink;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[n][e] *= shrink;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float ref = top[n] == kNoScore ? 0.f : top[n];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const float p = __builtin_amdgcn_exp2f((sc[i][n][d] - ref) * a.scale_log2);
                    sum[n] += p;
                    const __bf16 hi = (__bf16)p;
                    weight[n][4 * i + d] = LO && m >= 8 ? (__bf16)(p - (float)hi) : hi;
                    if (!LO) weight_low[n][4 * i + d] = (__bf16)(p - (float)hi);
                }
        }
        if (__ballot(hole)) {   // (see attend_general_kernel: values that are not finite and not everyone's)
            bool odd = false;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) odd |= not_finite(v[i][j]);
            if (__ballot(odd)) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        bf16x8 on;
#pragma unroll
                        for (int d = 0; d < 8; ++d) on[d] = (keep[n] >> d) & 1 ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll
                        for (int side = 0; side < 2; ++side) {
                            const f32x4 some = __builtin_amdgcn_mfma_f32_16x16x32_bf16(where_not_below(column(v, e), side ? 0xff80 : 0x7f80), on, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                            for (int d = 0; d < 4; ++d) o[n][e][d] += some[d] > 0.f ? (side ? -__builtin_inff() : __builtin_inff()) : 0.f;
                            __builtin_amdgcn_sched_barrier(0);   // (one after the other: few registers, and time does not matter here)
                        }
                    }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i][j] = finite_only(v[i][j]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bf16x8 x = column(v, e);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                o[n][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, weight[n], o[n][e], 0, 0, 0);
                if (!LO) o[n][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, weight_low[n], o[n][e], 0, 0, 0);
            }
        }
        load_v(next, k0 + kStep, block_next);
        here[0] = next[0];
        here[1] = next[1];
    }
    // join the waves: O's lane has dimensions 32 kq + 8 d + e of its row
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        sum[n] += __shfl_xor(sum[n], 16);
        sum[n] += __shfl_xor(sum[n], 32);
        if (kq == 0 && (!LO || m < 8)) wave_m[wave][n * kCols + m] = top[n], wave_l[wave][n * kCols + m] = sum[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = n * kCols + (LO ? m & 7 : m);
        float all = kNoScore;
#pragma unroll
        for (int j = 0; j < 4; ++j) all = fmaxf(all, wave_m[j][at]);
        const float mine = __builtin_amdgcn_exp2f((top[n] - (all == kNoScore ? 0.f : all)) * a.scale_log2);
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int d = 0; d < 4; ++d) o[n][e][d] = (LO ? o[n][e][d] + across_8(o[n][e][d]) : o[n][e][d]) * mine;
        if (!LO || m < 8)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int e = 0; e < 8; e += 4)
                    *reinterpret_cast<f32x4 *>(&wave_o[wave][at][32 * kq + 8 * d + e]) = f32x4{o[n][e][d], o[n][e + 1][d], o[n][e + 2][d], o[n][e + 3][d]};
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows / 16 + (kRows < 16); ++i) {
        const int row = 16 * i + (tid >> 4), d0 = 8 * (tid & 15);
        if (row >= rows) break;
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
        finish_row<__bf16>(a, src, split, tr.t0 + row / G, h * G + row % G, Hq, d0, best, total, x);
    }
}

template <int NT, bool LO>
void launch_rows_of(const AttendArgs &a, uint32_t blocks, hipStream_t st)
{
    const int shift = a.src.cache.block_shift, pages = shift < 0 ? 0 : shift >= 4 ? 1 : 2;
    const auto launch = [&](auto kernel) { kernel<<<blocks, kRowsThreads, 0, st>>>(a); };
    if (a.src.cache.k_rotated) launch(pages == 0 ? attend_rows_kernel<NT, LO, 0, false, false> : pages == 1 ? attend_rows_kernel<NT, LO, 1, false, false> : attend_rows_kernel<NT, LO, 2, false, false>);
    else if (a.half) launch(pages == 0 ? attend_rows_kernel<NT, LO, 0, true, true> : pages == 1 ? attend_rows_kernel<NT, LO, 1, true, true> : attend_rows_kernel<NT, LO, 2, true, true>);
    else launch(pages == 0 ? attend_rows_kernel<NT, LO, 0, true, false> : pages == 1 ? attend_rows_kernel<NT, LO, 1, true, false> : attend_rows_kernel<NT, LO, 2, true, false>);
}

}  // namespace

tri_status launch_attend_rows(AttendArgs a, int32_t rows, hipStream_t st)
{
    a.first_groups = (uint32_t)((int64_t)a.src.n_split * a.src.cache.n_kv_heads * a.src.cache.n_seqs);
    const uint32_t blocks = a.first_groups + (uint32_t)((int64_t)a.other.n_split * a.other.cache.n_kv_heads * a.other.cache.n_seqs);
    if (rows <= 8) launch_rows_of<1, true>(a, blocks, st);
    else if (rows <= 16) launch_rows_of<2, true>(a, blocks, st);
    else launch_rows_of<2, false>(a, blocks, st);
    return hip_status("attend_rows_kernel");
}

}  // namespace tri
