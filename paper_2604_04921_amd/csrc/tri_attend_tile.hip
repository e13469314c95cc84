// Attention with many rows per KV head (chunks of prompts, batches behind a shared prefix): bf16, contiguous caches and pages of any size.
#include <type_traits>

#include "tri_attend_common.h"
#include "tri_serve4.h"

namespace tri {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kWaves = 4, kRows = 32 * kWaves;   // rows of a workgroup
constexpr int kTileKeys = 64, kKeys = kTileKeys / kWaves;   // keys of a tile, and those of them that a wave brings
static_assert(kRows == kTileRows && kKeys == 16, "");
constexpr float kStaleBits = 8.f;   // powers of two by which a score may pass the maximum that weights are relative to

// Rotates a lane's 64 elements of a row: x[c][e] is dimension 16 c + 8 h + e.
template <bool HALF>
__device__ __forceinline__ void rotate_q(float (*x)[8], int32_t pos, int h, const uint64_t *turns)
{
#pragma unroll
    for (int c = 0; c < (HALF ? 4 : 8); ++c)
#pragma unroll
        for (int e = 0; e < (HALF ? 8 : 4); ++e) {
            const uint64_t w = turns[HALF ? 16 * c + 8 * h + e : 8 * c + 4 * h + e];
            float cs, sn;
            turn_fast(phase_of(pos, (uint32_t)w, (uint32_t)(w >> 32)), &cs, &sn);
            float &r = HALF ? x[c][e] : x[c][2 * e], &i = HALF ? x[(c + 4) & 7][e] : x[c][(2 * e + 1) & 7];
            const float re = r, im = i;
            r = fmaf(re, cs, -(im * sn));
            i = fmaf(re, sn, im * cs);
        }
}

// What is done to keys on their way to the first product.  What has been turned is no bf16 number any more, and where scores are large, rounding it to one shows: outputs 0.0064 and 0.0071 off (root mean square, relative;
// two pre-RoPE caches) and 0.0034 (q alone turned), where the outputs' own rounding is 0.0017.  The product then runs in fp16, three bits more at the same rate: 0.0021, 0.0022 and 0.0023, for 70 -> 80, 47 -> 53 and
// 28 -> 31 us.  Rows of q are brought to [1, 2) by a power of two, those of K only where fp16 would not hold them, and the scores get the powers back.
enum Keys { kAsTheyAre, kWiden, kTurn };   // q as it came; q turned, keys bf16 numbers made fp16; both turned

// The power of two that x / unit_of(x) has a magnitude of [1, 2) with, for x of at least 2^-113; infinities and NaN stay what they are.
__device__ __forceinline__ float unit_of(float x)
{
    const int e = (int)((__float_as_uint(x) >> 23) & 255) - 127;
    return x == 0.f ? 1.f : __uint_as_float((uint32_t)(min(max(e, -113), 113) + 127) << 23);
}
__device__ __forceinline__ float over(float unit) { return __uint_as_float((254u << 23) - __float_as_uint(unit)); }   // 1 / unit
__device__ __forceinline__ bf16x8 narrow_f16(const float *x, float by)   // (the bits; the type is that of all operands)
{
    f16x8 u;
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = (_Float16)(x[e] * by);
    return __builtin_bit_cast(bf16x8, u);
}

template <bool F16>
__device__ __forceinline__ f32x16 scores(bf16x8 k, bf16x8 q, f32x16 sum)
{
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, k), __builtin_bit_cast(f16x8, q), sum, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q, sum, 0, 0, 0);
}

struct TileBuffer {
    __bf16 k[kTileKeys * kHeadDim], v[kTileKeys * kHeadDim];
    int32_t pos[kTileKeys];
    float unit[kTileKeys];     // fp16: what a key's scores are multiplied by
    int32_t lim[3 * kWaves];   // of every wave's keys: highest and lowest position, and which are there (a bit each; bit 16: a unit is not one)
};

// A workgroup has four waves of 32 rows each (token, query head of the group) and goes through the keys 64 at a time, K and V lying in LDS for all four.  S^T[key][row] = K Q^T runs on
// v_mfma_f32_32x32x16_bf16, or _f16 where queries or keys are turned on the way (see Keys), O^T[dim][row] = V^T P^T on the former: a row is a lane's column throughout, so its maximum and sum are in-lane but for one exchange of the lane's halves, and the weights are the second product's
// operand where the first leaves its scores (lane half h holds keys 8 (i / 4) + 4 h + i % 4; the V operand takes its keys in that order, from transposing LDS reads).  K and V go from memory to LDS without passing
// through registers; a tile's loads are under way while the last one is worked on.  The weights are rounded to bf16 once:
// values are bf16 numbers, the instruction takes both operands in one type, and a second product for what is taken off would make half as many matrix instructions again where these bound the kernel (unlike with few
// rows).  Every key's rounding is its own, so it adds to an output about what its own rounding does: 0.0023 (root mean square, relative) where that alone is 0.0017.
// Measured: two chunks of 1024 tokens over up to 8192 keys in pages of 64, 8 x 4 heads, 227 GFLOP: 259 to 270 us, 840 to 875 TFLOP/s (a library product of 8192 x 8192 matrices runs at 1355 here).  The matrix pipe is busy 35 % of the
// time, the vector pipe with softmax 41 %, LDS 33 %, and the two hardly overlap: a wave issues in order, and there are two to a SIMD.  64 rows to a wave (one to a SIMD) took 577 us when 32 took
// 322, eight waves to a workgroup 382; the loads' issue is a quarter of the time (without them, on stale tiles, 245 of 322).  Without neighbours on one XCD two prompts' 256 sequences take 379 us, with 229.
// That is with queries and keys as they are.  Two chunks of 1024 over 8192 keys each, contiguous, take 294 us so, 383 with queries turned on the way and 452 with keys too: every row tile turns its keys again, and what
// does not fit is spilled (6 to 9 registers with queries turned, 11 to 21 with keys).
// FOUR: keys and values are held in 4 bits.  A lane brings 32 elements of a row, which have one scale.  Values are written into LDS as the bf16 numbers that they stand for, exactly; keys as they are, with their scales, for
// v_mfma_scale_f32_32x32x64_f8f6f4, which takes queries as e4m3 numbers: two to an element, four bits each, which is all a bf16 number has, or three where queries are turned, and sums as attend4_rows_kernel says.  Weights are
// bf16 numbers, as above.  Two chunks of 1024 tokens over 5000 to 7168 keys (227 GF) take 270 us, 840 TFLOP/s, where a large library product in bf16 has 1344; with keys as bf16 numbers in LDS, which is four times the reads and as
// many conversions as values are, 291.  That is with queries as they are, where it spills three or four registers; with queries turned on the way it spills 31 to 33, of the third part, and two chunks of 1024 tokens over 8192 keys
// take 387.  No unit bounds it (vector instructions 42 % of the time, matrix 31 %, LDS 37 %; waits 37 % of the waves' time): without its exponentials, its first products, its writes to LDS or its
// loads it takes 7, 6, 6 and 12 % less.  Issuing the next tile's first product among the exponentials, with three tiles of keys in LDS, takes as long (266 to 267), and rows straight from memory without LDS 440 and more.
template <int PAGES, Keys KEYS, bool HALF, bool FOUR = false>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_tile_kernel(AttendArgs a)
{
    constexpr bool TURN = KEYS == kTurn, F16 = KEYS != kAsTheyAre && !FOUR;
    constexpr int kParts = KEYS == kAsTheyAre ? 2 : 3;   // FOUR: e4m3 numbers to an element of q
    constexpr int kLanes = 64 / kKeys, kPieces = 16 / kLanes;   // F16: lanes to a row of K, pieces to a lane
    __shared__ __align__(16) uint64_t turns[kBands];
    // (two objects and two copies of the loop's body: the compiler then knows that reading one does not have to wait for the loads into the other)
    __shared__ __align__(16) TileBuffer buf0, buf1;
    __shared__ int32_t wave_last[kWaves], wave_end[kWaves];
    const CacheView &c = a.src.cache;
    const int H = c.n_kv_heads, G = a.group_size, Hq = H * G;
    // Row tiles of the same keys run next to each other on one XCD (workgroups go to the eight in turn), where the keys stay in its L2.
    const uint32_t x = blockIdx.x & 7, y = blockIdx.x >> 3;
    const int rt0 = a.row_tiles - 1 - y % a.row_tiles;   // (a prompt's last rows have the most keys: they begin first)
    const Unit unit_here = unit_of(a.src, (y / a.row_tiles) * 8 + x);
    const int split = unit_here.split, head = unit_here.h, s = unit_here.s;
    if (split >= a.src.n_split) return;
    const TokenRange tr = tokens_of(a, a.src, s);
    const int rows = tr.n * G, r0 = rt0 * kRows;
    if (r0 >= rows) return;
    const KeyRange range = keys_of_split(a, a.src, s, head, split);
    if (range.lo >= range.hi && a.part_o) {
        no_keys(a, a.src, split, tr.t0, r0, min(rows - r0, kRows), head, Hq);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const int k_lo = __builtin_amdgcn_readfirstlane(range.lo);
    int k_hi = __builtin_amdgcn_readfirstlane(range.hi);
    const int64_t base = (int64_t)a.layer * c.stride_layer + (int64_t)head * c.stride_head;
    const int64_t pbase = (int64_t)a.layer * c.pos_stride_layer + (int64_t)head * c.pos_stride_head;
    const uint32_t sb = FOUR ? (uint32_t)c.stride_slot / 2u : (uint32_t)c.stride_slot * 2u;
    // Lane offsets, as the part that the others follow from by exclusive or: the compiler would keep all of them in registers that it does not have (fresh() hides that
    // they stay the same from tile to tile).  Pieces of 16 bytes lie in LDS at their number exclusive-or the row (K) or twice the row (V), so that eight lanes of a 16-byte
    // read of neighbouring rows, and sixteen of a transposing 8-byte read of four rows, meet different banks.
    const uint32_t row4 = lane >> 4;
    const uint32_t piece_k = ((lane & 15) ^ row4) * 16, piece_v = ((lane & 15) ^ (2 * row4)) * 16, from_row = row4 * sb;
    const int in_block = PAGES ? (1 << c.block_shift) - 1 : 0;
    auto is_block = [&](int b) { return (b >= 0) & ((a.src.n_blocks == 0) | (b < a.src.n_blocks)); };
    // the block of key k0, or (PAGES 2: below sixteen slots) of the lane's key of the sixteen from k0 on
    auto block_at = [&](int k0) {
        if (PAGES == 2) k0 += lane_again() & 15;
        return PAGES ? c.block_table[(int64_t)s * c.max_blocks + (min(k0, max(k_hi - 1, 0)) >> c.block_shift)] : 0;
    };
    int32_t pos_new = 0;
    uint32_t there_new = 0;
    uint4 k_new, v_new;              // FOUR: elements 32 (lane & 3) and on of the wave's key lane / 4, and its words of scales
    uint32_t k_scale_new = 0, v_scale_new = 0;
    auto load4 = [&](int k0, int block_loaded) __attribute__((always_inline)) {
        int n = __builtin_amdgcn_readfirstlane(min(max(k_hi - k0, 0), kKeys));
        const uint32_t l = lane_again(), row = l >> 2;
        if (PAGES == 2) {   // keys that are not there bring the pool's first row, with scales of zero
            const bool mine = ((int)(l & 15) < n) & is_block(block_loaded);
            there_new = (uint32_t)__ballot(mine) & 0xffffu;
            const bool there = (there_new >> row) & 1;
            const int b = __shfl(block_loaded, (int)row), in = (k0 + row) & in_block;
            const int64_t at = (there ? base + (int64_t)b * c.stride_sb + slot_offset(c, in) : base) / 2 + 16 * (l & 3);
            k_new = *reinterpret_cast<const uint4 *>((const char *)c.k + at);
            v_new = *reinterpret_cast<const uint4 *>((const char *)c.v + at);
            const int64_t word = pbase + (there ? (int64_t)b * c.pos_stride_sb + in : 0);
            k_scale_new = there ? a.k_scale[word] : 0;
            v_scale_new = there ? a.v_scale[word] : 0;
            pos_new = a.causal ? c.pos[pbase + (mine ? (int64_t)block_loaded * c.pos_stride_sb + ((k0 + (l & 15)) & in_block) : 0)] : 0;
            return;
        }
        int64_t kv, at;
        if (PAGES == 1) {
            const int block = __builtin_amdgcn_readfirstlane(block_loaded);
            const int in = k0 & in_block;
            if (!is_block(block)) n = 0;
            const int b = n ? block : 0;
            kv = base + (int64_t)b * c.stride_sb + (int64_t)in * c.stride_slot;
            at = pbase + (int64_t)b * c.pos_stride_sb + in;
        } else {
            kv = base + (int64_t)s * c.stride_sb + (int64_t)k0 * c.stride_slot;
            at = pbase + (int64_t)s * c.pos_stride_sb + k0;
        }
        there_new = (1u << n) - 1;
        const uint32_t bytes = __builtin_amdgcn_readfirstlane(n > 0 ? (n - 1) * sb + kHeadDim / 2 : 0), words = __builtin_amdgcn_readfirstlane(n * 4);   // (lanes beyond bring zeros)
        const auto rsrc = [&](const void *p, int64_t offset, uint32_t size) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((const char *)p) + offset, 0, size, 0x00027000); };
        const uint32_t from = row * sb + 16 * (l & 3);
        k_new = as_uint4(__builtin_amdgcn_raw_buffer_load_b128(rsrc(c.k, kv / 2, bytes), from, 0, 0));
        k_scale_new = __builtin_amdgcn_raw_buffer_load_b32(rsrc(a.k_scale, at * 4, words), row * 4, 0, 0);
        v_new = as_uint4(__builtin_amdgcn_raw_buffer_load_b128(rsrc(c.v, kv / 2, bytes), from, 0, 0));
        v_scale_new = __builtin_amdgcn_raw_buffer_load_b32(rsrc(a.v_scale, at * 4, words), row * 4, 0, 0);
        pos_new = __builtin_amdgcn_raw_buffer_load_b32(rsrc(c.pos, at * 4, a.causal ? words : 0), (l % kKeys) * 4, 0, 0);
    };
    auto load = [&](TileBuffer &to, int k0, int block_loaded) __attribute__((always_inline)) {   // k0: this wave's first key
        if constexpr (FOUR) return load4(k0, block_loaded);
        int n = __builtin_amdgcn_readfirstlane(min(max(k_hi - k0, 0), kKeys));
        if (PAGES == 2) {   // every row has an address of its own; keys that are not there bring the pool's first row, which put() clears
            const uint32_t l = lane_again();
            const bool mine = ((int)(l & 15) < n) & is_block(block_loaded);
            there_new = (uint32_t)__ballot(mine) & 0xffffu;
#pragma unroll
            for (int i = 0; i < kKeys / 4; ++i) {
                const int row = 4 * i + (l >> 4), b = __shfl(block_loaded, row);
                const int64_t at = ((there_new >> row) & 1 ? base + (int64_t)b * c.stride_sb + slot_offset(c, (k0 + row) & in_block) : base) * 2;
                typedef const __attribute__((address_space(1))) void global_void;
                __builtin_amdgcn_global_load_lds((global_void *)((const char *)c.k + at + ((l & 15) ^ row) * 16), (lds_void *)(to.k + (kKeys * wave + 4 * i) * kHeadDim), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((global_void *)((const char *)c.v + at + ((l & 15) ^ (2 * (row & 7))) * 16), (lds_void *)(to.v + (kKeys * wave + 4 * i) * kHeadDim), 16, 0, 0);
            }
            pos_new = a.causal || TURN ? c.pos[pbase + (mine ? (int64_t)block_loaded * c.pos_stride_sb + ((k0 + (l & 15)) & in_block) : 0)] : 0;
            return;
        }
        int64_t kv, at;
        if (PAGES == 1) {
            const int block = __builtin_amdgcn_readfirstlane(block_loaded);   // (here and not where it is asked for: that is a tile ago)
            const int in = k0 & in_block;
            if (!is_block(block)) n = 0;
            const int b = n ? block : 0;
            kv = base + (int64_t)b * c.stride_sb + (int64_t)in * c.stride_slot;
            at = pbase + (int64_t)b * c.pos_stride_sb + in;
        } else {
            kv = base + (int64_t)s * c.stride_sb + (int64_t)k0 * c.stride_slot;
            at = pbase + (int64_t)s * c.pos_stride_sb + k0;
        }
        there_new = (1u << n) - 1;
        const uint32_t bytes = __builtin_amdgcn_readfirstlane(n > 0 ? (n - 1) * sb + kHeadDim * 2 : 0);   // (lanes beyond it bring zeros)
        const auto kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((const char *)c.k) + kv * 2, 0, bytes, 0x00027000);
        const auto vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((const char *)c.v) + kv * 2, 0, bytes, 0x00027000);
        uint32_t row = from_row, pk = piece_k, pv = piece_v;
        fresh(row), fresh(pk), fresh(pv);
        const auto pr = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t *>(c.pos) + at, 0, __builtin_amdgcn_readfirstlane(a.causal || TURN ? n * 4 : 0), 0x00027000);
#pragma unroll
        for (int i = 0; i < kKeys / 4; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void *)(to.k + (kKeys * wave + 4 * i) * kHeadDim), 16, row + 4 * i * sb + (pk ^ (64 * i)), 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kKeys / 4; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void *)(to.v + (kKeys * wave + 4 * i) * kHeadDim), 16, row + 4 * i * sb + (pv ^ (128 * (i & 1))), 0, 0, 0);
        pos_new = __builtin_amdgcn_raw_buffer_load_b32(pr, (lane % kKeys) * 4, 0, 0);
    };
    // What the loads have brought, when it has come: the wave's own keys are turned where they lie, their positions written down.
    auto put = [&](TileBuffer &to) __attribute__((always_inline)) {
        bool scaled = false;
        if constexpr (FOUR) {
            // (pieces of 16 bytes lie at their number exclusive-or a quarter of the row, so that reads of one piece of sixteen neighbouring rows meet different banks)
            const uint32_t l = lane_again(), row = l >> 2, g = l & 3;
            uint4 *k = reinterpret_cast<uint4 *>(to.k) + (kKeys * wave + row) * 4, *v = reinterpret_cast<uint4 *>(to.v + (kKeys * wave + row) * kHeadDim);
            const uint32_t vw[4] = {v_new.x, v_new.y, v_new.z, v_new.w};
            k[g ^ ((row >> 2) & 3)] = k_new;
            if (g == 0) to.unit[kKeys * wave + row] = __uint_as_float(k_scale_new);
            const float scale = scale_at(v_scale_new, g);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[(4 * g + j) ^ (2 * (row & 7))] = read8(vw[j], scale);
        } else {
        if (PAGES == 2 && there_new != 0xffffu) {
            __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): the rows have come
            const uint32_t l = lane_again();
            if (!((there_new >> (l >> 2)) & 1)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(to.v + (kKeys * wave + (l >> 2)) * kHeadDim + 8 * ((l & 3) + 4 * i)) = make_uint4(0, 0, 0, 0);
            }
        }
        if (F16) {
            __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
            const int row = lane / kLanes;
            bf16x8 *k = reinterpret_cast<bf16x8 *>(to.k + (kKeys * wave + row) * kHeadDim);
            float v[kPieces][8];
#pragma unroll
            for (int i = 0; i < kPieces; ++i) widen8(__builtin_bit_cast(uint4, k[(lane % kLanes + kLanes * i) ^ row]), v[i]);
            if (TURN) {
                const int turn_pos = __shfl(pos_new, row);
#pragma unroll
                for (int i = 0; i < (HALF ? kPieces / 2 : kPieces); ++i)
#pragma unroll
                    for (int e = 0; e < (HALF ? 8 : 4); ++e) {
                        const int piece = lane % kLanes + kLanes * i;
                        const uint64_t t = turns[HALF ? 8 * piece + e : 4 * piece + e];
                        float cs, sn;
                        turn_fast(phase_of(turn_pos, (uint32_t)t, (uint32_t)(t >> 32)), &cs, &sn);
                        float &r = HALF ? v[i][e] : v[i][2 * e], &im = HALF ? v[(i + kPieces / 2) % kPieces][e] : v[i][(2 * e + 1) & 7];
                        const float re = r, im0 = im;
                        r = fmaf(re, cs, -(im0 * sn));
                        im = fmaf(re, sn, im0 * cs);
                    }
            }
            float most = 0.f, unit = 1.f;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[i][e]));
#pragma unroll
            for (int i = 1; i < kLanes; i *= 2) most = fmaxf(most, __shfl_xor(most, i));
            // fp16 as it is from 2^-6 (below 2^-14 of it bits are lost, 2^-19 of the row's largest at most) to 2^15
            scaled = __ballot(most >= 0x1p15f || (most < 0x1p-6f && most > 0.f));
            if (scaled) unit = unit_of(most);
            const float by = over(unit);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) k[(lane % kLanes + kLanes * i) ^ row] = narrow_f16(v[i], by);
            if (lane % kLanes == 0) to.unit[kKeys * wave + row] = unit;
        }
        }
        const bool there = (there_new >> (lane % kKeys)) & 1;   // (lanes kKeys apart hold the same)
        int32_t hi = there ? pos_new : -0x7fffffff - 1, lo = there ? pos_new : 0x7fffffff;
#pragma unroll
        for (int i = 1; i < kKeys; i *= 2) hi = max(hi, __shfl_xor(hi, i)), lo = min(lo, __shfl_xor(lo, i));
        if (lane < kKeys) to.pos[kKeys * wave + lane] = pos_new;
        if (lane == 0) to.lim[wave] = hi, to.lim[kWaves + wave] = lo, to.lim[2 * kWaves + wave] = there_new | (uint32_t)scaled << 16;
    };

    // The first tile is asked for before anything is known of the queries.
    int k0 = k_lo, ahead = block_at(k_lo + kKeys * wave);
    if (k0 < k_hi) {
        load(buf0, k0 + kKeys * wave, ahead);
        ahead = block_at(k0 + kTileKeys + kKeys * wave);
    }
    if (tid < kBands) turns[tid] = a.turns.w[tid];
    __syncthreads();

    // this lane's row: column `col` of S^T and O^T
    const int at = r0 + 32 * wave + col, r = min(at, rows - 1), t = tr.t0 + r / G, hq = head * G + r % G;
    const bool real = at < rows;
    const int32_t t_pos = a.causal ? a.pos[t] : 0x7fffffff;
    int32_t first_pos = t_pos, last_pos = real ? t_pos : -0x7fffffff - 1;
    bf16x8 q[8];
    i32x8 q8[FOUR ? kParts : 1][2];   // FOUR: the first and the last 64 dimensions, each 16 h to 16 h + 15 and those 32 further on
    uint32_t q_scale = 0;             // FOUR: a byte for every part
    float unit = 1.f;   // of the row's q
    if constexpr (FOUR) {
        const char *p = a.q + ((int64_t)t * a.q_stride_token + (int64_t)hq * a.q_stride_head) * 2 + 32 * h;
        float x[2][32], most = 0.f;   // x[i]: of the i-th 64 dimensions
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) widen8(*reinterpret_cast<const uint4 *>(p + 128 * i + 64 * (j / 2) + 16 * (j % 2)), x[i] + 8 * j);
        if constexpr (KEYS != kAsTheyAre) {
            const int32_t turn_pos = a.pos[t];
            const auto turn = [&](int f, float &re, float &im) {
                const uint64_t w = turns[f];
                float cs, sn;
                turn_fast(phase_of(turn_pos, (uint32_t)w, (uint32_t)(w >> 32)), &cs, &sn);
                const float x0 = re, y0 = im;
                re = fmaf(x0, cs, -(y0 * sn));
                im = fmaf(x0, sn, y0 * cs);
            };
            if (a.half) {
#pragma unroll
                for (int e = 0; e < 32; ++e) turn(32 * (e / 16) + 16 * h + e % 16, x[0][e], x[1][e]);
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) turn(32 * i + 16 * (e / 8) + 8 * h + e % 8, x[i][2 * e], x[i][2 * e + 1]);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 32; ++e) most = fmaxf(most, fabsf(x[i][e]));
        most = fmaxf(most, __shfl_xor(most, 32));
        // the first part of the row's largest is in [128, 256); a part's scale is 2^-4 of the last one's
        const int power = max((int)(__float_as_uint(most) >> 23), 127 - 99);
        const float by = __uint_as_float((uint32_t)(261 - power) << 23);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 32; ++e) x[i][e] *= by;
#pragma unroll
        for (int n = 0; n < kParts; ++n) {
            q_scale |= (uint32_t)(power - 7 - 4 * n) << (8 * n);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float *y = x[i] + 4 * j;
                    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
                    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
                    q8[n][i][j] = w;
                    y[0] = (y[0] - __builtin_amdgcn_cvt_f32_fp8(w, 0)) * 16.f;
                    y[1] = (y[1] - __builtin_amdgcn_cvt_f32_fp8(w, 1)) * 16.f;
                    y[2] = (y[2] - __builtin_amdgcn_cvt_f32_fp8(w, 2)) * 16.f;
                    y[3] = (y[3] - __builtin_amdgcn_cvt_f32_fp8(w, 3)) * 16.f;
                }
        }
    } else {
        const char *p = a.q + ((int64_t)t * a.q_stride_token + (int64_t)hq * a.q_stride_head) * 2 + 16 * h;
        if (F16) {
            float v[8][8], most = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) widen8(*reinterpret_cast<const uint4 *>(p + 32 * j), v[j]);
            if (a.rotate_q) {
                if (TURN ? HALF : (bool)a.half) rotate_q<true>(v, a.pos[t], h, turns);
                else rotate_q<false>(v, a.pos[t], h, turns);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[j][e]));
            unit = unit_of(fmaxf(most, __shfl_xor(most, 32)));
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = narrow_f16(v[j], over(unit));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = *reinterpret_cast<const bf16x8 *>(p + 32 * j);
        }
    }
#pragma unroll
    for (int i = 1; i < 32; i *= 2) first_pos = min(first_pos, __shfl_xor(first_pos, i)), last_pos = max(last_pos, __shfl_xor(last_pos, i));
    first_pos = __builtin_amdgcn_readfirstlane(first_pos);
    last_pos = __builtin_amdgcn_readfirstlane(last_pos);
    const bool idle = r0 + 32 * wave >= rows;
    // Keys at the end of the range that lie behind all rows' positions (the later part of a chunk's own tokens) are not loaded: the range ends with its last key that a row attends to, looked
    // for from the end, 1024 keys at a time, where the tokens behind these rows are one in 32 of the keys at least (it takes 3 us before the first tile).  A prompt of 8192 tokens over itself: 607 us, 815
    // without; chunks of 1024 tokens over 8192 keys, the longest rows of which have nothing to leave out, are equal.
    const int later = tr.n - min(tr.n, (r0 + kRows) / G);
    if (a.causal && a.src.scan && k_lo < k_hi && later >= (k_hi - k_lo) / 32 && later > 0) {
        if (lane == 0) wave_last[wave] = last_pos;
        __syncthreads();
        int32_t last = wave_last[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) last = max(last, wave_last[i]);
        int end = k_lo;
        for (int hi = k_hi; hi > k_lo && end == k_lo; hi -= 1024) {
            int mine = k_lo;   // behind the last attended key that this lane sees
            int32_t p[4];
            bool on[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = hi - 1 - tid - 256 * i, at = max(key, k_lo);
                const int b = PAGES ? block_of(c, a.src.n_blocks, s, at) : s;
                on[i] = (key >= k_lo) & (b >= 0);
                p[i] = c.pos[pbase + (int64_t)max(b, 0) * c.pos_stride_sb + (PAGES ? at & in_block : at)];
            }
#pragma unroll
            for (int i = 3; i >= 0; --i)
                if (on[i] & (p[i] <= last)) mine = hi - tid - 256 * i;
#pragma unroll
            for (int i = 1; i < 64; i *= 2) mine = max(mine, __shfl_xor(mine, i));
            if (lane == 0) wave_end[wave] = mine;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kWaves; ++i) end = max(end, wave_end[i]);
            __syncthreads();
        }
        k_hi = __builtin_amdgcn_readfirstlane(end);
    }

    f32x16 o[4];
    float top = kNoScore, sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
    // the lane's operands in a tile: dimension group j of its K row at at_k ^ 32 j; of the V rows of a step, dimensions 32 j + col at at_v ^ 64 j
    const uint32_t row_v0 = 4 * h + ((lane & 15) >> 2);
    const uint32_t at_k = col * 256 + (h ^ (col & 15)) * 16;
    const uint32_t at_v = row_v0 * 256 + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (2 * row_v0)) * 16) + (lane & 1) * 8;

    // mask: some of the tile's keys are not everyone's; scaled: some have units
    auto compute = [&](const TileBuffer &from, const bool mask, const bool scaled) __attribute__((always_inline)) {
        uint32_t ak = at_k, av = at_v;
        fresh(ak), fresh(av);
        f32x16 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
        bf16x8 k[FOUR ? 1 : 2][8], v[2][4];   // v[u][j]: dimensions 32 j + col, the keys of weight[u]
        auto values = [&](int U) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t at = av ^ (64 * j);
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((const char *)from.v + at + (32 * 256 * U + 16 * 256 * u)));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((const char *)from.v + at + (32 * 256 * U + 16 * 256 * u + 8 * 256)));
                    v[u][j] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
        };
        if constexpr (FOUR) {
            uint4 k4[2][2];   // [u][i]: the i-th 64 dimensions
            uint32_t k_scale[2];
            const uint32_t row = lane_again() & 31, half = lane_again() >> 5;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int i = 0; i < 2; ++i) k4[u][i] = reinterpret_cast<const uint4 *>(from.k)[(32 * u + row) * 4 + ((2 * i + half) ^ ((row >> 2) & 3))];
                k_scale[u] = __float_as_uint(from.unit[32 * u + row]) >> (8 * half);   // bytes 0 and 2
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const i32x8 x{(int)k4[u][i].x, (int)k4[u][i].y, (int)k4[u][i].z, (int)k4[u][i].w, 0, 0, 0, 0};
                    const auto product = [&](auto part) {
                        constexpr int n = decltype(part)::value;
                        if constexpr (n < kParts) {
                            if (i == 0) sc[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, q8[n][0], sc[u], 4, 0, 0, k_scale[u], n, q_scale);
                            else sc[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, q8[n][1], sc[u], 4, 0, 2, k_scale[u], n, q_scale);
                        }
                    };
                    product(std::integral_constant<int, 2>()), product(std::integral_constant<int, 1>()), product(std::integral_constant<int, 0>());
                }
                if (u == 0) {
                    values(0);   // asked for ahead of the softmax
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_s_setprio(0);
        } else {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) k[u][j] = *reinterpret_cast<const bf16x8 *>((const char *)from.k + (ak ^ (32 * j)) + 32 * 256 * u);
        __builtin_amdgcn_sched_barrier(0);   // all reads under way before the first product waits for one
        __builtin_amdgcn_s_setprio(1);   // (the products of a wave go before the other's softmax: 263 -> 258 us for two chunks of 1024 tokens over 8192 keys)
#pragma unroll
        for (int j = 0; j < 8; ++j) sc[0] = scores<F16>(k[0][j], q[j], sc[0]);
        values(0);   // asked for ahead of the softmax
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 8; ++j) sc[1] = scores<F16>(k[1][j], q[j], sc[1]);
        __builtin_amdgcn_s_setprio(0);
        }
        if (F16 && scaled) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[u][i] *= from.unit[32 * u + 8 * (i / 4) + 4 * h + i % 4];
        }
        const float scale = F16 ? a.scale_log2 * unit : a.scale_log2;
        uint32_t keep = ~0u;   // bit 16 u + i: key 32 u + 8 (i / 4) + 4 h + i % 4 is attended to
        bool hole = false;
        if (mask) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int first = 32 * u + 8 * g + 4 * h;
                    const uint32_t there = (uint32_t)from.lim[2 * kWaves + first / kKeys] >> (first % kKeys);
                    const int4 p4 = *reinterpret_cast<const int4 *>(&from.pos[first]);
                    const int32_t p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const int i = 4 * g + d;
                        const bool on = ((there >> d) & 1) & (p[d] <= t_pos);   // (not causal: t_pos is the highest there is)
                        keep &= on ? ~0u : ~(1u << (16 * u + i));
                        sc[u][i] = on ? sc[u][i] : kNoScore;
                        hole |= ((there >> d) & 1) & !on & real;
                    }
                }
        }
        float best = kNoScore;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) best = fmaxf(best, sc[u][i]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(best), __float_as_uint(best), false, false);
        best = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
        // weights are relative to a maximum that scores may pass by a factor of 2^8 before the sums are brought to the new one
        if (__ballot(best > top && !((best - top) * scale <= kStaleBits))) {
            const float next = fmaxf(top, best);
            const float shrink = next == kNoScore ? 1.f : __builtin_amdgcn_exp2f((top - next) * scale);
            top = next;
            sum *= shrink;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] *= shrink;
        }
        const float off = (top == kNoScore ? 0.f : top) * scale;
        const bool holes = __ballot(hole);
#pragma unroll
        for (int U = 0; U < 2; ++U) {
            bf16x8 weight[2];
            if (U == 1) values(1);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float p = __builtin_amdgcn_exp2f(fmaf(sc[U][i], scale, -off));
                sum += p;
                weight[i / 8][i % 8] = (__bf16)p;
            }
            if (holes) {   // (see attend_general_kernel: values that are not finite and not everyone's)
                bool odd = false;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) odd |= not_finite(__builtin_bit_cast(uint4, v[u][j]));
                if (__ballot(odd)) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
#pragma unroll
                        for (int side = 0; side < 2; ++side) {
                            f32x16 some;
#pragma unroll
                            for (int i = 0; i < 16; ++i) some[i] = 0.f;
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                bf16x8 on;
#pragma unroll
                                for (int d = 0; d < 8; ++d) on[d] = (keep >> (16 * U + 8 * u + d)) & 1 ? (__bf16)1.f : (__bf16)0.f;
                                some = __builtin_amdgcn_mfma_f32_32x32x16_bf16(where_not_below(v[u][j], side ? 0xff80 : 0x7f80), on, some, 0, 0, 0);
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[j][i] += some[i] > 0.f ? (side ? -__builtin_inff() : __builtin_inff()) : 0.f;
                            __builtin_amdgcn_sched_barrier(0);   // (one after the other: few registers, and time does not matter here)
                        }
#pragma unroll
                        for (int u = 0; u < 2; ++u) v[u][j] = __builtin_bit_cast(bf16x8, finite_only(__builtin_bit_cast(uint4, v[u][j])));
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[u][j], weight[u], o[j], 0, 0, 0);
        }
    };

    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): no load into LDS is under way when the workgroup ends without a tile
    if (k0 < k_hi) put(buf0);
    auto step = [&](TileBuffer &here, TileBuffer &next) __attribute__((always_inline)) {
        // This tile has come, what put() wrote of it is there, and the last one is read.  Both waits are said here.  A barrier does not wait for loads into LDS; and the wait for the wave's own LDS writes, which
        // the compiler sets ahead of barriers, it left out of this one on the way round the loop: other waves then met limits and positions of the tile before the last, or keys half turned.
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
        __syncthreads();
        const bool more = k0 + kTileKeys < k_hi;
        if (more) {
            load(next, k0 + kTileKeys + kKeys * wave, ahead);
            ahead = block_at(k0 + 2 * kTileKeys + kKeys * wave);
        }
        if (!idle) {
            const int32_t lim = here.lim[min(lane, 3 * kWaves - 1)];
            int32_t hi = -0x7fffffff - 1, lo = 0x7fffffff, any = 0, all = 0xffff;
#pragma unroll
            for (int i = 0; i < kWaves; ++i)
                hi = max(hi, __builtin_amdgcn_readlane(lim, i)), lo = min(lo, __builtin_amdgcn_readlane(lim, kWaves + i)), any |= __builtin_amdgcn_readlane(lim, 2 * kWaves + i), all &= __builtin_amdgcn_readlane(lim, 2 * kWaves + i);
            // (nothing to do where no key is there, or all are behind the last position of the wave's rows)
            if ((any & 0xffff) && lo <= last_pos) compute(here, all != 0xffff || hi > first_pos, any >> 16);
        }
        if (more) put(next);
        k0 += kTileKeys;
        return more;
    };
    if (k0 < k_hi)
        while (step(buf0, buf1) && step(buf1, buf0)) {
        }
    const float total = sum + __shfl_xor(sum, 32);
    if (!real) return;
    if (a.part_o) {
        const int64_t row = ((int64_t)(a.src.part0 + split) * a.n_tokens + t) * Hq + hq;
        if (h == 0) a.part_ml[row] = make_float2(top * unit, total);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4 *>(a.part_o + row * kHeadDim + 32 * j + 2 * i + 4 * h) = f32x4{o[j][i], o[j][i + 1], o[j][i + 2], o[j][i + 3]};
        return;
    }
    const float inv = 1.f / total;
    __bf16 *p = reinterpret_cast<__bf16 *>(a.out) + (int64_t)t * a.out_stride_token + (int64_t)hq * a.out_stride_head;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
            bf16x4 b;
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = (__bf16)(total != 0.f ? o[j][i + e] * inv : 0.f);
            *reinterpret_cast<bf16x4 *>(p + 32 * j + 2 * i + 4 * h) = b;
        }
}

}  // namespace

tri_status launch_attend_tile(const AttendArgs &a, int64_t groups, hipStream_t st)
{
    const uint32_t blocks = (uint32_t)groups;
    const int shift = a.src.cache.block_shift, pages = shift < 0 ? 0 : shift >= 4 ? 1 : 2;
    const auto launch = [&](auto kernel) { kernel<<<blocks, 64 * kWaves, 0, st>>>(a); };
    const auto of = [&](auto direct, auto paged, auto small) { pages == 0 ? launch(direct) : pages == 1 ? launch(paged) : launch(small); };
    if (!a.src.cache.k_rotated && a.half) of(attend_tile_kernel<0, kTurn, true>, attend_tile_kernel<1, kTurn, true>, attend_tile_kernel<2, kTurn, true>);
    else if (!a.src.cache.k_rotated) of(attend_tile_kernel<0, kTurn, false>, attend_tile_kernel<1, kTurn, false>, attend_tile_kernel<2, kTurn, false>);
    else if (a.rotate_q) of(attend_tile_kernel<0, kWiden, false>, attend_tile_kernel<1, kWiden, false>, attend_tile_kernel<2, kWiden, false>);
    else of(attend_tile_kernel<0, kAsTheyAre, false>, attend_tile_kernel<1, kAsTheyAre, false>, attend_tile_kernel<2, kAsTheyAre, false>);
    return hip_status("attend_tile_kernel");
}

tri_status launch_attend4_tile(const AttendArgs &a, int64_t groups, hipStream_t st)
{
    const uint32_t blocks = (uint32_t)groups;
    const int shift = a.src.cache.block_shift;
    const auto launch = [&](auto kernel) { kernel<<<blocks, 64 * kWaves, 0, st>>>(a); };
    const auto of = [&](auto direct, auto paged, auto small) { shift < 0 ? launch(direct) : shift >= 4 ? launch(paged) : launch(small); };
    if (a.rotate_q) of(attend_tile_kernel<0, kWiden, false, true>, attend_tile_kernel<1, kWiden, false, true>, attend_tile_kernel<2, kWiden, false, true>);
    else of(attend_tile_kernel<0, kAsTheyAre, false, true>, attend_tile_kernel<1, kAsTheyAre, false, true>, attend_tile_kernel<2, kAsTheyAre, false, true>);
    return hip_status("attend_tile_kernel");
}

}  // namespace tri
