// Appending a step's keys, values and positions to a cache, the rotation by position on the way (tri_append).
#include <algorithm>
#include <cmath>

#include "tri_serve.h"

namespace tri {

BandTurns band_turns(double theta)
{
    // theta^(-f/64), as fractions of 2^64, by products of two earlier ones (64 calls of powl take 17 us, longer than the kernels of a small step; the products in long
    // double 0.6 us or, where the linker had put the code elsewhere, 3.4; so 0.4).  The root is off by 2^-64 of itself and enters f times, as does a product's rounding: 2 f 2^-64 theta^(-f/64), at most 11 * 2^-64 for theta of 100
    // and more, of which w has 1 / 2 pi.
    const auto times = [](uint64_t x, uint64_t y) { return (uint64_t)(((unsigned __int128)x * y + ((uint64_t)1 << 63)) >> 64); };
    const uint64_t turn = (uint64_t)(18446744073709551616.0L / 6.283185307179586476925286766559L + 0.5L);   // 2^64 / 2 pi
    uint64_t power[kBands];
    power[1] = (uint64_t)(powl((long double)theta, -2.0L / kHeadDim) * 18446744073709551616.0L);   // (below 2^64: theta is above 1)
    for (int f = 2; f < kBands; ++f) power[f] = times(power[f / 2], power[f - f / 2]);
    BandTurns t;
    t.w[0] = turn;
    for (int f = 1; f < kBands; ++f) t.w[f] = times(power[f], turn);
    return t;
}

namespace {

constexpr int kAppendThreads = 256;

template <typename T>
struct Piece;   // 16 bytes of a row as floats
template <>
struct Piece<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void get(const uint4 &u, float *x)
    {
        x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 put(const float *x)
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    static __device__ __forceinline__ void turn(uint32_t phase, float *c, float *s) { turn_exact(phase, c, s); }
};
template <>
struct Piece<__bf16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void get(const uint4 &u, float *x)
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    static __device__ __forceinline__ uint4 put(const float *x)
    {
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        bf16x8 b;
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = (__bf16)x[i];
        return __builtin_bit_cast(uint4, b);
    }
    static __device__ __forceinline__ void turn(uint32_t phase, float *c, float *s) { turn_fast(phase, c, s); }
};

// A thread takes two 16-byte pieces of one K row and of its V row, half a row apart: both parts of its bands lie in them in either
// pair layout.  Pure streaming: a row is read and written once; the rotation (a sincos per band and row) is not what bounds it.
// A wave covers 8 (bf16) or 4 (fp32) neighbouring rows; the sequence of its first token is found by all lanes at once (the number of
// starts at or below it), the others' by going on from there.  The rows are asked for before that (four prompts' 19972 tokens, 8 KV heads, 164 MB read and written: 37 us with the
// loads behind the search, 28.5 with the rows in the caches).  Stores are non-temporal: from memory to memory that call takes 31 us (5.3 TB/s), 39 with plain ones, 34 with non-temporal
// loads, whatever the stores.  A single token's launch takes 3.1 us, 256 sequences' 4.9.
template <typename T>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a)
{
    constexpr int kElems = Piece<T>::n, kPieces = 64 / kElems;   // threads per row
    const CacheView &c = a.cache;
    const int S = c.n_seqs, H = c.n_kv_heads;
    const int64_t i = (int64_t)blockIdx.x * kAppendThreads + threadIdx.x;
    if (a.new_seq_len && i < S) {
        const int s = (int)i;
        const int n = clamp_len(a.head_len ? a.head_len[((int64_t)a.layer * S + s) * H] : c.seq_len[s], c.max_seq_len);
        int got = 1;
        if (a.start) got = max(clamp_to(a.start[s + 1], a.n_tokens) - clamp_to(a.start[s], a.n_tokens), 0);
        a.new_seq_len[s] = (int)min((int64_t)n + got, (int64_t)c.max_seq_len);
    }
    const int64_t row = i / kPieces;
    const int part = (int)(i % kPieces);
    const int t_first = (int)(((int64_t)blockIdx.x * kAppendThreads + (threadIdx.x & ~63)) / kPieces / H);
    if (t_first >= a.n_tokens) return;   // (the whole wave)
    const int t = (int)(row / H), h = (int)(row - (int64_t)t * H);
    // the rows are asked for before their place is known
    const int64_t from = ((int64_t)min(t, a.n_tokens - 1) * a.stride_token + (int64_t)h * a.stride_head + part * kElems) * (int64_t)sizeof(T);
    constexpr int64_t half_row = 64 * sizeof(T);
    uint4 k0 = *reinterpret_cast<const uint4 *>(a.k_new + from), k1 = *reinterpret_cast<const uint4 *>(a.k_new + from + half_row);
    const uint4 v0 = *reinterpret_cast<const uint4 *>(a.v_new + from), v1 = *reinterpret_cast<const uint4 *>(a.v_new + from + half_row);
    const int32_t pos = a.pos[min(t, a.n_tokens - 1)];
    int s = t, first = t;
    if (a.start) {
        s = 0;
        for (int j = 0; j < S; j += 64) {
            const int e = j + (int)(threadIdx.x & 63);
            s += __popcll(__ballot(e < S && a.start[min(e, S - 1) + 1] <= t_first));
        }
        while (s < S && a.start[s + 1] <= t) ++s;
        if (s >= S || t >= a.n_tokens) return;
        first = a.start[s];
        if (t < first) return;
    }
    if (t >= a.n_tokens || s >= S) return;
    const int len = clamp_len(a.head_len ? a.head_len[((int64_t)a.layer * S + s) * H + h] : c.seq_len[s], c.max_seq_len);
    const int64_t slot = (int64_t)len + (t - first);
    if (slot >= c.max_seq_len) return;
    int n = (int)slot;
    int64_t block = s;
    if (c.block_shift >= 0) {
        block = block_of(c, a.n_blocks, s, n);
        if (block < 0) return;
        n &= (1 << c.block_shift) - 1;
    }
    const int64_t to = ((int64_t)a.layer * c.stride_layer + (int64_t)h * c.stride_head + block * c.stride_sb + slot_offset(c, n) + part * kElems) *
                       (int64_t)sizeof(T);
    if (a.rotate) {
        float x[kElems], y[kElems];
        Piece<T>::get(k0, x);
        Piece<T>::get(k1, y);
        if (a.half) {   // bands part * kElems + e: real parts in the first half of the row
#pragma unroll
            for (int e = 0; e < kElems; ++e) {
                const uint64_t w = a.turns.w[part * kElems + e];
                float cs, sn;
                Piece<T>::turn(phase_of(pos, (uint32_t)w, (uint32_t)(w >> 32)), &cs, &sn);
                const float re = x[e], im = y[e];
                x[e] = fmaf(re, cs, -(im * sn));
                y[e] = fmaf(re, sn, im * cs);
            }
        } else {
#pragma unroll
            for (int e = 0; e < kElems / 2; ++e) {
                const int f = part * (kElems / 2) + e;
                float cs, sn;
                Piece<T>::turn(phase_of(pos, (uint32_t)a.turns.w[f], (uint32_t)(a.turns.w[f] >> 32)), &cs, &sn);
                const float re = x[2 * e], im = x[2 * e + 1];
                x[2 * e] = fmaf(re, cs, -(im * sn));
                x[2 * e + 1] = fmaf(re, sn, im * cs);
                Piece<T>::turn(phase_of(pos, (uint32_t)a.turns.w[32 + f], (uint32_t)(a.turns.w[32 + f] >> 32)), &cs, &sn);
                const float re2 = y[2 * e], im2 = y[2 * e + 1];
                y[2 * e] = fmaf(re2, cs, -(im2 * sn));
                y[2 * e + 1] = fmaf(re2, sn, im2 * cs);
            }
        }
        k0 = Piece<T>::put(x);
        k1 = Piece<T>::put(y);
    }
    char *dk = (char *)c.k + to, *dv = (char *)c.v + to;
    store_stream16(dk, k0);
    store_stream16(dk + half_row, k1);
    store_stream16(dv, v0);
    store_stream16(dv + half_row, v1);
    if (part == 0)
        const_cast<int32_t *>(c.pos)[(int64_t)a.layer * c.pos_stride_layer + (int64_t)h * c.pos_stride_head + block * c.pos_stride_sb + n] = pos;
}

}  // namespace

int64_t append_threads(int64_t rows, int32_t dtype) { return rows * (dtype == TRI_BF16 ? 8 : 16); }

tri_status launch_append(const AppendArgs &a, int32_t dtype, hipStream_t st)
{
    const int64_t threads = std::max<int64_t>(append_threads((int64_t)a.n_tokens * a.cache.n_kv_heads, dtype), a.new_seq_len ? a.cache.n_seqs : 0);
    if (threads == 0) return TRI_OK;
    const uint32_t blocks = (uint32_t)((threads + kAppendThreads - 1) / kAppendThreads);
    if (dtype == TRI_BF16) append_kernel<__bf16><<<blocks, kAppendThreads, 0, st>>>(a);
    else append_kernel<float><<<blocks, kAppendThreads, 0, st>>>(a);
    return hip_status("append_kernel");
}

}  // namespace tri
