// Attention of many query rows over the keys of one KV head, on the matrix unit (gfx950, wave64): what the prompt and the
// tree kernels share.
//
// A wave holds 32 query rows and goes over the keys in tiles of 32.  Scores are formed transposed, S^T = K.Q^T, and so
// is the output, O^T = V^T.P^T: the 32x32 result of the matrix instruction gives lane l the column l % 32 and the rows
// 8*(i/4) + 4*(l/32) + i%4, i = 0..15.  A lane therefore holds 16 scores of ONE query, its maximum needs the other half of
// the wave only where it rises, a factor on the accumulators is a plain per-lane product, and, because the order of the keys inside a
// product is free as long as both operands agree, the scores of a lane are the second operand as they are: no lane exchange between
// the two products.  V is wanted with the keys of a lane consecutive; the transposing LDS read (four keys of
// 16 columns per 16 lanes) does that for bf16, an fp32 product takes one key per half of the wave and needs none.
//
// K and V rows go from memory to LDS without passing registers, 16 bytes a lane, tiles in turn.  A 16-byte piece p of row r lies at
// piece p ^ swizzle(r): rows are 128 to 512 bytes long, so without it the same piece of all rows would share its banks.
#pragma once

#include "l2kv_device.hpp"

namespace l2kv {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_char_t;

constexpr int kTile = 32;                    // query rows and keys of one matrix instruction
// Weights are relative to a reference that lies this far (in powers of two) above a row's largest score at the time, and that is moved when a
// score passes it: they are at most 1, as are the factors of a move, so sums of weights times values leave the range of fp32 only where those of a
// plain softmax do, and most tiles leave the accumulators alone.  bf16: 16, so that a row's largest weight is between 2^-16 and 1 (8 instead of
// 16: 1.3 % longer); weights are rounded relative to themselves, wherever they lie, the exponent's argument, of up to 32 near the top, is off by 2^-20 at
// most beside their 2^-8, and what falls below 2^-126 is below 2^-110 of the largest (at the other end, products of values below 2^-110 may be
// lost, an error below any result's use).  fp32, where the argument's bits are
// the weight's: 0, the largest score itself; products take so long there that moving the accumulators costs little (three prompts of 511 to
// 1533 tokens, 4 heads of 64: 35.9 -> 36.7 us).
template <typename E> constexpr float kHeadroom = E::kBytes == 2 ? 16.0f : 0.0f;

template <typename E, int D> struct AttnRow {
    static constexpr int kBytes = D * E::kBytes;                     // 128, 256 or 512
    static constexpr int kPieces = kBytes / 16;
    static constexpr int kQWords = D * E::kBytes / 8;                // 32-bit words a lane holds of its half of a query row
    static constexpr int kDTiles = D / kTile;
    // Where piece p of row r of a tile lies: K is read 32 rows at one piece, so 16 consecutive rows go to different pieces; V
    // (bf16) eight rows of four consecutive pieces, (fp32) rows r and r + 4 of eight consecutive pieces.
    __device__ static __forceinline__ int k_swizzle(int r) { return kPieces == 8 ? (r >> 1) & 7 : r & 15; }
    __device__ static __forceinline__ int v_swizzle(int r) {
        if constexpr (E::kBytes == 4) return kPieces == 8 ? 0 : ((r >> 2) & 1) << 3;
        else if constexpr (kPieces == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
        else return ((r & 3) << 2) | ((r >> 2) & 3);
    }
};

// 16 bytes per lane from base + offset to LDS, lane after lane from `lds` on, not waited for.  (Written out because the compiler waits for
// loads of this kind in front of every transposing read, also of the other tile; no register is written, so
// nothing but the wait below depends on when it is done.)  m0, which says where in LDS, has its old content again behind it: it is reserved, so
// that the compiler cannot be told that it changes.  The pause makes five wait states, which a vector load wants behind a vector
// instruction that wrote its scalar address (a reload of a spilled one, say) and which the compiler does not see to in here.
// kOnce: what is not read again soon passes the caches by.
template <bool kOnce> __device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t lds) {
    uint32_t m0;
    if constexpr (kOnce)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %2, %3 nt\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0) : "s"(lds), "v"(offset), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0) : "s"(lds), "v"(offset), "s"(base) : "memory");
}
// This wave's loads to LDS are done, but for the last `tiles` tiles of kLoads each (at most kMost of them stay on their way).
template <int kLoads, int kMost>
__device__ __forceinline__ void wait_loads_to_lds(int32_t tiles) {
    constexpr auto left = [](int n) { return (kWaitVmcnt0 | (n & 15) | (n >> 4) << 14); };
    static_assert(kLoads * kMost < 64, "what the counter of loads can hold");
    if (kMost >= 2 && tiles >= 2) __builtin_amdgcn_s_waitcnt(left(2 * kLoads * (kMost >= 2)));
    else if (kMost >= 1 && tiles >= 1) __builtin_amdgcn_s_waitcnt(left(kLoads * (kMost >= 1)));
    else __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    static_assert(kMost <= 2, "the cases above");
    asm volatile("" ::: "memory");
}

// Rows [k0, k0 + kRows) of a matrix of `rows` rows to LDS, by kWaves waves; rows behind the end are copies of the last.
template <typename E, int D, int kRows, int kWaves, bool kIsV, bool kOnce>
__device__ __forceinline__ void stage_rows(const char* base, int64_t k0, int64_t rows, uint32_t lds, int wave, int lane) {
    using R = AttnRow<E, D>;
    constexpr int kRowsPerChunk = 1024 / R::kBytes, kLanesPerRow = R::kPieces;
    constexpr int kChunks = kRows / kRowsPerChunk;
    static_assert(kChunks % kWaves == 0, "every wave copies as many chunks");
    const char* from = base + k0 * R::kBytes;
    const int64_t left = rows - k0;
    const int last = left < kRows ? (int)left - 1 : kRows - 1;
    if constexpr (R::kBytes == 512) asm volatile("" : "+v"(lane));       // places in the tile are worked out again every time: registers
#pragma unroll
    for (int n = 0; n < kChunks / kWaves; ++n) {
        const int chunk = n * kWaves + wave;
        const int r = chunk * kRowsPerChunk + lane / kLanesPerRow;
        const int piece = (lane % kLanesPerRow) ^ (kIsV ? R::v_swizzle(r) : R::k_swizzle(r));
        const int src = r < last ? r : last;
        load_to_lds<kOnce>(from, (uint32_t)(src * R::kBytes + piece * 16), lds + chunk * 1024);
    }
}

// Where a lane finds its operands in a tile of 32 rows.  Steps along the row flip bits of the piece, steps of whole rows are constant
// distances (both swizzles repeat after 16 rows), so a few registers and the offsets of the read instructions cover a tile.
template <typename E, int D> struct TileAddress {
    using R = AttnRow<E, D>;
    int k, v[2];
    __device__ __forceinline__ explicit TileAddress(int lane) {
        const int half = lane / kTile, row = lane % kTile;
        k = row * R::kBytes + ((half ^ R::k_swizzle(row)) << 4);
        if constexpr (E::kBytes == 2) {
            // four keys of 16 columns per 16 lanes
            const int r = 4 * half + (lane % 16) / 4, column = (lane / 16 % 2) * 16 + (lane % 4) * 4;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                v[i] = (r + 8 * i) * R::kBytes + (((column / 8) ^ R::v_swizzle(r + 8 * i)) << 4) + (column % 8) * 2;
        } else {
            v[0] = v[1] = 4 * half * R::kBytes + (((row / 4) ^ R::v_swizzle(4 * half)) << 4) + (row % 4) * 4;
        }
    }
    // What is worked out from the places from here on is not held any longer than it is used: registers.
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(k), "+v"(v[0]), "+v"(v[1])); }
    // piece 2t + half of the lane's row of a K tile
    __device__ __forceinline__ u32x4_t key(const char* tile, int t) const {
        return *reinterpret_cast<const u32x4_t*>(tile + (k ^ (t << 5)));
    }
    // bf16: keys 16t + 8i + 4 half .. + 3 at column 32d + lane % 32
    __device__ __forceinline__ u32x2_t values(const char* tile, int t, int i, int d) const {
        typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
        return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(tile + t * 16 * R::kBytes + (v[i] ^ (d << 6)))));
    }
    // fp32: key 8 * (i / 4) + 4 half + i % 4 at column 32d + lane % 32
    __device__ __forceinline__ float value(const char* tile, int i, int d) const {
        return *reinterpret_cast<const float*>(tile + (8 * (i / 4) + i % 4) * R::kBytes + (v[0] ^ (d << 7)));
    }
};

// Query rows of one tile in registers: words of the pieces 2t + half of the lane's row.
template <typename E, int D> struct QueryTile { u32x4_t piece[AttnRow<E, D>::kQWords / 4]; };

template <typename E, int D>
__device__ __forceinline__ void load_query(QueryTile<E, D>& q, const char* row, int half) {
#pragma unroll
    for (int t = 0; t < AttnRow<E, D>::kQWords / 4; ++t) q.piece[t] = *reinterpret_cast<const u32x4_t*>(row + (2 * t + half) * 16);
}

// One piece of K times one of Q^T.
template <typename E> __device__ __forceinline__ f32x16_t score_product(const u32x4_t& k, const u32x4_t& q, f32x16_t s) {
    if constexpr (E::kBytes == 2) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q), s, 0, 0, 0);
    } else {
        // one product of two columns at a time: 8t + j and 8t + 4 + j
        const f32x4_t kf = __builtin_bit_cast(f32x4_t, k), qf = __builtin_bit_cast(f32x4_t, q);
#pragma unroll
        for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j], qf[j], s, 0, 0, 0);
        return s;
    }
}

// K tile . Q^T.
template <typename E, int D>
__device__ __forceinline__ void scores(const char* tile, const TileAddress<E, D>& at, const QueryTile<E, D>& q, f32x16_t& s) {
    s = f32x16_t{};
#pragma unroll
    for (int t = 0; t < AttnRow<E, D>::kQWords / 4; ++t) {
        if (AttnRow<E, D>::kBytes == 512 && t % 4 == 0) __builtin_amdgcn_sched_barrier(0);      // few operands on their way: registers
        s = score_product<E>(at.key(tile, t), q.piece[t], s);
    }
}

template <typename E> struct Weights;          // a tile's softmax weights as second operand of O^T = V^T.P^T
template <> struct Weights<BF16> { uint32_t w[8]; };
template <> struct Weights<F32> { float w[16]; };

// o += V^T tile . P^T, for rows of 512 bytes: few operands on their way, registers.
template <typename E, int D>
__device__ __forceinline__ void weighted_values(const char* tile, const TileAddress<E, D>& at, const Weights<E>& p, f32x16_t (&o)[D / kTile]) {
    if constexpr (E::kBytes == 2) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const u32x4_t w = {p.w[4 * t], p.w[4 * t + 1], p.w[4 * t + 2], p.w[4 * t + 3]};
#pragma unroll
            for (int d = 0; d < D / kTile; ++d) {
                if (d % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                const u32x2_t a = at.values(tile, t, 0, d), b = at.values(tile, t, 1, d);
                const u32x4_t v = {a[0], a[1], b[0], b[1]};
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, w), o[d], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int d = 0; d < D / kTile; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(at.value(tile, i, d), p.w[i], o[d], 0, 0, 0);
    }
}

// The values of a tile in registers, and o += V^T tile . P^T with them: shorter rows are read while the weights are worked out, so that the
// products do not wait (a prompt of 32768 tokens 7.9 -> 7.7 ms, trees of a batch 130 -> 121 us).
template <typename E, int D> struct ValueTile { u32x4_t v[2][D / kTile]; };
template <int D> struct ValueTile<F32, D> { float v[16][D / kTile]; };
template <typename E, int D>
__device__ __forceinline__ void load_values(const char* tile, const TileAddress<E, D>& at, ValueTile<E, D>& x) {
    if constexpr (E::kBytes == 2) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int d = 0; d < D / kTile; ++d) {
                const u32x2_t a = at.values(tile, t, 0, d), b = at.values(tile, t, 1, d);
                x.v[t][d] = u32x4_t{a[0], a[1], b[0], b[1]};
            }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int d = 0; d < D / kTile; ++d) x.v[i][d] = at.value(tile, i, d);
    }
}
template <typename E, int D>
__device__ __forceinline__ void weighted_values(const ValueTile<E, D>& x, const Weights<E>& p, f32x16_t (&o)[D / kTile]) {
    if constexpr (E::kBytes == 2) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const u32x4_t w = {p.w[4 * t], p.w[4 * t + 1], p.w[4 * t + 2], p.w[4 * t + 3]};
#pragma unroll
            for (int d = 0; d < D / kTile; ++d)
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x.v[t][d]), __builtin_bit_cast(bf16x8_t, w), o[d], 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int d = 0; d < D / kTile; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.v[i][d], p.w[i], o[d], 0, 0, 0);
    }
}

// Bits of the values of a word (two bf16, one fp32) that are not finite.
template <typename E> __device__ __forceinline__ uint32_t not_finite_bits(uint32_t w) {
    if constexpr (E::kBytes == 4) return (w & 0x7f800000u) == 0x7f800000u ? ~0u : 0u;
    else return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// Whether the 32 rows of a V tile hold an infinity or a NaN (the same answer in all lanes).
template <typename E, int D> __device__ __forceinline__ bool values_not_finite(const char* lds, int lane) {
    bool bad = false;
#pragma unroll 4
    for (int i = lane; i < kTile * AttnRow<E, D>::kPieces; i += kWaveSize) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(lds + i * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) bad |= not_finite_bits<E>(v[j]) != 0;
    }
    return __ballot(bad) != 0;
}

// The same of values in registers: an exponent of all ones and one more is the sign bit.  (bf16 rows of 256 bytes have none left for it.)
template <typename E, int D> __device__ __forceinline__ bool values_not_finite(const ValueTile<E, D>& x) {
    uint32_t any = 0;
    if constexpr (E::kBytes == 2) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) any |= (x.v[t][d][i] & 0x7f807f80u) + 0x00800080u;
        return __ballot((any & 0x80008000u) != 0) != 0;
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int d = 0; d < D / kTile; ++d) any |= (__builtin_bit_cast(uint32_t, x.v[i][d]) & 0x7f800000u) + 0x00800000u;
        return __ballot((any & 0x80000000u) != 0) != 0;
    }
}

// For a tile with hidden keys, where 0 times an infinity is not zero: the operand of 16 keys (bf16: t = 0, 1) or two (fp32: t = 0..15) with
// the finite values of the keys to keep, or the others; and the weights that go with it.
template <typename E, int D>
__device__ __forceinline__ u32x4_t values_operand(const char* tile, const TileAddress<E, D>& at, int t, int d) {
    if constexpr (E::kBytes == 2) {
        const u32x2_t a = at.values(tile, t, 0, d), b = at.values(tile, t, 1, d);
        return u32x4_t{a[0], a[1], b[0], b[1]};
    } else {
        return u32x4_t{__builtin_bit_cast(uint32_t, at.value(tile, t, d)), 0, 0, 0};
    }
}
template <typename E> __device__ __forceinline__ u32x4_t weights_operand(const Weights<E>& p, int t) {
    u32x4_t w = {0, 0, 0, 0};
    if constexpr (E::kBytes == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t first = p.w[i], second = p.w[4 + i];
            w[i] = t == 0 ? first : second;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[0] = i == t ? __builtin_bit_cast(uint32_t, p.w[i]) : w[0];
    }
    return w;
}
template <typename E> __device__ __forceinline__ f32x16_t value_product(const u32x4_t& v, const u32x4_t& w, const f32x16_t& c) {
    if constexpr (E::kBytes == 2)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, w), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, (uint32_t)v[0]), __builtin_bit_cast(float, (uint32_t)w[0]), c, 0, 0, 0);
}

// o += V^T.P^T over the finite values of a tile, in the order of weighted_values: a row that sees none of the others has the same
// bits whatever they are.  Returns whether there are others.
template <typename E, int D>
__device__ __forceinline__ bool finite_values(const char* tile, const TileAddress<E, D>& at, const Weights<E>& p, f32x16_t (&o)[D / kTile]) {
    uint32_t any = 0;
#pragma unroll 1
    for (int t = 0; t < (E::kBytes == 2 ? 2 : 16); ++t) {
        const u32x4_t w = weights_operand<E>(p, t);
#pragma unroll
        for (int d = 0; d < D / kTile; ++d) {
            u32x4_t v = values_operand<E, D>(tile, at, t, d);
#pragma unroll
            for (int i = 0; i < (E::kBytes == 2 ? 4 : 1); ++i) {
                const uint32_t bad = not_finite_bits<E>(v[i]);
                v[i] &= ~bad;
                any |= bad;
            }
            o[d] = value_product<E>(v, w, o[d]);
            __builtin_amdgcn_sched_barrier(0);                     // one product at a time: registers
        }
    }
    return __ballot(any != 0) != 0;
}

// The values that are not finite, one key at a time: where a bit of `seen` says so, its product is added.  Slow.
template <typename E, int D>
__device__ __forceinline__ void other_values(const char* tile, const TileAddress<E, D>& at, const Weights<E>& p, uint32_t seen,
                                             f32x16_t (&o)[D / kTile], int lane) {
    const int half = lane / kTile;
#pragma unroll 1
    for (int key = 0; key < kTile; ++key) {
        const bool mine = (key >> 2 & 1) == half, add = (seen >> key) & 1;
        const int t = E::kBytes == 2 ? key / 16 : key / 8 * 4 + key % 4;
        const int j = (key & 3) + 4 * (key >> 3 & 1);              // its place among 8 of the operand
        u32x4_t keep;
#pragma unroll
        for (int i = 0; i < 4; ++i) keep[i] = mine && (E::kBytes == 4 || j / 2 == i) ? (E::kBytes == 4 ? ~0u : (j % 2 == 0 ? 0xffffu : 0xffff0000u)) : 0u;
        const u32x4_t w = weights_operand<E>(p, t);
#pragma unroll
        for (int d = 0; d < D / kTile; ++d) {
            u32x4_t v = values_operand<E, D>(tile, at, t, d);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] &= keep[i] & not_finite_bits<E>(v[i]);
            const f32x16_t one = value_product<E>(v, w, f32x16_t{});
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] += add ? one[i] : 0.f;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Larger of a value and the one of the lane 32 away.
__device__ __forceinline__ float max_of_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// Running softmax of a wave's 32 query rows.
template <typename E, int D> struct RowState {
    f32x16_t o[D / kTile];
    float m;               // what weights are relative to, in powers of two (see kHeadroom); the same in both halves
    float l;               // sum of the weights of this lane's keys
    __device__ __forceinline__ void clear() {
        m = -__builtin_inff();
        l = 0.f;
#pragma unroll
        for (int d = 0; d < D / kTile; ++d) o[d] = f32x16_t{};
    }
};

// Scores of a tile of keys (hidden ones -inf) to weights, moving the reference where a score passes it.  scale: softmax scale
// times log2(e).  bf16 weights are rounded for the matrix unit, and the sum is taken over the ROUNDED ones, so the weights of a row sum
// to one exactly as they are applied: rounding one key that outweighs the rest has no effect at all.
template <typename E, int D>
__device__ __forceinline__ void softmax_step(RowState<E, D>& st, const f32x16_t& s, Weights<E>& p, float scale) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top *= scale;
    if (__ballot(top > st.m) != 0) {
        // each row by its own scores: what another row of the wave sees does not change its bits
        const float both = max_of_halves(top), m = both > st.m ? both + kHeadroom<E> : st.m;
        const float f = m == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(st.m - m);
        st.m = m;
        st.l *= f;
#pragma unroll
        for (int d = 0; d < D / kTile; ++d) st.o[d] *= f;
    }
    const float m = st.m == -__builtin_inff() ? 0.f : st.m;                // nothing seen yet: exp2(-inf) = 0
    float e[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale, -m));
    if constexpr (E::kBytes == 2) {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x2_t two = {e[2 * i], e[2 * i + 1]};
            p.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2_t));
            st.l = dot2_bf16(p.w[i], 0x3f803f80u, st.l);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p.w[i] = e[i];
            st.l += e[i];
        }
    }
}

}  // namespace l2kv
