// Rotary positions on the way into the cache: what l2kv_stream_append does for one token per sequence, for any number of packed tokens,
// with the rotation of queries and keys in it.
//
// Pair i of a token at position p is turned by the angle p * freq[i]: (x1, x2) -> a (x1 cos - x2 sin, x2 cos + x1 sin).  Angles reach a
// million radians at long contexts, where an fp32 angle is off by a twentieth of a radian, so they are formed in fp64 and reduced to one turn
// before sine and cosine.  The turn itself is done in fp64 as well and rounded to fp32, and for bf16 from there, which is how frameworks
// convert doubles (one rounding in its place, by a bit that says whether anything lies below: 0 to 7 % longer, and one element in 65536
// that lies beside a middle on the other side of it than theirs); the key's norm, which decides whether it is kept, is that of the row as
// stored, and four fp64 operations an element hide behind the memory (two bytes in, two out).
//
// A workgroup takes some tokens: their angles once into LDS, for all heads; then rows of Q, K and V, 16 elements a lane in two pieces
// of 8, neighbouring lanes side by side: of what is turned pieces u and u + rot/16 (the two halves belong together; interleaved pairs
// lie in one piece), of the rest, which is copied, and of V the same behind it.  (Two pieces side by side a lane, where nothing belongs
// together: 3.4 TB/s instead of 4.2 for fp32 rows of 128 of which 16 elements are turned.)
//
// Bound by memory: 36768 bf16 tokens of 32 + 8 + 8 heads of 128 take 173 to 179 us, 5.05 to 5.25 TB/s in and out (a large copy: 4.80), 183 without the
// rows that are on their way ahead; 64 fp32 tokens of 8 + 4 + 4 heads of 64 take 4.4 to 4.8 us, a launch and three loads that wait for one another.
#include "l2kv_device.hpp"
#include "l2kv_host.hpp"
#include "row_norm.hpp"

namespace l2kv {
namespace {

constexpr int kRotThreads = 256, kRotWaves = kRotThreads / kWaveSize;
// Most tokens of a workgroup, and most rows from more than 4 of them: heads are few where 4 tokens leave lanes idle (32768 fp32 tokens of 1 + 1 + 1
// heads of 64 21.7 us, 17.3 with 16 of them; 8 + 8 + 8 heads 92 and, with 8, 98).  Rows of 512 bytes fill the lanes, and the LDS of more
// angles costs workgroups (bf16, D 256, 4 + 1 + 1 heads: 47 us, 55 with 16).
constexpr int rot_tokens(int row_bytes) { return row_bytes <= 256 ? 16 : 4; }
constexpr int kRotRows = 96;
constexpr int64_t kNoSlot = -1, kNoSequence = -2;

// Slot of token t: its place among its sequence's tokens behind the occupied slots; kNoSlot where they are full, kNoSequence for a token
// that no sequence has.  For a wave, t the same in all lanes.
__device__ __forceinline__ int64_t token_slot(const RotaryArgs& a, int64_t t, int lane) {
    if (a.token_off == nullptr) return t;
    int32_t lo = 0, count = a.n_seq;
    while (count > 1) {                                            // the last sequence that starts at or before t, 64 candidates a step
        const int32_t step = (int32_t)(((int64_t)count + kWaveSize - 1) / kWaveSize);
        const int64_t mine = lo + (int64_t)lane * step;
        const bool at_or_before = (int64_t)lane * step < count && a.token_off[mine] <= t;
        const uint64_t found = __ballot(at_or_before);
        const int32_t last = found == 0 ? 0 : 63 - __builtin_clzll(found);
        const int32_t left = count - last * step;
        lo += last * step;
        count = left < step ? left : step;
    }
    const Range tokens = clamped_range(a.token_off, lo, a.total_tokens), slots = clamped_range(a.slot_off, lo, a.total_slots);
    const int64_t at = t - tokens.first;
    if (at < 0 || at >= tokens.count) return kNoSequence;
    const int64_t have = a.lens_in[lo] < 0 ? 0 : a.lens_in[lo];
    return have + at < slots.count ? slots.first + have + at : kNoSlot;
}

// 8 elements: 16 bytes of bf16, 32 of fp32.
template <typename E> struct Piece { Words<E::kBytes * 2> w; };
template <typename E> __device__ __forceinline__ Piece<E> load_piece(const char* p) { return {load_words_stream<E::kBytes * 2>(p)}; }
template <typename E> __device__ __forceinline__ float piece_element(const Piece<E>& p, int i) {
    if constexpr (E::kBytes == 4) return __builtin_bit_cast(float, p.w.w[i]);
    else return i % 2 == 0 ? bf16_lo(p.w.w[i / 2]) : bf16_hi(p.w.w[i / 2]);
}
template <typename E> __device__ __forceinline__ Piece<E> make_piece(const float (&x)[8]) {
    Piece<E> p;
    if constexpr (E::kBytes == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p.w.w[i] = __builtin_bit_cast(uint32_t, x[i]);
    } else {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 4; ++i) p.w.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x[2 * i], x[2 * i + 1]}, bf16x2_t));
    }
    return p;
}

template <typename E, int D, bool kInterleaved>
__global__ __launch_bounds__(kRotThreads)
void rotary_kernel(const RotaryArgs a) {
    constexpr int kLanes = D / 16, kRows = kWaveSize / kLanes;     // lanes of a row, rows of a wave
    constexpr int kRowBytes = D * E::kBytes, kPiece = 8 * E::kBytes;
    constexpr int kTokens = rot_tokens(kRowBytes);
    __shared__ __attribute__((aligned(16))) double angle[kTokens][D / 2][2];
    __shared__ int64_t slot_of[kTokens];
    __shared__ __attribute__((aligned(16))) char key_rows[kRotWaves][kRows * kRowBytes];

    const int lane = threadIdx.x % kWaveSize;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens_per_block;
    const int tokens = (int)(a.total_tokens - t0 < a.tokens_per_block ? a.total_tokens - t0 : a.tokens_per_block);

    if (a.lens_out != nullptr) {
        for (int64_t s = (int64_t)blockIdx.x * kRotThreads + threadIdx.x; s < a.n_seq; s += (int64_t)gridDim.x * kRotThreads) {
            const int64_t n = clamped_range(a.token_off, s, a.total_tokens).count, room = clamped_range(a.slot_off, s, a.total_slots).count;
            const int64_t have = a.lens_in[s] < 0 ? 0 : a.lens_in[s];
            const int64_t end = have + n < room ? have + n : room;
            a.lens_out[s] = (int32_t)(end > have ? end : have);
        }
    }
    const int heads = a.Hq + 2 * a.Hkv, u = lane % kLanes;
    const int rows = tokens * heads;
    // Rows are on their way while the angles are worked out, and while the rows before them are.
    struct Place { int row, t, h, kv, p0, p1; bool is_q, is_k, turn; };
    auto place_of = [&](int first) {
        Place at;
        at.row = first + lane / kLanes < rows ? first + lane / kLanes : rows - 1;          // the last ones are done twice
        at.t = at.row / heads, at.h = at.row - at.t * heads;
        at.is_q = at.h < a.Hq, at.is_k = !at.is_q && at.h < a.Hq + a.Hkv;
        at.kv = at.is_q ? 0 : (at.is_k ? at.h - a.Hq : at.h - a.Hq - a.Hkv);
        const int turned = at.is_q || at.is_k ? a.rot / 16 : 0;                            // lanes, of two pieces each
        at.turn = u < turned;
        at.p0 = at.turn ? u : u + turned, at.p1 = at.turn ? u + turned : u + kLanes;
        return at;
    };
    Piece<E> next0, next1;
    auto load_rows = [&](const Place& at) {
        const char* src = at.is_q ? a.Q + ((t0 + at.t) * a.q_stride + (int64_t)at.h * D) * E::kBytes
                        : at.is_k ? a.K + ((t0 + at.t) * a.k_stride + (int64_t)at.kv * D) * E::kBytes
                                  : a.V + ((t0 + at.t) * a.v_stride + (int64_t)at.kv * D) * E::kBytes;
        next0 = load_piece<E>(src + at.p0 * kPiece);
        next1 = load_piece<E>(src + at.p1 * kPiece);
    };
    Place place = place_of(wave * kRows);
    if (wave * kRows < rows) load_rows(place);
    for (int t = wave; t < tokens; t += kRotWaves) {
        const int64_t slot = token_slot(a, t0 + t, lane);
        if (lane == 0) slot_of[t] = slot;
    }
    const int pairs = a.rot / 2;
    for (int i = threadIdx.x; i < tokens * pairs; i += kRotThreads) {
        const int t = i / pairs, f = i - t * pairs;
        const double theta = (double)a.positions[t0 + t] * a.freqs[f];
        // less whole turns: 2 pi in two parts, so that the difference is as exact as the angle
        const double turns = __builtin_rint(theta * 0.15915494309189533577);
        const double rest = __builtin_fma(-turns, 2.4492935982947064e-16, __builtin_fma(-turns, 6.283185307179586, theta));
        double s, c;
        sincospi(rest * 0.31830988618379067154, &s, &c);
        angle[t][f][0] = c * a.amplitude;
        angle[t][f][1] = s * a.amplitude;
    }
    __syncthreads();

    for (int first = wave * kRows; first < rows; first += kRotWaves * kRows) {
        const auto [row, t, h, kv, p0, p1, is_q, is_k, turn] = place;
        const int64_t slot = slot_of[t];
        Piece<E> x = next0, y = next1;
        if (first + kRotWaves * kRows < rows) {
            place = place_of(first + kRotWaves * kRows);
            load_rows(place);
        }
        if (turn) {
            float r0[8], r1[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int pair = !kInterleaved ? 8 * u + i : (i < 4 ? 4 * p0 + i : 4 * p1 + i - 4);
                const double c = angle[t][pair][0], s = angle[t][pair][1];
                double x1, x2;
                if constexpr (kInterleaved) {
                    x1 = piece_element<E>(i < 4 ? x : y, 2 * i % 8);
                    x2 = piece_element<E>(i < 4 ? x : y, 2 * i % 8 + 1);
                } else {
                    x1 = piece_element<E>(x, i);
                    x2 = piece_element<E>(y, i);
                }
                const float a1 = (float)(x1 * c - x2 * s), a2 = (float)(x2 * c + x1 * s);
                if constexpr (kInterleaved) {
                    (i < 4 ? r0 : r1)[2 * i % 8] = a1;
                    (i < 4 ? r0 : r1)[2 * i % 8 + 1] = a2;
                } else {
                    r0[i] = a1;
                    r1[i] = a2;
                }
            }
            x = make_piece<E>(r0);
            y = make_piece<E>(r1);
        }
        const bool store = is_q ? slot != kNoSequence : slot >= 0;
        char* to = is_q ? a.Qr + ((t0 + t) * (int64_t)a.Hq + h) * kRowBytes : (is_k ? a.Kc : a.Vc) + (kv * a.total_slots + slot) * kRowBytes;
        if (store) {
            store_words<E::kBytes * 2>(to + p0 * kPiece, x.w);
            store_words<E::kBytes * 2>(to + p1 * kPiece, y.w);
        }
        if (__ballot(is_k) == 0) continue;
        // norms of the keys among the rows: 16 lanes a row, one chunk each
        char* const keys = key_rows[wave];
        store_words<E::kBytes * 2>(keys + lane / kLanes * kRowBytes + p0 * kPiece, x.w);
        store_words<E::kBytes * 2>(keys + lane / kLanes * kRowBytes + p1 * kPiece, y.w);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int r0 = 0; r0 < kRows; r0 += 4) {
            const int r = r0 + lane / 16;
            float sum = 0.f;
            {
#pragma clang fp contract(off)
                const char* chunk = keys + r * kRowBytes + (lane % 16) * (kRowBytes / 16);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    float v;
                    if constexpr (E::kBytes == 4) v = reinterpret_cast<const float*>(chunk)[i];
                    else v = bf16_lo(reinterpret_cast<const uint16_t*>(chunk)[i]);
                    const float sq = v * v;
                    sum = sum + sq;                                // 0 + x is x
                }
                sum = row16_tree_sum(sum);
            }
            const int krow = first + r;
            if (lane % 16 == 0 && krow < rows) {
                const int kt = krow / heads, kh = krow - kt * heads - a.Hq;
                const int64_t kslot = slot_of[kt];
                if (kh >= 0 && kh < a.Hkv && kslot >= 0) {
                    a.norms_c[kh * a.total_slots + kslot] = sum;
                    a.pos_c[kh * a.total_slots + kslot] = a.positions[t0 + kt];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

}  // namespace

l2kv_status rotary_dispatch(RotaryArgs a, l2kv_dtype dt, int32_t D, bool interleaved, hipStream_t stream) {
    // Enough tokens for some rows a lane group, but workgroups for the whole chip: few tokens one to each.
    const int heads = a.Hq + 2 * a.Hkv;
    a.tokens_per_block = rot_tokens(D * (dt == L2KV_F32 ? 4 : 2));
    while (a.tokens_per_block > 4 && a.tokens_per_block * heads > kRotRows) a.tokens_per_block /= 2;
    while (a.tokens_per_block > 1 && a.total_tokens < a.tokens_per_block * (int64_t)device_compute_units()) a.tokens_per_block /= 2;
    const int64_t blocks = (a.total_tokens + a.tokens_per_block - 1) / a.tokens_per_block;
    if (blocks > (1 << 24) - 1) return L2KV_ERR_SHAPE;             // a launch has fewer than 2^32 lanes
    const dim3 grid((unsigned)blocks);
#define L2KV_ROT(E, D_)                                                                                     \
    do {                                                                                                    \
        if (interleaved) hipLaunchKernelGGL((rotary_kernel<E, D_, true>), grid, dim3(kRotThreads), 0, stream, a); \
        else hipLaunchKernelGGL((rotary_kernel<E, D_, false>), grid, dim3(kRotThreads), 0, stream, a);       \
    } while (0)
    if (dt == L2KV_F32) {
        if (D == 64) L2KV_ROT(F32, 64);
        else L2KV_ROT(F32, 128);
    } else if (D == 64) {
        L2KV_ROT(BF16, 64);
    } else if (D == 128) {
        L2KV_ROT(BF16, 128);
    } else {
        L2KV_ROT(BF16, 256);
    }
#undef L2KV_ROT
    return launch_status();
}

}  // namespace l2kv
