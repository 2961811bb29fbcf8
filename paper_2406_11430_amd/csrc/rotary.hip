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
// Heads are normed on the way (kMore): the sum of squares in fp64 over the lanes of a row, weights in LDS as doubles, so that a normed element
// costs two products more, and slots may be found by a table of pages.
//
// Bound by memory: 36768 bf16 tokens of 32 + 8 + 8 heads of 128 take 173 to 179 us, 5.05 to 5.25 TB/s in and out (a large copy: 4.80), 183 without the
// rows that are on their way ahead; 64 fp32 tokens of 8 + 4 + 4 heads of 64 take 4.4 to 4.8 us, a launch and three loads that wait for one another.
// With norms, into pages: the 36768 tokens 189 us (204 with a branch for every element), 64 tokens of 32 + 8 + 8 heads of 128 5.3 to 7 us.
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
// that no sequence has.  For a wave, t the same in all lanes.  kMore: there may be pages.
template <bool kMore> __device__ __forceinline__ int64_t token_slot(const RotaryArgs& a, int64_t t, int lane) {
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
    const Range tokens = clamped_range(a.token_off, lo, a.total_tokens);
    const int64_t at = t - tokens.first;
    if (at < 0 || at >= tokens.count) return kNoSequence;
    const int64_t have = a.lens_in[lo] < 0 ? 0 : a.lens_in[lo];
    if constexpr (kMore) {
        if (a.page_table != nullptr) {
            const int64_t row = have + at, index = row >> a.page_shift;
            if (index >= a.max_pages || (a.ends != nullptr && row >= a.ends[lo])) return kNoSlot;
            const int32_t page = a.page_table[(int64_t)lo * a.max_pages + index];
            return page < 0 || page >= a.n_pages ? kNoSlot : ((int64_t)page << a.page_shift) + (row & ((1 << a.page_shift) - 1));
        }
    }
    const Range slots = clamped_range(a.slot_off, lo, a.total_slots);
    return have + at < slots.count ? slots.first + have + at : kNoSlot;
}

// Where sequences s0 .. s0 + 63 end after the call, a lane each (in the last lane the first): as far as there is room, and in pages only as
// far as there are pages and as the sequence's end allows.  Of new rows in many pages the whole wave looks for one that is missing (32768 tokens of 32 + 8 + 8 heads of 128 in pages
// of 16, one entry after the other by a single lane: 390 us, 168 so).
constexpr int64_t kFewPages = 4;
template <bool kMore> __device__ __forceinline__ void write_lens(const RotaryArgs& a, int64_t s0, int lane) {
    const int64_t s = s0 + (kWaveSize - 1 - lane);
    const bool mine = s < a.n_seq;
    const int64_t n = mine ? clamped_range(a.token_off, s, a.total_tokens).count : 0, have = !mine || a.lens_in[s] < 0 ? 0 : a.lens_in[s];
    if constexpr (kMore) {
        if (a.page_table != nullptr) {
            auto held = [&](int64_t entry) { return a.page_table[entry] >= 0 && a.page_table[entry] < a.n_pages; };
            const int64_t first = have >> a.page_shift, behind = ((have + n - 1) >> a.page_shift) + 1;
            const int64_t wanted = n == 0 ? 0 : (behind < a.max_pages ? behind : a.max_pages) - first, entry = s * a.max_pages + first;
            int64_t there = 0;
            if (wanted <= kFewPages)
                while (there < wanted && held(entry + there)) ++there;
            for (uint64_t many = __ballot(wanted > kFewPages); many != 0; many &= many - 1) {
                const int whose = __builtin_ctzll(many);
                const int64_t e0 = __shfl(entry, whose), count = __shfl(wanted, whose);
                int64_t i = 0;
                uint64_t missing = 0;
                for (; i < count && missing == 0; i += missing == 0 ? kWaveSize : __builtin_ctzll(missing))
                    missing = __ballot(i + lane >= count || !held(e0 + i + lane));
                if (lane == whose) there = i;                      // what is behind the last entry counts as missing
            }
            const int64_t pages = (first + there) << a.page_shift, given = mine && a.ends != nullptr ? a.ends[s] : pages;
            const int64_t room = given < pages ? given : pages, end = have + n < room ? have + n : room;
            if (mine) a.lens_out[s] = (int32_t)(end > have ? end : have);
            return;
        }
    }
    if (!mine) return;
    const int64_t room = clamped_range(a.slot_off, s, a.total_slots).count, end = have + n < room ? have + n : room;
    a.lens_out[s] = (int32_t)(end > have ? end : have);
}

// Sum over the kLanes (4, 8 or 16) consecutive lanes that share a row, in every one of them the same.
template <int CTRL> __device__ __forceinline__ double dpp_read(double v) {
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CTRL, 0xf, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int kLanes> __device__ __forceinline__ double sum_of_row(double v) {
    v += dpp_read<kDppXor1>(v);
    v += dpp_read<kDppXor2>(v);
    if constexpr (kLanes >= 8) v += dpp_read<kDppHalfMirror>(v);
    if constexpr (kLanes >= 16) v += dpp_read<kDppMirror>(v);
    return v;
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

template <typename E, int D, bool kInterleaved, bool kMore>
__global__ __launch_bounds__(kRotThreads)
void rotary_kernel(const RotaryArgs a) {
    constexpr int kLanes = D / 16, kRows = kWaveSize / kLanes;     // lanes of a row, rows of a wave
    constexpr int kRowBytes = D * E::kBytes, kPiece = 8 * E::kBytes;
    constexpr int kTokens = rot_tokens(kRowBytes);
    __shared__ __attribute__((aligned(16))) double angle[kTokens][D / 2][2];
    __shared__ int64_t slot_of[kTokens];
    __shared__ __attribute__((aligned(16))) double weights[kMore ? 2 : 1][kMore ? D : 2];    // of queries, of keys; ones where there are none
    __shared__ __attribute__((aligned(16))) char key_rows[kRotWaves][kRows * kRowBytes];

    const int lane = threadIdx.x % kWaveSize;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens_per_block;
    const int tokens = (int)(a.total_tokens - t0 < a.tokens_per_block ? a.total_tokens - t0 : a.tokens_per_block);

    if (a.lens_out != nullptr) {
        // by the last waves: the first ones look for slots
        for (int64_t s0 = (int64_t)blockIdx.x * kRotThreads + (kRotWaves - 1 - wave) * kWaveSize; s0 < a.n_seq; s0 += (int64_t)gridDim.x * kRotThreads)
            write_lens<kMore>(a, s0, lane);
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
        const int64_t slot = token_slot<kMore>(a, t0 + t, lane);
        if (lane == 0) slot_of[t] = slot;
    }
    const int pairs = a.rot / 2;
    for (int i = (threadIdx.x + kRotThreads - kWaveSize) % kRotThreads; i < tokens * pairs; i += kRotThreads) {      // from the second wave on
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
    if constexpr (kMore) {
        for (int i = threadIdx.x; i < 2 * D; i += kRotThreads) {
            const float* const w = i < D ? a.q_weight : a.k_weight;
            weights[i / D][i % D] = w != nullptr ? (double)w[i % D] : 1.0;
        }
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
        // kMore: elements times their weight over the root of the mean square (heads that are not normed: times one), without a branch
        // for each of them.
        [[maybe_unused]] double root = 1.0;
        const bool normed = kMore && (is_q ? a.q_weight != nullptr : is_k && a.k_weight != nullptr);
        if constexpr (kMore) {
            if (__ballot(normed) != 0) {
                double sum = 0.0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double p = piece_element<E>(x, i), q = piece_element<E>(y, i);
                    sum = __builtin_fma(p, p, __builtin_fma(q, q, sum));
                }
                const double mean = sum_of_row<kLanes>(sum) * (1.0 / D) + a.eps;
                // The instruction is good to 2^-14 at least; a step leaves 3/2 of the error's square: 2^-27.4, 2^-54.2, and the third
                // takes off what the roundings of the second left.
                double r = __builtin_amdgcn_rsq(mean);
#pragma unroll
                for (int i = 0; i < 3; ++i) r = __builtin_fma(r * 0.5, __builtin_fma(-mean * r, r, 1.0), r);
                root = !normed ? 1.0 : mean == __builtin_inf() ? 0.0 : r;
            }
        }
        [[maybe_unused]] const double* const w0 = weights[kMore && !is_q ? 1 : 0] + (kMore ? 8 * p0 : 0);
        [[maybe_unused]] const double* const w1 = weights[kMore && !is_q ? 1 : 0] + (kMore ? 8 * p1 : 0);
        auto element = [&](bool second, int i) -> double {
            const double v = piece_element<E>(second ? y : x, i);
            if constexpr (kMore) return v * (second ? w1 : w0)[i] * root;
            return v;
        };
        if (turn) {
            float r0[8], r1[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int pair = !kInterleaved ? 8 * u + i : (i < 4 ? 4 * p0 + i : 4 * p1 + i - 4);
                const double c = angle[t][pair][0], s = angle[t][pair][1];
                double x1, x2;
                if constexpr (kInterleaved) {
                    x1 = element(i >= 4, 2 * i % 8);
                    x2 = element(i >= 4, 2 * i % 8 + 1);
                } else {
                    x1 = element(false, i);
                    x2 = element(true, i);
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
        } else if (normed) {
            float r0[8], r1[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                r0[i] = (float)element(false, i);
                r1[i] = (float)element(true, i);
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
    const bool more = a.q_weight != nullptr || a.k_weight != nullptr || a.page_table != nullptr;
#define L2KV_ROT(E, D_)                                                                                                       \
    do {                                                                                                                      \
        auto kernel = more ? (interleaved ? rotary_kernel<E, D_, true, true> : rotary_kernel<E, D_, false, true>)             \
                           : (interleaved ? rotary_kernel<E, D_, true, false> : rotary_kernel<E, D_, false, false>);          \
        hipLaunchKernelGGL(kernel, grid, dim3(kRotThreads), 0, stream, a);                                                    \
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
