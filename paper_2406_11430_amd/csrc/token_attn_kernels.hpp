// Attention of single tokens over rows in pages: l2kv_paged_attn where sequences have one new token as a rule.
//
// A read stream of the rows of every (token, KV head), as decode attention over a slot cache is (decode_kernels.hpp): 16 lanes share a row,
// a wave takes 16 rows of K and V at a time (32 of 128 bytes), with the next ones on their way in registers, and every row group
// runs its own softmax.  All rows of all items lie end to end and every workgroup takes an equal stretch of them (rows_attn_kernels.hpp),
// so lengths need not be alike and no order has to be known; what a stretch has of an item that others have parts of goes to memory
// and a second kernel joins the parts.
//
// The rows that a wave takes at a time lie in one page, or in two (rows of 128 bytes, pages of 16): where a page begins is the same in all
// lanes and worked out in scalar registers, its number asked for one step ahead.  Pages in no order cost nothing here (119.0 us, in the order
// of the plane 118.2, with an earlier kernel of the same reads).
//
// Bound by memory: 64 sequences of 500 to 4000 rows (bf16, D 128, 8 KV heads of 4 query heads) 102 us, 5.8 TB/s, of which the stream takes 95 and the join
// 4; one of 131072 rows 89 us, 6.0 TB/s (a bare read: 7.2).  One of 2048 rows with 32 KV heads 12 us: launch, three loads that wait for one
// another, 34 MB, join.  Other rows and groups, the same 64 sequences, TB/s: bf16 D 64 with groups of 1, 4, 8 5.7, 5.1, 3.8 (products on the vector
// unit), D 128 6.2, 5.8, 5.3, D 256 with 1 to 4 6.5, 6.4, 6.4, 6.2; fp32 D 64 with 1, 4, 8 6.2, 6.1, 5.2, D 128 with 1, 4, 6, 8 6.5, 6.4, 6.2, 5.9: one wave a
// SIMD is enough for the long rows.  The kernel of many rows (loads to LDS, products on the matrix unit) takes 116 to 160 us for the first of these in eight shapes.
#pragma once

#include "decode_kernels.hpp"
#include "rows_attn_kernels.hpp"

namespace l2kv {

constexpr int kTokenRows = 8;              // of a part: query heads of a KV head, at most

template <typename E, int D> struct TokenGeometry : DecodeGeometry<E, D> {
    using Geo = DecodeGeometry<E, D>;
    static constexpr int kBlock = kDecWaves * Geo::kTileRows;          // rows of a workgroup's step
    static constexpr int kPages = Geo::kTileRows / 16;                 // pages that a wave's rows may lie in
};

// Where a wave's rows are: offset into a plane, in bytes, of each 16 of them.
template <typename E, int D> struct TokenPlace { int64_t at[TokenGeometry<E, D>::kPages]; };

template <typename E, int D, int G>
__global__ __launch_bounds__(kDecThreads)
void token_attn_kernel(const RowsArgs a) {
    using Geo = TokenGeometry<E, D>;
    using L = RowsLength<kRowsPaged, Geo::kBlock>;
    typedef const __attribute__((address_space(4))) int32_t table_t;   // not written while the kernel runs
    constexpr int W = Geo::kWords, EPL = Geo::kElems, kLanesPerRow = Geo::kLanesPerRow, kGroups = Geo::kGroups, kRowBytes = D * E::kBytes;
    constexpr bool kBf16 = E::kBytes == 2;
    constexpr float kLowest = -__FLT_MAX__;
    constexpr int kVec = G * D <= kDecThreads ? 1 : (G * D <= 2 * kDecThreads ? 2 : 4);
    static_assert(G * D <= 4 * kDecThreads && G <= kTokenRows, "output elements per thread");
    // Groups of 6 to 8 heads form their scores on the matrix unit, as in decode_item: with that many the vector unit bounds a stream of
    // products and cross-lane sums (64 sequences of 500 to 4000 rows, 8 KV heads of 8 query heads 128 us, 115 so; of 6 110 and 105).  A tile
    // of K, the weights and the factors of a rescaling pass through LDS, in the place of the sums after the loop.
    constexpr bool kMfma = kBf16 && D == 128 && G >= 6;
    constexpr int kKtFloats = kDecWaves * 16 * kKtRow / 4;
    static_assert(!kMfma || kKtFloats + kDecWaves * G * 16 + kDecWaves * 8 <= kGroups * G * D, "room for what the loop keeps");
    __shared__ __attribute__((aligned(16))) float s_acc[kGroups * G * D];
    __shared__ float s_m[kGroups * G], s_l[kGroups * G];

    const int lane = threadIdx.x % kWaveSize, c = lane % kRowLanes, rg = lane / kRowLanes;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const uint32_t lane_off = rg * Geo::kSlotBytes + c * Pieces<W>::kBytes;

    RowsItem it;
    int64_t end, stretch = 0;
    if (a.workgroups == 0) {
        if (!rows_own_item<kRowsPaged, Geo::kBlock>(a, it, lane)) return;
        end = L::kExtra + L::keys(a, it.q, it.block);
    } else {
        if (threadIdx.x == 0) a.joins[blockIdx.x].parts = 0;       // until an item begins here that ends elsewhere
        if (!rows_stretch_item<kRowsPaged, Geo::kBlock>(a, it, stretch, end, lane)) return;
    }
    for (int slot = 0;; slot = 1) {                                // one item after the other
        const int64_t keys = L::keys(a, it.q, it.block), item_end = it.start + L::kExtra + keys;
        const int64_t here_end = (end < item_end ? end : item_end) - it.start;
        const int32_t first_block = it.at <= L::kExtra ? 0 : (int32_t)((it.at - L::kExtra + Geo::kBlock - 1) / Geo::kBlock);
        const int32_t end_block = here_end <= L::kExtra ? 0 : (int32_t)((here_end - L::kExtra + Geo::kBlock - 1) / Geo::kBlock);
        const bool whole = it.at == 0 && item_end <= end;
        const int64_t token = it.q.q_first + it.block;
        const int32_t n = (int32_t)(keys < it.q.n_rows ? keys : it.q.n_rows);
        const char* const Kh = a.K + (int64_t)it.head * a.kv_head_stride * E::kBytes;
        const char* const Vh = a.V + (int64_t)it.head * a.kv_head_stride * E::kBytes;
        table_t* const table = (table_t*)(uintptr_t)(a.page_table + (int64_t)it.seq * a.max_pages);

        uint32_t qw[kMfma ? 1 : G][W];
        float qf[kBf16 ? 1 : G][kBf16 ? 1 : EPL];
        const char* const Q = a.Q + (token * a.q_stride + (int64_t)it.head * G * D) * E::kBytes;
        [[maybe_unused]] bf16x8_t qa[4];                       // head c, elements 32j + 8rg ..
        [[maybe_unused]] float cm[4], cl[4];                   // heads 4rg + i: maximum, and the weights of row c of the tiles
        [[maybe_unused]] char* const kt = reinterpret_cast<char*>(s_acc) + wave * 16 * kKtRow;
        [[maybe_unused]] float* const sp = s_acc + kKtFloats + wave * G * 16;
        [[maybe_unused]] float* const sa = s_acc + kKtFloats + kDecWaves * G * 16 + wave * 8;
        if constexpr (kMfma) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x4_t raw = {0u, 0u, 0u, 0u};
                if (c < G) raw = *reinterpret_cast<const u32x4_t*>(Q + c * kRowBytes + (j * 4 + rg) * 16);
                qa[j] = __builtin_bit_cast(bf16x8_t, raw);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) cm[i] = kLowest, cl[i] = 0.f;
        }
#pragma unroll
        for (int g = 0; g < (kMfma ? 0 : G); ++g) {
            const Words<W> raw = cached_words<W>(Q + g * kRowBytes + (c % kLanesPerRow) * Pieces<W>::kBytes);
#pragma unroll
            for (int w = 0; w < W; ++w) qw[g][w] = raw.w[w];
            if constexpr (!kBf16) widen_words<E, W>(raw, qf[g]);
        }
        // the lowest number and not minus infinity where there is no row yet: no difference of two is NaN
        float m[G], l[G], acc[G][EPL];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            m[g] = kLowest;
            l[g] = 0.f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) acc[g][e] = 0.f;
        }

        // Page numbers of the rows of one of the wave's tiles (rows behind the last: the last's), and where those pages have them.
        struct Numbers { int32_t page[Geo::kPages]; };
        auto ask = [&](int32_t tile) {
            Numbers p;
#pragma unroll
            for (int i = 0; i < Geo::kPages; ++i) {
                const uint32_t row = (uint32_t)tile * Geo::kTileRows + 16 * i;
                p.page[i] = table[(row < (uint32_t)n ? row : (uint32_t)n - 1) >> a.page_shift];
            }
            return p;
        };
        auto place = [&](const Numbers& p, int32_t tile) {
            const uint32_t first = (uint32_t)tile * Geo::kTileRows;
            TokenPlace<E, D> t;
#pragma unroll
            for (int i = 0; i < Geo::kPages; ++i) {
                const int32_t page = p.page[i] < 0 ? 0 : (p.page[i] < a.n_pages ? p.page[i] : a.n_pages - 1);
                t.at[i] = (((int64_t)page << a.page_shift) + ((first + 16 * i) & ((1 << a.page_shift) - 1))) * kRowBytes;
            }
            return t;
        };
        constexpr int kPerPage = kDecLoads / Geo::kPages;          // loads of a lane in a page's 16 rows
        constexpr int kStep = kRowsPerWaveLoad * Geo::kSlotBytes;  // bytes that a wave loads at a time
        auto load = [&](Tile<E, D>& t, const TokenPlace<E, D>& p) {
#pragma unroll
            for (int u = 0; u < kDecLoads; ++u) t.k[u] = stream_words<W>(Kh + p.at[u / kPerPage] + (lane_off + u % kPerPage * kStep));
#pragma unroll
            for (int u = 0; u < kDecLoads; ++u) t.v[u] = stream_words<W>(Vh + p.at[u / kPerPage] + (lane_off + u % kPerPage * kStep));
        };
        // Rows behind the last are the last again; the last tile of an item only.
        auto load_last = [&](Tile<E, D>& t, int32_t first) {
#pragma unroll
            for (int u = 0; u < kDecLoads; ++u) {
                int32_t row = first + (u * kRowsPerWaveLoad + rg) * Geo::kRowsPerSlot + c / kLanesPerRow;
                row = row < n ? row : n - 1;
                int32_t page = a.page_table[(int64_t)it.seq * a.max_pages + (row >> a.page_shift)];
                page = page < 0 ? 0 : (page < a.n_pages ? page : a.n_pages - 1);
                const int64_t at = (((int64_t)page << a.page_shift) + (row & ((1 << a.page_shift) - 1))) * kRowBytes + (c % kLanesPerRow) * Pieces<W>::kBytes;
                t.k[u] = stream_words<W>(Kh + at);
                t.v[u] = stream_words<W>(Vh + at);
            }
        };

        // Rows behind the last have no weight, and no value: 0 times an infinity is not zero.
        auto hide = [&](Tile<E, D>& t, int32_t first) {
#pragma unroll
            for (int u = 0; u < kDecLoads; ++u) {
                const bool there = first + (u * kRowsPerWaveLoad + rg) * Geo::kRowsPerSlot + c / kLanesPerRow < n;
#pragma unroll
                for (int w = 0; w < W; ++w) t.v[u].w[w] = there ? t.v[u].w[w] : 0u;
            }
        };
        auto consume_mfma = [&](Tile<E, D>& t, int32_t first, bool last) {
            if constexpr (kMfma) {
                if (last) hide(t, first);
                // the tile of K, rows a little apart, to the layout of the operand: row c, elements 32j + 8rg ..
#pragma unroll
                for (int u = 0; u < kDecLoads; ++u)
                    *reinterpret_cast<u32x4_t*>(kt + (u * kRowsPerWaveLoad + rg) * kKtRow + c * 16) = u32x4_t{t.k[u].w[0], t.k[u].w[1], t.k[u].w[2], t.k[u].w[3]};
                __builtin_amdgcn_wave_barrier();
                f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(kt + c * kKtRow + (j * 4 + rg) * 16);
                    sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qa[j], __builtin_bit_cast(bf16x8_t, w), sc, 0, 0, 0);
                }
                const bool there = !last || first + c < n;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float si = there ? sc[i] : -INFINITY;
                    const float mn = fmaxf(cm[i], row16_max(si) * a.scale);
                    const float alpha = fast_exp2(cm[i] - mn), pi = fast_exp2(fmaf(si, a.scale, -mn));
                    cl[i] = fmaf(cl[i], alpha, pi);
                    cm[i] = mn;
                    if (const int g = 4 * rg + i; g < G) {
                        sp[g * 16 + (c % 4) * 4 + c / 4] = pi;     // [head][row group of the row][load of the row]
                        if (c == 0) sa[g] = alpha;
                    }
                }
                __builtin_amdgcn_wave_barrier();
                float pw[G][kDecLoads];
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const f32x4_t pg = *reinterpret_cast<const f32x4_t*>(sp + g * 16 + rg * 4);
#pragma unroll
                    for (int u = 0; u < kDecLoads; ++u) pw[g][u] = pg[u];
                    const float alpha = sa[g];
#pragma unroll
                    for (int e = 0; e < EPL; ++e) acc[g][e] *= alpha;
                }
#pragma unroll
                for (int u = 0; u < kDecLoads; ++u) {
                    float vx[EPL];
                    widen_words<E, W>(t.v[u], vx);
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int e = 0; e < EPL; ++e) acc[g][e] = fmaf(pw[g][u], vx[e], acc[g][e]);
                }
                __builtin_amdgcn_wave_barrier();                   // the next tile goes where this one was
            }
        };
        auto consume_vector = [&](Tile<E, D>& t, int32_t first, bool last) {
            // Query heads at a time, whose scores and weights are in registers together: half of 5 to 8 (64 sequences of 500 to 4000 rows, 8 KV heads
            // of 8 query heads 134 us, 128 so).
            if constexpr (!kMfma) {
                constexpr int kPass = G > 4 ? (G + 1) / 2 : G;
                if (last) hide(t, first);
#pragma unroll
                for (int g0 = 0; g0 < G; g0 += kPass) {
                    float s[kPass][kDecLoads], p[kPass][kDecLoads];
#pragma unroll
                    for (int u = 0; u < kDecLoads; ++u) {
                        float kx[kBf16 ? 1 : EPL];
                        if constexpr (!kBf16) widen_words<E, W>(t.k[u], kx);
#pragma unroll
                        for (int i = 0; i < kPass; ++i) {
                            if (g0 + i >= G) continue;
                            float x;
                            if constexpr (kBf16) {
                                x = dot2_bf16(qw[g0 + i][0], t.k[u].w[0], 0.f);
#pragma unroll
                                for (int w = 1; w < W; ++w) x = dot2_bf16(qw[g0 + i][w], t.k[u].w[w], x);
                            } else {
                                x = qf[g0 + i][0] * kx[0];
#pragma unroll
                                for (int e = 1; e < EPL; ++e) x = fmaf(qf[g0 + i][e], kx[e], x);
                            }
                            s[i][u] = x;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kPass; ++i)
#pragma unroll
                        for (int u = 0; u < kDecLoads; ++u)
                            if (g0 + i < G) s[i][u] = row_tree_sum<kLanesPerRow>(s[i][u]);
                    if (last) {
#pragma unroll
                        for (int u = 0; u < kDecLoads; ++u) {
                            const bool there = first + (u * kRowsPerWaveLoad + rg) * Geo::kRowsPerSlot + c / kLanesPerRow < n;
#pragma unroll
                            for (int i = 0; i < kPass; ++i)
                                if (g0 + i < G) s[i][u] = there ? s[i][u] : -INFINITY;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kPass; ++i) {
                        const int g = g0 + i;
                        if (g >= G) continue;
                        float top = s[i][0];
#pragma unroll
                        for (int u = 1; u < kDecLoads; ++u) top = fmaxf(top, s[i][u]);
                        const float mn = fmaxf(m[g], top * a.scale);
                        const float alpha = fast_exp2(m[g] - mn);
                        m[g] = mn;
                        asm volatile("" : "+v"(m[g]));                     // one head after the other, as in decode_item
                        l[g] *= alpha;
#pragma unroll
                        for (int e = 0; e < EPL; ++e) acc[g][e] *= alpha;
                        float sum = 0.f;
#pragma unroll
                        for (int u = 0; u < kDecLoads; ++u) {
                            p[i][u] = fast_exp2(fmaf(s[i][u], a.scale, -m[g]));
                            sum += p[i][u];
                        }
                        l[g] += sum;
                    }
#pragma unroll
                    for (int u = 0; u < kDecLoads; ++u) {
                        float vx[EPL];
                        widen_words<E, W>(t.v[u], vx);
#pragma unroll
                        for (int i = 0; i < kPass; ++i) {
                            if (g0 + i >= G) continue;
#pragma unroll
                            for (int e = 0; e < EPL; ++e) acc[g0 + i][e] = fmaf(p[i][u], vx[e], acc[g0 + i][e]);
                        }
                    }
                    if (g0 + kPass < G) __builtin_amdgcn_sched_barrier(0);
                }
            }
        };

        auto consume = [&](Tile<E, D>& t, int32_t first, bool last) {
            if constexpr (kMfma) consume_mfma(t, first, last);
            else consume_vector(t, first, last);
        };

        // Full tiles in two registers' worth in turn: the next is asked for before the one at hand is worked on, the page numbers of the one after
        // it as well, and no branch stands between a load and its use.
        {
            constexpr int32_t kStride = kDecWaves;                     // tiles between a wave's
            constexpr int32_t kRows = Geo::kTileRows;
            int32_t tile = first_block * kDecWaves + wave;
            const int32_t tiles = end_block * kDecWaves, full = n / kRows < tiles ? n / kRows : tiles;
            if (tile < full) {
                Tile<E, D> ta, tb;
                Numbers next = ask(tile);
                load(ta, place(next, tile));
                next = ask(tile + kStride);
                __builtin_amdgcn_sched_barrier(0);
                while (tile + 2 * kStride < full) {
                    load(tb, place(next, tile + kStride));
                    next = ask(tile + 2 * kStride);
                    __builtin_amdgcn_sched_barrier(0);
                    consume(ta, 0, false);
                    __builtin_amdgcn_sched_barrier(0);
                    load(ta, place(next, tile + 2 * kStride));
                    next = ask(tile + 3 * kStride);
                    __builtin_amdgcn_sched_barrier(0);
                    consume(tb, 0, false);
                    __builtin_amdgcn_sched_barrier(0);
                    tile += 2 * kStride;
                }
                if (tile + kStride < full) {
                    load(tb, place(next, tile + kStride));
                    __builtin_amdgcn_sched_barrier(0);
                    consume(ta, 0, false);
                    consume(tb, 0, false);
                    tile += 2 * kStride;
                } else {
                    consume(ta, 0, false);
                    tile += kStride;
                }
            }
            if (n % kRows != 0 && tile == full && tile < tiles) {
                Tile<E, D> tt;
                load_last(tt, tile * kRows);
                consume(tt, tile * kRows, true);
            }
        }

        if constexpr (kMfma) {
            // to the layout of the row groups, which share the maximum; the sum of weights counts once
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float sum = row16_tree_sum(cl[i]);
                if (const int g = 4 * rg + i; g < G && c == 0) {
                    sa[g] = cm[i];
                    sp[g] = sum;
                }
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int g = 0; g < G; ++g) {
                m[g] = sa[g];
                l[g] = rg == 0 ? sp[g] : 0.f;
            }
            __syncthreads();                                       // nobody reads the loop's part of it any more
        }
        // the row groups of the workgroup through LDS
        const int grp = (wave * kRowsPerWaveLoad + rg) * Geo::kRowsPerSlot + c / kLanesPerRow, cr = c % kLanesPerRow;
#pragma unroll
        for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) s_acc[(grp * G + g) * D + slice_elem<E, W>(cr, e)] = acc[g][e];
            if (cr == 0) {
                s_m[grp * G + g] = m[g];
                s_l[grp * G + g] = l[g];
            }
        }
        __syncthreads();
        if (const int o0 = threadIdx.x * kVec; o0 < G * D) {
            const int g = o0 / D, d = o0 % D;
            float mx = kLowest, num[kVec] = {}, den = 0.f;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) mx = fmaxf(mx, s_m[i * G + g]);
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                const float w = fast_exp2(s_m[i * G + g] - mx);
#pragma unroll
                for (int k = 0; k < kVec; ++k) num[k] = fmaf(w, s_acc[(i * G + g) * D + d + k], num[k]);
                den = fmaf(w, s_l[i * G + g], den);
            }
            if (whole) {
                const float f = den == 0.f ? 0.f : 1.f / den;      // no row: zeros
                char* const to = a.O + ((token * (a.Hkv * G) + it.head * G + g) * D + d) * E::kBytes;
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    if constexpr (kBf16) reinterpret_cast<__bf16*>(to)[k] = (__bf16)(num[k] * f);
                    else reinterpret_cast<float*>(to)[k] = num[k] * f;
                }
            } else {
                float* const to = a.partial + (((int64_t)blockIdx.x * 2 + slot) * kTokenRows + g) * rows_partial_floats(D);
#pragma unroll
                for (int k = 0; k < kVec; ++k) to[d + k] = num[k];
                if (d == 0) *reinterpret_cast<float2*>(to + D) = make_float2(mx, den);
            }
        }
        if (item_end >= end) {
            if (it.at == 0 && item_end > end && threadIdx.x == 0)
                a.joins[blockIdx.x] = RowsJoin{token * (a.Hkv * G) + it.head * G, (int32_t)quotient(item_end - 1, stretch) - (int32_t)blockIdx.x + 1, G, slot, 0};
            return;
        }
        rows_next_item<kRowsPaged>(a, it, item_end);
        __syncthreads();                                           // before the next item's results go where this one's were
    }
}

template <typename E, int D>
l2kv_status token_attn_launch(const RowsArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)(a.workgroups == 0 ? (int64_t)a.n_blocks * a.Hkv : a.workgroups)), block(kDecThreads);
#define L2KV_TOKEN(G_) case G_: hipLaunchKernelGGL((token_attn_kernel<E, D, G_>), grid, block, 0, stream, a); break
    switch (a.G) {
        L2KV_TOKEN(1); L2KV_TOKEN(2); L2KV_TOKEN(3); L2KV_TOKEN(4);
        default:
            if constexpr (D <= 128) {
                switch (a.G) {
                    L2KV_TOKEN(5); L2KV_TOKEN(6); L2KV_TOKEN(7); L2KV_TOKEN(8);
                    default: return L2KV_ERR_SHAPE;
                }
            } else {
                return L2KV_ERR_SHAPE;
            }
    }
#undef L2KV_TOKEN
    if (a.workgroups > 1) {
        if (l2kv_status st = launch_status(); st != L2KV_OK) return st;
        const dim3 join_grid((unsigned)((a.G * (D / 4) + kJoinThreads - 1) / kJoinThreads), (unsigned)a.workgroups);
        hipLaunchKernelGGL((rows_join_kernel<E, D, kTokenRows>), join_grid, dim3(kJoinThreads), 0, stream, a);
    }
    return launch_status();
}

}  // namespace l2kv
