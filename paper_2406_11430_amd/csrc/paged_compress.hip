// Compaction of a cache in pages: of every plane and sequence the rows with the lowest (norm bits, row), in the order of the rows, into the
// pages of another table (arXiv 2406.11430, Sec. 1: keep the lowest-norm keys and their values).
//
// A workgroup selects for each (plane, sequence), with the norms in registers straight from their pages; kept rows are then copied from page to
// page, 16 bytes a lane, with norms and token ids.  Short sequences take one launch for both (select_copy_paged_kernel).  Few and longer sequences are selected from by several workgroups each, in three launches that
// put the norms into one line per plane on the way (8 planes of 131072 rows, a tenth kept, 92 us with one workgroup a plane, 47 so; of 1000000
// 722 and 232).  Many longer sequences, and very many, have their norms gathered first (4 bytes a row beside the 2 * row bytes of each kept
// one) for the selection of ragged batches.  Source and destination are
// other pages, so rows that several sequences share are only read, and nothing has to be read before it is written over.
//
// Bound by memory: 64 sequences of 1k to 8k bf16 rows of 128 in 8 planes, half kept, 254 us, 4.9 TB/s in and out with 15 us of selection (rows of
// pages in order 217, as from plane to slots; pages in no order cost the difference, of 16 rows and of 256 alike).  Four
// planes of 777 rows 6.7 us, a launch of dependent loads.
#include "paged_rows.hpp"

namespace l2kv {
namespace {

constexpr int kPcThreads = 256, kPcWaves = kPcThreads / kWaveSize, kPcScan = 1024;
constexpr int kPcUnroll = 2;
template <int kRowBytes> constexpr int kPcRowsPerBlock = kPcWaves * RowCopy<kRowBytes>::kRowsPerWave * kPcUnroll;

// Where the rows of the sequences begin in a line, and the kept ones; what goes beyond the lines' ends is left out.  One workgroup.
__global__ __launch_bounds__(kPcScan)
void compress_offsets_kernel(const PagedCompressArgs a, CompressScratch w) {
    __shared__ int64_t waves[2][kPcScan / kWaveSize];
    const int lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
    int64_t rows = 0, kept = 0;
    for (int32_t s0 = 0; s0 < a.n_seq; s0 += kPcScan) {
        const int32_t s = s0 + (int32_t)threadIdx.x;
        Rows r = {0, 0};
        if (s < a.n_seq) r = rows_of(a, s);
        int64_t have = r.have, keep = r.keep;
#pragma unroll
        for (int d = 1; d < kWaveSize; d *= 2) {
            const int64_t h = __shfl_up(have, d), k = __shfl_up(keep, d);
            have += lane >= d ? h : 0;
            keep += lane >= d ? k : 0;
        }
        if (lane == kWaveSize - 1) waves[0][wave] = have, waves[1][wave] = keep;
        __syncthreads();
        int64_t before[2] = {rows, kept};
        for (int i = 0; i < kPcScan / kWaveSize; ++i) {
            if (i < wave) before[0] += waves[0][i], before[1] += waves[1][i];
            rows += waves[0][i], kept += waves[1][i];
        }
        const int64_t first = before[0] + have - r.have, out = before[1] + keep - r.keep;
        if (s < a.n_seq) {
            const Held h = held_of(a, r, first, out);
            w.in_off[s] = h.in_first;
            w.out_off[s] = h.out_first;
            a.lens_out[s] = (int32_t)h.keep;
            if (s == a.n_seq - 1) {
                w.in_off[s + 1] = h.in_first + h.have;
                w.out_off[s + 1] = h.out_end;
            }
        }
        __syncthreads();
    }
}

// The last sequence that begins at or before j, 64 candidates a step; j the same in all lanes.
__device__ __forceinline__ int32_t sequence_at(const int64_t* off, int32_t n_seq, int64_t j, int lane) {
    int32_t lo = 0, count = n_seq;
    while (count > 1) {
        const int32_t step = (count + kWaveSize - 1) / kWaveSize;
        const bool at_or_before = (int64_t)lane * step < count && off[lo + (int64_t)lane * step < n_seq ? lo + lane * step : n_seq - 1] <= j;
        const uint64_t found = __ballot(at_or_before);
        const int32_t last = found == 0 ? 0 : 63 - __builtin_clzll(found);
        lo += last * step;
        count = count - last * step < step ? count - last * step : step;
    }
    return lo;
}
// The same for j of this lane, from a sequence that begins at or before it.
__device__ __forceinline__ int32_t sequence_from(const int64_t* off, int32_t n_seq, int32_t s, int64_t j) {
    int32_t lo = s, hi = n_seq;                                    // off[lo] <= j, and off[hi] > j where hi < n_seq
    while (hi - lo > 1) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (off[mid] <= j) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Grid (256 rows, planes): norms from their pages into the line.
__global__ __launch_bounds__(kPcThreads)
void compress_gather_kernel(const PagedCompressArgs a, CompressScratch w, int64_t first_plane) {
    const int lane = threadIdx.x % kWaveSize;
    const int64_t plane = first_plane + blockIdx.y, base = (int64_t)blockIdx.x * kPcThreads + threadIdx.x - lane, j = base + lane;
    const int64_t end = w.in_off[a.n_seq];
    if (base >= end) return;
    int32_t s = sequence_at(w.in_off, a.n_seq, base, lane);
    if (s + 1 < a.n_seq && w.in_off[s + 1] < base + kWaveSize) s = sequence_from(w.in_off, a.n_seq, s, j < end ? j : end - 1);
    if (j >= end) return;
    const int64_t slots = (int64_t)a.n_pages << a.page_shift;
    w.norms[plane * a.total_rows + j] = a.norms_c[plane * slots + slot_of(a.table_in, a.max_in, s, j - w.in_off[s], a.page_shift, a.n_pages)];
}

// Grid (chunks of kept rows, planes): K and V of a row by the same lanes, whose places then count for both, two rows a lane on their way (alternate
// workgroups of K and of V with four rows 272 us, so 266: 64 sequences of 1k to 8k bf16 rows of 128 in 8 planes, half kept).
template <int kRowBytes>
__global__ __launch_bounds__(kPcThreads)
void compress_copy_kernel(const PagedCompressArgs a, CompressScratch w, int64_t first_plane) {
    using P = RowCopy<kRowBytes>;
    const int64_t plane = first_plane + blockIdx.y, slots = (int64_t)a.n_pages << a.page_shift;
    const int lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize, c = lane % P::kLanes, rg = lane / P::kLanes;
    const int64_t end = w.out_off[a.n_seq];
    const int64_t wave_first = (int64_t)blockIdx.x * kPcRowsPerBlock<kRowBytes> + wave * (P::kRowsPerWave * kPcUnroll);
    if (wave_first >= end) return;
    // which rows, before it is known whose they are
    int64_t at[kPcUnroll], row[kPcUnroll];
#pragma unroll
    for (int u = 0; u < kPcUnroll; ++u) {
        at[u] = wave_first + u * P::kRowsPerWave + rg;
        row[u] = w.kept[plane * a.total_kept + (at[u] < end ? at[u] : end - 1)];
    }
    const int32_t s0 = sequence_at(w.out_off, a.n_seq, wave_first, lane);
    // all rows of a wave are one sequence's as a rule
    const bool alone = s0 + 1 >= a.n_seq || w.out_off[s0 + 1] >= wave_first + P::kRowsPerWave * kPcUnroll;
    int64_t src[kPcUnroll], dst[kPcUnroll];
    bool live[kPcUnroll];
    auto place = [&](int u, int32_t s, int64_t out_first, int64_t kept, int64_t have) {
        const int64_t out = at[u] - out_first;
        live[u] = at[u] < end && out < kept;
        int64_t r = row[u] < have ? row[u] : have - 1;             // inside the sequence whatever is there
        r = r < 0 ? 0 : r;
        const int32_t page = a.table_out[(int64_t)s * a.max_out + (live[u] ? out >> a.page_shift : 0)];
        src[u] = plane * slots + slot_of(a.table_in, a.max_in, s, r, a.page_shift, a.n_pages);
        live[u] = live[u] && page >= 0 && page < a.n_pages;        // nothing is written where there is no page
        dst[u] = plane * slots + ((int64_t)(live[u] ? page : 0) << a.page_shift) + (out & ((1 << a.page_shift) - 1));
    };
    if (alone) {
        const int32_t s = __builtin_amdgcn_readfirstlane(s0);
        const int64_t out_first = w.out_off[s], kept = a.lens_out[s], have = have_of(a, w, s);
#pragma unroll
        for (int u = 0; u < kPcUnroll; ++u) place(u, s, out_first, kept, have);
    } else {
#pragma unroll
        for (int u = 0; u < kPcUnroll; ++u) {
            const int32_t s = sequence_from(w.out_off, a.n_seq, s0, at[u] < end ? at[u] : end - 1);
            place(u, s, w.out_off[s], a.lens_out[s], have_of(a, w, s));
        }
    }
    Words<P::kWords> k[kPcUnroll], v[kPcUnroll];
#pragma unroll
    for (int u = 0; u < kPcUnroll; ++u) k[u] = load_words_stream<P::kWords, P::kStride>(a.Kc + src[u] * kRowBytes + c * 16);
#pragma unroll
    for (int u = 0; u < kPcUnroll; ++u) v[u] = load_words_stream<P::kWords, P::kStride>(a.Vc + src[u] * kRowBytes + c * 16);
    float norm[kPcUnroll] = {};
    int32_t pos[kPcUnroll] = {};
    if (c == 0) {
#pragma unroll
        for (int u = 0; u < kPcUnroll; ++u) norm[u] = a.norms_c[src[u]], pos[u] = a.pos_c[src[u]];
    }
#pragma unroll
    for (int u = 0; u < kPcUnroll; ++u) {
        if (!live[u]) continue;
        store_words_stream<P::kWords, P::kStride>(a.Kc + dst[u] * kRowBytes + c * 16, k[u]);
        store_words_stream<P::kWords, P::kStride>(a.Vc + dst[u] * kRowBytes + c * 16, v[u]);
        if (c == 0) {
            a.norms_c[dst[u]] = norm[u];
            a.pos_c[dst[u]] = pos[u];
        }
    }
}

}  // namespace

size_t paged_compress_least_bytes(int64_t n_planes, int64_t n_seq, int64_t total_rows, int64_t total_kept) {
    return (size_t)(16 * (n_seq + 1) + 4 * n_planes * (total_rows + total_kept) + 15) / 16 * 16;
}
size_t paged_compress_workspace_bytes(int64_t n_planes, int64_t n_seq, int64_t total_rows, int64_t total_kept) {
    return paged_compress_least_bytes(n_planes, n_seq, total_rows, total_kept) + select_paged_split_bytes(n_planes, n_seq, total_rows);
}

l2kv_status paged_compress_dispatch(const PagedCompressArgs& a, l2kv_dtype dt, int32_t D, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const CompressScratch w(workspace, a.n_planes, a.n_seq, a.total_rows);
    constexpr int64_t kMaxY = 65535;
    const int row_bytes = D * (dt == L2KV_F32 ? 4 : 2);
    if (select_copy_paged_applies(a, row_bytes)) return select_copy_paged_dispatch(a, row_bytes, stream);
    if (a.max_len <= kPagedSelectRows && a.n_seq <= kPagedSelectSeq) {
        if (l2kv_status st = select_paged_dispatch(a, w, stream); st != L2KV_OK) return st;
    } else if (select_paged_split_applies(a) && workspace_bytes >= paged_compress_workspace_bytes(a.n_planes, a.n_seq, a.total_rows, a.total_kept)) {
        char* const scratch = static_cast<char*>(workspace) + paged_compress_least_bytes(a.n_planes, a.n_seq, a.total_rows, a.total_kept);
        if (l2kv_status st = select_paged_split_dispatch(a, w, scratch, stream); st != L2KV_OK) return st;
    } else {
        hipLaunchKernelGGL(compress_offsets_kernel, dim3(1), dim3(kPcScan), 0, stream, a, w);
        if (l2kv_status st = launch_status(); st != L2KV_OK) return st;
        const unsigned gather = (unsigned)((a.total_rows + kPcThreads - 1) / kPcThreads);
        for (int64_t p0 = 0; p0 < a.n_planes; p0 += kMaxY) {
            const unsigned planes = (unsigned)(a.n_planes - p0 < kMaxY ? a.n_planes - p0 : kMaxY);
            hipLaunchKernelGGL(compress_gather_kernel, dim3(gather, planes), dim3(kPcThreads), 0, stream, a, w, p0);
            if (l2kv_status st = launch_status(); st != L2KV_OK) return st;
        }
        const int64_t step = (int64_t{1} << 21) / a.n_seq;         // planes of a launch: it has fewer than 2^32 lanes
        for (int64_t p0 = 0; p0 < a.n_planes; p0 += step) {
            const int32_t planes = (int32_t)(a.n_planes - p0 < step ? a.n_planes - p0 : step);
            if (l2kv_status st = select_ragged_dispatch(w.norms + p0 * a.total_rows, planes, a.n_seq, a.total_rows, w.in_off, w.out_off, a.total_kept,
                                                        a.max_len, L2KV_KEEP_LOWEST, w.kept + p0 * a.total_kept, stream);
                st != L2KV_OK)
                return st;
        }
    }
    const int64_t per_block = row_bytes == 128 ? kPcRowsPerBlock<128> : kPcRowsPerBlock<256>;
    static_assert(kPcRowsPerBlock<256> == kPcRowsPerBlock<512>, "one chunk size for rows of 16 lanes");
    const unsigned chunks = (unsigned)((a.total_kept + per_block - 1) / per_block);
    for (int64_t p0 = 0; p0 < a.n_planes; p0 += kMaxY) {
        const dim3 grid(chunks, (unsigned)(a.n_planes - p0 < kMaxY ? a.n_planes - p0 : kMaxY));
        switch (row_bytes) {
            case 128: hipLaunchKernelGGL((compress_copy_kernel<128>), grid, dim3(kPcThreads), 0, stream, a, w, p0); break;
            case 256: hipLaunchKernelGGL((compress_copy_kernel<256>), grid, dim3(kPcThreads), 0, stream, a, w, p0); break;
            default: hipLaunchKernelGGL((compress_copy_kernel<512>), grid, dim3(kPcThreads), 0, stream, a, w, p0); break;
        }
        if (l2kv_status st = launch_status(); st != L2KV_OK) return st;
    }
    return L2KV_OK;
}

}  // namespace l2kv
