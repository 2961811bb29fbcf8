// Rows of the sequences of a compaction in pages, as the selection and the copy see them.
#pragma once

#include "l2kv_device.hpp"
#include "l2kv_host.hpp"

namespace l2kv {

// In the workspace of a compaction: where the kept rows of the sequences begin in a line of all of them, and (long sequences) the rows;
// norms in the order of the rows; kept rows.
struct CompressScratch {
    int64_t *in_off, *out_off;             // [n_seq + 1]
    float* norms;                          // [n_planes][total_rows]
    int32_t* kept;                         // [n_planes][total_kept]
    __host__ __device__ CompressScratch(void* workspace, int64_t n_planes, int64_t n_seq, int64_t total_rows) {
        in_off = static_cast<int64_t*>(workspace);
        out_off = in_off + n_seq + 1;
        norms = reinterpret_cast<float*>(out_off + n_seq + 1);
        kept = reinterpret_cast<int32_t*>(norms + n_planes * total_rows);
    }
};

// Rows and kept rows of a sequence, as far as lengths, bounds and pages go.
struct Rows { int64_t have, keep; };
__device__ __forceinline__ Rows rows_of(const PagedCompressArgs& a, int64_t s) {
    int64_t have = a.lens_in[s], keep = a.keep[s];
    const int64_t room = (int64_t)a.max_in << a.page_shift, to = (int64_t)a.max_out << a.page_shift;
    have = have < room ? have : room;
    have = have < a.max_len ? have : a.max_len;
    have = have < 0 ? 0 : have;
    keep = keep < have ? keep : have;
    keep = keep < to ? keep : to;
    return Rows{have, keep < 0 ? 0 : keep};
}

// What the bounds of all rows and of all kept ones leave of a sequence with `rows` rows and `kept` kept ones before it: past the end of the
// line nothing is kept, of this sequence and of those behind it.
struct Held { int64_t in_first, have, out_first, keep, out_end; };
__device__ __forceinline__ Held held_of(const PagedCompressArgs& a, const Rows& r, int64_t rows, int64_t kept) {
    Held h;
    h.in_first = rows < a.total_rows ? rows : a.total_rows;
    h.have = rows + r.have < a.total_rows ? r.have : a.total_rows - h.in_first;
    h.out_first = kept < a.total_kept ? kept : a.total_kept;
    h.out_end = kept + r.keep < a.total_kept ? kept + r.keep : a.total_kept;
    h.keep = h.out_end - h.out_first < h.have ? h.out_end - h.out_first : h.have;
    return h;
}

// Rows that the selection saw.
__device__ __forceinline__ int64_t have_of(const PagedCompressArgs& a, const CompressScratch& w, int32_t s) {
    const Rows r = rows_of(a, s);
    const int64_t left = a.total_rows - w.in_off[s];
    return r.have < left ? r.have : left;
}

__device__ __forceinline__ int64_t slot_of(const int32_t* table, int32_t max_pages, int32_t seq, int64_t row, int32_t shift, int32_t n_pages) {
    int32_t p = table[(int64_t)seq * max_pages + (row >> shift)];
    p = p < 0 ? 0 : (p < n_pages ? p : n_pages - 1);
    return ((int64_t)p << shift) + (row & ((1 << shift) - 1));
}

// Selection straight from the pages, for sequences that a workgroup holds in registers (select.hip).
constexpr int64_t kPagedSelectRows = 32768, kPagedSelectSeq = 1024;
l2kv_status select_paged_dispatch(const PagedCompressArgs& a, const CompressScratch& w, hipStream_t stream);

// Selection and copy of short sequences in one launch: whether these are such, and the launch.
bool select_copy_paged_applies(const PagedCompressArgs& a, int32_t row_bytes);
l2kv_status select_copy_paged_dispatch(const PagedCompressArgs& a, int32_t row_bytes, hipStream_t stream);

// Selection of few and longer ones, each by several workgroups: whether it is one of those, what it needs beside the scratch memory above,
// 16-aligned (0: there is no such selection of these sizes), and the launch.
bool select_paged_split_applies(const PagedCompressArgs& a);
size_t select_paged_split_bytes(int64_t n_planes, int64_t n_seq, int64_t total_rows);
l2kv_status select_paged_split_dispatch(const PagedCompressArgs& a, const CompressScratch& w, void* scratch, hipStream_t stream);

}  // namespace l2kv
