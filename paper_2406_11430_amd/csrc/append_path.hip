// The accepted path of a drafted tree into the slot cache: rows of node tensors, in the order of the path, behind the occupied slots of their
// sequence, with norms and token ids.  A copy of rows, 16 lanes a row (8 for rows of 128 bytes), bound by launch and by the chain of
// loads in front of the rows; every path is a row of the launch, so that nothing has to be searched.  64 paths of up to 9 tokens in 64 planes
// of 256-byte rows, 19 MB in and out, take 7.7 us with two rows of a lane on their way (8.3 with one); one path of 3 in 8 planes 2.6.
#include "l2kv_device.hpp"
#include "l2kv_host.hpp"

namespace l2kv {
namespace {

constexpr int kPathThreads = 256, kPathAhead = 2;      // rows that a lane moves at a time

template <int kRowBytes>
__global__ __launch_bounds__(kPathThreads)
void append_path_kernel(const char* __restrict__ Kt, const char* __restrict__ Vt, const float* __restrict__ norms_t,
                        const int32_t* __restrict__ pos_t, int32_t n_planes, int64_t total_nodes,
                        const int64_t* __restrict__ node_off, const int32_t* __restrict__ path, int32_t max_path,
                        const int32_t* __restrict__ path_lens, const int64_t* __restrict__ slot_off, int64_t total_slots,
                        const int32_t* __restrict__ lens_in, int32_t* __restrict__ lens_out, char* __restrict__ Kc,
                        char* __restrict__ Vc, float* __restrict__ norms_c, int32_t* __restrict__ pos_c) {
    using P = RowCopy<kRowBytes>;
    constexpr int kRows = kPathThreads / P::kLanes;
    const int c = threadIdx.x % P::kLanes, r = threadIdx.x / P::kLanes;
    const int64_t seq = blockIdx.x;
    const Range nodes = clamped_range(node_off, seq, total_nodes), slots = clamped_range(slot_off, seq, total_slots);
    const int64_t have = lens_in[seq] < 0 ? 0 : lens_in[seq];
    int64_t n = path_lens[seq];
    n = n > max_path ? max_path : n;
    if (n > slots.count - have) n = slots.count - have;
    if (n < 0 || nodes.count == 0) n = 0;
    if (blockIdx.y == 0 && threadIdx.x == 0) lens_out[seq] = (int32_t)(have + n);
    // rows of all planes, K and V side by side: plane after plane within a path position; some on their way at a time
    const int64_t rows = n * n_planes, step = (int64_t)gridDim.y * kRows;
    for (int64_t first = (int64_t)blockIdx.y * kRows + r; first < rows; first += kPathAhead * step) {
        Words<P::kWords> k[kPathAhead], v[kPathAhead];
        int64_t src[kPathAhead], dst[kPathAhead];
        float norm[kPathAhead];
        int32_t pos[kPathAhead];
#pragma unroll
        for (int u = 0; u < kPathAhead; ++u) {
            const int64_t i = first + u * step < rows ? first + u * step : first;          // behind the end: the first again
            const int64_t plane = (i | n) >> 32 == 0 ? (int64_t)((uint32_t)i / (uint32_t)n) : i / n, j = i - plane * n;
            int64_t node = path[seq * max_path + j];
            node = node < 0 ? 0 : (node < nodes.count ? node : nodes.count - 1);
            src[u] = plane * total_nodes + nodes.first + node, dst[u] = plane * total_slots + slots.first + have + j;
        }
#pragma unroll
        for (int u = 0; u < kPathAhead; ++u) {
            k[u] = load_words_stream<P::kWords, P::kStride>(Kt + src[u] * kRowBytes + c * 16);
            v[u] = load_words_stream<P::kWords, P::kStride>(Vt + src[u] * kRowBytes + c * 16);
            norm[u] = norms_t[src[u]];
            pos[u] = pos_t[src[u]];
        }
#pragma unroll
        for (int u = 0; u < kPathAhead; ++u) {
            store_words<P::kWords, P::kStride>(Kc + dst[u] * kRowBytes + c * 16, k[u]);
            store_words<P::kWords, P::kStride>(Vc + dst[u] * kRowBytes + c * 16, v[u]);
            if (c == 0) {
                norms_c[dst[u]] = norm[u];
                pos_c[dst[u]] = pos[u];
            }
        }
    }
}

}  // namespace

l2kv_status append_path_dispatch(const void* Kt, const void* Vt, const float* norms_t, const int32_t* pos_t, l2kv_dtype dt, int32_t n_planes,
                                 int32_t n_seq, int32_t D, int64_t total_nodes, const int64_t* node_off, const int32_t* path,
                                 int32_t max_path, const int32_t* path_lens, const int64_t* slot_off, int64_t total_slots,
                                 const int32_t* lens_in, int32_t* lens_out, void* Kc, void* Vc, float* norms_c, int32_t* pos_c,
                                 hipStream_t stream) {
    const int row_bytes = D * (dt == L2KV_F32 ? 4 : 2);
    if (n_seq > (1 << 24) - 1) return L2KV_ERR_SHAPE;              // a launch has fewer than 2^32 lanes
    const int64_t rows_per_block = kPathAhead * kPathThreads / (row_bytes == 128 ? 8 : 16);
    int64_t y = ((int64_t)max_path * n_planes + rows_per_block - 1) / rows_per_block;
    if (y > 65535) y = 65535;                                      // the rest in further rounds
    const dim3 grid((unsigned)n_seq, (unsigned)y);
#define L2KV_PATH(RB)                                                                                                        \
    hipLaunchKernelGGL((append_path_kernel<RB>), grid, dim3(kPathThreads), 0, stream, static_cast<const char*>(Kt),          \
                       static_cast<const char*>(Vt), norms_t, pos_t, n_planes, total_nodes, node_off, path, max_path, \
                       path_lens, slot_off, total_slots, lens_in, lens_out, static_cast<char*>(Kc), static_cast<char*>(Vc),  \
                       norms_c, pos_c)
    switch (row_bytes) {
        case 128: L2KV_PATH(128); break;
        case 256: L2KV_PATH(256); break;
        case 512: L2KV_PATH(512); break;
        default: return L2KV_ERR_SHAPE;
    }
#undef L2KV_PATH
    return launch_status();
}

}  // namespace l2kv
