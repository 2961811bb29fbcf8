// Pages of a cache that sequences share: forking, reserving room (with copies of pages that others hold too) and releasing.
//
// A page has refs[page] holders, the entries of page tables that name it; those without any are numbered in free_pages[0 .. free_count),
// the next to be handed out last.  Which page an entry gets, and where a released page goes, is decided by the order of the entries
// (sequence after sequence, page after page) and by nothing else: counts are added up with atomics, whose order does not
// matter, and of the entries that name one page the last is found with an atomic maximum.
//
// The tables are small (64 sequences of 500 pages: 128 KB) and every decision needs all those before it, so one workgroup works through them,
// 1024 sequences and then 1024 entries at a time; the copies are a launch of their own behind it.
#include "l2kv_device.hpp"
#include "l2kv_host.hpp"

namespace l2kv {
namespace {

constexpr int kPageThreads = 1024, kPageWaves = kPageThreads / kWaveSize;
constexpr int kForkThreads = 256, kCopyThreads = 256;

// In the workspace: of every page how many of its holders are left when the entries at hand are taken off, and the last of those entries;
// pages to copy, {from, to} (from -1: none), and their number.
struct PagesScratch {
    int32_t *left, *last;
    int2* copies;
    int32_t* n_copies;
    __host__ __device__ PagesScratch(void* workspace, int64_t n_pages) {
        n_copies = static_cast<int32_t*>(workspace);
        copies = reinterpret_cast<int2*>(n_copies + 4);
        left = reinterpret_cast<int32_t*>(copies + n_pages);
        last = left + n_pages;
    }
};

struct PagesShared {
    int32_t first[kPageThreads];           // of a sequence: index of its first entry
    int64_t upto[kPageThreads];            // entries of the sequences up to it
    int64_t waves[kPageWaves];
    int64_t news[kPageThreads];            // reserving: new pages wanted up to the end of a sequence
    int32_t need[kPageThreads];            // of them by itself
    bool others[kPageThreads];             // it would write a page that others hold as well
    int32_t handed;                        // new pages handed out
};

// Inclusive prefix sum over the workgroup, of numbers whose sum is below 2^31 within a wave.
__device__ __forceinline__ int64_t block_prefix(uint32_t v, int64_t (&waves)[kPageWaves], int64_t& total) {
    const int lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
    const uint32_t mine = wave_inclusive_sum(v);
    __syncthreads();                       // what was in `waves` is not read any more
    if (lane == kWaveSize - 1) waves[wave] = mine;
    __syncthreads();
    int64_t before = 0;
    total = 0;
    for (int w = 0; w < kPageWaves; ++w) {
        before += w < wave ? waves[w] : 0;
        total += waves[w];
    }
    return before + mine;
}

// The entries of up to 1024 sequences laid end to end.  `range` gives the first entry of a sequence and how many there are.
template <typename F> __device__ __forceinline__ int64_t lay_out(PagesShared& sh, int32_t s0, int32_t n_seq, F&& range) {
    int32_t first = 0, count = 0;
    const int64_t s = (int64_t)s0 + threadIdx.x;
    if (s < n_seq) range((int32_t)s, first, count);
    int64_t total;
    const int64_t upto = block_prefix((uint32_t)count, sh.waves, total);
    sh.first[threadIdx.x] = first;
    sh.upto[threadIdx.x] = upto;
    __syncthreads();
    return total;
}
struct Entry { int32_t seq; int64_t at; bool last_of_seq; };                  // sequence among the 1024, place in the table
__device__ __forceinline__ Entry entry_of(const PagesShared& sh, int32_t s0, int32_t max_pages, int64_t e) {
    int32_t lo = 0;                                                       // the first whose entries reach beyond e
#pragma unroll
    for (int step = kPageThreads / 2; step > 0; step /= 2) lo = sh.upto[lo + step - 1] <= e ? lo + step : lo;
    const int64_t before = lo == 0 ? 0 : sh.upto[lo - 1];
    return Entry{lo, (int64_t)(s0 + lo) * max_pages + sh.first[lo] + (e - before), e + 1 == sh.upto[lo]};
}
__device__ __forceinline__ bool is_page(int32_t p, int32_t n_pages) { return p >= 0 && p < n_pages; }

template <typename T> __device__ __forceinline__ T device_load(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void device_store(int32_t* p, int32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ int32_t device_add(int32_t* p, int32_t v) { return __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Runs `visit` for every entry that `range` gives, all lanes together (an entry that is not there: e = -1).
template <typename R, typename F>
__device__ __forceinline__ void for_entries(PagesShared& sh, const PagesArgs& a, R&& range, F&& visit) {
    for (int32_t s0 = 0; s0 < a.n_seq; s0 += kPageThreads) {
        const int64_t total = lay_out(sh, s0, a.n_seq, range);
        for (int64_t e0 = 0; e0 < total; e0 += kPageThreads) {
            const int64_t e = e0 + threadIdx.x;
            Entry x = {0, -1, false};
            if (e < total) x = entry_of(sh, s0, a.max_pages, e);
            visit(s0, x);
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(kForkThreads)
void pages_init_kernel(const PagesArgs a) {
    const int64_t i = (int64_t)blockIdx.x * kForkThreads + threadIdx.x, step = (int64_t)gridDim.x * kForkThreads;
    for (int64_t e = i; e < (int64_t)a.n_seq * a.max_pages; e += step) a.table[e] = -1;
    for (int64_t p = i; p < a.n_pages; p += step) {
        a.refs[p] = 0;
        a.free_pages[p] = a.n_pages - 1 - (int32_t)p;
    }
    if (i == 0) *a.free_count = a.n_pages;
}

// A lane an entry of the new table: one holder more.
__global__ __launch_bounds__(kForkThreads)
void pages_fork_kernel(const int32_t* __restrict__ table_in, const int32_t* __restrict__ lens_in, int32_t n_in,
                       const int32_t* __restrict__ parents, const PagesArgs a, int32_t* __restrict__ lens_out) {
    const int64_t n = (int64_t)a.n_seq * a.max_pages, step = (int64_t)gridDim.x * kForkThreads;
    for (int64_t e = (int64_t)blockIdx.x * kForkThreads + threadIdx.x; e < n; e += step) {
        const int64_t s = n <= 0xffffffffLL ? (uint32_t)e / (uint32_t)a.max_pages : e / a.max_pages, i = e - s * a.max_pages;
        const int32_t parent = parents[s];
        int32_t page = -1, len = 0;
        if (parent >= 0 && parent < n_in) {
            len = lens_in[parent] < 0 ? 0 : lens_in[parent];
            const int64_t room = (int64_t)a.max_pages << a.page_shift;
            len = len < room ? len : (int32_t)room;
            if (i << a.page_shift < len) page = table_in[(int64_t)parent * a.max_pages + i];
            if (!is_page(page, a.n_pages)) page = -1;
        }
        a.table[e] = page;
        if (page >= 0) device_add(a.refs + page, 1);
        if (i == 0) lens_out[s] = len;
    }
}

// Room for rows from[s] .. to[s]-1 of every sequence.  An entry without a page gets one, and one whose page others hold as well gets
// a copy in its place, except that of the holders of a page that all ask for it in this call the last keeps it.
__global__ __launch_bounds__(kPageThreads)
void pages_reserve_kernel(const PagesArgs a, const int32_t* __restrict__ from, const int32_t* __restrict__ to, int32_t* __restrict__ ends,
                          void* workspace) {
    __shared__ PagesShared sh;
    const PagesScratch w(workspace, a.n_pages);
    auto range = [&](int32_t s, int32_t& first, int32_t& count) {
        const int64_t b = from[s], e = to[s];
        if (b < 0 || e <= b || e > (int64_t)a.max_pages << a.page_shift) return;
        first = (int32_t)(b >> a.page_shift);
        count = (int32_t)((e - 1) >> a.page_shift) - first + 1;
    };
    for_entries(sh, a, range, [&](int32_t, const Entry& x) {
        const int32_t p = x.at < 0 ? -1 : a.table[x.at];
        if (!is_page(p, a.n_pages)) return;
        device_store(w.left + p, device_load(a.refs + p));           // the same whoever does it
        device_store(w.last + p, -1);
    });
    __threadfence();
    __syncthreads();
    for_entries(sh, a, range, [&](int32_t, const Entry& x) {
        const int32_t p = x.at < 0 ? -1 : a.table[x.at];
        if (!is_page(p, a.n_pages)) return;
        device_add(w.left + p, -1);
        __hip_atomic_fetch_max(w.last + p, (int32_t)x.at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    __threadfence();
    __syncthreads();
    int64_t have = *a.free_count;
    have = have < 0 ? 0 : (have > a.n_pages ? a.n_pages : have);
    int64_t base = 0;                                          // new pages wanted by the sequences before these
    if (threadIdx.x == 0) sh.handed = 0;
    auto wants = [&](int64_t at, int32_t p) {
        return at >= 0 && (!is_page(p, a.n_pages) || device_load(w.left + p) > 0 || device_load(w.last + p) != (int32_t)at);
    };
    for (int32_t s0 = 0; s0 < a.n_seq; s0 += kPageThreads) {
        const int64_t total = lay_out(sh, s0, a.n_seq, range);
        sh.news[threadIdx.x] = 0;
        sh.need[threadIdx.x] = 0;
        sh.others[threadIdx.x] = false;
        __syncthreads();
        // how many are wanted up to the end of each sequence, then who gets one
        int64_t sum = 0;
        for (int pass = 0; pass < 2; ++pass) {
            sum = base;
            for (int64_t e0 = 0; e0 < total; e0 += kPageThreads) {
                const int64_t e = e0 + threadIdx.x;
                Entry x = {0, -1, false};
                if (e < total) x = entry_of(sh, s0, a.max_pages, e);
                const int32_t p = x.at < 0 ? -1 : a.table[x.at];
                const bool want = wants(x.at, p);
                int64_t these;
                const int64_t upto = sum + block_prefix(want ? 1u : 0u, sh.waves, these);
                sum += these;
                if (pass == 0) {
                    if (want) __hip_atomic_fetch_add(&sh.need[x.seq], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                    if (x.last_of_seq) sh.news[x.seq] = upto;
                } else if (want && sh.news[x.seq] <= have) {
                    const int32_t raw = a.free_pages[have - upto];
                    const int32_t page = is_page(raw, a.n_pages) ? raw : 0;
                    w.copies[upto - 1] = make_int2(is_page(p, a.n_pages) ? p : -1, page);
                    if (is_page(p, a.n_pages)) device_add(a.refs + p, -1);
                    device_store(a.refs + page, 1);
                    a.table[x.at] = page;
                    __hip_atomic_fetch_max(&sh.handed, (int32_t)upto, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                }
            }
            __threadfence();
            __syncthreads();
        }
        base = sum;
        // The last holder of a page keeps it only if the others got their copies.
        for (int64_t e = threadIdx.x; e < total; e += kPageThreads) {
            const Entry x = entry_of(sh, s0, a.max_pages, e);
            const int32_t p = a.table[x.at];
            if (sh.news[x.seq] > have && is_page(p, a.n_pages) && device_load(a.refs + p) != 1) sh.others[x.seq] = true;
        }
        __syncthreads();
        if (const int32_t s = s0 + (int32_t)threadIdx.x; s < a.n_seq) {
            int32_t first, count = 0;
            range(s, first, count);
            const bool fits = count > 0 && (sh.news[threadIdx.x] <= have || (sh.need[threadIdx.x] == 0 && !sh.others[threadIdx.x]));
            ends[s] = fits ? to[s] : from[s];
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        *a.free_count = (int32_t)(have - sh.handed);
        *w.n_copies = sh.handed;
    }
}

// Rows of copied pages, K and V, norms and token ids of all planes: a workgroup a stretch of rows of one page and plane.
template <int kRowBytes>
__global__ __launch_bounds__(kCopyThreads)
void pages_copy_kernel(char* __restrict__ Kc, char* __restrict__ Vc, float* __restrict__ norms_c, int32_t* __restrict__ pos_c, int32_t n_planes,
                       int64_t total_slots, int32_t page_shift, int32_t n_pages, void* workspace) {
    using P = RowCopy<kRowBytes>;
    constexpr int kRows = kCopyThreads / P::kLanes;            // 16, or 32 short ones; a page has 16 or more
    const PagesScratch w(workspace, n_pages);
    const int32_t count = *w.n_copies;
    const int c = threadIdx.x % P::kLanes, r = threadIdx.x / P::kLanes;
    const int64_t per_page = ((int64_t)1 << page_shift) > kRows ? ((int64_t)1 << page_shift) / kRows : 1, items = count * per_page * n_planes;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int64_t pair = i / (per_page * n_planes), rest = i - pair * per_page * n_planes, plane = rest / per_page;
        const int64_t row = (rest - plane * per_page) * kRows + r;
        const int2 p = w.copies[pair];
        if (p.x < 0 || row >= (int64_t)1 << page_shift) continue;
        const int64_t src = plane * total_slots + ((int64_t)p.x << page_shift) + row, dst = plane * total_slots + ((int64_t)p.y << page_shift) + row;
        const Words<P::kWords> k = load_words_stream<P::kWords, P::kStride>(Kc + src * kRowBytes + c * 16);
        const Words<P::kWords> v = load_words_stream<P::kWords, P::kStride>(Vc + src * kRowBytes + c * 16);
        store_words<P::kWords, P::kStride>(Kc + dst * kRowBytes + c * 16, k);
        store_words<P::kWords, P::kStride>(Vc + dst * kRowBytes + c * 16, v);
        if (c == 0) {
            norms_c[dst] = norms_c[src];
            pos_c[dst] = pos_c[src];
        }
    }
}

// Entries behind the rows to keep give up their pages.
__global__ __launch_bounds__(kPageThreads)
void pages_release_kernel(const PagesArgs a, const int32_t* __restrict__ keep, void* workspace) {
    __shared__ PagesShared sh;
    const PagesScratch w(workspace, a.n_pages);
    auto range = [&](int32_t s, int32_t& first, int32_t& count) {
        const int64_t rows = keep[s] < 0 ? 0 : keep[s], from = (rows + (1 << a.page_shift) - 1) >> a.page_shift;
        if (from >= a.max_pages) return;
        first = (int32_t)from;
        count = a.max_pages - first;
    };
    for_entries(sh, a, range, [&](int32_t, const Entry& x) {
        const int32_t p = x.at < 0 ? -1 : a.table[x.at];
        if (is_page(p, a.n_pages)) device_store(w.last + p, -1);
    });
    __threadfence();
    __syncthreads();
    for_entries(sh, a, range, [&](int32_t, const Entry& x) {
        const int32_t p = x.at < 0 ? -1 : a.table[x.at];
        if (!is_page(p, a.n_pages)) return;
        device_add(a.refs + p, -1);
        __hip_atomic_fetch_max(w.last + p, (int32_t)x.at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    __threadfence();
    __syncthreads();
    auto freed = [&](const Entry& x, int32_t p) {
        return x.at >= 0 && is_page(p, a.n_pages) && device_load(a.refs + p) <= 0 && device_load(w.last + p) == (int32_t)x.at;
    };
    int64_t all = 0, sum = 0;
    for_entries(sh, a, range, [&](int32_t, const Entry& x) {
        int64_t these;
        (void)block_prefix(freed(x, x.at < 0 ? -1 : a.table[x.at]) ? 1u : 0u, sh.waves, these);
        all += these;
    });
    int64_t have = *a.free_count;
    have = have < 0 ? 0 : (have > a.n_pages ? a.n_pages : have);
    __syncthreads();
    for_entries(sh, a, range, [&](int32_t, const Entry& x) {
        const int32_t p = x.at < 0 ? -1 : a.table[x.at];
        const bool mine = freed(x, p);
        int64_t these;
        const int64_t upto = sum + block_prefix(mine ? 1u : 0u, sh.waves, these);
        sum += these;
        if (mine && have + all - upto < a.n_pages) a.free_pages[have + all - upto] = p;       // the first on top
        if (x.at >= 0) a.table[x.at] = -1;
    });
    if (threadIdx.x == 0) *a.free_count = (int32_t)(have + all < a.n_pages ? have + all : a.n_pages);
}

}  // namespace

size_t pages_workspace_bytes(int64_t n_pages) { return 16 + (size_t)n_pages * 16; }

l2kv_status pages_init_dispatch(const PagesArgs& a, hipStream_t stream) {
    const int64_t n = (int64_t)a.n_seq * a.max_pages > a.n_pages ? (int64_t)a.n_seq * a.max_pages : a.n_pages;
    const int64_t blocks = (n + kForkThreads - 1) / kForkThreads;
    hipLaunchKernelGGL(pages_init_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(kForkThreads), 0, stream, a);
    return launch_status();
}

l2kv_status pages_fork_dispatch(const int32_t* table_in, const int32_t* lens_in, int32_t n_in, const int32_t* parents, const PagesArgs& out,
                                int32_t* lens_out, hipStream_t stream) {
    const int64_t blocks = ((int64_t)out.n_seq * out.max_pages + kForkThreads - 1) / kForkThreads;
    hipLaunchKernelGGL(pages_fork_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(kForkThreads), 0, stream, table_in, lens_in, n_in,
                       parents, out, lens_out);
    return launch_status();
}

l2kv_status pages_reserve_dispatch(const PagesArgs& a, const int32_t* from, const int32_t* to, int32_t* ends, l2kv_dtype dt, int32_t n_planes,
                                   int32_t D, void* Kc, void* Vc, float* norms_c, int32_t* pos_c, void* workspace, hipStream_t stream) {
    hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(kPageThreads), 0, stream, a, from, to, ends, workspace);
    if (l2kv_status st = launch_status(); st != L2KV_OK) return st;
    const int64_t rows = (int64_t)a.n_seq * n_planes << a.page_shift, blocks = (rows + 15) / 16;
    const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048));
    const int64_t slots = (int64_t)a.n_pages << a.page_shift;
#define L2KV_COPY(RB)                                                                                                             \
    hipLaunchKernelGGL((pages_copy_kernel<RB>), grid, dim3(kCopyThreads), 0, stream, static_cast<char*>(Kc), static_cast<char*>(Vc), norms_c, \
                       pos_c, n_planes, slots, a.page_shift, a.n_pages, workspace)
    switch (D * (dt == L2KV_F32 ? 4 : 2)) {
        case 128: L2KV_COPY(128); break;
        case 256: L2KV_COPY(256); break;
        default: L2KV_COPY(512); break;
    }
#undef L2KV_COPY
    return launch_status();
}

l2kv_status pages_release_dispatch(const PagesArgs& a, const int32_t* keep, void* workspace, hipStream_t stream) {
    hipLaunchKernelGGL(pages_release_kernel, dim3(1), dim3(kPageThreads), 0, stream, a, keep, workspace);
    return launch_status();
}

}  // namespace l2kv
