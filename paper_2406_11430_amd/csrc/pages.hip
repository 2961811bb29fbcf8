// Pages of a cache that sequences share: forking, reserving room (with copies of pages that others hold too) and releasing.
//
// A page has refs[page] holders, the entries of page tables that name it; those without any are numbered in free_pages[0 .. free_count),
// the next to be handed out last.  Which page an entry gets, and where a released page goes, is decided by the order of the entries
// (sequence after sequence, page after page) and by nothing else: counts are added up with atomics, whose order does not
// matter, and of the entries that name one page the last is found with an atomic maximum.
//
// The tables are small (64 sequences of 500 pages: 128 KB) and every decision needs all those before it, so one workgroup works through them,
// 1024 sequences and 2048 entries at a time; up to 8192 entries stay in LDS from phase to phase.  It is bound by the
// memory round trips that follow one another and by the fetch of its own instructions.  The copies are a launch of their own behind it.
// One more row for each of 64 sequences 8 us with the (empty) copy; release, fork and reservation of 32 branches of 1000 to 2000 rows with 34 MB copied, 32 us:
// 5 + 2 + 7 and the copy 13, at 5.2 TB/s.  A reservation is one workgroup's whatever its size, and grows with it: 64 new sequences of 64 pages 24 us, of 140
// 49, of 250 (beyond what LDS keeps) 79, of 8192 2300; one of 8192 40.  (Releases of that many are spread: pages_release_begin_kernel.)
#include "l2kv_device.hpp"
#include "l2kv_host.hpp"

namespace l2kv {
namespace {

constexpr int kPageThreads = 1024, kKeptEntries = 8192, kPageWaves = kPageThreads / kWaveSize;
constexpr int kForkThreads = 256, kCopyThreads = 256;

// In the workspace: of every page how many of its holders are left when the entries at hand are taken off, and the last of those entries;
// pages to copy, {from, to}, and their number.  (A release of large tables has the free pages before it, and those freed by each
// workgroup, in the same places.)
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
    int32_t upto[kPageThreads];            // entries of the sequences up to it
    int32_t waves[kPageWaves];
    int32_t news[kPageThreads];            // reserving: new pages wanted up to the end of a sequence
    int32_t need[kPageThreads];            // of them by itself
    bool others[kPageThreads];             // it would write a page that others hold as well
    int32_t handed, copied;                // new pages handed out, those of them that are copies
    // entries that are looked at in every phase (place in the table, page, sequence), where they are few enough
    int32_t at[kKeptEntries], page[kKeptEntries];
    uint16_t seq[kKeptEntries];
    bool flag[kKeptEntries];               // wants a new page, gives its page back: found out once
    int32_t top[kPageThreads];             // the first pages to be handed out, asked for ahead
};

// Where there are few entries, what is asked about their pages is counted in LDS, in the room that more entries would take: open addressing,
// page, number of entries that name it, the last of them.  (Counted in memory, two round trips more: a step of 32 branches with
// copies 35.3 us, 33.2 so.)  And as all of them come at once,
// what one pass has found out of them the next has in registers (32.0).
constexpr int kSeenEntries = 2048, kSeenSlots = 4096, kSeenBits = 12;
static_assert(kSeenEntries + kSeenSlots + kSeenSlots / 2 <= kKeptEntries, "room for pages, numbers and last entries");
struct Seen {
    PagesShared& sh;
    __device__ __forceinline__ int32_t* page(uint32_t i) const { return sh.at + kSeenEntries + i; }
    __device__ __forceinline__ int32_t* number(uint32_t i) const { return sh.page + kSeenEntries + i; }
    __device__ __forceinline__ int32_t* last(uint32_t i) const {
        return (i < kSeenSlots / 2 ? sh.at : sh.page) + kSeenEntries + kSeenSlots + i % (kSeenSlots / 2);
    }
    __device__ __forceinline__ void clear() const {
        for (uint32_t i = threadIdx.x; i < kSeenSlots; i += kPageThreads) *page(i) = -1, *number(i) = 0, *last(i) = -1;
    }
    static __device__ __forceinline__ uint32_t first(int32_t p) { return (uint32_t)p * 2654435769u >> (32 - kSeenBits); }
    __device__ __forceinline__ void add(int32_t p, int32_t at) const {
        uint32_t i = first(p);
        for (;; i = (i + 1) % kSeenSlots) {                    // half of the slots stay free
            int32_t was = -1;
            if (__hip_atomic_compare_exchange_strong(page(i), &was, p, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) || was == p) break;
        }
        (void)__hip_atomic_fetch_add(number(i), 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        (void)__hip_atomic_fetch_max(last(i), at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    // of a page that was added
    __device__ __forceinline__ uint32_t find(int32_t p) const {
        uint32_t i = first(p);
        while (*page(i) != p) i = (i + 1) % kSeenSlots;
        return i;
    }
};

// Inclusive prefix sum over the workgroup, and the sum of all; below 2^31.
__device__ __forceinline__ int32_t block_prefix(int32_t v, int32_t (&waves)[kPageWaves], int32_t& total) {
    const int lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
    const int32_t mine = (int32_t)wave_inclusive_sum((uint32_t)v);
    __syncthreads();                       // what was in `waves` is not read any more
    if (lane == kWaveSize - 1) waves[wave] = mine;
    __syncthreads();
    const int32_t all = (int32_t)wave_inclusive_sum((uint32_t)waves[lane % kPageWaves]);      // of each 16 lanes' copies; the first are enough
    total = __builtin_amdgcn_readlane(all, kPageWaves - 1);
    return mine + (wave == 0 ? 0 : __shfl(all, wave - 1));
}

// Counts and numbers of pages are this workgroup's alone while it runs: atomics and loads of its own scope, which the die's L2 answers.
__device__ __forceinline__ int32_t own_load(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void own_store(int32_t* p, int32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void own_add(int32_t* p, int32_t v) { (void)__hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void own_max(int32_t* p, int32_t v) { (void)__hip_atomic_fetch_max(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

// The same of what this workgroup has loaded before: not from the L1, which additions by way of the L2 may have left behind.
__device__ __forceinline__ int32_t own_load_again(int32_t* p) { return __hip_atomic_fetch_or(p, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ bool is_page(int32_t p, int32_t n_pages) { return p >= 0 && p < n_pages; }

// kPer consecutive entries of a lane: place in the table (-1: none), sequence among the 1024 at hand, page (-1: none), whether it is its
// sequence's last.  (Two: a kernel that works through eight is 33 KB of instructions that every call fetches anew, 41 us a step of 32 branches,
// 31 so; with one tables of 64 sequences of 250 pages take 114 us, 100 with two.)
constexpr int kPer = 2, kEntries = kPageThreads * kPer;
static_assert(kSeenEntries <= kEntries, "few entries come once");
struct Entries {
    int32_t at[kPer], seq[kPer], page[kPer];
    bool last[kPer];
    __device__ __forceinline__ void load(const PagesShared& sh, const PagesArgs& a, int32_t s0, int32_t e0, int32_t total) {
        const int32_t first = e0 + (int32_t)threadIdx.x * kPer;
        int32_t lo = 0;                                        // the first sequence whose entries reach beyond it
#pragma unroll
        for (int step = kPageThreads / 2; step > 0; step /= 2) lo = sh.upto[lo + step - 1] <= first ? lo + step : lo;
        int32_t begin = lo == 0 ? 0 : sh.upto[lo - 1], end = sh.upto[lo], index = sh.first[lo];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int32_t e = first + k;
            at[k] = -1, page[k] = -1, seq[k] = lo, last[k] = false;
            if (e >= total) continue;
            while (end <= e) ++lo, begin = end, end = sh.upto[lo], index = sh.first[lo];
            seq[k] = lo;
            at[k] = (s0 + lo) * a.max_pages + index + (e - begin);
            last[k] = e + 1 == end;
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (at[k] >= 0) page[k] = a.table[at[k]];
#pragma unroll
        for (int k = 0; k < kPer; ++k) page[k] = is_page(page[k], a.n_pages) ? page[k] : -1;
    }
    __device__ __forceinline__ void keep(PagesShared& sh, int32_t e0) const {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int32_t e = e0 + (int32_t)threadIdx.x * kPer + k;
            if (e >= kKeptEntries) continue;
            sh.at[e] = at[k];
            sh.page[e] = page[k];
            sh.seq[e] = (uint16_t)seq[k];
        }
    }
    __device__ __forceinline__ void kept(const PagesShared& sh, int32_t e0, int32_t total) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int32_t e = e0 + (int32_t)threadIdx.x * kPer + k;
            at[k] = -1, page[k] = -1, seq[k] = 0, last[k] = false;
            if (e >= total) continue;
            at[k] = sh.at[e];
            page[k] = sh.page[e];
            seq[k] = sh.seq[e];
            last[k] = e + 1 == sh.upto[seq[k]];
        }
    }
};

// The entries of up to 1024 sequences from s0 on, laid end to end; `range` gives the first entry of a sequence and how many there are.
template <typename R> __device__ __forceinline__ int32_t lay_out(PagesShared& sh, int32_t s0, int32_t n_seq, R&& range) {
    int32_t first = 0, count = 0;
    if (const int32_t s = s0 + (int32_t)threadIdx.x; s < n_seq) range(s, first, count);
    int32_t total;
    const int32_t upto = block_prefix(count, sh.waves, total);
    sh.first[threadIdx.x] = first;
    sh.upto[threadIdx.x] = upto;
    __syncthreads();
    return total;
}

// All entries that `range` gives, 1024 sequences and kEntries entries at a time.  Where they fit they are kept, and nothing of the
// tables and ranges is read again.
template <typename R> struct AllEntries {
    PagesShared& sh;
    const PagesArgs& a;
    R range;
    int32_t total;
    bool kept, few;
    __device__ __forceinline__ AllEntries(PagesShared& sh_, const PagesArgs& a_, R range_) : sh(sh_), a(a_), range(range_) {
        Seen{sh}.clear();
        total = lay_out(sh, 0, a.n_seq, range);
        kept = a.n_seq <= kPageThreads && total <= kKeptEntries;
        few = kept && total <= kSeenEntries;
        if (!kept) return;
        for (int32_t e0 = 0; e0 < total; e0 += kEntries) {
            Entries x;
            x.load(sh, a, 0, e0, total);
            x.keep(sh, e0);
        }
        __syncthreads();
    }
    // of the sequences from s0 on, which are laid out
    template <typename F> __device__ __forceinline__ void each_of(int32_t s0, F&& visit) {
        for (int32_t e0 = 0; e0 < total; e0 += kEntries) {
            Entries x;
            if (kept) x.kept(sh, e0, total);
            else x.load(sh, a, s0, e0, total);
            visit(x, e0);
        }
        __syncthreads();
    }
    // What find(x, flags) says of a lane's entries, and how many it is true of: found out the first time, and again where it is not kept.
    template <typename F> __device__ __forceinline__ int32_t flags_of(const Entries& x, int32_t e0, bool first, bool (&flags)[kPer], F&& find) {
        bool* const at = sh.flag + (kept ? e0 + (int32_t)threadIdx.x * kPer : 0);
        if (first || !kept) {
            find(x, flags);
            if (kept) {
#pragma unroll
                for (int k = 0; k < kPer; ++k)
                    if (e0 + (int32_t)threadIdx.x * kPer + k < kKeptEntries) at[k] = flags[k];
            }
        } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) flags[k] = x.at[k] >= 0 && at[k];
        }
        int32_t n = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k) n += flags[k] ? 1 : 0;
        return n;
    }
    template <typename F> __device__ __forceinline__ void each(F&& visit) {
        for (int32_t s0 = 0; s0 < a.n_seq; s0 += kPageThreads) {
            if (!kept) total = lay_out(sh, s0, a.n_seq, range);
            each_of(s0, visit);
        }
    }
};

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
        if (page >= 0) (void)__hip_atomic_fetch_add(a.refs + page, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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
    // the rows of the first sequences beside the number of free pages, not behind it
    const bool early = (int32_t)threadIdx.x < a.n_seq;
    const int32_t early_from = early ? from[threadIdx.x] : 0, early_to = early ? to[threadIdx.x] : 0;
    int32_t have = *a.free_count;
    have = have < 0 ? 0 : (have > a.n_pages ? a.n_pages : have);
    const int32_t top = (int32_t)threadIdx.x < have ? a.free_pages[have - 1 - (int32_t)threadIdx.x] : -1;
    int32_t own_from = 0, own_to = 0;                          // of the sequence that `range` was asked about last
    auto range = [&](int32_t s, int32_t& first, int32_t& count) {
        const int64_t b = own_from = s < kPageThreads ? early_from : from[s], e = own_to = s < kPageThreads ? early_to : to[s];
        if (b < 0 || e <= b || e > (int64_t)a.max_pages << a.page_shift) return;
        first = (int32_t)(b >> a.page_shift);
        count = (int32_t)((e - 1) >> a.page_shift) - first + 1;
    };
    AllEntries all(sh, a, range);
    // Pages that have one holder are that entry's own: nothing has to be counted for them (the same entry twice in a table has two).
    bool shared = false;
    all.each([&](const Entries& x, int32_t) {
        int32_t refs[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) refs[k] = x.page[k] < 0 ? 1 : own_load(a.refs + x.page[k]);
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            if (x.page[k] < 0) continue;
            shared |= refs[k] != 1;
            if (all.few) continue;
            own_store(w.left + x.page[k], refs[k] - 1);             // the same whoever does it: without the one who asks
            own_store(w.last + x.page[k], -1);
        }
    });
    shared = __syncthreads_or(shared) != 0;
    const Seen seen{sh};
    if (shared && all.few) {
        all.each([&](const Entries& x, int32_t) {
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (x.page[k] >= 0) seen.add(x.page[k], x.at[k]);
        });
    } else if (shared) {
        all.each([&](const Entries& x, int32_t) {
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                if (x.page[k] < 0) continue;
                own_add(w.left + x.page[k], -1);
                own_max(w.last + x.page[k], x.at[k]);
            }
        });
    }
    sh.top[threadIdx.x] = top;
    // Which entries want a new page: those without one, and of a page's holders all but the last if all of them ask, else all.
    auto wanted = [&](const Entries& x, bool (&want)[kPer]) {
        int32_t left[kPer], last[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            left[k] = -1, last[k] = x.at[k];
            if (!shared || x.page[k] < 0) continue;
            if (all.few) {
                const uint32_t i = seen.find(x.page[k]);
                left[k] = own_load(a.refs + x.page[k]) - 1 - *seen.number(i);
                last[k] = *seen.last(i);
            } else {
                left[k] = own_load(w.left + x.page[k]);
                last[k] = own_load(w.last + x.page[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k) want[k] = x.at[k] >= 0 && (x.page[k] < 0 || left[k] >= 0 || last[k] != x.at[k]);
    };
    int32_t base = 0;                                          // new pages wanted by the sequences before these
    bool once_want[kPer];                                      // of few entries: what the first pass has found out of the lane's
    int32_t once_upto = 0;
    if (threadIdx.x == 0) sh.handed = sh.copied = 0;
    for (int32_t s0 = 0; s0 < a.n_seq; s0 += kPageThreads) {
        if (!all.kept) all.total = lay_out(sh, s0, a.n_seq, range);
        sh.news[threadIdx.x] = 0;
        sh.need[threadIdx.x] = 0;
        sh.others[threadIdx.x] = false;
        __syncthreads();
        // how many are wanted up to the end of each sequence
        int32_t sum = base;
        all.each_of(s0, [&](const Entries& x, int32_t e0) {
            bool want[kPer];
            const int32_t mine = all.flags_of(x, e0, true, want, wanted);
            int32_t these, so_far = sum + block_prefix(mine, sh.waves, these) - mine;
            sum += these;
            once_upto = so_far;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                once_want[k] = want[k];
                so_far += want[k] ? 1 : 0;
                if (want[k]) (void)__hip_atomic_fetch_add(&sh.need[x.seq[k]], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                if (x.last[k]) sh.news[x.seq[k]] = so_far;
            }
        });
        const int32_t end = sum;
        // who gets one
        sum = base;
        all.each_of(s0, [&](const Entries& x, int32_t e0) {
            bool want[kPer];
            int32_t so_far = once_upto;
            if (all.few) {
#pragma unroll
                for (int k = 0; k < kPer; ++k) want[k] = once_want[k];
            } else {
                const int32_t mine = all.flags_of(x, e0, false, want, wanted);
                int32_t these;
                so_far = sum + block_prefix(mine, sh.waves, these) - mine;
                sum += these;
            }
            int32_t page[kPer], number[kPer], most = 0;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                so_far += want[k] ? 1 : 0;
                number[k] = want[k] && sh.news[x.seq[k]] <= have ? so_far : 0;
                if (number[k] > 0) page[k] = number[k] <= kPageThreads ? sh.top[number[k] - 1] : a.free_pages[have - number[k]];
            }
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                if (number[k] == 0) continue;
                const int32_t fresh = is_page(page[k], a.n_pages) ? page[k] : 0;
                if (x.page[k] >= 0) {
                    own_add(a.refs + x.page[k], -1);
                    // in no order: copies do not meet
                    w.copies[__hip_atomic_fetch_add(&sh.copied, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)] = make_int2(x.page[k], fresh);
                }
                own_store(a.refs + fresh, 1);
                a.table[x.at[k]] = fresh;
                if (all.kept) sh.page[e0 + (int32_t)threadIdx.x * kPer + k] = -1;      // not asked about below
                most = number[k];
            }
            if (most > 0) (void)__hip_atomic_fetch_max(&sh.handed, most, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        });
        // The last holder of a page keeps it only if the others got their copies.
        if (end > have) {
            all.each_of(s0, [&](const Entries& x, int32_t) {
#pragma unroll
                for (int k = 0; k < kPer; ++k)
                    if (x.page[k] >= 0 && sh.news[x.seq[k]] > have && own_load_again(a.refs + x.page[k]) != 1) sh.others[x.seq[k]] = true;
            });
        }
        base = end;
        if (const int32_t s = s0 + (int32_t)threadIdx.x; s < a.n_seq) {
            // (a lane's sequence is the one that it laid out)
            const bool fits = own_from >= 0 && own_to > own_from && own_to <= (int64_t)a.max_pages << a.page_shift && (sh.news[threadIdx.x] <= have || (sh.need[threadIdx.x] == 0 && !sh.others[threadIdx.x]));
            ends[s] = fits ? own_to : own_from;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        *a.free_count = have - sh.handed;
        *w.n_copies = sh.copied;
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
        if (row >= (int64_t)1 << page_shift) continue;
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
    int32_t have = *a.free_count;
    auto range = [&](int32_t s, int32_t& first, int32_t& count) {
        const int64_t rows = keep[s] < 0 ? 0 : keep[s], from = (rows + (1 << a.page_shift) - 1) >> a.page_shift;
        if (from >= a.max_pages) return;
        first = (int32_t)from;
        count = a.max_pages - first;
    };
    AllEntries every(sh, a, range);
    const Seen seen{sh};
    if (!every.few) {
        every.each([&](const Entries& x, int32_t) {
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (x.page[k] >= 0) own_store(w.last + x.page[k], -1);
        });
    }
    every.each([&](const Entries& x, int32_t) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            if (x.page[k] < 0) continue;
            if (every.few) {
                seen.add(x.page[k], x.at[k]);
            } else {
                own_add(a.refs + x.page[k], -1);
                own_max(w.last + x.page[k], x.at[k]);
            }
        }
    });
    // Of the entries that name a page without holders the last gives it back; the first of these on top.
    auto freed = [&](const Entries& x, bool (&mine)[kPer]) {
        int32_t refs[kPer], last[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            refs[k] = x.page[k] < 0 ? 1 : own_load(a.refs + x.page[k]);
            last[k] = x.page[k] < 0 || every.few ? 0 : own_load(w.last + x.page[k]);
        }
        if (every.few) {
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                if (x.page[k] < 0) continue;
                const uint32_t i = seen.find(x.page[k]);
                refs[k] -= *seen.number(i), last[k] = *seen.last(i);
                if (last[k] == x.at[k]) own_store(a.refs + x.page[k], refs[k]);      // asked about once; who is not the last does not look
            }
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k) mine[k] = x.page[k] >= 0 && refs[k] <= 0 && last[k] == x.at[k];
    };
    have = have < 0 ? 0 : (have > a.n_pages ? a.n_pages : have);
    int32_t all = 0, sum = 0;
    if (!every.few) {
        every.each([&](const Entries& x, int32_t e0) {
            bool mine[kPer];
            int32_t these;
            (void)block_prefix(every.flags_of(x, e0, true, mine, freed), sh.waves, these);
            all += these;
        });
    }
    every.each([&](const Entries& x, int32_t e0) {
        bool mine[kPer];
        int32_t these;
        int32_t upto = sum + block_prefix(every.flags_of(x, e0, every.few, mine, freed), sh.waves, these);
        sum += these;
        if (every.few) all = these;                            // few entries come once, all together
#pragma unroll
        for (int k = kPer - 1; k >= 0; --k) {
            if (mine[k]) {
                if (have + all - upto < a.n_pages) a.free_pages[have + all - upto] = x.page[k];
                --upto;
            }
            if (x.at[k] >= 0) a.table[x.at[k]] = -1;
        }
    });
    if (threadIdx.x == 0) *a.free_count = have + all < a.n_pages ? have + all : a.n_pages;
}

// The same for large tables, by many workgroups with a stretch of the table each and a launch for every phase: 64 sequences of 8192 pages 24 us,
// of 140 or 250 18.
struct LargeRelease {
    int32_t *have, *counts;                // free pages before, pages freed by each workgroup
    __device__ __forceinline__ explicit LargeRelease(const PagesScratch& w) : have(w.n_copies + 1), counts(reinterpret_cast<int32_t*>(w.copies)) {}
};
template <typename F>
__device__ __forceinline__ void for_stretch(const PagesArgs& a, const int32_t* keep, F&& visit) {
    const int64_t all = (int64_t)a.n_seq * a.max_pages, each = (all + gridDim.x - 1) / gridDim.x;
    const int64_t first = blockIdx.x * each, end = first + each < all ? first + each : all;
    for (int64_t e0 = first; e0 < end; e0 += kPageThreads) {
        const int64_t e = e0 + threadIdx.x;
        int32_t at = -1, page = -1;
        if (e < end) {
            const uint32_t s = (uint32_t)e / (uint32_t)a.max_pages, i = (uint32_t)e - s * (uint32_t)a.max_pages;
            const int64_t rows = keep[s] < 0 ? 0 : keep[s];
            if (i >= (rows + (1 << a.page_shift) - 1) >> a.page_shift) {
                at = (int32_t)e;
                page = a.table[e];
                page = is_page(page, a.n_pages) ? page : -1;
            }
        }
        visit(at, page);
    }
}

__global__ __launch_bounds__(kPageThreads)
void pages_release_begin_kernel(const PagesArgs a, const int32_t* __restrict__ keep, void* workspace) {
    const PagesScratch w(workspace, a.n_pages);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        const int32_t have = *a.free_count;
        *LargeRelease(w).have = have < 0 ? 0 : (have > a.n_pages ? a.n_pages : have);
    }
    for_stretch(a, keep, [&](int32_t, int32_t page) {
        if (page >= 0) w.last[page] = -1;
    });
}
__global__ __launch_bounds__(kPageThreads)
void pages_release_holders_kernel(const PagesArgs a, const int32_t* __restrict__ keep, void* workspace) {
    const PagesScratch w(workspace, a.n_pages);
    for_stretch(a, keep, [&](int32_t at, int32_t page) {
        if (page < 0) return;
        (void)__hip_atomic_fetch_add(a.refs + page, -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        (void)__hip_atomic_fetch_max(w.last + page, at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
}
__global__ __launch_bounds__(kPageThreads)
void pages_release_count_kernel(const PagesArgs a, const int32_t* __restrict__ keep, void* workspace) {
    const PagesScratch w(workspace, a.n_pages);
    int32_t n = 0;
    for_stretch(a, keep, [&](int32_t at, int32_t page) { n += page >= 0 && a.refs[page] <= 0 && w.last[page] == at; });
    __shared__ int32_t waves[kPageWaves];
    int32_t all;
    (void)block_prefix(n, waves, all);
    if (threadIdx.x == 0) LargeRelease(w).counts[blockIdx.x] = all;
}
__global__ __launch_bounds__(kPageThreads)
void pages_release_end_kernel(const PagesArgs a, const int32_t* __restrict__ keep, void* workspace) {
    const PagesScratch w(workspace, a.n_pages);
    const LargeRelease r(w);
    __shared__ int32_t waves[kPageWaves];
    const int32_t have = *r.have, mine = threadIdx.x < gridDim.x ? r.counts[threadIdx.x] : 0;      // kLargeWorkgroups at most
    int32_t all, sum;
    (void)block_prefix(mine, waves, all);
    (void)block_prefix(threadIdx.x < blockIdx.x ? mine : 0, waves, sum);
    for_stretch(a, keep, [&](int32_t at, int32_t page) {
        const bool freed = page >= 0 && a.refs[page] <= 0 && w.last[page] == at;
        int32_t these;
        const int32_t upto = sum + block_prefix(freed ? 1 : 0, waves, these);
        sum += these;
        if (freed && have + all - upto < a.n_pages) a.free_pages[have + all - upto] = page;
        if (at >= 0) a.table[at] = -1;
    });
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.free_count = have + all < a.n_pages ? have + all : a.n_pages;
}

// Entries that one workgroup looks at in the time of the three launches more, and those that a workgroup of many has.
constexpr int64_t kLargeEntries = 4096, kLargeEach = 2048, kLargeWorkgroups = kPageThreads;

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
    // as if every sequence had a page copied, and a workgroup for each compute unit at least
    const int64_t rows = (int64_t)a.n_seq * n_planes << a.page_shift, blocks = (rows + 15) / 16;
    const dim3 grid((unsigned)(blocks < 256 ? 256 : (blocks < 2048 ? blocks : 2048)));
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
    const int64_t entries = (int64_t)a.n_seq * a.max_pages;
    if (entries > kLargeEntries) {
        int64_t n = (entries + kLargeEach - 1) / kLargeEach;
        n = n < kLargeWorkgroups ? n : kLargeWorkgroups;
        n = n < 2 * (int64_t)a.n_pages ? n : 2 * (int64_t)a.n_pages;       // that their counts have room for
        for (auto kernel : {pages_release_begin_kernel, pages_release_holders_kernel, pages_release_count_kernel, pages_release_end_kernel}) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(kPageThreads), 0, stream, a, keep, workspace);
            if (l2kv_status st = launch_status(); st != L2KV_OK) return st;
        }
        return L2KV_OK;
    }
    hipLaunchKernelGGL(pages_release_kernel, dim3(1), dim3(kPageThreads), 0, stream, a, keep, workspace);
    return launch_status();
}

}  // namespace l2kv
