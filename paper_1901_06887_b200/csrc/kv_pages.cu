// The pages of a cache: handed out, shared, given back, moved together, and copied.
//
// A page's reference counts the rows whose table holds it; a page nobody holds is free.  Pages are handed out lowest first, in the order of
// the call's rows, so that results are the same every time.  A shared page is always full: a fork shares the full pages of its parent and copies the
// one that is partly filled, so nothing that a row appends is seen by another.
//
// Split.  Bookkeeping is a handful of dependent steps over small integers (who comes first, which pages are free, who gets which, write), so it
// is one launch of one team: a CTA, or a cluster of eight where there is more to read than a CTA takes quickly.  What the steps hand on lies in shared
// memory where one CTA is the team and it fits (SMALL), else in scratch: every trip to device memory between two steps costs half a microsecond.  Free pages are
// found by a scan of the references: every warp counts its stretch, the counts are added up, every warp lists its stretch.
//
// Cost.  Bookkeeping is latency: one call behind the other, 64 rows of some 30 pages are forked and released in 13.1 and given a token each in 5.4 us (8 rows of a
// small model: 7.7 and 5.1).  Copies are bytes: 254 MB in and out in 41 us, 6.2 TB/s; many pages of 1, 2, 4 or 8 heads of 128 at 6.5 to 6.7 (a warp takes a head:
// pages of fewer than four heads leave warps idle, which other CTAs make up for).
#include "lm_device.cuh"
#include "lm_host.h"

namespace mt {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kTeam = 8;                      // CTAs of a large call
constexpr int kFew = 4;                       // tokens that a thread adds by itself
constexpr int kSmall = 1024, kSmallRows = 4096, kSmallList = 4096;            // places, rows and free pages that SMALL holds

__device__ __forceinline__ uint32_t remote_u32(const void* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return v;
}

struct Shared {
    int warp_free[kWarps];                    // free pages of each warp's stretch, then those before it in the CTA
    int free, holes;                          // of this CTA
    long long scan[2][kWarps];
};

// What the steps of a call hand on.
struct SmallHand {
    int32_t rows[kSmall], other[kSmall], owner[kSmallRows], info[kSmall], list[kSmallList];
    long long place[2 * kSmall];
};
struct Hand {
    SmallHand* small;
    const int32_t *rows, *other;              // of the call
    int32_t *owner, *info;
    long long* place;
    int32_t *near, *far;                      // free pages: the first `most_near` of them, the rest
    int most_near;
    __device__ __forceinline__ void put(int rank, int page) const {
        if (rank < most_near) near[rank] = page; else far[rank] = page;
    }
};
// (written by another CTA of the team, perhaps)
template <bool SMALL, class T>
__device__ __forceinline__ T fetch(const T* p) { return SMALL ? *p : __ldcg(p); }
template <bool SMALL>
__device__ __forceinline__ int free_page(const Hand& h, long long rank) { return rank < h.most_near ? h.near[rank] : __ldcg(h.far + rank); }

struct Team {
    int rank, size, warp, lane;               // warp: of the whole team
    int thread, threads;
    __device__ __forceinline__ void sync() const {
        if (size > 1) cluster_sync_all(); else __syncthreads();
    }
};
__device__ __forceinline__ Team team_of(int size) {
    Team t;
    t.rank = size > 1 ? blockIdx.x : 0;       // one cluster is the whole grid
    t.size = size;
    t.lane = threadIdx.x & 31;
    t.warp = t.rank * kWarps + (threadIdx.x >> 5);
    t.thread = t.rank * kThreads + threadIdx.x;
    t.threads = size * kThreads;
    return t;
}

// --- free pages
struct Stretch {
    int begin, end;
};
__device__ __forceinline__ Stretch stretch_of(const Team& t, int n_pages) {
    const int64_t each = (((int64_t)n_pages + t.size * kWarps - 1) / (t.size * kWarps) + 127) / 128 * 128;
    const int64_t a = each * t.warp, b = a + each;
    return {(int)min(a, (int64_t)n_pages), (int)min(b, (int64_t)n_pages)};
}
// Bit e: page at + e is free.  Pages behind the end are not.
__device__ __forceinline__ uint32_t free_of_four(const int32_t* refs, int at, int end) {
    uint32_t m = 0;
    if (at + 3 < end) {
        const int4 r = __ldcg(reinterpret_cast<const int4*>(refs + at));
        m = (r.x <= 0 ? 1u : 0u) | (r.y <= 0 ? 2u : 0u) | (r.z <= 0 ? 4u : 0u) | (r.w <= 0 ? 8u : 0u);
    } else {
        for (int e = 0; e < 4; ++e)
            if (at + e < end && __ldcg(refs + at + e) <= 0) m |= 1u << e;
    }
    return m;
}
// (returns the mask of the lane's first four pages, which for_stretch need not read again)
__device__ __forceinline__ uint32_t count_free(const Team& t, Shared& s, const int32_t* refs, int n_pages) {
    const Stretch x = stretch_of(t, n_pages);
    const uint32_t first = x.begin + 4 * t.lane < x.end ? free_of_four(refs, x.begin + 4 * t.lane, x.end) : 0;
    int n = __popc(first);
    for (int at = x.begin + 128 + 4 * t.lane; at < x.end; at += 128) n += __popc(free_of_four(refs, at, x.end));
#pragma unroll
    for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    if (t.lane == 0) s.warp_free[threadIdx.x >> 5] = n;
    __syncthreads();
    if (threadIdx.x < 32) {
        const int v = s.warp_free[threadIdx.x];
        int incl = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, d);
            if (t.lane >= d) incl += y;
        }
        s.warp_free[threadIdx.x] = incl - v;
        if (threadIdx.x == 31) { s.free = incl; s.holes = 0; }
    }
    return first;
}
// (behind a sync of the team) free pages before this CTA's first, and all of them
__device__ __forceinline__ void total_free(const Team& t, const Shared& s, int& before, int& all) {
    before = 0;
    all = 0;
    for (int r = 0; r < t.size; ++r) {
        const int n = t.size > 1 ? (int)remote_u32(&s.free, r) : s.free;
        if (r < t.rank) before += n;
        all += n;
    }
}
// f(first page of four, mask of the free ones, number of free pages before them), for this warp's stretch
template <class F>
__device__ __forceinline__ void for_stretch(const Team& t, const Shared& s, const int32_t* refs, int n_pages, uint32_t first, int before, F f) {
    const Stretch x = stretch_of(t, n_pages);
    int run = before + s.warp_free[threadIdx.x >> 5];
    for (int base = x.begin; base < x.end; base += 128) {
        const int at = base + 4 * t.lane;
        const uint32_t m = base == x.begin ? first : at < x.end ? free_of_four(refs, at, x.end) : 0;
        const int n = __popc(m);
        int incl = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, d);
            if (t.lane >= d) incl += y;
        }
        if (at < x.end) f(at, m, run + incl - n);
        run += __shfl_sync(0xffffffffu, incl, 31);
    }
}
__device__ __forceinline__ void list_free(const Team& t, const Shared& s, const int32_t* refs, int n_pages, uint32_t first, int before, const Hand& list, int most) {
    for_stretch(t, s, refs, n_pages, first, before, [&](int at, uint32_t m, int rank) {
        for (; m && rank < most; m &= m - 1, ++rank) list.put(rank, at + __ffs(m) - 1);
    });
}

// Sums of the CTA's values before this thread's, and of all, two at a time.
__device__ __forceinline__ void scan_block(Shared& s, long long (&v)[2], long long (&all)[2]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long incl[2] = {v[0], v[1]};
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long y0 = __shfl_up_sync(0xffffffffu, incl[0], d), y1 = __shfl_up_sync(0xffffffffu, incl[1], d);
        if (lane >= d) { incl[0] += y0; incl[1] += y1; }
    }
    if (lane == 31) { s.scan[0][warp] = incl[0]; s.scan[1][warp] = incl[1]; }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        long long of_warps = s.scan[k][lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, of_warps, d);
            if (lane >= d) of_warps += y;
        }
        const long long before = __shfl_sync(0xffffffffu, of_warps, (warp + 31) & 31);
        all[k] = __shfl_sync(0xffffffffu, of_warps, 31);
        v[k] = (warp ? before : 0) + incl[k] - v[k];
    }
    __syncthreads();
}

struct Params {
    mt_kv_pages k;
    int shift;                                // log2 of page_tokens
    int n;
    const int32_t *rows, *other;              // fork: children, parents; reserve: rows, counts; release: rows
    int32_t* copies;
    int64_t* slots;
    int64_t n_slots;
    OpStatus status;
    int team;
    // scratch
    int32_t *owner, *free_list, *info, *staged;
    long long* place;
};

__device__ __forceinline__ bool in(int x, int n) { return (unsigned)x < (unsigned)n; }
__device__ __forceinline__ int pages_of(const Params& p, int len) { return (int)(((unsigned)len + p.k.page_tokens - 1) >> p.shift); }
__device__ __forceinline__ bool good_length(const Params& p, int len) { return len >= 0 && (int64_t)len <= (int64_t)p.k.table_width << p.shift; }
__device__ __forceinline__ int32_t* table_row(const Params& p, int row) { return p.k.tables + (int64_t)row * p.k.table_width; }
__device__ __forceinline__ void give_back(const Params& p, int page, int i) {
    const bool there = in(page, p.k.n_pages);
    const bool held = there && atomicSub(p.k.refs + page, 1) > 0;              // nobody held it: the table is not the pages'
    if (there && !held) atomicAdd(p.k.refs + page, 1);
    if (!held) raise_status(p.status, MT_ERR_INVALID_ARG, i);
}
// The rows of a call: owner[row] is the first place of the call that names it.
template <bool SMALL>
__device__ __forceinline__ Hand hand_of(const Params& p, uint8_t* shared) {
    SmallHand* const s = reinterpret_cast<SmallHand*>(shared);
    if (SMALL) return {s, s->rows, s->other, s->owner, s->info, s->place, s->list, p.free_list, kSmallList};
    return {nullptr, p.rows, p.other, p.owner, p.info, p.place, nullptr, p.free_list, 0};
}
// owner[row] of the rows of the call: nobody yet.
template <bool SMALL>
__device__ __forceinline__ void clear_owners(const Params& p, const Hand& h, const Team& t, bool both) {
    if (SMALL) {
        SmallHand* const s = h.small;
        if ((int)threadIdx.x < p.n) {
            s->rows[threadIdx.x] = p.rows[threadIdx.x];
            if (p.other) s->other[threadIdx.x] = p.other[threadIdx.x];
        }
        for (int r = threadIdx.x; r < p.k.n_rows; r += kThreads) h.owner[r] = 0x7fffffff;
    } else {
        for (int i = t.thread; i < p.n; i += t.threads) {
            const int r = p.rows[i];
            if (in(r, p.k.n_rows)) h.owner[r] = 0x7fffffff;
            const int o = both ? p.other[i] : -1;
            if (in(o, p.k.n_rows)) h.owner[o] = 0x7fffffff;
        }
    }
}
__device__ __forceinline__ void claim_rows(const Params& p, const Hand& h, const Team& t) {
    for (int i = t.thread; i < p.n; i += t.threads) {
        const int r = h.rows[i];
        if (in(r, p.k.n_rows)) atomicMin(h.owner + r, i);
    }
}

template <bool SMALL>
__global__ void __launch_bounds__(kThreads) fork_kernel(const Params p) {
    extern __shared__ __align__(16) uint8_t shared[];
    const Hand h = hand_of<SMALL>(p, shared);
    __shared__ Shared s;
    const Team t = team_of(p.team);
    const int warps = t.size * kWarps;
    pdl_launch_dependents();
    pdl_wait();
    clear_owners<SMALL>(p, h, t, true);
    const uint32_t mask = count_free(t, s, p.k.refs, p.k.n_pages);
    t.sync();
    claim_rows(p, h, t);
    int before, n_free;
    total_free(t, s, before, n_free);
    list_free(t, s, p.k.refs, p.k.n_pages, mask, before, h, p.n);
    t.sync();
    // what a pair needs: info = tokens, -1 refused, -2 nothing to do; a parent that is a child too is read before it changes
    for (int i = t.warp; i < p.n; i += warps) {
        const int child = h.rows[i], parent = h.other[i];
        bool ok = in(child, p.k.n_rows) && in(parent, p.k.n_rows) && fetch<SMALL>(h.owner + child) == i;
        int len = 0;
        if (ok) {
            len = p.k.lengths[parent];
            ok = good_length(p, len) && good_length(p, p.k.lengths[child]);
        }
        if (ok) {
            const int pages = pages_of(p, len);
            const int32_t* const from = table_row(p, parent);
            int32_t* const to = fetch<SMALL>(h.owner + parent) != 0x7fffffff ? p.staged + (int64_t)i * p.k.table_width : nullptr;
            bool mine = true;
            for (int c = t.lane; c < pages; c += 32) {
                const int page = from[c];
                if (!in(page, p.k.n_pages)) mine = false;
                if (to) to[c] = page;
            }
            ok = __all_sync(0xffffffffu, mine);
        }
        if (t.lane == 0) {
            if (!ok) raise_status(p.status, MT_ERR_INVALID_ARG, i);
            h.info[i] = !ok ? -1 : child == parent ? -2 : len;
        }
    }
    t.sync();
    if (t.rank == 0) {                        // who gets which of the free pages
        long long run = 0, all[2];
        for (int i0 = 0; i0 < p.n; i0 += kThreads) {
            const int i = i0 + threadIdx.x;
            const int len = i < p.n ? fetch<SMALL>(h.info + i) : -1;
            long long v[2] = {len > 0 && (len & (p.k.page_tokens - 1)) ? 1 : 0, 0};
            scan_block(s, v, all);
            if (i < p.n) h.place[i] = run + v[0];
            run += all[0];
        }
    }
    t.sync();
    for (int i = t.warp; i < p.n; i += warps) {
        const int child = h.rows[i], parent = h.other[i], len = fetch<SMALL>(h.info + i);
        const int part = len & (p.k.page_tokens - 1), whole = len >> p.shift;
        int from = -1, fresh = -1;
        bool go = len >= 0;
        if (go && part) {
            const long long at = fetch<SMALL>(h.place + i);
            if (at < n_free) {
                fresh = free_page<SMALL>(h, at);
            } else {
                go = false;
                if (t.lane == 0) raise_status(p.status, MT_ERR_OOM, i);
            }
        }
        if (go) {
            const int32_t* const src = fetch<SMALL>(h.owner + parent) != 0x7fffffff ? p.staged + (int64_t)i * p.k.table_width : table_row(p, parent);
            int32_t* const row = table_row(p, child);
            const int old = pages_of(p, p.k.lengths[child]);
            const int now = whole + (part ? 1 : 0);
            for (int c = t.lane; c < max(old, now); c += 32) {
                if (c < old) give_back(p, row[c], i);
                if (c < whole) {
                    const int page = __ldcg(src + c);
                    atomicAdd(p.k.refs + page, 1);
                    row[c] = page;
                } else if (c < now) {
                    row[c] = fresh;
                    p.k.refs[fresh] = 1;
                }
            }
            if (part) from = __ldcg(src + whole);
            __syncwarp();
            if (t.lane == 0) p.k.lengths[child] = len;
        }
        if (t.lane < 3) p.copies[(int64_t)i * 3 + t.lane] = t.lane == 0 ? from : t.lane == 1 ? fresh : fresh >= 0 ? part : 0;
    }
}

template <bool SMALL>
__global__ void __launch_bounds__(kThreads) reserve_kernel(const Params p) {
    extern __shared__ __align__(16) uint8_t shared[];
    const Hand h = hand_of<SMALL>(p, shared);
    __shared__ Shared s;
    const Team t = team_of(p.team);
    const int warps = t.size * kWarps;
    pdl_launch_dependents();
    pdl_wait();
    clear_owners<SMALL>(p, h, t, false);
    const uint32_t mask = count_free(t, s, p.k.refs, p.k.n_pages);
    t.sync();
    claim_rows(p, h, t);
    int before, n_free;
    total_free(t, s, before, n_free);
    t.sync();
    int most = p.k.n_pages;                   // free pages that are wanted
    if (t.rank == 0) {                        // place[2 i]: pages of the rows before, place[2 i + 1]: their tokens
        long long pages = 0, tokens = 0, all[2];
        for (int i0 = 0; i0 < p.n; i0 += kThreads) {
            const int i = i0 + threadIdx.x;
            int need = 0, count = 0;
            if (i < p.n) {
                const int row = h.rows[i];
                count = h.other[i];
                bool ok = in(row, p.k.n_rows) && fetch<SMALL>(h.owner + row) == i && count >= 0;
                int len = 0;
                if (ok) {
                    len = p.k.lengths[row];
                    ok = good_length(p, len) && (int64_t)len + count <= (int64_t)p.k.table_width << p.shift;
                }
                if (ok) need = pages_of(p, len + count) - pages_of(p, len);
                else raise_status(p.status, MT_ERR_INVALID_ARG, i);
                h.info[i] = ok ? len : -1;
                count = max(count, 0);
            }
            long long v[2] = {need, count};
            scan_block(s, v, all);
            if (i < p.n) { h.place[2 * (int64_t)i] = pages + v[0]; h.place[2 * (int64_t)i + 1] = tokens + v[1]; }
            pages += all[0];
            tokens += all[1];
        }
        for (int64_t x = tokens + threadIdx.x; x < p.n_slots; x += kThreads) p.slots[x] = -1;
        if (t.size == 1) most = (int)min(pages, (long long)most);
    }
    list_free(t, s, p.k.refs, p.k.n_pages, mask, before, h, most);
    t.sync();
    // Place i, by `size` lanes of which this is `lane`: a warp, or, for a few tokens, a thread.
    auto place = [&](int i, int lane, int size) {
        const int len = fetch<SMALL>(h.info + i), row = h.rows[i], count = max(h.other[i], 0);
        const long long first = fetch<SMALL>(h.place + 2 * (int64_t)i), out = fetch<SMALL>(h.place + 2 * (int64_t)i + 1);
        bool go = len >= 0;
        int had = 0, need = 0;
        if (go) {
            had = pages_of(p, len);
            need = pages_of(p, len + count) - had;
            if (need > 0 && first + need > n_free) {
                go = false;
                if (lane == 0) raise_status(p.status, MT_ERR_OOM, i);
            }
        }
        if (go && out + count > p.n_slots) {  // the caller has no room for their slots
            go = false;
            if (lane == 0) raise_status(p.status, MT_ERR_INVALID_ARG, i);
        }
        const int64_t last = go && had > 0 && (len & (p.k.page_tokens - 1)) ? table_row(p, row)[had - 1] : 0;      // the page that is partly filled
        if (go && count > 0 && (uint64_t)last >= (uint64_t)p.k.n_pages) {
            go = false;
            if (lane == 0) raise_status(p.status, MT_ERR_INVALID_ARG, i);
        }
        if (go) {
            for (int c = lane; c < need; c += size) {
                const int page = free_page<SMALL>(h, first + c);
                table_row(p, row)[had + c] = page;
                p.k.refs[page] = 1;
            }
            if (lane == 0) p.k.lengths[row] = len + count;
        }
        for (int c = lane; c < count && out + c < p.n_slots; c += size) {
            const int at = len + c, col = at >> p.shift;
            const int64_t page = !go ? 0 : col < had ? last : free_page<SMALL>(h, first + col - had);
            p.slots[out + c] = go ? (page << p.shift) + (at & (p.k.page_tokens - 1)) : -1;
        }
    };
    for (int i = t.thread; i < p.n; i += t.threads)
        if (h.other[i] <= kFew) place(i, 0, 1);
    for (int i = t.warp; i < p.n; i += warps)
        if (h.other[i] > kFew) place(i, t.lane, 32);
}

template <bool SMALL>
__global__ void __launch_bounds__(kThreads) release_kernel(const Params p) {
    extern __shared__ __align__(16) uint8_t shared[];
    const Hand h = hand_of<SMALL>(p, shared);
    const Team t = team_of(p.team);
    pdl_launch_dependents();
    pdl_wait();
    clear_owners<SMALL>(p, h, t, false);
    t.sync();
    claim_rows(p, h, t);
    t.sync();
    for (int i = t.warp; i < p.n; i += t.size * kWarps) {
        const int row = h.rows[i];
        const bool ok = in(row, p.k.n_rows) && fetch<SMALL>(h.owner + row) == i;
        const int len = ok ? p.k.lengths[row] : -1;
        if (!ok || !good_length(p, len)) {
            if (t.lane == 0) raise_status(p.status, MT_ERR_INVALID_ARG, i);
            continue;
        }
        const int pages = pages_of(p, len);
        for (int c = t.lane; c < pages; c += 32) give_back(p, table_row(p, row)[c], i);
        __syncwarp();
        if (t.lane == 0) p.k.lengths[row] = 0;
    }
}

// Used pages behind the first `used` ones go to the holes among these, the i-th to the i-th.
__global__ void __launch_bounds__(kThreads) compact_kernel(const Params p) {
    __shared__ Shared s;
    const Team t = team_of(p.team);
    int32_t *const holes = p.free_list, *const high = p.staged, *const moved = p.owner;
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t mask = count_free(t, s, p.k.refs, p.k.n_pages);
    t.sync();
    int before, n_free;
    total_free(t, s, before, n_free);
    const int used = p.k.n_pages - n_free;
    int mine = 0;
    for_stretch(t, s, p.k.refs, p.k.n_pages, mask, before, [&](int at, uint32_t m, int rank) {
        for (int e = 0; e < 4 && at + e < p.k.n_pages; ++e) {
            const int page = at + e;
            if (page >= used) moved[page] = page;
            if (m >> e & 1) {
                if (page < used) { holes[rank] = page; ++mine; }
                ++rank;
            } else if (page >= used) {
                high[used - 1 - (page - rank)] = page;       // the last used page first: how many there are is not known yet
            }
        }
    });
    if (mine) atomicAdd(&s.holes, mine);
    t.sync();
    int n_holes = 0;
    for (int r = 0; r < t.size; ++r) n_holes += t.size > 1 ? (int)remote_u32(&s.holes, r) : s.holes;
    const int moves = min(n_holes, p.n);
    for (int i = t.thread; i < p.n; i += t.threads) {
        int from = -1, to = -1;
        if (i < moves) {
            from = __ldcg(high + (n_holes - 1 - i));
            to = __ldcg(holes + i);
            p.k.refs[to] = p.k.refs[from];
            p.k.refs[from] = 0;
            moved[from] = to;
        }
        p.copies[(int64_t)i * 3] = from;
        p.copies[(int64_t)i * 3 + 1] = to;
        p.copies[(int64_t)i * 3 + 2] = i < moves ? p.k.page_tokens : 0;
    }
    t.sync();
    for (int row = t.warp; row < p.k.n_rows; row += t.size * kWarps) {
        const int len = p.k.lengths[row];
        if (!good_length(p, len)) {
            if (t.lane == 0) raise_status(p.status, MT_ERR_INVALID_ARG, row);
            continue;
        }
        const int pages = pages_of(p, len);
        int32_t* const r = table_row(p, row);
        for (int c = t.lane; c < pages; c += 32) {
            const int page = r[c];
            if (page >= used && page < p.k.n_pages) r[c] = __ldcg(moved + page);
        }
    }
}

// ------------------------------------------------------------------------------------------------ copies
constexpr int kCopyThreads = 128;
constexpr int kAhead = 8;                     // vectors of a lane under way
constexpr int kCachesPerLaunch = 64, kFewCaches = 8;                           // (the block of 64 costs a launch a microsecond on the host)
struct CopyCache {
    uint8_t* codes[2];                        // keys, values
    uint8_t* params[2];
    int heads, row;                           // bytes of a token's codes
};
template <int CACHES>
struct CopyParams {
    const int32_t* copies;
    int n, n_pages, page_tokens;
    OpStatus status;
    CopyCache c[CACHES];
};
static_assert(sizeof(CopyParams<kCachesPerLaunch>) <= 4096, "");

template <int CACHES>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyParams<CACHES> p) {
    pdl_launch_dependents();
    pdl_wait();
    const CopyCache& c = p.c[blockIdx.y >> 1];
    const int kv = blockIdx.y & 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t head_codes = (int64_t)p.page_tokens * c.row, head_params = (int64_t)p.page_tokens * 4;
    for (int i = blockIdx.x; i < p.n; i += gridDim.x) {
        const int from = p.copies[(int64_t)i * 3], to = p.copies[(int64_t)i * 3 + 1], tokens = p.copies[(int64_t)i * 3 + 2];
        if (from == -1 && to == -1) continue;
        if (!in(from, p.n_pages) || !in(to, p.n_pages) || tokens < 0 || tokens > p.page_tokens) {
            if (threadIdx.x == 0) raise_status(p.status, MT_ERR_INVALID_ARG, i);
            continue;
        }
        if (from == to) continue;
        const int vecs = tokens * c.row / 16;
        for (int h = warp; h < c.heads; h += kCopyThreads / 32) {
            const uint4* const src = reinterpret_cast<const uint4*>(c.codes[kv] + ((int64_t)from * c.heads + h) * head_codes);
            uint4* const dst = reinterpret_cast<uint4*>(c.codes[kv] + ((int64_t)to * c.heads + h) * head_codes);
            const uint32_t* const ps = reinterpret_cast<const uint32_t*>(c.params[kv] + ((int64_t)from * c.heads + h) * head_params);
            uint32_t* const pd = reinterpret_cast<uint32_t*>(c.params[kv] + ((int64_t)to * c.heads + h) * head_params);
            for (int v0 = lane; v0 < vecs; v0 += 32 * kAhead) {
                uint4 x[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) if (v0 + 32 * k < vecs) x[k] = __ldcs(src + v0 + 32 * k);
#pragma unroll
                for (int k = 0; k < kAhead; ++k) if (v0 + 32 * k < vecs) __stcs(dst + v0 + 32 * k, x[k]);
            }
            for (int v = lane; v < tokens; v += 32) pd[v] = ps[v];
        }
    }
}

// kernels: [0] for a call that is SMALL, [1] for others
cudaError_t launch_team(void (*const (&kernels)[2])(Params), Params& p, int64_t work, bool small, cudaStream_t s) {
    p.team = work > (1 << 16) ? kTeam : 1;    // words a thread of a single CTA reads: 64
    small = small && p.team == 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.team);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = small ? sizeof(SmallHand) : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.team;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.team > 1 ? 2 : 1;
    ++g_kernel_launches;
    return cudaLaunchKernelEx(&cfg, kernels[small ? 0 : 1], p);
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

cudaError_t configure_kv_pages() {
    cudaError_t e = cudaFuncSetAttribute(fork_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SmallHand));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(reserve_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SmallHand));
    return e == cudaSuccess ? cudaFuncSetAttribute(release_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SmallHand)) : e;
}

mt_status launch_kv_pages(const KvPagesArgs& a, cudaStream_t s) {
    Params p;
    p.k = a.k;
    p.shift = 0;
    while ((1 << p.shift) < a.k.page_tokens) ++p.shift;
    p.n = a.n;
    p.rows = a.rows; p.other = a.other; p.copies = a.copies; p.slots = a.slots; p.n_slots = a.n_slots; p.status = a.status;
    const size_t n = (size_t)a.n, pages = (size_t)a.k.n_pages, rows = (size_t)a.k.n_rows, width = (size_t)a.k.table_width;
    const bool fork = a.what == KvPagesArgs::kFork, reserve = a.what == KvPagesArgs::kReserve, compact = a.what == KvPagesArgs::kCompact;
    const size_t owner = round_up(4 * (compact ? pages : rows)), list = fork ? round_up(4 * n) : round_up(4 * pages);
    const size_t info = round_up(4 * n), place = round_up(16 * n), staged = fork ? round_up(4 * n * width) : compact ? round_up(4 * pages) : 0;
    uint8_t* w;
    const mt_status st = op_scratch(s, owner + list + info + place + staged, &w);
    if (st != MT_OK) return st;
    p.owner = reinterpret_cast<int32_t*>(w);
    p.free_list = reinterpret_cast<int32_t*>(w + owner);
    p.info = reinterpret_cast<int32_t*>(w + owner + list);
    p.place = reinterpret_cast<long long*>(w + owner + list + info);
    p.staged = reinterpret_cast<int32_t*>(w + owner + list + info + place);
    const int64_t of_rows = (int64_t)(n * width);
    const bool small = a.n <= kSmall && a.k.n_rows <= kSmallRows;
    void (*const forks[2])(Params) = {fork_kernel<true>, fork_kernel<false>};
    void (*const reserves[2])(Params) = {reserve_kernel<true>, reserve_kernel<false>};
    void (*const releases[2])(Params) = {release_kernel<true>, release_kernel<false>};
    void (*const compacts[2])(Params) = {compact_kernel, compact_kernel};
    const cudaError_t e = fork ? launch_team(forks, p, (int64_t)pages + 3 * of_rows, small, s)
                        : reserve ? launch_team(reserves, p, 2 * (int64_t)pages, small, s)
                        : compact ? launch_team(compacts, p, 2 * (int64_t)pages + (int64_t)(rows * width), false, s)
                                  : launch_team(releases, p, of_rows, small, s);
    return e == cudaSuccess ? MT_OK : MT_ERR_CUDA;
}

template <int CACHES>
static cudaError_t copy_in(const mt_kv_cache* const* caches, int m, const int32_t* copies, int n, const OpStatus& status, cudaStream_t s) {
    CopyParams<CACHES> p;
    p.copies = copies; p.n = n; p.n_pages = caches[0]->n_pages; p.page_tokens = caches[0]->page_tokens; p.status = status;
    for (int i = 0; i < m; ++i) {
        const mt_kv_cache& c = *caches[i];
        p.c[i] = {{static_cast<uint8_t*>(c.k_codes), static_cast<uint8_t*>(c.v_codes)},
                  {static_cast<uint8_t*>(c.k_params), static_cast<uint8_t*>(c.v_params)}, c.kv_heads, c.head_dim / 2};
    }
    return launch_pdl(copy_kernel<CACHES>, dim3((unsigned)(n < 4096 ? n : 4096), (unsigned)(2 * m)), dim3(kCopyThreads), 0, s, p);
}

cudaError_t launch_kv_copy(const mt_kv_cache* const* caches, int n_caches, const int32_t* copies, int n, const OpStatus& status, cudaStream_t s) {
    for (int c0 = 0; c0 < n_caches; c0 += kCachesPerLaunch) {
        const int m = n_caches - c0 < kCachesPerLaunch ? n_caches - c0 : kCachesPerLaunch;
        const cudaError_t e = m <= kFewCaches ? copy_in<kFewCaches>(caches + c0, m, copies, n, status, s)
                                              : copy_in<kCachesPerLaunch>(caches + c0, m, copies, n, status, s);
        if (e != cudaSuccess) return e;
        if (n_caches - c0 <= kCachesPerLaunch) break;
    }
    return cudaSuccess;
}

}  // namespace mt
