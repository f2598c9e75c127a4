// The pages of a paged cache: the append of new tokens' K and V rows, and the upkeep of the page table -- forking branches, reserving
// pages for new tokens, giving pages back, compacting the pool, copying pages (paper Section 3.2: B branches of one question share their
// prompt and part ways while they generate; a branch that ends leaves its memory to others).
//
// State, all on the device: a page table [B][columns] of page numbers (anything outside [0, pages) is no page), a reference count per
// page = the number of table entries that name it (a page without references is free), and a length per branch.  Whole numbers
// throughout; where pages are chosen the lowest numbers come first, so every call has one right result whatever the order of
// its threads.  References are counted with integer atomics, whose order changes nothing.
#include <algorithm>

#include "lotts_common.h"

namespace lotts {

typedef unsigned p_u32x4 __attribute__((ext_vector_type(4)));
typedef int p_i32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxBranches = 4096;
constexpr int kMaxPages = 1 << 24;
constexpr int kUpkeepThreads = 1024;
constexpr int kUpkeepWaves = kUpkeepThreads / kWave;

// ---------------------------------------------------------------------------------------------
// kv_append_paged: a wavefront a token, its 16-byte pieces over the lanes
// ---------------------------------------------------------------------------------------------
struct AppendPagedParams {
    const unsigned char *Knew, *Vnew;
    unsigned char *Kpages, *Vpages;
    const int32_t *table, *kv_len, *q_start;
    long long new_t, new_h, page_p, page_h, page_t, table_stride;  // bytes; table: entries
    int B, T, R, Hkv, pieces, n, shift, pages, columns;            // pieces: of a row; n: of a token
    FastDiv d_r, d_pieces;
};

// The branch whose new tokens row t of the step belongs to; B if it is nobody's.  A wavefront looks at 64 ends at a time, first of
// every 64th branch, then of those 64: for more than 64 branches two loads one after the other, where a search by halves has twelve.
__device__ __forceinline__ int branch_of(const int32_t* q_start, int B, int t, int lane) {
    int first = 0;
    if (B > kWave) {
        const int b = (lane + 1) * kWave;
        first = kWave * __popcll(__ballot(b <= B && q_start[min(b, B)] <= t));
        if (first >= B) return B;
    }
    const int b = first + lane;
    return min(B, first + __popcll(__ballot(b < B && q_start[min(b, B - 1) + 1] <= t)));
}

__global__ __launch_bounds__(256) void kv_append_paged_kernel(const AppendPagedParams p) {
    const int lane = threadIdx.x & (kWave - 1);
    const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
    if (t >= p.T) return;
    constexpr int AT = 2;  // pieces of K and of V that a lane has in flight
    const unsigned char *ks = p.Knew + t * p.new_t, *vs = p.Vnew + t * p.new_t;
    p_u32x4 k[AT], v[AT];
    long long to[AT];
    auto request = [&](int i0) {
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            const int i = i0 + j * kWave + lane;
            const int h = quot(i, p.d_pieces), c = i - h * p.pieces;
            to[j] = h * p.page_h + c * 16;
            if (i < p.n) {
                k[j] = *reinterpret_cast<const p_u32x4*>(ks + h * p.new_h + c * 16);
                v[j] = *reinterpret_cast<const p_u32x4*>(vs + h * p.new_h + c * 16);
            }
        }
    };
    request(0);  // the source does not depend on where it goes
    int b, pos;
    if (p.q_start) {
        b = branch_of(p.q_start, p.B, t, lane);
        if (b >= p.B || t < p.q_start[b]) return;
        pos = p.kv_len[b] - (p.q_start[b + 1] - t);
    } else {
        b = quot(t, p.d_r);
        pos = p.kv_len[b] - ((b + 1) * p.R - t);
    }
    if (pos < 0 || pos >> p.shift >= p.columns) return;
    const int page = p.table[b * p.table_stride + (pos >> p.shift)];
    if (page < 0 || page >= p.pages) return;
    const long long at = page * p.page_p + (pos & ((1 << p.shift) - 1)) * p.page_t;
    unsigned char *kd = p.Kpages + at, *vd = p.Vpages + at;
    for (int i0 = 0; i0 < p.n; i0 += AT * kWave) {
        if (i0 > 0) request(i0);
#pragma unroll
        for (int j = 0; j < AT; ++j)
            if (i0 + j * kWave + lane < p.n) {
                *reinterpret_cast<p_u32x4*>(kd + to[j]) = k[j];
                *reinterpret_cast<p_u32x4*>(vd + to[j]) = v[j];
            }
    }
}

// ---------------------------------------------------------------------------------------------
// upkeep
// ---------------------------------------------------------------------------------------------
struct UpkeepParams {
    int32_t *table, *refs, *kv_len;
    const int32_t* arg;  // new tokens, parents or lengths to keep
    int32_t *out, *count, *list;
    long long table_stride;
    int B, columns, pages, shift, cols, log_cols;
};

__device__ __forceinline__ bool is_page(int e, int pages) { return (unsigned)e < (unsigned)pages; }

// Exclusive prefix sum over the workgroup; *total gets the sum.  sums: kUpkeepWaves words of LDS, free again behind the next barrier.
__device__ __forceinline__ unsigned group_scan(unsigned v, unsigned* sums, unsigned* total) {
    const unsigned incl = wave_incl_scan_u32(v);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    if (lane == kWave - 1) sums[wave] = incl;
    __syncthreads();
    const unsigned s = wave_incl_scan_u32(lane < kUpkeepWaves ? sums[lane] : 0);
    *total = __builtin_amdgcn_readlane(s, kUpkeepWaves - 1);
    const unsigned before = wave > 0 ? __builtin_amdgcn_readlane(s, wave - 1) : 0;
    return before + incl - v;
}

// Walks over the reference counts in ascending order, kChunk at a time: f(page, before, is) is called for every page number below `pages`
// with the number of pages before it that `pick` picked, and whether it is one; stops behind a chunk once `enough` are
// found.  Returns how many were.  A wavefront's ballots count its 64 neighbours, LDS holds the counts of a chunk's pieces.
constexpr int kWalk = 16;                      // pages a thread looks at in a chunk
constexpr int kChunk = kWalk * kUpkeepThreads;
__device__ __forceinline__ void load_chunk(const int32_t* refs, int pages, int at, int (&r)[kWalk]) {
#pragma unroll
    for (int j = 0; j < kWalk; ++j) {
        const int i = at + j * kUpkeepThreads + (int)threadIdx.x;
        r[j] = i < pages ? refs[i] : 0;
    }
}
// r: the first chunk's counts, requested by the caller, who has had other things to wait for.
template <typename Pick, typename F>
__device__ __forceinline__ int walk(const int32_t* refs, int pages, int enough, int* counts, int (&r)[kWalk], Pick pick, F f) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid & (kWave - 1);
    int found = 0;
    for (int at = 0; at < pages && found < enough; at += kChunk) {
        if (at > 0) load_chunk(refs, pages, at, r);
        unsigned long long mask[kWalk];
#pragma unroll
        for (int j = 0; j < kWalk; ++j) {
            const int i = at + j * kUpkeepThreads + tid;
            mask[j] = __ballot(i < pages && pick(i, r[j]));
            if (lane == 0) counts[j * kUpkeepWaves + wave] = __popcll(mask[j]);
        }
        __syncthreads();
        // kWalk * kUpkeepWaves = 4 * 64 counts: every wavefront scans all of them
        int before[kWalk * kUpkeepWaves / kWave], sum = 0;
#pragma unroll
        for (int k = 0; k < kWalk * kUpkeepWaves / kWave; ++k) {
            const int c = counts[k * kWave + lane], incl = (int)wave_incl_scan_u32((unsigned)c);
            before[k] = found + sum + incl - c;
            sum += __builtin_amdgcn_readlane(incl, kWave - 1);
        }
#pragma unroll
        for (int j = 0; j < kWalk; ++j) {
            const int i = at + j * kUpkeepThreads + tid, slot = j * kUpkeepWaves + wave;
            const int base = __builtin_amdgcn_readlane(before[j * kUpkeepWaves / kWave], slot % kWave);
            if (i < pages) f(i, base + __popcll(mask[j] & ((1ull << lane) - 1)), (mask[j] >> lane & 1) != 0);
        }
        found += sum;
        __syncthreads();
    }
    return found;
}

// kv_pages_reserve: one workgroup.  The columns that the branches' new tokens are written to form one list of slots, in the order of
// branches and columns; a slot wants a page if it has none or shares its own.  The pages wanted are counted, that many free ones are
// looked up in ascending order, and only then, if they are there, anything is changed.
__global__ __launch_bounds__(kUpkeepThreads) void kv_pages_reserve_kernel(const UpkeepParams p) {
    __shared__ int start[kMaxBranches];   // slots in front of a branch's
    __shared__ int length[kMaxBranches];  // its tokens before the call
    __shared__ unsigned sums[kUpkeepWaves];
    __shared__ int counts[kWalk * kUpkeepWaves];
    __shared__ int bad;
    __shared__ int list[kUpkeepThreads];
    const int tid = threadIdx.x;
    int r0[kWalk];
    load_chunk(p.refs, p.pages, 0, r0);  // whichever pages are free: on their way while the slots are found
    if (tid == 0) bad = 0;
    __syncthreads();
    const int per = (p.B + kUpkeepThreads - 1) / kUpkeepThreads, b0 = tid * per;  // consecutive branches
    auto span = [&](int b, int* first) {
        const int len = max(p.kv_len[b], 0), n = max(p.arg[b], 0);
        length[b] = len;
        *first = len >> p.shift;
        const long long end = (long long)len + n;
        if (n > 0 && end > (long long)p.columns << p.shift) bad = 1;
        return n > 0 ? (int)((end - 1) >> p.shift) - *first + 1 : 0;
    };
    int mine = 0, first;
    for (int b = b0; b < min(p.B, b0 + per); ++b) {
        const int n = span(b, &first);
        start[b] = n;
        p.out[2 * b] = p.out[2 * b + 1] = -1;
        mine += n;
    }
    unsigned slots;
    int at = (int)group_scan((unsigned)mine, sums, &slots);
    for (int b = b0; b < min(p.B, b0 + per); ++b) {
        const int n = start[b];
        start[b] = at;
        at += n;
    }
    __syncthreads();
    if (bad) {  // a branch's tokens would pass the table
        if (tid == 0) *p.count = -1;
        return;
    }
    // a slot's branch: the last one that starts at or before it and has slots (those without start where the next one does)
    struct Slot {
        int b, c, entry;
        bool shared, wanted;
    };
    auto slot_at = [&](int s) {
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (start[mid] <= s) lo = mid;
            else hi = mid - 1;
        }
        Slot x;
        x.b = lo;
        x.c = (length[lo] >> p.shift) + s - start[lo];
        x.entry = p.table[lo * p.table_stride + x.c];
        const bool none = !is_page(x.entry, p.pages);
        x.shared = !none && p.refs[x.entry] > 1;
        x.wanted = none || x.shared;
        return x;
    };
    if ((int)slots <= kUpkeepThreads) {
        // a slot a thread, looked at once, and the list in LDS: the usual step of every branch (64 branches x 5 tokens: 9.5 -> 9.2 us)
        Slot x = {};
        if (tid < (int)slots) x = slot_at(tid);
        unsigned wanted;
        const int rank = (int)group_scan(x.wanted, sums, &wanted);
        const int found = walk(p.refs, p.pages, (int)wanted, counts, r0, [](int, int r) { return r <= 0; },
                               [&](int i, int before, bool is) {
                                   if (is && before < (int)wanted) list[before] = i;
                               });
        if (tid == 0) *p.count = max(0, (int)wanted - found);
        if (found < (int)wanted) return;
        if (x.wanted) {
            const int page = list[rank];
            if (x.shared && (long long)x.c << p.shift < length[x.b]) {
                p.out[2 * x.b] = x.entry;
                p.out[2 * x.b + 1] = page;
            }
            p.table[x.b * p.table_stride + x.c] = page;
            p.refs[page] = 1;
            if (x.shared) atomicSub(p.refs + x.entry, 1);  // (everybody has looked at the references)
        }
        __syncthreads();
        for (int b = tid; b < p.B; b += kUpkeepThreads) p.kv_len[b] = length[b] + max(p.arg[b], 0);
        return;
    }
    int wanted = 0;
    for (int s0 = 0; s0 < (int)slots; s0 += kUpkeepThreads) wanted += __syncthreads_count(s0 + tid < (int)slots && slot_at(s0 + tid).wanted);
    const int found = walk(p.refs, p.pages, wanted, counts, r0, [](int, int r) { return r <= 0; },
                           [&](int i, int before, bool is) {
                               if (is && before < wanted) p.list[before] = i;
                           });
    if (tid == 0) *p.count = max(0, wanted - found);
    if (found < wanted) return;
    // (the list was written in front of walk's last barrier; with nothing wanted it is not read)
    unsigned rank0 = 0;
    for (int s0 = 0; s0 < (int)slots; s0 += kUpkeepThreads) {
        const bool in = s0 + tid < (int)slots;
        Slot x = {};
        if (in) x = slot_at(s0 + tid);
        unsigned n;
        const unsigned rank = rank0 + group_scan(in && x.wanted, sums, &n);
        if (in && x.wanted) {
            const int page = p.list[rank];
            p.list[rank] = x.shared ? x.entry : -1;  // what loses a reference, once no slot looks at references any more
            if (x.shared && (long long)x.c << p.shift < length[x.b]) {
                p.out[2 * x.b] = x.entry;
                p.out[2 * x.b + 1] = page;
            }
            p.table[x.b * p.table_stride + x.c] = page;
            p.refs[page] = 1;
        }
        rank0 += n;
        __syncthreads();
    }
    __syncthreads();
    for (int r = tid; r < wanted; r += kUpkeepThreads)
        if (p.list[r] >= 0) atomicSub(p.refs + p.list[r], 1);
    for (int b = tid; b < p.B; b += kUpkeepThreads) p.kv_len[b] = length[b] + max(p.arg[b], 0);
}

// kv_pages_free: a workgroup a branch
__global__ __launch_bounds__(256) void kv_pages_free_kernel(const UpkeepParams p) {
    const int b = blockIdx.x;
    const int now = p.kv_len[b], len = max(0, p.arg ? min(now, p.arg[b]) : now);
    int32_t* row = p.table + b * p.table_stride;
    for (int c = (int)(((long long)len + (1 << p.shift) - 1) >> p.shift) + threadIdx.x; c < p.columns; c += 256) {
        const int e = row[c];
        if (is_page(e, p.pages)) atomicSub(p.refs + e, 1);
        if (e != -1) row[c] = -1;
    }
    __syncthreads();
    if (threadIdx.x == 0) p.kv_len[b] = len;
}

// kv_pages_fork: a workgroup takes some columns of all rows, which it holds in LDS: rows may change places
constexpr int kForkEntries = 8192;
__global__ __launch_bounds__(256) void kv_pages_fork_kernel(const UpkeepParams p) {
    __shared__ int old[kForkEntries];
    __shared__ int parent[kMaxBranches], children[kMaxBranches];
    const int c0 = blockIdx.x * p.cols, tid = threadIdx.x;
    const bool lengths = c0 >= p.columns;  // the last workgroup's part
    const int n = lengths ? p.B : p.B << p.log_cols;
    constexpr int AT = 4;  // entries that a thread has in flight
    for (int e0 = tid; e0 < n; e0 += AT * 256) {
        int v[AT];
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            const int e = e0 + j * 256, b = e >> p.log_cols, c = c0 + (e & (p.cols - 1));
            v[j] = -1;
            if (e < n) v[j] = lengths ? p.kv_len[e] : c < p.columns ? p.table[b * p.table_stride + c] : -1;
        }
#pragma unroll
        for (int j = 0; j < AT; ++j)
            if (e0 + j * 256 < n) old[e0 + j * 256] = v[j];
    }
    for (int b = tid; b < p.B; b += 256) {
        const int from = p.arg[b];
        parent[b] = from >= p.B ? b : max(from, -1);
        children[b] = 0;
    }
    __syncthreads();
    if (lengths) {
        for (int b = tid; b < p.B; b += 256)
            if (parent[b] != b) p.kv_len[b] = parent[b] < 0 ? 0 : old[parent[b]];
        return;
    }
    for (int b = tid; b < p.B; b += 256)
        if (parent[b] >= 0 && parent[b] != b) atomicAdd(children + parent[b], 1);
    __syncthreads();
    // A page gains its row's children, all at once (not one by one, so that 48 branches of one parent do not queue 48 times), and loses a reference for
    // every row that is replaced; where a row is replaced by the same page, the two meet.
    for (int e = tid; e < n; e += 256) {
        const int b = e >> p.log_cols, ci = e & (p.cols - 1), from = parent[b], was = old[e];
        if (c0 + ci >= p.columns) continue;
        const int gain = children[b] - (from != b ? 1 : 0);
        if (gain != 0 && is_page(was, p.pages)) atomicAdd(p.refs + was, gain);
        if (from == b) continue;
        const int is = from < 0 ? -1 : old[(from << p.log_cols) + ci];
        if (was != is) p.table[b * p.table_stride + c0 + ci] = is;
    }
}

// kv_pages_compact: one workgroup counts the pages in use, pairs those behind that many with the free ones in front, and moves the
// references; a second launch renames the table's entries.  list: the new number of every page that moved.
__global__ __launch_bounds__(kUpkeepThreads) void kv_pages_compact_kernel(const UpkeepParams p) {
    __shared__ int counts[kWalk * kUpkeepWaves];
    const int tid = threadIdx.x;
    int r0[kWalk];
    load_chunk(p.refs, p.pages, 0, r0);
    const int live = walk(p.refs, p.pages, p.pages + 1, counts, r0, [](int, int r) { return r > 0; }, [](int, int, bool) {});
    if (p.pages > kChunk) load_chunk(p.refs, p.pages, 0, r0);  // (a pool of one chunk is in registers still)
    const int moves = walk(p.refs, live, live + 1, counts, r0, [](int, int r) { return r <= 0; },
                           [&](int i, int before, bool is) {
                               if (is) p.out[2 * before + 1] = i;
                           });
    if (p.pages > kChunk) load_chunk(p.refs, p.pages, 0, r0);
    walk(p.refs, p.pages, moves, counts, r0, [&](int i, int r) { return i >= live && r > 0; },
         [&](int i, int before, bool is) {
             if (is) p.out[2 * before] = i;
         });
    for (int i = live + tid; i < p.pages; i += kUpkeepThreads) p.list[i] = -1;  // an entry from `live` on that names a free page names none afterwards
    __syncthreads();
    for (int j = tid; j < moves; j += kUpkeepThreads) {
        const int src = p.out[2 * j], dst = p.out[2 * j + 1];
        p.refs[dst] = p.refs[src];
        p.refs[src] = 0;
        p.list[src] = dst;
    }
    if (tid == 0) {
        p.count[0] = moves;
        p.count[1] = live;
    }
}
__global__ __launch_bounds__(256) void kv_pages_rename_kernel(const UpkeepParams p) {
    const int live = p.count[1];
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= p.columns) return;
    int32_t* entry = p.table + blockIdx.y * p.table_stride + c;
    const int e = *entry;
    if (is_page(e, p.pages) && e >= live) *entry = p.list[e];
}

// kv_pages_copy: pieces of a page of one plane over the workgroups
struct CopyParams {
    unsigned char* pool;
    const int32_t *pairs, *count;
    long long plane_stride, page_stride, page_bytes, pieces;  // pieces: of a page, kCopyPiece bytes each
    int planes, pages, n;
};
constexpr int kCopyLoads = 4;
constexpr int kCopyPiece = 256 * 16 * kCopyLoads;
__global__ __launch_bounds__(256) void kv_pages_copy_kernel(const CopyParams p) {
    int n = p.n;
    if (p.count) n = max(0, min(n, p.count[0]));
    const long long units = (long long)n * p.planes * p.pieces;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const long long pp = u / p.pieces, pair = pp / p.planes;
        const int src = p.pairs[2 * pair], dst = p.pairs[2 * pair + 1];
        if (!is_page(src, p.pages) || !is_page(dst, p.pages) || src == dst) continue;
        unsigned char* plane = p.pool + (pp - pair * p.planes) * p.plane_stride;
        const long long at = (u - pp * p.pieces) * kCopyPiece + threadIdx.x * 16;
        p_u32x4 v[kCopyLoads];
#pragma unroll
        for (int j = 0; j < kCopyLoads; ++j)
            if (at + j * 4096 < p.page_bytes) v[j] = *reinterpret_cast<const p_u32x4*>(plane + src * p.page_stride + at + j * 4096);
#pragma unroll
        for (int j = 0; j < kCopyLoads; ++j)
            if (at + j * 4096 < p.page_bytes) *reinterpret_cast<p_u32x4*>(plane + dst * p.page_stride + at + j * 4096) = v[j];
    }
}

// Checks that the upkeep calls share.
static int upkeep(UpkeepParams* p, int32_t B, int32_t columns, int32_t pages, int32_t* table, int64_t table_stride, int32_t* refs) {
    if (B < 1 || B > kMaxBranches || columns < 1 || pages < 1 || pages > kMaxPages || table_stride < columns) return LOTTS_ERR_SHAPE;
    if (!table || !refs) return LOTTS_ERR_NULL;
    if ((((uintptr_t)table | (uintptr_t)refs) & 3) != 0) return LOTTS_ERR_SHAPE;
    *p = UpkeepParams{};
    p->table = table; p->refs = refs; p->table_stride = table_stride;
    p->B = B; p->columns = columns; p->pages = pages;
    return LOTTS_OK;
}
static int page_shift(int32_t page_tokens) {  // -1 if it is no power of two from 16 to 1024
    for (int s = 4; s <= 10; ++s)
        if (page_tokens == 1 << s) return s;
    return -1;
}

}  // namespace lotts

extern "C" int kv_append_paged(int32_t B, int32_t T, int32_t Hkv, int32_t D, int32_t page_tokens, int32_t pages, int32_t columns,
                               lotts_dtype dtype, const void* Knew, const void* Vnew, int64_t new_stride_t, int64_t new_stride_h, void* Kpages,
                               void* Vpages, int64_t page_stride_p, int64_t page_stride_h, int64_t page_stride_t, const int32_t* page_table,
                               int64_t table_stride, const int32_t* kv_len, const int32_t* q_start, void* stream) {
    using namespace lotts;
    if (dtype != LOTTS_BF16 && dtype != LOTTS_F32) return LOTTS_ERR_DTYPE;
    const long long es = dtype == LOTTS_BF16 ? 2 : 4;
    const int shift = page_shift(page_tokens);
    if (B < 1 || B > kMaxBranches || T < 1 || T > (1 << 25) || Hkv < 1 || D < 1 || D > 65536 || shift < 0 || pages < 1 || pages > kMaxPages || columns < 1 ||
        (long long)columns << shift > 0x7fffffffLL || table_stride < columns || ((long long)D * es) % 16 != 0)
        return LOTTS_ERR_SHAPE;
    if (!Knew || !Vnew || !Kpages || !Vpages || !page_table || !kv_len) return LOTTS_ERR_NULL;
    if (!q_start && T % B != 0) return LOTTS_ERR_SHAPE;
    const int64_t strides[5] = {new_stride_t, new_stride_h, page_stride_p, page_stride_h, page_stride_t};
    for (int64_t s : strides)
        if (s < 0 || (s * es) % 16 != 0) return LOTTS_ERR_SHAPE;
    if (new_stride_h < D || page_stride_t < D || (long long)Hkv * D > (1 << 24)) return LOTTS_ERR_SHAPE;
    if ((((uintptr_t)Knew | (uintptr_t)Vnew | (uintptr_t)Kpages | (uintptr_t)Vpages) & 15) != 0) return LOTTS_ERR_SHAPE;
    AppendPagedParams p;
    p.Knew = static_cast<const unsigned char*>(Knew);
    p.Vnew = static_cast<const unsigned char*>(Vnew);
    p.Kpages = static_cast<unsigned char*>(Kpages);
    p.Vpages = static_cast<unsigned char*>(Vpages);
    p.table = page_table; p.kv_len = kv_len; p.q_start = q_start;
    p.new_t = new_stride_t * es; p.new_h = new_stride_h * es;
    p.page_p = page_stride_p * es; p.page_h = page_stride_h * es; p.page_t = page_stride_t * es;
    p.table_stride = table_stride;
    p.B = B; p.T = T; p.R = T / B; p.Hkv = Hkv; p.pieces = (int)(D * es / 16); p.n = p.pieces * Hkv;
    p.shift = shift; p.pages = pages; p.columns = columns;
    p.d_r = fast_div(q_start ? 1 : p.R); p.d_pieces = fast_div(p.pieces);
    LOTTS_LAUNCH(kv_append_paged_kernel, dim3((unsigned)((T + 3LL) / 4)), dim3(256), (hipStream_t)stream, p);
    return check_launch();
}

extern "C" size_t kv_pages_workspace_bytes(int32_t pages) {
    return pages < 1 || pages > lotts::kMaxPages ? 0 : (size_t)pages * 4;
}

extern "C" int kv_pages_reserve(int32_t B, int32_t columns, int32_t pages, int32_t page_tokens, int32_t* page_table, int64_t table_stride,
                                int32_t* refs, int32_t* kv_len, const int32_t* new_tokens, int32_t* copies, int32_t* missing, void* workspace,
                                size_t workspace_bytes, void* stream) {
    using namespace lotts;
    UpkeepParams p;
    const int rc = upkeep(&p, B, columns, pages, page_table, table_stride, refs);
    if (rc != LOTTS_OK) return rc;
    p.shift = page_shift(page_tokens);
    if (p.shift < 0 || (long long)columns << p.shift > 0x7fffffffLL || (long long)B * columns > 0x7fffffffLL) return LOTTS_ERR_SHAPE;
    if (!kv_len || !new_tokens || !copies || !missing || !workspace) return LOTTS_ERR_NULL;
    if (workspace_bytes < kv_pages_workspace_bytes(pages)) return LOTTS_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 3) != 0) return LOTTS_ERR_SHAPE;
    p.kv_len = kv_len; p.arg = new_tokens; p.out = copies; p.count = missing;
    p.list = static_cast<int32_t*>(workspace);
    LOTTS_LAUNCH(kv_pages_reserve_kernel, dim3(1), dim3(kUpkeepThreads), (hipStream_t)stream, p);
    return check_launch();
}

extern "C" int kv_pages_free(int32_t B, int32_t columns, int32_t pages, int32_t page_tokens, int32_t* page_table, int64_t table_stride,
                             int32_t* refs, int32_t* kv_len, const int32_t* keep, void* stream) {
    using namespace lotts;
    UpkeepParams p;
    const int rc = upkeep(&p, B, columns, pages, page_table, table_stride, refs);
    if (rc != LOTTS_OK) return rc;
    p.shift = page_shift(page_tokens);
    if (p.shift < 0) return LOTTS_ERR_SHAPE;
    if (!kv_len) return LOTTS_ERR_NULL;
    p.kv_len = kv_len; p.arg = keep;
    LOTTS_LAUNCH(kv_pages_free_kernel, dim3((unsigned)B), dim3(256), (hipStream_t)stream, p);
    return check_launch();
}

extern "C" int kv_pages_fork(int32_t B, int32_t columns, int32_t pages, int32_t* page_table, int64_t table_stride, int32_t* refs, int32_t* kv_len,
                             const int32_t* parent, void* stream) {
    using namespace lotts;
    UpkeepParams p;
    const int rc = upkeep(&p, B, columns, pages, page_table, table_stride, refs);
    if (rc != LOTTS_OK) return rc;
    if (!kv_len || !parent) return LOTTS_ERR_NULL;
    p.kv_len = kv_len; p.arg = parent;
    p.log_cols = 6;
    while (B << p.log_cols > 4 * 256 && p.log_cols > 2) --p.log_cols;  // one trip to memory, if that leaves 16 bytes of a row
    while (B << p.log_cols > kForkEntries) --p.log_cols;
    p.cols = 1 << p.log_cols;
    LOTTS_LAUNCH(kv_pages_fork_kernel, dim3((unsigned)((columns + (long long)p.cols - 1) / p.cols + 1)), dim3(256), (hipStream_t)stream, p);
    return check_launch();
}

extern "C" int kv_pages_compact(int32_t B, int32_t columns, int32_t pages, int32_t* page_table, int64_t table_stride, int32_t* refs, int32_t* moves,
                                int32_t* counts, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lotts;
    UpkeepParams p;
    int rc = upkeep(&p, B, columns, pages, page_table, table_stride, refs);
    if (rc != LOTTS_OK) return rc;
    if (!moves || !counts || !workspace) return LOTTS_ERR_NULL;
    if (workspace_bytes < kv_pages_workspace_bytes(pages)) return LOTTS_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 3) != 0) return LOTTS_ERR_SHAPE;
    p.out = moves; p.count = counts;
    p.list = static_cast<int32_t*>(workspace);
    LOTTS_LAUNCH(kv_pages_compact_kernel, dim3(1), dim3(kUpkeepThreads), (hipStream_t)stream, p);
    rc = check_launch();
    if (rc != LOTTS_OK) return rc;
    LOTTS_LAUNCH(kv_pages_rename_kernel, dim3((unsigned)((columns + 255LL) / 256), (unsigned)B), dim3(256), (hipStream_t)stream, p);
    return check_launch();
}

extern "C" int kv_pages_copy(void* pool, int32_t planes, int32_t pages, int64_t plane_stride, int64_t page_stride, int64_t page_bytes,
                             const int32_t* pairs, int32_t n, const int32_t* count, void* stream) {
    using namespace lotts;
    if (planes < 1 || pages < 1 || pages > kMaxPages || n < 1 || page_bytes < 16 || page_bytes % 16 != 0 || page_bytes > (1LL << 40) ||
        page_stride < page_bytes || page_stride % 16 != 0 || plane_stride < 0 || plane_stride % 16 != 0)
        return LOTTS_ERR_SHAPE;
    if ((long long)n * planes > (1LL << 36)) return LOTTS_ERR_SHAPE;  // pieces in 64 bits
    if (!pool || !pairs) return LOTTS_ERR_NULL;
    if (((uintptr_t)pool & 15) != 0) return LOTTS_ERR_SHAPE;
    CopyParams p;
    p.pool = static_cast<unsigned char*>(pool);
    p.pairs = pairs; p.count = count;
    p.plane_stride = plane_stride; p.page_stride = page_stride; p.page_bytes = page_bytes;
    p.pieces = (page_bytes + kCopyPiece - 1) / kCopyPiece;
    p.planes = planes; p.pages = pages; p.n = n;
    const long long units = (long long)n * planes * p.pieces;
    LOTTS_LAUNCH(kv_pages_copy_kernel, dim3((unsigned)std::min<long long>(units, 8 * kNumCU)), dim3(256), (hipStream_t)stream, p);
    return check_launch();
}
