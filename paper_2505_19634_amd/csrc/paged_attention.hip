// verify_attention_paged: causal attention of the new tokens of every branch against the branch's paged cache.  The branches of a call
// may have different numbers of new tokens: a chunk of a prompt that is being read, the drafts of a verification step, one token of
// plain decoding (paper Section 2: the target verifies the drafts in one parallel forward; Section 3.2: B branches of one question,
// whose prompt's pages they share).
//
// A branch's query rows of one KV head -- n new tokens x G query heads, the heads of a token next to each other -- are stacked, and a
// workgroup takes a tile of that stack.  Row r of the stack is token r / G; it sees the keys in front of position L - n + r / G + 1.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "lotts_common.h"

namespace lotts {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int kPgMaxBranches = 4096;
constexpr int kPgMaxPages = 1 << 24;
constexpr int kPgGroup = 16;         // keys that lie in one page whatever the page size
constexpr int kNarrowTile = 32;      // keys of a tile of a narrow item: one wavefront's at a time
constexpr int kWideTile = 64;        // keys of a tile of a wide item: the workgroup's
constexpr int kWideRows = 256;       // rows of a wide item
// Places in the sequence of work (below) of a narrow tile, a wide tile, and what starting on an item costs.  Measured where both are in a call: a tile
// of 32 keys for up to 32 rows 0.27 us at D = 64, 0.6 at 128; one of 64 keys for 256 rows 1.25 and 2.2.  (At 2 : 5, a chunk of 500 beside 31 branches, D = 64,
// kept some workgroups 34 us and others 68.)
constexpr int kNarrowCost = 2, kStartCost = 6;
constexpr int wide_cost(int D) { return D == 64 ? 9 : 7; }
constexpr int kMaxWideCost = 9;
// Places of a worker below which there are no more workers than items, and for narrow items that take more than this on average: 4 tiles, one for each
// wavefront.  (With 32 for both: 16 branches of 512 tokens 22.6 us against 13.2, 64 of 700 22.6 against 16.0, one of 2000 17.4 against 10.6; 2 tiles are
// no faster; with 8 for both one branch of 300 tokens 9.2 against 8.3.)  A cut of a wide item moves 256 rows.
constexpr int kMinPiece = 32, kMinNarrowPiece = 8;
constexpr int kApartPlaces = 280;    // places of a worker below which items are cut one by one
constexpr int kMaxWorkers = 2 * kNumCU;  // (paged_plan has when there are so many)
constexpr int kMergeGroup = 8;       // partials that are merged at a time

struct PagedParams {
    const void *Q, *K, *V;
    const int32_t *table, *kv_len, *q_start;
    long long q_t, q_h;                 // bytes
    long long page_p, page_h, page_t;   // bytes
    long long table_stride;
    int B, T, R, Hq, Hkv, G, pages, columns, shift;
    int items;                          // item slots of a KV head
    int workers;
    float scale_log2;                   // scale * log2(e)
    float scale;
    FastDiv d_g;
    void* O;
    float* lse;
    long long o_t, o_h;                 // bytes
    void* ws;                           // partials: 2 * workers slots of part_rows rows of D floats, then as many of (maximum, sum)
    unsigned ws_bytes, off_ml, off_o;
    int part_rows;
    unsigned long long* cells;          // arrivals: [2][2 * workers], (call tag << 16) | arrivals
    unsigned long long tag;
};

// A branch of the call: its first row of Q, its new tokens and all its tokens (both brought into the range that the arguments allow, so
// that nothing is addressed out of bounds whatever the device data say).
struct Branch {
    int first, n, L;
};
__host__ __device__ __forceinline__ Branch branch_at(const PagedParams& p, int b) {
    Branch r;
    int end;
    if (p.q_start) {
        r.first = min(max(p.q_start[b], 0), p.T);
        end = min(max(p.q_start[b + 1], r.first), p.T);
    } else {
        r.first = b * p.R;
        end = r.first + p.R;
    }
    r.n = end - r.first;
    r.L = min(max(p.kv_len[b], 0), p.columns << p.shift);
    return r;
}
// Keys that row t of Q sees if it is one of the branch's new tokens, never more than the branch has; -1 if it is not: where q_start does not ascend,
// a search for the branch that t belongs to may end at one that does not hold it.
__host__ __device__ __forceinline__ int keys_of_row(const Branch& br, int t) {
    return t < br.first || t - br.first >= br.n ? -1 : max(0, br.L - br.n + (t - br.first) + 1);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* base, unsigned bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, 0x00020000);
}
// Partials cross workgroups, and with them XCDs, inside the launch: sc0 sc1, past every cache that is not shared (system scope; device scope is sc1 alone).
constexpr int kDevScope = 17;
__device__ __forceinline__ void part_store4(__amdgpu_buffer_rsrc_t r, unsigned at, float4 v) {
    u32x4 u;
    u[0] = __float_as_uint(v.x); u[1] = __float_as_uint(v.y); u[2] = __float_as_uint(v.z); u[3] = __float_as_uint(v.w);
    __builtin_amdgcn_raw_buffer_store_b128(u, r, (int)at, 0, kDevScope);
}
__device__ __forceinline__ void part_store2(__amdgpu_buffer_rsrc_t r, unsigned at, float2 v) {
    u32x2 u;
    u[0] = __float_as_uint(v.x); u[1] = __float_as_uint(v.y);
    __builtin_amdgcn_raw_buffer_store_b64(u, r, (int)at, 0, kDevScope);
}
__device__ __forceinline__ float4 part_load4(__amdgpu_buffer_rsrc_t r, unsigned at) {
    const u32x4 u = __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, kDevScope);
    return make_float4(__uint_as_float(u[0]), __uint_as_float(u[1]), __uint_as_float(u[2]), __uint_as_float(u[3]));
}
__device__ __forceinline__ float2 part_load2(__amdgpu_buffer_rsrc_t r, unsigned at) {
    const u32x2 u = __builtin_amdgcn_raw_buffer_load_b64(r, (int)at, 0, kDevScope);
    return make_float2(__uint_as_float(u[0]), __uint_as_float(u[1]));
}

// ---------------------------------------------------------------------------------------------
// The work of a call.  A KV head's items -- the row tiles of its branches, one after the other -- form a sequence in which every key tile
// takes as many places as it takes time, all heads' sequences follow one another, and worker w of W gets the w-th of equal pieces of
// the whole, whatever the branches' lengths and numbers of new tokens are.  Where a piece ends inside an item, the item has a partial
// result from either side.  Nothing of this is known to the host: every workgroup finds its piece from the lengths of all branches,
// 64 item slots at a time, a lane each.
//   Items are narrow (all rows of a branch, at most NARROW_TILES * 32: the keys are dealt to the wavefronts) or wide (kWideRows rows: the rows
//   are dealt to them).  The slots of branch b begin at floor(q_start[b] * G / kWideRows) + b, which leaves room for its ceil(n * G / kWideRows)
//   items and needs no sum over the branches; a narrow branch uses the first of its slots.  Without wide items a slot is a branch.
// ---------------------------------------------------------------------------------------------
struct Items {        // of the lane
    unsigned end;     // places of the head's sequence up to the end of this item
    int b, first, n, L, row0, tiles, cost;
};
template <bool WIDE>
__device__ __forceinline__ int first_slot(const PagedParams& p, int b) {
    if (!WIDE) return b;
    const int first = p.q_start ? min(max(p.q_start[b], 0), p.T) : b * p.R;
    return (int)((long long)first * p.G / kWideRows) + b;
}
template <int D, bool WIDE, int NARROW_TILES>
__device__ __forceinline__ Items items_at(const PagedParams& p, int base, unsigned before, int lane) {
    const int slot = base + lane;
    Items t;
    int b = min(slot, p.B - 1);
    if (WIDE) {  // the last branch whose slots begin at or before this one
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (first_slot<true>(p, mid) <= slot) lo = mid;
            else hi = mid - 1;
        }
        b = lo;
    }
    const Branch br = branch_at(p, b);
    const int rows = br.n * p.G;
    const bool narrow = !WIDE || rows <= NARROW_TILES * 32;
    const int j = slot - first_slot<WIDE>(p, b);
    t.row0 = j * kWideRows;
    const bool there = slot < p.items && (narrow ? j == 0 && rows > 0 : j >= 0 && t.row0 < rows);
    const int end = narrow ? rows : min(t.row0 + kWideRows, rows);
    const int keys = max(1, br.L - br.n + quot(max(end, 1) - 1, p.d_g) + 1);
    t.b = b; t.first = br.first; t.n = br.n; t.L = br.L;
    t.tiles = narrow ? (keys - 1) / kNarrowTile + 1 : (keys - 1) / kWideTile + 1;
    t.cost = there ? kStartCost + t.tiles * (narrow ? kNarrowCost : wide_cost(D)) : 0;
    t.end = before + wave_incl_scan_u32((unsigned)t.cost);
    return t;
}

// Pieces: any rising function of w does as long as all agree on it.
struct Pieces {
    double places;
    int workers;
    __device__ __forceinline__ long long start(int w) const { return (long long)(places * w / workers); }
    __device__ __forceinline__ int worker(long long at) const {
        int w = min((int)((double)at * workers / places), workers - 1);
        while (w > 0 && start(w) > at) --w;
        while (w + 1 < workers && start(w + 1) <= at) ++w;
        return w;
    }
};

// A part of an item: rows [row0, row0 + nrows) of the stack of (branch, KV head) against the key tiles [lo, hi) of its `tiles`.
struct Segment {
    int b, kvh, first, n, L, row0, nrows;
    int lo, hi, tiles;
    int part, parts;              // the item is worked on in `parts` pieces, this is the part-th
    int slot0, slot1, slot_step;  // where their results lie: slot0, then slot1 + i * slot_step
    __device__ __forceinline__ int slot(int i) const { return i == 0 ? slot0 : slot1 + i * slot_step; }
};

// Output quad c4 of row r of a segment: normalised and rounded; the first quad's thread stores the lse.
__device__ __forceinline__ void store_out(const PagedParams& p, const Segment& g, int r, int c4, float4 o, float M, float l) {
    const int i = quot(g.row0 + r, p.d_g), h = g.kvh * p.G + g.row0 + r - i * p.G;
    const float inv = l == 0.f ? 0.f : 1.0f / l;  // a row that sees nothing is 0
    bf16x4 v;
    v[0] = (__bf16)(o.x * inv);
    v[1] = (__bf16)(o.y * inv);
    v[2] = (__bf16)(o.z * inv);
    v[3] = (__bf16)(o.w * inv);
    *reinterpret_cast<bf16x4*>((unsigned char*)p.O + (long long)(g.first + i) * p.o_t + h * p.o_h + c4 * 8) = v;
    if (p.lse && c4 == 0) p.lse[(long long)(g.first + i) * p.Hq + h] = (M * p.scale_log2 + log2f(l)) * 0.69314718055994530942f;
}

// Merges partials [from, from + count) of the segment's item -- every STEP-th of them -- in their order: into the output, or in place of the first.
template <int D, int WAVES>
__device__ __forceinline__ void merge_parts(const PagedParams& p, const Segment& g, __amdgpu_buffer_rsrc_t rs, int from, int count, int step, bool last) {
    constexpr int F4 = D / 4, CH = 8;
    for (int e = threadIdx.x; e < g.nrows * F4; e += WAVES * kWave) {  // (a row's quads lie in one wavefront: what is read comes in front of what is written)
        const int r = e / F4, c4 = e - r * F4;
        float M = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        unsigned first_at = 0;
        for (int s0 = 0; s0 < count; s0 += CH) {
            float2 ml[CH];
            float4 v[CH];
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                ml[j] = make_float2(-INFINITY, 0.f);
                v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (s0 + j < count) {
                    const unsigned row = (unsigned)g.slot(from + (s0 + j) * step) * p.part_rows + r;
                    if (s0 + j == 0) first_at = row;
                    ml[j] = part_load2(rs, p.off_ml + row * 8u);
                    v[j] = part_load4(rs, p.off_o + (row * D + c4 * 4) * 4u);
                }
            }
            float Mn = M;
#pragma unroll
            for (int j = 0; j < CH; ++j) Mn = fmaxf(Mn, ml[j].x);
            const float Mu = Mn == -INFINITY ? 0.f : Mn, a = __builtin_amdgcn_exp2f((M - Mu) * p.scale_log2);
            l *= a;
            o.x *= a; o.y *= a; o.z *= a; o.w *= a;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const float w = __builtin_amdgcn_exp2f((ml[j].x - Mu) * p.scale_log2);
                l += ml[j].y * w;
                o.x += v[j].x * w; o.y += v[j].y * w; o.z += v[j].z * w; o.w += v[j].w * w;
            }
            M = Mn;
        }
        if (last) {
            store_out(p, g, r, c4, o, M, l);
        } else {
            part_store4(rs, p.off_o + (first_at * D + c4 * 4) * 4u, o);
            if (c4 == 0) part_store2(rs, p.off_ml + first_at * 8u, make_float2(M, l));
        }
    }
}

// The workgroup's partial of a cut item is written: it counts itself, and whoever comes last merges -- kMergeGroup neighbours first, then what
// these have left.  Every wavefront waits for its stores before the count.  A cell starts at the call's tag, which is larger than that
// of any earlier call, and goes back to zero: a captured launch is replayed with its tag.
template <int D, int WAVES>
__device__ __forceinline__ void arrive(const PagedParams& p, const Segment& g, __amdgpu_buffer_rsrc_t rs, int* sh) {
    auto last_of = [&](unsigned long long* cell, int count) {
        __builtin_amdgcn_s_waitcnt(0);  // the wavefront's stores are in memory
        __syncthreads();
        if (threadIdx.x == 0) {
            atomicMax(cell, p.tag);
            const bool last = atomicAdd(cell, 1ull) + 1 == p.tag + count;
            if (last) __hip_atomic_store(cell, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *sh = last;
        }
        __syncthreads();
        const bool last = *sh != 0;
        __syncthreads();
        return last;
    };
    const int group = g.part / kMergeGroup, first = group * kMergeGroup, members = min(kMergeGroup, g.parts - first);
    const bool one_group = g.parts <= kMergeGroup;
    if (members > 1) {
        if (!last_of(p.cells + g.slot(first), members)) return;
        merge_parts<D, WAVES>(p, g, rs, first, members, 1, one_group);
    }
    if (one_group) return;
    const int groups = (g.parts - 1) / kMergeGroup + 1;
    if (!last_of(p.cells + 2 * p.workers + g.slot(0), groups)) return;
    merge_parts<D, WAVES>(p, g, rs, 0, groups, kMergeGroup, true);
}

// A branch's entry for a key.  (Both kinds of item look up 64 tiles' at a time, a lane each, so that no tile waits for its entry.)
__device__ __forceinline__ int page_entry(const PagedParams& p, const int32_t* row, int key) { return row[min(key >> p.shift, p.columns - 1)]; }

// 16 keys of a page: the buffer ends behind the last one that there is, so that keys behind it, and those without a page, read as zeros.
__device__ __forceinline__ unsigned group_bytes(const PagedParams& p, int entry, int key, int keys, int row_bytes) {
    const int n = (unsigned)entry < (unsigned)p.pages ? min(keys - key, kPgGroup) : 0;
    return n > 0 ? (unsigned)(n - 1) * (unsigned)p.page_t + row_bytes : 0;
}
__device__ __forceinline__ long long group_at(const PagedParams& p, int entry, int key, int kvh) {
    return (long long)((unsigned)entry < (unsigned)p.pages ? entry : 0) * p.page_p + kvh * p.page_h + (key & ((1 << p.shift) - 1)) * p.page_t;
}

// ---------------------------------------------------------------------------------------------
// bf16
// ---------------------------------------------------------------------------------------------
template <int D>
struct Tile {
    static constexpr int KS = D / 16;             // MFMA k-steps of the QK^T contraction
    static constexpr int DB = D / 32;             // 32-wide blocks of the head dimension
    static constexpr int LPR = D / 8;             // lanes per key row of a load
    static constexpr int RPI = kWave / LPR;       // key rows per load instruction
    static constexpr int NLD = kPgGroup / RPI;    // load instructions per 16 keys
    static constexpr int OSTRIDE = D + 4;         // floats per row of a parked output
};
// LDS of a wavefront with a narrow item: its tiles, and its output when the states meet.
template <int D>
__host__ __device__ constexpr int narrow_slab(int stages) {
    return std::max(stages * kNarrowTile * D * 4, (32 * Tile<D>::OSTRIDE * 4 + 255) / 256 * 256);
}

// Maximum of a lane's and its partner's 32 lanes away.
__device__ __forceinline__ float max_halves(float v) {
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// One row tile's step: scores of 32 keys, mask, running maximum (of the products as they are; differences from it are scaled, so that the largest
// weight is 1 whatever the scale) and sum; the weights come back in the order in which the product with V takes them.  Register i of a lane is key (i / 4) * 8 + hh * 4 + i % 4 of
// the tile, for row `lane % 32`; vis: keys in front of it are seen; have: bit g: 16 keys from 16 g on lie in a page.
template <int DB>
__device__ __forceinline__ void softmax_step(f32x16& s, f32x16 (&o)[DB], float& m, float& l, bf16x8 (&pf)[2], float scale, int vis, int have, bool masked) {
    if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (i >> 2) * 8 + (i & 3) < vis && (have >> (i >> 3) & 1) ? s[i] : -INFINITY;
    }
    float mx = m;
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i]);
    const float m_new = max_halves(mx), base = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f((m - base) * scale);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float w = __builtin_amdgcn_exp2f((s[i] - base) * scale);
        sum += w;
        pf[i >> 3][i & 7] = (__bf16)w;  // the second product takes bf16 on both sides: a half step, 2^-8 of each weight; the sum keeps fp32
    }
    l = l * alpha + sum;
    m = m_new;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {  // (seldom, once some hundred keys have gone by)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    }
}

// Key tiles get into LDS by the loads themselves, 16 bytes a lane: lane i of a load writes piece i behind
// the load's base, so rows cannot be padded; instead piece c of row r lies at c ^ spread(r), which the lane that loads it picks.  Both the 16-byte row
// reads of K (32 rows, one piece) and the transposing reads of V (8 rows, 4 neighbouring pieces) then meet every bank equally often.
template <int D>
__device__ __forceinline__ int spread(int r) {
    if (D == 128) return (r & 3) << 2 | (r >> 2 & 3);  // 16 pieces a row
    return (r >> 1 & 1) << 2 | (r >> 2 & 3);           // 8 pieces a row, two rows next to each other
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // M0 is on the clobber list on purpose
template <bool ONCE>  // what is read once passes the caches by
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, unsigned off, unsigned lds_base) {
    if (ONCE) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, 0 offen nt lds" : : "v"(off), "s"(lds_base), "s"(r) : "m0");
    else asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" : : "v"(off), "s"(lds_base), "s"(r) : "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ unsigned lds_address(const void* at) {
    return __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) const void*)at);
}

constexpr int kStages = 4;     // tiles in LDS: one whose V is read, one whose K is read, two on their way
// A wide item's weights are exp2(score * scale - maximum * scale), the latter rounded: it is kept up to 2^26, where that is a factor of 4 at most that all
// weights of a row share.  Rows whose scores the scale takes further get a smaller scale: scores that differ by some 2^-20 of the
// largest are 2^6 apart all the same, and the largest has all the weight.  (A difference first and then the product costs 7 % of a chunk's time.)
constexpr float kMaxScaled = 67108864.f;
constexpr float kRescale = 8.f;  // a running maximum may be behind the true one by a factor of 2^8 before the state is rescaled

// Pieces of a tile at an address in LDS, K rows and V rows ROW bytes apart.  (What differs between the pieces of a lane lies in bits of the address that
// its row does not touch: one register and an exclusive or.)
template <int D>
__device__ __forceinline__ unsigned lane_of_k(int lane) {
    return (lane & 31) * (D * 2) + ((lane >> 5) ^ spread<D>(lane & 15)) * 16;
}
template <int D>
__device__ __forceinline__ bf16x8 read_k(unsigned at, int i) {  // A operand of K Q^T: key lane % 32, the i-th 16 of the head dimension
    return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(at ^ (i * 32));
}
template <int D>
__device__ __forceinline__ unsigned lane_of_v(int lane) {
    const int blk = lane >> 4, i16 = lane & 15, r = (blk >> 1) * 4 + (i16 >> 2);
    return r * (D * 2) + (((blk & 1) * 2 + (i16 >> 1 & 1)) ^ spread<D>(r)) * 16 + (i16 & 1) * 8;
}
template <int D>
__device__ __forceinline__ bf16x8 read_v(unsigned at, int kk, int db) {  // A operand of V^T P^T: 32 columns from 32 db on, the kk-th 16 keys
    union {
        short4v s[2];
        bf16x8 v;
    } f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
        f.s[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(uintptr_t)((at ^ (db * 64 + h * 32)) + (kk * 16 + h * 8) * (D * 2)));
    return f.v;
}

// Infinities and NaN in V.  A row's weight for a later token of its chunk is 0, but the product with V takes it all the same, and 0 times an infinity is
// NaN.  So where some rows of an item do not see a key, what is not finite in the key's row of V is taken out of LDS before the products, and the rows that
// see it get NaN in its columns afterwards.  (Looking costs the drafts of 16 branches 0.2 %, a prompt of 2039 0.8 %, one of 1500 with as many KV heads as
// query heads 2.3 %, 31.4 us for 30.7; with NaN all over V these take 53, 58 and 85 us.  Adding the values themselves, by conditions an element, made the
// wide kernels 10 KB larger and a prompt 2 us slower.)
__device__ __forceinline__ unsigned not_finite(unsigned two) {  // bits 15 and 31: of a bf16 whose exponent's bits are all set
    return ((two & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
// 16 bytes of every lane, at an address in LDS; whether anything was taken out.
__device__ __forceinline__ bool keep_finite(unsigned at) {
    __attribute__((address_space(3))) u32x4* piece = (__attribute__((address_space(3))) u32x4*)(uintptr_t)at;
    u32x4 v = *piece;
    if (__builtin_expect(__ballot((not_finite(v[0]) | not_finite(v[1]) | not_finite(v[2]) | not_finite(v[3])) != 0) == 0, 1)) return false;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] &= ~((not_finite(v[i]) >> 15) * 0xffffu);
    *piece = v;
    return true;
}
// Columns of V that the lane looks after, and the first key in whose row they are not finite.
template <int D>
struct NotFinite {
    static constexpr int C = D / kWave;
    int first[C];
    __device__ __forceinline__ NotFinite() {
#pragma unroll
        for (int i = 0; i < C; ++i) first[i] = 0x7fffffff;
    }
    __device__ __forceinline__ void look(const PagedParams& p, const int32_t* row, int kvh, int from, int to) {  // the later, the larger the keys
#pragma unroll 4
        for (int key = from; key < to; ++key) {
            const int e = page_entry(p, row, key);
            const bool there = (unsigned)e < (unsigned)p.pages;  // (in no page: that of page 0 is read for nothing)
            const unsigned short* v = reinterpret_cast<const unsigned short*>((const unsigned char*)p.V + group_at(p, e, key, kvh)) + (threadIdx.x & (kWave - 1)) * C;
#pragma unroll
            for (int i = 0; i < C; ++i)
                if (there && (v[i] & 0x7f80) == 0x7f80) first[i] = min(first[i], key);
        }
    }
    // at: D words of LDS that are the wavefront's.
    __device__ __forceinline__ void publish(unsigned at) const {
#pragma unroll
        for (int i = 0; i < C; ++i) *(__attribute__((address_space(3))) int*)(uintptr_t)(at + ((threadIdx.x & (kWave - 1)) * C + i) * 4) = first[i];
    }
    // The outputs of the lane's row, which sees the keys in front of lim.
    static __device__ __forceinline__ void mark(unsigned at, int lim, f32x16 (&o)[D / 32]) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u32x4 k = *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)(at + (db * 32 + q * 8 + (threadIdx.x & 32) / 8) * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[db][q * 4 + i] = (int)k[i] < lim ? NAN : o[db][q * 4 + i];
            }
    }
};

// A narrow item's part: wavefront w takes tiles lo + w, lo + w + WAVES, ..., through STAGES slabs of its own: with two, the next tile is on its way while
// one is worked on; with one, the other wavefronts' are.
template <int D, int TW, int WAVES, int STAGES>
__device__ __forceinline__ void narrow_segment(const PagedParams& p, const Segment& g, unsigned char* lds, float (*sh_m)[32], float (*sh_l)[32], int* sh_bad, int (*sh_first)[D], int* sh) {
    using X = Tile<D>;
    constexpr int ROW = D * 2, HALF = kNarrowTile * ROW, SLAB = narrow_slab<D>(STAGES), LOADS = 4 * X::NLD;  // of a tile
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid & (kWave - 1);
    const int ln = lane & 31, hh = lane >> 5;
    const int32_t* row = p.table + g.b * p.table_stride;
    const int keys = min(g.L, max(0, g.L - g.n + quot(g.nrows - 1, p.d_g) + 1)), before = g.L - g.n;
    const int n_tiles = g.lo + wave < g.hi ? (g.hi - 1 - g.lo - wave) / WAVES + 1 : 0;
    const int v_row = lane / X::LPR, v_slot = lane % X::LPR;
    const unsigned slab = lds_address(lds) + wave * SLAB, row_off = (unsigned)v_row * (unsigned)p.page_t;
    const unsigned piece = (v_slot ^ spread<D>(v_row)) * 16;  // of the first load; the others' differ in the bits that spread() takes from the row's upper part
    // Lane i knows of the wavefront's tile ahead_from + i where its two groups of 16 keys lie and how many bytes of them there are (none
    // without a page, and behind the last key).
    unsigned ahead_lo[2], ahead_hi[2], ahead_bytes[2];
    int ahead_from = 0;
    auto look_ahead = [&](int it) {
        ahead_from = it;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int key = (g.lo + wave + (it + lane) * WAVES) * kNarrowTile + h * kPgGroup, e = page_entry(p, row, key);
            const long long at = group_at(p, e, key, g.kvh);
            ahead_lo[h] = (unsigned)at;
            ahead_hi[h] = (unsigned)(at >> 32);
            ahead_bytes[h] = group_bytes(p, e, key, keys, D * 2) | ((unsigned)e < (unsigned)p.pages ? 1u : 0u);  // (a multiple of 16; bit 0: it has a page)
        }
    };
    auto fetch = [&](int it) {
        if (it - ahead_from >= kWave) look_ahead(it);
        const int x = it - ahead_from;
        const unsigned stage = slab + (STAGES > 1 ? (it & 1) * 2 * HALF : 0);
        int have = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long long at = (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane(ahead_hi[h], x) << 32 | (unsigned)__builtin_amdgcn_readlane(ahead_lo[h], x));
            const unsigned bytes = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_readlane(ahead_bytes[h], x));
            have |= (int)(bytes & 1) << h;
            const __amdgpu_buffer_rsrc_t kr = buffer((const unsigned char*)p.K + at, bytes & ~1u), vr = buffer((const unsigned char*)p.V + at, bytes & ~1u);
#pragma unroll
            for (int i = 0; i < X::NLD; ++i) {
                const unsigned off = row_off + (unsigned)(i * X::RPI) * (unsigned)p.page_t + (piece ^ spread<D>(i * X::RPI) * 16);
                load_to_lds<true>(kr, off, stage + h * kPgGroup * ROW + i * 1024);
                load_to_lds<true>(vr, off, stage + HALF + h * kPgGroup * ROW + i * 1024);
            }
        }
        return have;
    };
    int have_next = 0;
    if (n_tiles > 0) {
        look_ahead(0);
        have_next = fetch(0);
    }
    bf16x8 qf[TW][X::KS];
    int lim[TW];
#pragma unroll
    for (int t = 0; t < TW; ++t) {
        const int r = min(t * 32 + ln, g.nrows - 1), i = quot(r, p.d_g);
        lim[t] = before + i + 1;
        const unsigned char* qp = (const unsigned char*)p.Q + (long long)(g.first + i) * p.q_t + (g.kvh * p.G + r - i * p.G) * p.q_h;
#pragma unroll
        for (int s = 0; s < X::KS; ++s) qf[t][s] = *reinterpret_cast<const bf16x8*>(qp + (2 * s + hh) * 16);
    }
    const bool two = TW > 1 && g.nrows > 32;
    bool taken_out = false;
    const int unseen = g.n > 1 ? (before + 1) & -X::RPI : 0x7fffffff;  // keys that not all rows see, and those that a load brings with them
    const unsigned kat = slab + lane_of_k<D>(lane), vat = slab + HALF + lane_of_v<D>(lane);
    f32x16 oacc[TW][X::DB];
    float m_run[TW], l_run[TW];
#pragma unroll
    for (int t = 0; t < TW; ++t) {
        m_run[t] = -INFINITY;
        l_run[t] = 0.f;
#pragma unroll
        for (int db = 0; db < X::DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[t][db][i] = 0.f;
    }
    for (int it = 0; it < n_tiles; ++it) {
        const int kb = (g.lo + wave + it * WAVES) * kNarrowTile, have = have_next;
        const unsigned stage = STAGES > 1 ? (it & 1) * 2 * HALF : 0;
        if (STAGES > 1 && it + 1 < n_tiles) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile before has been read
            have_next = fetch(it + 1);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        if (__builtin_expect(kb + kNarrowTile > unseen, 0)) {
#pragma unroll 1
            for (int key = max(kb, unseen); key < min(kb + kNarrowTile, keys); key += X::RPI)
                taken_out |= keep_finite(slab + stage + HALF + (key - kb) * ROW + lane * 16);
        }
        const bool masked = have != 3 || kb + kNarrowTile > before + 1;
        bf16x8 kf[X::KS], pf[TW][2];
#pragma unroll
        for (int s = 0; s < X::KS; ++s) kf[s] = read_k<D>(kat + stage, s);
#pragma unroll
        for (int t = 0; t < TW; ++t) {
            if (t > 0 && !two) continue;
            f32x16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
            for (int k = 0; k < X::KS; ++k) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], qf[t][k], s, 0, 0, 0);
            softmax_step<X::DB>(s, oacc[t], m_run[t], l_run[t], pf[t], p.scale_log2, lim[t] - kb - hh * 4, have, masked);
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int db = 0; db < X::DB; ++db) {
                const bf16x8 v = read_v<D>(vat + stage, kk, db);
#pragma unroll
                for (int t = 0; t < TW; ++t)
                    if (t == 0 || two) oacc[t][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[t][kk], oacc[t][db], 0, 0, 0);
            }
        if (STAGES == 1 && it + 1 < n_tiles) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            have_next = fetch(it + 1);
        }
    }
    if (__builtin_expect(taken_out, 0)) {
        NotFinite<D> bad;
#pragma unroll 1
        for (int it = 0; it < n_tiles; ++it) {
            const int kb = (g.lo + wave + it * WAVES) * kNarrowTile;
            bad.look(p, row, g.kvh, max(kb, unseen), min(kb + kNarrowTile, keys));
        }
        bad.publish(lds_address(sh_first[wave]));
    }
    sh_bad[wave] = taken_out;
    // the wavefronts' states of a row tile meet in LDS, in their order
    const __amdgpu_buffer_rsrc_t rs = buffer(p.ws, p.ws_bytes);
    constexpr int F4 = D / 4, QPT = 32 * F4 / (WAVES * kWave), RSTEP = WAVES * kWave / F4;
    const int c4 = tid % F4, row0 = tid / F4;
    float* obuf = reinterpret_cast<float*>(lds + wave * SLAB);
#pragma unroll
    for (int t = 0; t < TW; ++t) {
        if (t > 0 && !two) continue;
        if (t > 0) __syncthreads();  // the row tile before has been read
        const float l = l_run[t] + shfl_xor_f(l_run[t], 32);
        if (hh == 0) {
            sh_m[wave][ln] = m_run[t];
            sh_l[wave][ln] = l;
        }
#pragma unroll
        for (int db = 0; db < X::DB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<float4*>(obuf + ln * X::OSTRIDE + db * 32 + q * 8 + hh * 4) =
                    make_float4(oacc[t][db][q * 4], oacc[t][db][q * 4 + 1], oacc[t][db][q * 4 + 2], oacc[t][db][q * 4 + 3]);
        __syncthreads();
        const bool any_bad = __ballot(sh_bad[lane % WAVES] != 0) != 0;
#pragma unroll
        for (int q = 0; q < QPT; ++q) {
            const int rt = row0 + q * RSTEP, r = t * 32 + rt;
            if (r >= g.nrows) continue;
            float M = -INFINITY, sum = 0.f;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) M = fmaxf(M, sh_m[v][rt]);
            const float Mu = M == -INFINITY ? 0.f : M;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int v = 0; v < WAVES; ++v) {
                const float f = __builtin_amdgcn_exp2f((sh_m[v][rt] - Mu) * p.scale_log2);
                const float4 ov = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(lds + v * SLAB) + rt * X::OSTRIDE + c4 * 4);
                sum += sh_l[v][rt] * f;
                o.x += ov.x * f; o.y += ov.y * f; o.z += ov.z * f; o.w += ov.w * f;
            }
            if (__builtin_expect(any_bad, 0)) {
                const int sees = before + quot(r, p.d_g) + 1;
#pragma unroll 1
                for (int v = 0; v < WAVES; ++v) {
                    if (!sh_bad[v]) continue;
                    const int4 k = *reinterpret_cast<const int4*>(&sh_first[v][c4 * 4]);
                    o.x = k.x < sees ? NAN : o.x;
                    o.y = k.y < sees ? NAN : o.y;
                    o.z = k.z < sees ? NAN : o.z;
                    o.w = k.w < sees ? NAN : o.w;
                }
            }
            if (g.parts == 1) {
                store_out(p, g, r, c4, o, M, sum);
            } else {
                const unsigned at = (unsigned)g.slot(g.part) * p.part_rows + r;
                part_store4(rs, p.off_o + (at * D + c4 * 4) * 4u, o);
                if (c4 == 0) part_store2(rs, p.off_ml + at * 8u, make_float2(M, sum));
            }
        }
    }
    if (g.parts > 1) arrive<D, WAVES>(p, g, rs, sh);
    __syncthreads();  // the slabs are free
}

// ---- wide items ----
// Loads of a wavefront for its keys of a tile, K or V.
template <int D>
__device__ constexpr int wide_loads() {
    return D == 128 ? 2 : 1;
}

// The products of a wide item are written as instructions, on vector registers, so that a slot of the loop below holds what it was given.  (Left to choose, the
// compiler put the scores into accumulation registers, Q into scratch memory and the waits for that into the loop.)  It does not know how long
// these take: what reads a result on the vector units is kept behind two later products, or behind mfma_done(), which hands the result on (a wait
// without it is no reason for the compiler to keep what reads the result behind the wait).
__device__ __forceinline__ void mfma_first(f32x16& d, const bf16x8& a, const bf16x8& b) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_onto(f32x16& d, const bf16x8& a, const bf16x8& b) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_done(f32x16& d) { asm volatile("s_nop 15\n\ts_nop 15" : "+v"(d)); }
template <int N>
__device__ __forceinline__ void mfma_done(f32x16 (&d)[N]) {
    static_assert(N == 2 || N == 4, "blocks of the head dimension");
    if constexpr (N == 2) asm volatile("s_nop 15\n\ts_nop 15" : "+v"(d[0]), "+v"(d[1]));
    else asm volatile("s_nop 15\n\ts_nop 15" : "+v"(d[0]), "+v"(d[1]), "+v"(d[2]), "+v"(d[3]));
}

// The loop over a wide item's tiles for a wavefront with a row tile.  arrive(): the next tile is in LDS for everybody; request(j, v, i): load i of the
// wavefront's part of tile j's K or V.  In a step 32 keys are weighed and multiplied with V while the next 32 are multiplied with Q and their maximum
// is found.  Two wavefronts share a SIMD, each issues in order: a product takes 32 cycles of the matrix unit beside whatever comes behind it, but a
// vector instruction that needs the one before it waits 8 cycles (independent ones take 4 to 8 by their length, an exponential 9).  So the step is
// written down as slots of one product each, and a pair of weights goes through three of them -- scaled, exponential, rounded and summed -- so
// that nothing in a slot depends on anything else in it; scheduling barriers keep the slots apart.  Loads go out a few a step: all of a tile's at
// once held the wavefronts 1000 to 1600 cycles a tile.  (4 wavefronts of two row tiles, a SIMD each: a prompt of 2039 tokens,
// 16 / 2 heads, 81 us against 62 with 8; 2 chunks of 2048 alike.)
template <int D, typename Arrive, typename Request>
__device__ __forceinline__ void wide_rows(const PagedParams& p, int lo, int hi, const bf16x8 (&qf)[Tile<D>::KS], int lim,
                                          int first_lim, unsigned kat, unsigned vat, f32x16 (&o)[Tile<D>::DB], float& m, float& l, Arrive arrive, Request request) {
    using X = Tile<D>;
    constexpr int ROW = D * 2, HALF = kWideTile * ROW, STAGE = 2 * HALF;
    constexpr int QS = X::KS, VS = 2 * X::DB;   // slots: products of 32 keys with K and with V
    constexpr int LOADS = wide_loads<D>(), EARLY = LOADS / 2;  // of a wavefront and operand; those beside products with K
    constexpr int AHEAD = 3;                    // slots between a read from LDS and its use
    constexpr int PAIRS = 8;                    // pairs of weights: the first half goes into the first half of the products with V
    constexpr int SPAN = QS + X::DB - (D == 64 ? 3 : 2);  // slots over which they begin: done two slots before their product
    constexpr int LOOK = QS + 2, LOOKS = VS - 3;  // slots that look at the next scores: two products behind the last one that makes them, up to the last but one
    float row_scale = p.scale_log2, negm = 0.f, mx = -INFINITY, l2 = 0.f;  // l2: the sums of every second weight
    f32x16 sa, sb;  // scores as products leave them, in turns: of the keys that are weighed, of the next ones
    bf16x8 pf[2];
    const float scale = p.scale_log2, rescale = fminf(kRescale / scale, 3.0e38f);  // (finite however small the scale: the first maximum always counts)
    auto read_k = [&](unsigned st, int i) { return lotts::read_k<D>(st + kat, i); };
    auto read_v = [&](unsigned st, int i) { return lotts::read_v<D>(st + vat, i / X::DB, i % X::DB); };
    // (Every result is pinned where it is computed: the compiler would move it down to its use, behind the mask's branch.)
    auto scale_pair = [&](f32x16& c, int q) {
        const int x = q * 2;
        float u = __builtin_fmaf(c[x], row_scale, negm), v = __builtin_fmaf(c[x + 1], row_scale, negm);
        asm volatile("" : "+v"(u), "+v"(v));
        c[x] = u;
        c[x + 1] = v;
    };
    auto weigh_pair = [&](f32x16& c, int q) {
        const int x = q * 2;
        float u = __builtin_amdgcn_exp2f(c[x]), v = __builtin_amdgcn_exp2f(c[x + 1]);
        asm volatile("" : "+v"(u), "+v"(v));
        c[x] = u;
        c[x + 1] = v;
    };
    auto sum_pair = [&](f32x16& c, int q) {
        const int x = q * 2;
        // the second product takes bf16 on both sides: a half step, 2^-8 of each weight; the sum keeps fp32
        const f32x2 pair = {c[x], c[x + 1]};
        unsigned u = __builtin_bit_cast(unsigned, __builtin_convertvector(pair, bf16x2));
        l += c[x];
        l2 += c[x + 1];
        asm volatile("" : "+v"(l), "+v"(l2), "+v"(u));
        u32x4 all = __builtin_bit_cast(u32x4, pf[x >> 3]);
        all[(x & 7) >> 1] = u;
        pf[x >> 3] = __builtin_bit_cast(bf16x8, all);
    };
    auto look = [&](const f32x16& n, int r) {  // a pair of the next scores
        const int x = r * 2;
        mx = fmaxf(fmaxf(mx, n[x]), n[x + 1]);
        asm volatile("" : "+v"(mx));
    };
    // what goes beside the product of slot i
    auto beside = [&](f32x16& c, const f32x16& n, int i) {
#pragma unroll
        for (int q = 0; q < PAIRS; ++q) {
            if (q * SPAN / PAIRS + 2 == i) sum_pair(c, q);
            if (q * SPAN / PAIRS + 1 == i) weigh_pair(c, q);
            if (q * SPAN / PAIRS == i) scale_pair(c, q);
        }
        if (i >= LOOK) {
#pragma unroll
            for (int r = 0; r < PAIRS; ++r)
                if (LOOK + r * LOOKS / PAIRS == i) look(n, r);
        }
    };
    auto mask = [&](f32x16& n, int kb, int have) {
        if ((have & 3) == 3 && kb + 32 <= first_lim) return;
        mfma_done(n);
        const int hh = (threadIdx.x & 32) >> 5;
        const int vis = lim - kb - hh * 4;
#pragma unroll
        for (int x = 0; x < 16; ++x) n[x] = (x >> 2) * 8 + (x & 3) < vis && (have >> (x >> 3) & 1) ? n[x] : -INFINITY;
    };
    bool rise = false;
    auto find_rise = [&] {
        mx = max_halves(mx);
        rise = mx > m + rescale;
    };
    auto settle = [&] {  // o and l follow where the maximum has risen much
        if (__builtin_amdgcn_ballot_w64(rise) != 0) {
            mfma_done(o);
            const float m_new = rise ? mx : m;
            const float base = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f((m - base) * scale);
            m = m_new;
            row_scale = fabsf(base) * scale > kMaxScaled ? kMaxScaled / fabsf(base) : scale;
            negm = -base * row_scale;
            l *= alpha;
            l2 *= alpha;
#pragma unroll
            for (int db = 0; db < X::DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
        }
        mx = -INFINITY;
    };
    auto multiply_k = [&](f32x16& n, int i, const bf16x8& k) {
        if (i == 0) mfma_first(n, k, qf[i]);
        else mfma_onto(n, k, qf[i]);
    };
    auto multiply_v = [&](int i, const bf16x8& v) { mfma_onto(o[i % X::DB], v, pf[i / X::DB]); };
    bf16x8 k0[AHEAD];  // the first pieces of K of the step ahead
    int have;
    unsigned st = lo % kStages * STAGE;
    // Step j: the scores in c, of the keys at st, are weighed and multiplied with V, those of the j-th 32 keys of all go into n.
    auto step = [&](f32x16& c, f32x16& n, int j) {
        const unsigned before = st;
        st = (j >> 1) % kStages * STAGE + (j & 1) * 32 * ROW;
        have >>= 2;
        bf16x8 f[QS + VS];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) f[i] = k0[i];
#pragma unroll
        for (int i = 0; i < QS; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            f[i + AHEAD] = i + AHEAD < QS ? read_k(st, i + AHEAD) : read_v(before, i + AHEAD - QS);
            multiply_k(n, i, f[i]);
            beside(c, n, i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = 0; r < EARLY; ++r)
                if (i == (2 * r + 1) * QS / (2 * (EARLY > 0 ? EARLY : 1))) request((j >> 1) + 2, j & 1, r);
        }
        if (D == 64) asm volatile("s_nop 1");  // (the first half's last weights were rounded in the slot before)
        mask(n, j * 32, have);
        const unsigned after = ((j + 1) >> 1) % kStages * STAGE + ((j + 1) & 1) * 32 * ROW;
        // the tile of the next step's K, so that its first pieces are read beside the products with V
        if ((j & 1) != 0 && j + 1 < 2 * hi) have = arrive(false, after) << 2;
#pragma unroll
        for (int i = 0; i < VS; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i + AHEAD < VS) f[QS + i + AHEAD] = read_v(before, i + AHEAD);
            else k0[i + AHEAD - VS] = read_k(after, i + AHEAD - VS);
            multiply_v(i, f[QS + i]);
            beside(c, n, QS + i);
            if (i == VS - 1) find_rise();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = EARLY; r < LOADS; ++r)
                if (i == (2 * (r - EARLY) + 1) * VS / (2 * (LOADS - EARLY))) request((j >> 1) + 2, j & 1, r);
        }
        settle();
    };
    // the last scores: nothing is left to multiply with Q
    auto finish = [&](f32x16& c) {
#pragma unroll
        for (int q = 0; q < PAIRS; ++q) scale_pair(c, q);
#pragma unroll
        for (int q = 0; q < PAIRS; ++q) weigh_pair(c, q);
#pragma unroll
        for (int q = 0; q < PAIRS; ++q) sum_pair(c, q);
        asm volatile("s_nop 1");
#pragma unroll
        for (int i = 0; i < VS; ++i) {
            const bf16x8 v = read_v(st, i);
            multiply_v(i, v);
        }
        mfma_done(o);
    };
    have = arrive(true, st);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) request(lo + 2, 0, i);
#pragma unroll
    for (int i = 0; i < QS; ++i) {
        const bf16x8 k = read_k(st, i);
        multiply_k(sa, i, k);
    }
    mfma_done(sa);
    mask(sa, lo * kWideTile, have);
#pragma unroll
    for (int r = 0; r < PAIRS; ++r) look(sa, r);
    find_rise();
    settle();
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) k0[i] = read_k(st + 32 * ROW, i);
    for (int it = lo; it + 1 < hi; ++it) {
        step(sa, sb, 2 * it + 1);
        step(sb, sa, 2 * it + 2);
    }
    step(sa, sb, 2 * hi - 1);
    finish(sb);
    l += l2;
}

// The workgroup loads a tile together, 8 keys a wavefront; wavefront w takes row tile w of the item.
template <int D, int WAVES>
__device__ __forceinline__ void wide_segment(const PagedParams& p, const Segment& g, unsigned char* lds, int* sh, int* sh_bad) {
    using X = Tile<D>;
    constexpr int KEYS = kWideTile / WAVES, LOADS = wide_loads<D>();
    static_assert(WAVES * 32 == kWideRows && KEYS * WAVES == kWideTile && KEYS <= kPgGroup && KEYS == LOADS * X::RPI, "a row tile and some keys of a tile for every wavefront");
    constexpr int ROW = D * 2, HALF = kWideTile * ROW, STAGE = 2 * HALF;  // bytes
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid & (kWave - 1);
    const int ln = lane & 31, hh = lane >> 5;
    const int32_t* row = p.table + g.b * p.table_stride;
    const int before = g.L - g.n;  // row r of the stack sees the keys in front of before + r / G + 1
    const int keys = max(0, before + quot(g.row0 + g.nrows - 1, p.d_g) + 1);
    const int first_lim = before + quot(min(g.row0 + wave * 32, g.row0 + g.nrows - 1), p.d_g) + 1;  // what all rows of the wavefront see
    const int v_row = lane / X::LPR, v_slot = lane % X::LPR;
    // Lane i knows of tile ahead_from + i: where the wavefront's keys lie, how many bytes of them there are (none without a page, and behind
    // the last key), and which of the tile's four groups have a page.
    unsigned ahead_lo = 0, ahead_hi = 0, ahead_bytes = 0;
    int ahead_have = 0, ahead_from = 0;
    auto look_ahead = [&](int it) {
        ahead_from = it;
        ahead_have = 0;
        const int kb = (it + lane) * kWideTile;
#pragma unroll
        for (int i = 0; i < kWideTile / kPgGroup; ++i) {
            const int e = page_entry(p, row, kb + i * kPgGroup);
            if ((unsigned)e < (unsigned)p.pages) ahead_have |= 1 << i;
            if (i == wave * KEYS / kPgGroup) {
                const int key = kb + wave * KEYS;
                const long long at = group_at(p, e, key, g.kvh);
                ahead_lo = (unsigned)at;
                ahead_hi = (unsigned)(at >> 32);
                ahead_bytes = group_bytes(p, e, key, min(keys, key + KEYS), D * 2);
            }
        }
    };
    const unsigned row_off = (unsigned)v_row * (unsigned)p.page_t;
    unsigned piece = (v_slot ^ spread<D>(wave * KEYS + v_row)) * 16;  // of the first load; the others' differ in the bits that spread() takes from the row's upper part
    const unsigned to = lds_address(lds) + wave * KEYS * ROW;
    int have_0 = 0, have_1 = 0;  // of the tile that arrives next and of the one behind it
    const unsigned long long k_to_v = (unsigned long long)p.V - (unsigned long long)p.K;
    unsigned long long at = 0;
    unsigned bytes = 0, stage = 0;
    // Tiles behind the last one are requested too, with no bytes in range: every wait counts the same loads.
    auto request = [&](int it, int v, int i) {
        if (i == 0 && v == 0) {
            if (it - ahead_from >= kWave) look_ahead(it);
            const int x = it - ahead_from;
            at = (unsigned long long)(unsigned)__builtin_amdgcn_readlane(ahead_hi, x) << 32 | (unsigned)__builtin_amdgcn_readlane(ahead_lo, x);
            bytes = __builtin_amdgcn_readlane(ahead_bytes, x);
            have_1 = __builtin_amdgcn_readlane(ahead_have, x);
            stage = to + it % kStages * STAGE;
        }
        unsigned first = piece;
        asm volatile("" : "+v"(first));  // (formed where it is used: four offsets are three registers more)
        load_to_lds<false>(buffer((const unsigned char*)p.K + (long long)(at + (k_to_v & (unsigned long long)-(long long)v)), bytes), row_off + (unsigned)(i * X::RPI) * (unsigned)p.page_t + (first ^ spread<D>(i * X::RPI) * 16),
                    stage + v * HALF + i * 1024);
    };
    const int unseen = (before + quot(g.row0, p.d_g) + 1) & -KEYS;  // keys that not all rows see, and those that a wavefront loads with them
    int until_unseen = max(0, (unseen - wave * KEYS + kWideTile - 1) / kWideTile) - g.lo;  // tiles to arrive in front of the first one in which the wavefront has such keys
    sh_bad[wave] = 0;  // (whether the wavefront has taken something out of V)
    look_ahead(g.lo);
#pragma unroll
    for (int tile = 0; tile < 2; ++tile) {
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) request(g.lo + tile, v, i);
        if (tile == 0) have_0 = have_1;
    }
    // The next tile is in LDS for everybody; everybody has left the tile before the last behind, whose stage the next requests take.  Loads behind
    // the tile's that are on their way: K and V of the next one at first, then K and half of V of the next one.
    auto arrive_tile = [&](bool first, unsigned stage_at) {
        if (__builtin_expect(--until_unseen < 0, 0)) {
            if (first) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS) : "memory");
            else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS + LOADS / 2) : "memory");
            bool taken_out = false;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) taken_out |= keep_finite(to + stage_at + HALF + i * 1024 + lane * 16);
            if (taken_out) sh_bad[wave] = 1;
        }
        if (first) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS + LOADS / 2) : "memory");
        const int have = have_0;
        have_0 = have_1;
        return have;
    };
    const int q_row = min(g.row0 + wave * 32 + ln, g.row0 + g.nrows - 1), q_token = quot(q_row, p.d_g), lim = before + q_token + 1;
    const unsigned char* qp = (const unsigned char*)p.Q + (long long)(g.first + q_token) * p.q_t + (g.kvh * p.G + q_row - q_token * p.G) * p.q_h;
    bf16x8 qf[X::KS];
#pragma unroll
    for (int s = 0; s < X::KS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qp + (2 * s + hh) * 16);
    const unsigned kat = lds_address(lds) + lane_of_k<D>(lane), vat = lds_address(lds) + HALF + lane_of_v<D>(lane);
    f32x16 oacc[X::DB];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int db = 0; db < X::DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;
    if (wave * 32 < g.nrows) {
        wide_rows<D>(p, g.lo, g.hi, qf, lim, first_lim, kat, vat, oacc, m_run, l_run, arrive_tile, request);
    } else {  // no rows: the loads and the meetings alone, in the same order
        arrive_tile(true, g.lo % kStages * STAGE);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) request(g.lo + 2, 0, i);
        for (int j = g.lo; j + 1 < g.hi; ++j) {
#pragma unroll
            for (int i = 0; i < LOADS / 2; ++i) request(j + 2, 1, i);
            arrive_tile(false, (j + 1) % kStages * STAGE);
#pragma unroll
            for (int i = LOADS / 2; i < LOADS; ++i) request(j + 2, 1, i);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) request(j + 3, 0, i);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // (everybody has met behind the last tile that anything was taken out of)
    if (__builtin_expect(__ballot(sh_bad[lane & (WAVES - 1)] != 0) != 0, 0)) {
        NotFinite<D> bad;
        bad.look(p, row, g.kvh, max(g.lo * kWideTile, unseen), min(g.hi * kWideTile, keys));
        __syncthreads();  // (the tiles have been read)
        bad.publish(lds_address(lds) + wave * D * 4);
        NotFinite<D>::mark(lds_address(lds) + wave * D * 4, lim, oacc);
    }
    const __amdgpu_buffer_rsrc_t rs = buffer(p.ws, p.ws_bytes);
    const float l = l_run + shfl_xor_f(l_run, 32);
    const int r = wave * 32 + ln;
    if (r < g.nrows && g.parts > 1) {
        const unsigned at = (unsigned)g.slot(g.part) * p.part_rows + r;
#pragma unroll
        for (int db = 0; db < X::DB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                part_store4(rs, p.off_o + (at * D + db * 32 + q * 8 + hh * 4) * 4u, make_float4(oacc[db][q * 4], oacc[db][q * 4 + 1], oacc[db][q * 4 + 2], oacc[db][q * 4 + 3]));
        if (hh == 0) part_store2(rs, p.off_ml + at * 8u, make_float2(m_run, l));
    } else if (r < g.nrows) {
        const int i = quot(g.row0 + r, p.d_g), h = g.kvh * p.G + g.row0 + r - i * p.G;
        const float inv = l == 0.f ? 0.f : 1.0f / l;  // a row that sees nothing is 0
        unsigned char* op = (unsigned char*)p.O + (long long)(g.first + i) * p.o_t + h * p.o_h;
#pragma unroll
        for (int db = 0; db < X::DB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (__bf16)(oacc[db][q * 4 + e] * inv);
                *reinterpret_cast<bf16x4*>(op + (db * 32 + q * 8 + hh * 4) * 2) = v;
            }
        if (p.lse && hh == 0) p.lse[(long long)(g.first + i) * p.Hq + h] = (m_run * p.scale_log2 + log2f(l)) * 0.69314718055994530942f;
    }
    if (g.parts > 1) arrive<D, WAVES>(p, g, rs, sh);
    __syncthreads();
}

template <bool WIDE>
__host__ __device__ constexpr int paged_waves() {
    return WIDE ? 8 : 4;
}
template <int D, int NARROW_TILES, bool WIDE, bool TWO>
__global__ __launch_bounds__(paged_waves<WIDE>() * kWave, TWO || WIDE ? 2 : 1) void paged_attn_kernel(const PagedParams p) {
    constexpr int WAVES = paged_waves<WIDE>();
    constexpr int STAGES = WIDE || (TWO && D == 128) ? 1 : 2, NARROW_LDS = WAVES * narrow_slab<D>(STAGES), WIDE_LDS = kStages * kWideTile * 2 * D * 2;
    __shared__ __attribute__((aligned(256))) unsigned char lds[WIDE && WIDE_LDS > NARROW_LDS ? WIDE_LDS : NARROW_LDS];
    __shared__ float sh_m[WAVES][32], sh_l[WAVES][32];
    __shared__ int sh, sh_bad[WAVES];  // sh_bad: whether a wavefront has taken something out of V; sh_first: NotFinite's, of a narrow item
    __shared__ __attribute__((aligned(16))) int sh_first[WAVES][D];
    const int lane = threadIdx.x & (kWave - 1);
    const int per_xcd = p.workers / kNumXCD;  // neighbours in the sequence share an XCD and with it a KV head's keys in its L2
    const int w = (int)(blockIdx.x % kNumXCD) * per_xcd + (int)(blockIdx.x / kNumXCD);
    int base = 0;
    Items items = items_at<D, WIDE, NARROW_TILES>(p, 0, 0, lane);
    unsigned total = __builtin_amdgcn_readlane(items.end, kWave - 1);
    int number = __popcll(__ballot(items.cost > 0));
    for (int s = kWave; s < p.items; s += kWave) {
        const Items more = items_at<D, WIDE, NARROW_TILES>(p, s, total, lane);
        total = __builtin_amdgcn_readlane(more.end, kWave - 1);
        number += __popcll(__ballot(more.cost > 0));
    }
    if (total == 0) return;
    // Every piece has at least one tile of an item that it lies in: whoever counts an item's parts counts on that.
    constexpr int LEAST = WIDE ? kMaxWideCost + 1 : kNarrowCost + 2;
    Pieces pieces;
    pieces.places = (double)total * p.Hkv;
    const double all = (double)number * p.Hkv;  // items
    const double least = !WIDE && pieces.places > kMinPiece * all ? kMinNarrowPiece : kMinPiece;
    pieces.workers = (int)fmax(1.0, fmin(fmin((double)p.workers, pieces.places / LEAST), fmax(all, pieces.places / least)));  // (an item's start is no reason to wait for another's)
    // Short calls with wide items are cut item by item: a cut costs as much as 2 to 4 tiles (256 rows of partial outputs out and in), and a piece of the sequence
    // mostly ends one item and begins another, with a cut on either side.  Each worker gets one part of one item, of about `size` places (0.6: what the last
    // part of an item lacks on average, so that the parts come to a little less than the workers).  Against pieces of the sequence, us, 16 / 2 heads, D = 128:
    // prompts of 200, 400, 850, 2039 and 3000 tokens 29.6, 33, 40, 47.6, 69.5 here, 29.7, 44, 47, 56, 93 there; 4 prompts of 500 36 and 57; 500 behind
    // 11500 80 and 103; 1000 behind 8000 96 and 102 (16 / 16 heads, D = 64: 70 both).  It loses where parts come down to a tile or two each: a prompt of 100
    // with 40 / 8 heads 26 and 14, 99 new of 1244 57 and 47 (16 / 2: 54 and 46), 61 of 7000 with 16 / 2 68 and 61.
    bool apart = false;
    double size = 0.0;
    unsigned parts_total = 0;
    auto parts_of = [&](Items& t, unsigned before) {
        t.cost = t.cost > 0 ? max(1, (int)ceil((t.cost - kStartCost) / size)) : 0;
        t.end = before + wave_incl_scan_u32((unsigned)t.cost);
    };
    if (WIDE && all <= 0.75 * p.workers && pieces.places < kApartPlaces * (double)p.workers) {
        size = fmax(1.0, (pieces.places - all * kStartCost) / (p.workers - 0.6 * all));
        for (int s = 0; s < p.items; s += kWave) {
            Items more = items;
            if (s > 0) more = items_at<D, WIDE, NARROW_TILES>(p, s, 0, lane);
            parts_of(more, parts_total);
            parts_total = __builtin_amdgcn_readlane(more.end, kWave - 1);
        }
        apart = parts_total * (double)p.Hkv <= 2.0 * p.workers;  // as many slots for partials as there are
    }
    long long at, end;
    if (apart) {
        parts_of(items, 0);
        total = parts_total;
        at = w;
        end = (long long)total * p.Hkv;
    } else {
        if (w >= pieces.workers) return;
        at = pieces.start(w);
        end = pieces.start(w + 1);
    }
    while (at < end) {
        const int kvh = __builtin_amdgcn_readfirstlane((int)(at / total));
        const long long head = (long long)kvh * total;
        const unsigned within = __builtin_amdgcn_readfirstlane((unsigned)(at - head));
        auto load = [&](int from, unsigned before) {
            items = items_at<D, WIDE, NARROW_TILES>(p, base = from, before, lane);
            if (apart) parts_of(items, before);
        };
        // the item that has place `within`
        if (base > 0 && (unsigned)(__builtin_amdgcn_readlane(items.end, 0) - __builtin_amdgcn_readlane(items.cost, 0)) > within) load(0, 0);
        while ((unsigned)__builtin_amdgcn_readlane(items.end, kWave - 1) <= within) load(base + kWave, __builtin_amdgcn_readlane(items.end, kWave - 1));
        const int i = __builtin_ctzll(__ballot(items.end > within));
        Segment g;
        g.b = __builtin_amdgcn_readlane(items.b, i);
        g.kvh = kvh;
        g.first = __builtin_amdgcn_readlane(items.first, i);
        g.n = __builtin_amdgcn_readlane(items.n, i);
        g.L = __builtin_amdgcn_readlane(items.L, i);
        g.row0 = __builtin_amdgcn_readlane(items.row0, i);
        g.tiles = __builtin_amdgcn_readlane(items.tiles, i);
        const unsigned item_end = __builtin_amdgcn_readlane(items.end, i);
        const int cost = __builtin_amdgcn_readlane(items.cost, i), rows = g.n * p.G;
        const bool narrow = !WIDE || rows <= NARROW_TILES * 32;
        if (narrow) g.row0 = 0;
        g.nrows = min(p.part_rows, narrow ? rows : min(kWideRows, rows - g.row0));  // (what max_new allows)
        if (apart) {
            g.part = (int)(within - (item_end - cost));
            g.parts = min(cost, g.tiles);
            g.lo = (int)((long long)g.tiles * g.part / g.parts);
            g.hi = g.part < g.parts ? (int)((long long)g.tiles * (g.part + 1) / g.parts) : g.lo;
            g.slot0 = g.slot1 = (int)(head + item_end - cost);
            g.slot_step = 1;
            at += p.workers;
        } else {
            const int each = narrow ? kNarrowCost : wide_cost(D);
            const long long tile0 = head + item_end - cost + kStartCost;
            auto tile_from = [&](long long place) { return place <= tile0 ? 0 : (int)min((long long)g.tiles, (place - tile0 + each - 1) / each); };
            g.lo = tile_from(at);
            g.hi = tile_from(end);
            int w0 = w;
            g.parts = 1;
            if (g.lo < g.hi && (g.lo > 0 || g.hi < g.tiles)) {
                w0 = g.lo > 0 ? pieces.worker(tile0) : w;
                g.parts = (g.hi < g.tiles ? pieces.worker(tile0 + (long long)(g.tiles - 1) * each) : w) - w0 + 1;
            }
            g.part = w - w0;
            // a worker has at most one item that it begins and does not end, and one that it goes on with
            g.slot0 = 2 * w0 + 1;
            g.slot1 = 2 * w0;
            g.slot_step = 2;
            at = head + item_end;
        }
        g.lo = __builtin_amdgcn_readfirstlane(g.lo);
        g.hi = __builtin_amdgcn_readfirstlane(g.hi);
        if (g.lo >= g.hi) continue;
        if constexpr (WIDE) {
            if (narrow) narrow_segment<D, NARROW_TILES, WAVES, STAGES>(p, g, lds, sh_m, sh_l, sh_bad, sh_first, &sh);
            else wide_segment<D, WAVES>(p, g, lds, &sh, sh_bad);
        } else {
            narrow_segment<D, NARROW_TILES, WAVES, STAGES>(p, g, lds, sh_m, sh_l, sh_bad, sh_first, &sh);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// fp32: fp32 arithmetic throughout, a workgroup per row of a head.  A key row is D / 4 lanes of 16 bytes; a wavefront takes every
// WAVES-th chunk of 4 * 256 / D keys (no chunk is larger than 16 keys: it lies in one page) and keeps a running state per D / 4 lanes;
// the states meet at the end.  The maximum is that of the scores as they are and the differences from it are scaled, so that the largest weight is 1
// whatever the scale.
// ---------------------------------------------------------------------------------------------
template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void paged_f32_kernel(const PagedParams p) {
    constexpr int LPK = D / 4, KPL = kWave / LPK, NJ = 4, CHUNK = NJ * KPL;
    __shared__ __attribute__((aligned(16))) float sh_acc[WAVES][D];
    __shared__ float sh_ml[WAVES][2];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid & (kWave - 1);
    const int grp = lane / LPK, c4 = lane % LPK;
    const int t = blockIdx.x / p.Hq, h = blockIdx.x - t * p.Hq, kvh = quot(h, p.d_g);
    // a tile of a stack is a row of a head here: the branch is the one whose tokens t is among
    int b;
    if (p.q_start) {
        int first = 0;
        if (p.B > kWave) {
            const int e = (lane + 1) * kWave;
            first = kWave * __popcll(__ballot(e <= p.B && p.q_start[min(e, p.B)] <= t));
            if (first >= p.B) return;
        }
        b = first + __popcll(__ballot(first + lane < p.B && p.q_start[min(first + lane, p.B - 1) + 1] <= t));
        if (b >= p.B) return;
    } else {
        b = t / p.R;
    }
    b = __builtin_amdgcn_readfirstlane(b);
    const int n = keys_of_row(branch_at(p, b), t);
    if (n < 0) return;
    const float scale = p.scale;
    const float4 qv = *reinterpret_cast<const float4*>((const unsigned char*)p.Q + t * p.q_t + h * p.q_h + c4 * 16);
    const int32_t* row = p.table + b * p.table_stride;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    for (int j0 = wave * CHUNK; j0 < n; j0 += WAVES * CHUNK) {
        const int e = __builtin_amdgcn_readfirstlane(row[j0 >> p.shift]);
        if ((unsigned)e >= (unsigned)p.pages) continue;  // no page: nothing to see
        const unsigned char* kp = (const unsigned char*)p.K + e * p.page_p + kvh * p.page_h + c4 * 16;
        const unsigned char* vp = (const unsigned char*)p.V + e * p.page_p + kvh * p.page_h + c4 * 16;
        float4 kv[NJ], vv[NJ];
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            const int j = min(j0 + i * KPL + grp, n - 1);  // keys behind the last one re-read it; masked below
            const long long off = (j & ((1 << p.shift) - 1)) * p.page_t;
            kv[i] = *reinterpret_cast<const float4*>(kp + off);
            vv[i] = *reinterpret_cast<const float4*>(vp + off);
        }
        float s[NJ], mx = m;
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            s[i] = qv.x * kv[i].x + qv.y * kv[i].y + qv.z * kv[i].z + qv.w * kv[i].w;
#pragma unroll
            for (int d = LPK / 2; d >= 1; d >>= 1) s[i] += shfl_xor_f(s[i], d);
            s[i] = j0 + i * KPL + grp < n ? s[i] : -INFINITY;
            mx = fmaxf(mx, s[i]);
        }
        const float mu = mx == -INFINITY ? 0.f : mx;
        const float alpha = expf((m - mu) * scale);
        l *= alpha;
        acc.x *= alpha; acc.y *= alpha; acc.z *= alpha; acc.w *= alpha;
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            const float pv = expf((s[i] - mu) * scale);
            if (j0 + i * KPL + grp >= n) vv[i] = make_float4(0.f, 0.f, 0.f, 0.f);  // an infinity counts once
            l += pv;
            acc.x += pv * vv[i].x; acc.y += pv * vv[i].y; acc.z += pv * vv[i].z; acc.w += pv * vv[i].w;
        }
        m = mx;
    }
#pragma unroll
    for (int d = LPK; d < kWave; d <<= 1) {
        const float mo = shfl_xor_f(m, d), lo = shfl_xor_f(l, d);
        const float4 ao = make_float4(shfl_xor_f(acc.x, d), shfl_xor_f(acc.y, d), shfl_xor_f(acc.z, d), shfl_xor_f(acc.w, d));
        const float M = fmaxf(m, mo);
        const float wa = m == -INFINITY ? 0.f : expf((m - M) * scale), wb = mo == -INFINITY ? 0.f : expf((mo - M) * scale);
        l = l * wa + lo * wb;
        acc.x = acc.x * wa + ao.x * wb; acc.y = acc.y * wa + ao.y * wb; acc.z = acc.z * wa + ao.z * wb; acc.w = acc.w * wa + ao.w * wb;
        m = M;
    }
    if (lane == 0) {
        sh_ml[wave][0] = m;
        sh_ml[wave][1] = l;
    }
    if (grp == 0) *reinterpret_cast<float4*>(&sh_acc[wave][c4 * 4]) = acc;
    __syncthreads();
    if (tid < D) {
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, sh_ml[w][0]);
        float lsum = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float wgt = (sh_ml[w][0] == -INFINITY) ? 0.f : expf((sh_ml[w][0] - M) * scale);
            lsum += sh_ml[w][1] * wgt;
            o += sh_acc[w][tid] * wgt;
        }
        reinterpret_cast<float*>((unsigned char*)p.O + t * p.o_t + h * p.o_h)[tid] = lsum == 0.f ? 0.f : o / lsum;
        if (p.lse && tid == 0) p.lse[(long long)t * p.Hq + h] = M * scale + logf(lsum);
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
static int paged_desc(const lotts_paged_desc* in, bool uniform, lotts_paged_desc* d, int* shift) {
    if (!in) return LOTTS_ERR_NULL;
    *d = *in;
    if (d->dtype != LOTTS_F32 && d->dtype != LOTTS_BF16) return LOTTS_ERR_DTYPE;
    if (d->B < 1 || d->B > kPgMaxBranches || d->T < 1 || d->Hq < 1 || d->Hkv < 1 || d->Hq % d->Hkv != 0) return LOTTS_ERR_SHAPE;
    if (d->D != 64 && d->D != 128) return LOTTS_ERR_SHAPE;
    if (d->max_new < 1 || d->max_new > d->T) return LOTTS_ERR_SHAPE;
    if (uniform && (d->T % d->B != 0 || d->max_new != d->T / d->B)) return LOTTS_ERR_SHAPE;
    if (d->pages < 1 || d->pages > kPgMaxPages || d->columns < 1) return LOTTS_ERR_SHAPE;
    *shift = -1;
    for (int s = 4; s <= 10; ++s)
        if (d->page_tokens == 1 << s) *shift = s;
    if (*shift < 0 || (long long)d->columns << *shift > 0x3fffffffLL) return LOTTS_ERR_SHAPE;
    if (!(d->scale >= 0.0f) || d->scale > 3.0e38f) return LOTTS_ERR_SHAPE;
    const long long D = d->D, es = d->dtype == LOTTS_BF16 ? 2 : 4;
    // 0 selects the dense layout
    if (!d->q_stride_h) d->q_stride_h = D;
    if (!d->q_stride_t) d->q_stride_t = d->Hq * D;
    if (!d->o_stride_h) d->o_stride_h = D;
    if (!d->o_stride_t) d->o_stride_t = d->Hq * D;
    if (!d->page_stride_t) d->page_stride_t = D;
    if (!d->page_stride_h) d->page_stride_h = d->page_tokens * D;
    if (!d->page_stride_p) d->page_stride_p = d->Hkv * d->page_tokens * D;
    if (!d->table_stride) d->table_stride = d->columns;
    const long long st[] = {d->q_stride_t, d->q_stride_h, d->o_stride_t, d->o_stride_h, d->page_stride_p, d->page_stride_h, d->page_stride_t};
    for (long long s : st)
        if (s < 0 || (s * es) % 16 != 0) return LOTTS_ERR_SHAPE;
    if (d->q_stride_h < D || d->o_stride_h < D || d->page_stride_t < D || d->table_stride < d->columns) return LOTTS_ERR_SHAPE;
    if (d->page_stride_t * es > (1LL << 26)) return LOTTS_ERR_SHAPE;  // 16 keys of a page: 32-bit offsets
    // the sequence of work of a KV head in 32 bits (were every branch as long as the table allows)
    const long long G = d->Hq / d->Hkv, slots = (long long)d->T * G / kWideRows + d->B;
    if (((long long)d->columns << *shift) / kNarrowTile * kMaxWideCost + kMaxWideCost + kStartCost > 0x7fffffffLL / slots) return LOTTS_ERR_SHAPE;
    if ((long long)d->T * d->Hq >= (1LL << 24)) return LOTTS_ERR_SHAPE;  // a grid holds fewer than 2^24 workgroups of 256 threads
    return LOTTS_OK;
}

constexpr int kPgTagShift = 16;
static std::atomic<unsigned long long> g_paged_tag{0};

// Which kernel, how many workers, and where the partials lie: [arrival cells][(maximum, sum)][outputs].
struct PagedPlan {
    bool wide, two;
    int narrow_tiles, workers, items, part_rows;
    size_t off_ml, off_o, bytes;
};
static PagedPlan paged_plan(const lotts_paged_desc& d) {
    PagedPlan pl = {};
    const long long G = d.Hq / d.Hkv, rows = d.max_new * G;
    // (Steps for which the caller leaves max_new at T, us: 1024 branches of 128 tokens with 3 new ones, 16 / 2 heads, 107 against 43, 256 of 1024 with 4 59
    // against 47, 64 ragged ones up to 8192 67 against 60.5, 16 of 4096 with 40 / 8 heads 46 against 47; 16 of 2000 with 6 new ones, 48 rows, 19 against 24.)
    pl.wide = rows > 64;
    pl.narrow_tiles = rows > 32 ? 2 : 1;
    // Two workgroups a unit, each with one slab a wavefront at D = 128, where there are so many items that a worker has several: one's start on an item, lengths
    // to table to keys, passes while the other works (1024 branches of 128 tokens 48.5 -> 35.1 us, 256 of 1024 51.4 -> 47, 512 of 500 55.4 ->
    // 46).  With fewer items there would be more cuts: 16 branches x 8 heads of 4096 48.5 -> 51.2, 64 x 2 of 4096 48.5 -> 52.7.
    pl.two = !pl.wide && pl.narrow_tiles == 1 && (long long)d.B * d.Hkv >= 2 * kNumCU;
    pl.workers = pl.two ? 2 * kNumCU : kNumCU;
    pl.items = (int)(pl.wide ? d.T * G / kWideRows + d.B : d.B);
    pl.part_rows = (int)std::min<long long>(kWideRows, (rows + 7) / 8 * 8);
    const size_t slots = 2 * (size_t)pl.workers;
    pl.off_ml = 4 * (size_t)kMaxWorkers * sizeof(unsigned long long);  // (whatever the call: the cells are nothing else, ever)
    pl.off_o = pl.off_ml + slots * pl.part_rows * 8;
    // A workspace for more branches and more new tokens serves fewer: twice the workers' partials of up to 32 rows are more than the partials of 33 to 56.
    const size_t at_least = (long long)d.B * d.Hkv >= 2 * kNumCU ? 2 * (size_t)kMaxWorkers * std::min(pl.part_rows, 32) : 0;
    pl.bytes = pl.off_ml + std::max(slots * pl.part_rows, at_least) * (8 + (size_t)d.D * 4);
    return pl;
}

}  // namespace lotts

extern "C" size_t verify_attention_paged_workspace_bytes(const lotts_paged_desc* desc) {
    using namespace lotts;
    lotts_paged_desc d;
    int shift;
    if (paged_desc(desc, false, &d, &shift) != LOTTS_OK) return 0;
    return d.dtype == LOTTS_F32 ? 256 : paged_plan(d).bytes;
}

extern "C" int verify_attention_paged(const lotts_paged_desc* desc, const void* Q, const void* Kpages, const void* Vpages, const int32_t* page_table,
                                      const int32_t* kv_len, const int32_t* q_start, void* O, float* lse, void* workspace, size_t workspace_bytes,
                                      void* stream) {
    using namespace lotts;
    lotts_paged_desc d;
    int shift;
    const int rc = paged_desc(desc, !q_start, &d, &shift);
    if (rc != LOTTS_OK) return rc;
    if (!Q || !Kpages || !Vpages || !page_table || !kv_len || !O || !workspace) return LOTTS_ERR_NULL;
    if ((((uintptr_t)Q | (uintptr_t)Kpages | (uintptr_t)Vpages | (uintptr_t)O | (uintptr_t)workspace) & 15) != 0) return LOTTS_ERR_SHAPE;
    if ((((uintptr_t)page_table | (uintptr_t)kv_len | (uintptr_t)q_start | (uintptr_t)lse) & 3) != 0) return LOTTS_ERR_SHAPE;
    const PagedPlan pl = paged_plan(d);
    if (workspace_bytes < (d.dtype == LOTTS_F32 ? 256 : pl.bytes)) return LOTTS_ERR_WORKSPACE;
    const long long es = d.dtype == LOTTS_BF16 ? 2 : 4;
    PagedParams p;
    p.Q = Q; p.K = Kpages; p.V = Vpages; p.table = page_table; p.kv_len = kv_len; p.q_start = q_start; p.O = O; p.lse = lse;
    p.q_t = d.q_stride_t * es; p.q_h = d.q_stride_h * es; p.o_t = d.o_stride_t * es; p.o_h = d.o_stride_h * es;
    p.page_p = d.page_stride_p * es; p.page_h = d.page_stride_h * es; p.page_t = d.page_stride_t * es;
    p.table_stride = d.table_stride;
    p.B = d.B; p.T = d.T; p.R = d.T / d.B; p.Hq = d.Hq; p.Hkv = d.Hkv; p.G = d.Hq / d.Hkv;
    p.pages = d.pages; p.columns = d.columns; p.shift = shift;
    const double scale = d.scale > 0.0f ? (double)d.scale : 1.0 / sqrt((double)d.D);
    p.scale = (float)scale;
    p.scale_log2 = (float)std::min(scale * 1.4426950408889634074, 3.4e38);
    p.d_g = fast_div(p.G);
    p.items = pl.items; p.workers = pl.workers; p.part_rows = pl.part_rows;
    p.ws = workspace; p.ws_bytes = (unsigned)pl.bytes; p.off_ml = (unsigned)pl.off_ml; p.off_o = (unsigned)pl.off_o;
    p.cells = static_cast<unsigned long long*>(workspace);
    p.tag = (g_paged_tag.fetch_add(1, std::memory_order_relaxed) + 1) << kPgTagShift;
    const hipStream_t s = (hipStream_t)stream;
    if (d.dtype == LOTTS_F32) {
        const dim3 grid((unsigned)((long long)d.T * d.Hq));
        // A row's keys are a chain of loads: few rows take 16 wavefronts each, so that the chain is short; many fill the chip with 4.  (80 rows of up to
        // 700 keys: 11.7 us a call with 4, 7.4 with 16.)
        if ((long long)d.T * d.Hq <= 2 * kNumCU) {
            if (d.D == 64) LOTTS_LAUNCH((paged_f32_kernel<64, 16>), grid, dim3(16 * kWave), s, p);
            else LOTTS_LAUNCH((paged_f32_kernel<128, 16>), grid, dim3(16 * kWave), s, p);
        } else {
            if (d.D == 64) LOTTS_LAUNCH((paged_f32_kernel<64, 4>), grid, dim3(4 * kWave), s, p);
            else LOTTS_LAUNCH((paged_f32_kernel<128, 4>), grid, dim3(4 * kWave), s, p);
        }
        return check_launch();
    }
    const dim3 grid((unsigned)pl.workers), block(paged_waves<false>() * kWave);
    if (pl.wide) {
        if (d.D == 64) LOTTS_LAUNCH((paged_attn_kernel<64, 1, true, false>), grid, dim3(paged_waves<true>() * kWave), s, p);
        else LOTTS_LAUNCH((paged_attn_kernel<128, 1, true, false>), grid, dim3(paged_waves<true>() * kWave), s, p);
    } else if (pl.narrow_tiles == 2) {
        if (d.D == 64) LOTTS_LAUNCH((paged_attn_kernel<64, 2, false, false>), grid, block, s, p);
        else LOTTS_LAUNCH((paged_attn_kernel<128, 2, false, false>), grid, block, s, p);
    } else if (pl.two) {
        if (d.D == 64) LOTTS_LAUNCH((paged_attn_kernel<64, 1, false, true>), grid, block, s, p);
        else LOTTS_LAUNCH((paged_attn_kernel<128, 1, false, true>), grid, block, s, p);
    } else {
        if (d.D == 64) LOTTS_LAUNCH((paged_attn_kernel<64, 1, false, false>), grid, block, s, p);
        else LOTTS_LAUNCH((paged_attn_kernel<128, 1, false, false>), grid, block, s, p);
    }
    return check_launch();
}
