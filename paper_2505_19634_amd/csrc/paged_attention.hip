// verify_attention_paged: causal attention of the new tokens of every branch against the branch's paged cache.  The branches of a call
// may have different numbers of new tokens: a chunk of a prompt that is being read, the drafts of a verification step, one token of
// plain decoding (paper Section 2: the target verifies the drafts in one parallel forward; Section 3.2: B branches of one question,
// whose prompt's pages they share).
//
// A branch's query rows of one KV head -- n new tokens x G query heads, the heads of a token next to each other -- are stacked, and a
// workgroup takes a tile of that stack.  Row r of the stack is token r / G; it sees the keys in front of position L - n + r / G + 1.
#include <algorithm>
#include <cmath>

#include "lotts_common.h"

namespace lotts {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kPgMaxBranches = 4096;
constexpr int kPgMaxPages = 1 << 24;
constexpr int kPgThreads = 256;
constexpr int kPgWaves = kPgThreads / kWave;
constexpr int kPgGroup = 16;  // keys that lie in one page whatever the page size: what one wavefront loads of a tile

struct PagedParams {
    const void *Q, *K, *V;
    const int32_t *table, *kv_len, *q_start;
    void* O;
    float* lse;
    long long q_t, q_h, o_t, o_h;       // bytes
    long long page_p, page_h, page_t;   // bytes
    long long table_stride;
    int B, T, R, Hq, Hkv, G, pages, columns, shift;
    int tiles;                          // row tiles of a KV head, at most
    float scale_log2;                   // scale * log2(e)
    FastDiv d_hkv, d_g;
};

// A branch of the call: its first row of Q, its new tokens and all its tokens (both brought into the range that the arguments allow, so
// that nothing is addressed out of bounds whatever the device data say).
struct Branch {
    int b, first, n, L;
};
__device__ __forceinline__ Branch branch_at(const PagedParams& p, int b) {
    Branch r;
    r.b = b;
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
// Row tiles: branch b's are numbers floor(q_start[b] * G / rows) + b and on; enough for its ceil(n * G / rows), and no sum over the branches
// is needed to find whose a number is.
__device__ __forceinline__ int first_tile(const PagedParams& p, int b, int rows) {
    const int first = p.q_start ? min(max(p.q_start[b], 0), p.T) : b * p.R;
    return (int)((long long)first * p.G / rows) + b;
}
__device__ __forceinline__ int branch_of_tile(const PagedParams& p, int tile, int rows, int lane) {
    int first = 0;
    if (p.B > kWave) {
        const int b = lane * kWave;
        first = kWave * max(0, __popcll(__ballot(b < p.B && first_tile(p, min(b, p.B - 1), rows) <= tile)) - 1);
    }
    const int b = first + lane;
    return max(0, first + __popcll(__ballot(b < p.B && first_tile(p, min(b, p.B - 1), rows) <= tile)) - 1);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* base, unsigned bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, 0x00020000);
}

// ---------------------------------------------------------------------------------------------
// bf16
// ---------------------------------------------------------------------------------------------
template <int D, int TW>
__global__ __launch_bounds__(kPgThreads, 1) void paged_attn_kernel(const PagedParams p) {
    constexpr int KT = 64;                  // keys of a tile
    constexpr int ROWS = kPgWaves * TW * 32;
    constexpr int KS = D / 16, DB = D / 32;
    constexpr int LPR = D / 8, RPI = kWave / LPR, NLD = kPgGroup / RPI;
    constexpr int KSTRIDE = D * 2 + 16, VSTRIDE = D * 2 + 64;
    __shared__ __attribute__((aligned(16))) unsigned char kslab[KT * KSTRIDE];
    __shared__ __attribute__((aligned(16))) unsigned char vslab[KT * VSTRIDE];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid & (kWave - 1);
    const int ln = lane & 31, hh = lane >> 5;
    const int id = (int)blockIdx.x, item = quot(id, p.d_hkv), kvh = id - item * p.Hkv;
    const int tile_no = p.tiles - 1 - item;  // the rows that see most first
    const int b = __builtin_amdgcn_readfirstlane(branch_of_tile(p, tile_no, ROWS, lane));
    const Branch br = branch_at(p, b);
    const int rows = br.n * p.G, row0 = (tile_no - first_tile(p, b, ROWS)) * ROWS;
    if (row0 < 0 || row0 >= rows) return;
    const int before = br.L - br.n;  // row r sees the keys in front of before + r / G + 1

    // the wavefront's rows
    bf16x8 qf[TW][KS];
    int lim[TW];
#pragma unroll
    for (int t = 0; t < TW; ++t) {
        const int r = min(row0 + (wave * TW + t) * 32 + ln, rows - 1);
        const int i = quot(r, p.d_g), g = r - i * p.G;
        lim[t] = before + i + 1;
        const unsigned char* qp = (const unsigned char*)p.Q + (br.first + i) * p.q_t + (kvh * p.G + g) * p.q_h;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[t][s] = *reinterpret_cast<const bf16x8*>(qp + (2 * s + hh) * 16);
    }
    const int last = quot(min(row0 + ROWS, rows) - 1, p.d_g);
    const int keys = max(0, before + last + 1), n_tiles = (keys + KT - 1) / KT;

    const int v_row = lane / LPR, v_chunk = lane % LPR;
    const int blk = lane >> 4, i16 = lane & 15;
    const int tr_off = ((blk >> 1) * 4 + (i16 >> 2)) * VSTRIDE + ((blk & 1) * 16 + (i16 & 3) * 4) * 2;
    const int32_t* row = p.table + b * p.table_stride;
    auto entry = [&](int key) { return __builtin_amdgcn_readfirstlane(row[min(key >> p.shift, p.columns - 1)]); };
    u32x4 kst[NLD], vst[NLD];
    int have = 0, have_next = 0;  // which groups of a tile lie in a page
    auto fetch = [&](int kb) {
        have_next = 0;
        int e = 0;
#pragma unroll
        for (int g = 0; g < KT / kPgGroup; ++g) {
            const int eg = entry(kb + g * kPgGroup);
            if ((unsigned)eg < (unsigned)p.pages) have_next |= 1 << g;
            if (g == wave) e = eg;
        }
        const int key = kb + wave * kPgGroup;
        const int n = (have_next >> wave & 1) ? min(keys - key, kPgGroup) : 0;
        // keys behind the last one, and those without a page, are out of the buffer's range: they read as zeros
        const unsigned bytes = n > 0 ? (unsigned)((n - 1) * p.page_t) + D * 2 : 0;
        const long long at = (n > 0 ? e : 0) * p.page_p + kvh * p.page_h + (key & ((1 << p.shift) - 1)) * p.page_t;
        const __amdgpu_buffer_rsrc_t kr = buffer((const unsigned char*)p.K + at, bytes), vr = buffer((const unsigned char*)p.V + at, bytes);
#pragma unroll
        for (int i = 0; i < NLD; ++i) {
            const unsigned off = (unsigned)((i * RPI + v_row) * p.page_t) + v_chunk * 16;
            kst[i] = __builtin_amdgcn_raw_buffer_load_b128(kr, (int)off, 0, 0);
            vst[i] = __builtin_amdgcn_raw_buffer_load_b128(vr, (int)off, 0, 0);
        }
    };

    f32x16 oacc[TW][DB];
    float m_run[TW], l_run[TW];
#pragma unroll
    for (int t = 0; t < TW; ++t) {
        m_run[t] = -INFINITY;
        l_run[t] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[t][db][i] = 0.f;
    }
    if (n_tiles > 0) fetch(0);
    for (int it = 0; it < n_tiles; ++it) {
        const int kb = it * KT;
        __syncthreads();  // the tile before has been read
#pragma unroll
        for (int i = 0; i < NLD; ++i) {
            *reinterpret_cast<u32x4*>(kslab + (wave * kPgGroup + i * RPI + v_row) * KSTRIDE + v_chunk * 16) = kst[i];
            *reinterpret_cast<u32x4*>(vslab + (wave * kPgGroup + i * RPI + v_row) * VSTRIDE + v_chunk * 16) = vst[i];
        }
        have = have_next;
        __syncthreads();
        if (it + 1 < n_tiles) fetch(kb + KT);
#pragma unroll
        for (int half = 0; half < KT / 32; ++half) {
            bf16x8 kf[KS];
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[s] = *reinterpret_cast<const bf16x8*>(kslab + (half * 32 + ln) * KSTRIDE + (2 * s + hh) * 16);
            bf16x8 pf[TW][2];
#pragma unroll
            for (int t = 0; t < TW; ++t) {
                // S^T[key][row]; register i of this lane is key kb + half * 32 + (i / 4) * 8 + hh * 4 + i % 4 for row ln
                f32x16 acc;
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
                for (int s = 0; s < KS; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[t][s], acc, 0, 0, 0);
                const int vis = lim[t] - (kb + half * 32) - hh * 4;
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float sc = acc[i] * p.scale_log2;
                    sc = (i >> 2) * 8 + (i & 3) < vis && (have >> (half * 2 + (i >> 3)) & 1) ? sc : -INFINITY;
                    acc[i] = sc;
                    mx = fmaxf(mx, sc);
                }
                mx = fmaxf(mx, shfl_xor_f(mx, 32));
                const float m_new = fmaxf(m_run[t], mx);
                const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
                const float alpha = __builtin_amdgcn_exp2f(m_run[t] - m_use);
                float psum = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float pv = __builtin_amdgcn_exp2f(acc[i] - m_use);
                    psum += pv;
                    pf[t][i >> 3][i & 7] = (__bf16)pv;
                }
                l_run[t] = l_run[t] * alpha + psum;
                m_run[t] = m_new;
                if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i) oacc[t][db][i] *= alpha;
                }
            }
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    union {
                        short4v s[2];
                        bf16x8 v;
                    } vf;
                    const unsigned char* ap = vslab + tr_off + (half * 32 + kk * 16) * VSTRIDE + db * 64;
                    vf.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(ap));
                    vf.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(ap + 8 * VSTRIDE));
#pragma unroll
                    for (int t = 0; t < TW; ++t) oacc[t][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.v, pf[t][kk], oacc[t][db], 0, 0, 0);
                }
        }
    }
#pragma unroll
    for (int t = 0; t < TW; ++t) {
        const float l = l_run[t] + shfl_xor_f(l_run[t], 32);
        const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);  // a row that sees nothing is 0; NaN stays
        const int r = row0 + (wave * TW + t) * 32 + ln;
        if (r >= rows) continue;
        const int i = quot(r, p.d_g), h = kvh * p.G + r - i * p.G;
        unsigned char* op = (unsigned char*)p.O + (br.first + i) * p.o_t + h * p.o_h;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (__bf16)(oacc[t][db][q * 4 + e] * inv);
                *reinterpret_cast<bf16x4*>(op + (db * 32 + q * 8 + hh * 4) * 2) = v;
            }
        if (p.lse && hh == 0) p.lse[(long long)(br.first + i) * p.Hq + h] = (m_run[t] + log2f(l)) * 0.69314718055994530942f;
    }
}

// ---------------------------------------------------------------------------------------------
// fp32: fp32 arithmetic throughout, a workgroup per row of a head.  A key row is D / 4 lanes of 16 bytes; a wavefront takes every
// fourth chunk of 4 * 256 / D keys (no chunk is larger than 16 keys: it lies in one page) and keeps a running state per D / 4 lanes;
// the states meet at the end.
// ---------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(kPgThreads) void paged_f32_kernel(const PagedParams p) {
    constexpr int LPK = D / 4, KPL = kWave / LPK, NJ = 4, CHUNK = NJ * KPL;
    __shared__ __attribute__((aligned(16))) float sh_acc[kPgWaves][D];
    __shared__ float sh_ml[kPgWaves][2];
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
    const Branch br = branch_at(p, b);
    if (t < br.first) return;
    const int n = max(0, br.L - br.n + (t - br.first) + 1);
    const float scale = p.scale_log2 * 0.69314718055994530942f;
    const float4 qv = *reinterpret_cast<const float4*>((const unsigned char*)p.Q + t * p.q_t + h * p.q_h + c4 * 16);
    const int32_t* row = p.table + b * p.table_stride;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    for (int j0 = wave * CHUNK; j0 < n; j0 += kPgWaves * CHUNK) {
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
            s[i] = j0 + i * KPL + grp < n ? s[i] * scale : -INFINITY;
            mx = fmaxf(mx, s[i]);
        }
        const float mu = mx == -INFINITY ? 0.f : mx;
        const float alpha = expf(m - mu);
        l *= alpha;
        acc.x *= alpha; acc.y *= alpha; acc.z *= alpha; acc.w *= alpha;
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            const float pv = expf(s[i] - mu);
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
        const float wa = m == -INFINITY ? 0.f : expf(m - M), wb = mo == -INFINITY ? 0.f : expf(mo - M);
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
        for (int w = 0; w < kPgWaves; ++w) M = fmaxf(M, sh_ml[w][0]);
        float lsum = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kPgWaves; ++w) {
            const float wgt = (sh_ml[w][0] == -INFINITY) ? 0.f : expf(sh_ml[w][0] - M);
            lsum += sh_ml[w][1] * wgt;
            o += sh_acc[w][tid] * wgt;
        }
        reinterpret_cast<float*>((unsigned char*)p.O + t * p.o_t + h * p.o_h)[tid] = lsum == 0.f ? 0.f : o / lsum;
        if (p.lse && tid == 0) p.lse[(long long)t * p.Hq + h] = M + logf(lsum);
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
    if ((long long)d->T * d->Hq >= (1LL << 24)) return LOTTS_ERR_SHAPE;  // a grid holds fewer than 2^24 workgroups of 256 threads
    return LOTTS_OK;
}

}  // namespace lotts

extern "C" size_t verify_attention_paged_workspace_bytes(const lotts_paged_desc* desc) {
    using namespace lotts;
    lotts_paged_desc d;
    int shift;
    if (paged_desc(desc, false, &d, &shift) != LOTTS_OK) return 0;
    return 256;
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
    if (workspace_bytes < verify_attention_paged_workspace_bytes(desc)) return LOTTS_ERR_WORKSPACE;
    const long long es = d.dtype == LOTTS_BF16 ? 2 : 4;
    PagedParams p;
    p.Q = Q; p.K = Kpages; p.V = Vpages; p.table = page_table; p.kv_len = kv_len; p.q_start = q_start; p.O = O; p.lse = lse;
    p.q_t = d.q_stride_t * es; p.q_h = d.q_stride_h * es; p.o_t = d.o_stride_t * es; p.o_h = d.o_stride_h * es;
    p.page_p = d.page_stride_p * es; p.page_h = d.page_stride_h * es; p.page_t = d.page_stride_t * es;
    p.table_stride = d.table_stride;
    p.B = d.B; p.T = d.T; p.R = d.T / d.B; p.Hq = d.Hq; p.Hkv = d.Hkv; p.G = d.Hq / d.Hkv;
    p.pages = d.pages; p.columns = d.columns; p.shift = shift;
    const double scale = d.scale > 0.0f ? (double)d.scale : 1.0 / sqrt((double)d.D);
    p.scale_log2 = (float)(scale * 1.4426950408889634074);
    p.d_hkv = fast_div(d.Hkv); p.d_g = fast_div(p.G);
    p.tiles = 0;
    const hipStream_t s = (hipStream_t)stream;
    if (d.dtype == LOTTS_F32) {
        const dim3 grid((unsigned)((long long)d.T * d.Hq));
        if (d.D == 64) LOTTS_LAUNCH(paged_f32_kernel<64>, grid, dim3(kPgThreads), s, p);
        else LOTTS_LAUNCH(paged_f32_kernel<128>, grid, dim3(kPgThreads), s, p);
        return check_launch();
    }
    constexpr int TW = 1, rows = kPgWaves * TW * 32;
    p.tiles = (int)((long long)d.T * p.G / rows) + d.B;
    const long long items = (long long)p.tiles * d.Hkv;
    if (items >= (1LL << 24)) return LOTTS_ERR_SHAPE;
    if (d.D == 64) LOTTS_LAUNCH((paged_attn_kernel<64, TW>), dim3((unsigned)items), dim3(kPgThreads), s, p);
    else LOTTS_LAUNCH((paged_attn_kernel<128, TW>), dim3((unsigned)items), dim3(kPgThreads), s, p);
    return check_launch();
}
