// skinny_gemm_mxfp4: Y[M][N] = X[M][K] W[N][K]^T for up to 256 new tokens of a verify forward against a weight matrix held in 4-bit microscaled
// numbers (mx.h): skinny_gemm with a quarter of the bytes to stream.  The elements become bf16, exactly, on their way to the matrix cores; fp32 sums,
// bf16 out.
//
// Lane (row, half) of a 32 x 32 x 16 product takes 8 of 16 k; which ones does not matter as long as both operands agree, so a lane takes a whole block of 32
// codes, 16 bytes, with its scale over four products, and the same 32 values of X.  W's rows are the product's rows, tokens its columns.
//
//   skinny_gemm_mxfp4_stream_kernel<MT, TG, KG, XD, ...>  a workgroup of eight wavefronts has 256 / KG weight rows and all tokens, or 512 and half of the tokens
//       beyond 128, for a range of K
//   skinny_gemm_mxfp4_direct_kernel  32 rows and 32 tokens, nothing shared: small matrices
//   skinny_gemm_mxfp4_reduce_kernel  where K is split across workgroups: sums the fp32 partials in their order
#include <algorithm>

#include "mx.h"

namespace lotts {

typedef float x_f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 x_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 x_bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk4 = 256;   // k of a row's 128 bytes of codes
constexpr int kWaves4 = 8;
constexpr unsigned kNowhere = 0x80000000u;  // an offset behind every buffer's end: reads as zeros

struct Gemm4Params {
    const unsigned char *X, *codes, *scales;
    __bf16* Y;
    float* part;                         // [ksplit][M][ldp] where K is split
    long long ldx, ld_codes, ld_scales;  // bytes
    long long ldy;                       // elements
    int M, N, K, ldp, tokens;
    int chunks, ksplit, nblocks, items;
    bool words;                          // four scales of a row are a load
    bool quads;                          // four columns of Y are a store
    FastDiv d_nblocks, d_ksplit;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer4(const void* base, bool any) { return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, any ? 0x7fffffff : 0, 0x00020000); }
// Pieces of 16 bytes lie exchanged within their row of 128 or 256 bytes, so that 32 rows' reads of one piece meet every bank equally often.
template <int BYTES>
__device__ __forceinline__ int spread4(int r) {
    return BYTES == 256 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
}

// MT: token tiles of 32; TG = 2: wavefronts in pairs own two row tiles together and half of the token tiles each; KG: groups of wavefronts with a share of the K
// range each, for the same rows; XD: steps of X in registers; WORDS: four scales of a row are a load; PARTS: half of the tokens, two row tiles a wavefront.
// Codes and X come through registers, codes two chunks of 256 k ahead (PARTS: one) and X XD steps of 64 k, on their way into LDS.  Of X three steps lie there: the one
// that is multiplied, the next one, whose first pieces are read before the barrier between them, and the one that is written; of the codes two chunks (PARTS:
// one, the wavefront's own).  A wavefront's loads come back in order: whoever waits for X waits for the codes requested before it, so both are far ahead, and
// requested a few at a time (all of a chunk's codes at once, with X two steps ahead: 64 tokens x 55296 x 5120 53 us).
template <int MT, int TG, int KG, int XD, bool WORDS, bool PARTS>
__global__ __launch_bounds__(kWaves4 * kWave, 2) void skinny_gemm_mxfp4_stream_kernel(const Gemm4Params p) {
    constexpr int GW = kWaves4 / KG, GT = GW * kWave;   // a group's wavefronts and threads
    constexpr int RT = PARTS ? 2 : TG, TT = MT / TG, ROWS = 32 * RT * GW / TG, WT = RT / TG;  // WT: row tiles whose codes a wavefront brings in
    constexpr int XK = 64, NS = kChunk4 / XK, XROW = XK * 2, XL = XROW / 16, XP = (MT * 32 * XL + GT - 1) / GT, XRP = GT / XL;  // steps of a chunk; lanes of a token, loads of a thread, tokens of a load
    static_assert(MT % TG == 0 && RT % TG == 0 && GW % TG == 0 && NS == 4 && 8 % XD == 0 && (!PARTS || TG == 1), "what wavefronts and steps share out");
    constexpr int XBUF = MT * 32 * XROW, WBUF = ROWS * 128, WBUFS = PARTS ? 1 : 2, WD = PARTS ? 1 : 2;
    constexpr int XBUFS = KG * (4 * XBUF + WBUFS * WBUF) <= 160 * 1024 ? 4 : 3, GROUP = XBUFS * XBUF + WBUFS * WBUF;  // (three do; of four a step knows its own)
    constexpr int PITCH = ROWS + 4, PARK = KG * 32 * PITCH * 4;  // a token tile's sums on the way out
    __shared__ __attribute__((aligned(1024))) unsigned char lds[KG * GROUP > PARK ? KG * GROUP : PARK];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid & (kWave - 1), ln = lane & 31, hh = lane >> 5;
    const int kg = wave / GW, wv = wave % GW, th = wv % TG, gt = tid % GT;
    // workgroups of one XCD take a run of the list [split][block][part]: they share X, and parts W, in its L2
    const int xcd = blockIdx.x % kNumXCD, each = p.items / kNumXCD, more = p.items % kNumXCD, i_xcd = blockIdx.x / kNumXCD;
    if (i_xcd >= each + (xcd < more)) return;
    const int item = xcd * each + min(xcd, more) + i_xcd, part = PARTS ? item & 1 : 0, sb = PARTS ? item >> 1 : item;
    const int split = quot(sb, p.d_nblocks), block = sb - split * p.nblocks;
    const int m0 = PARTS ? part * p.tokens : 0, M = PARTS ? min(p.tokens, p.M - m0) : p.M;
    const int c_lo = quot(split * p.chunks, p.d_ksplit), c_end = quot((split + 1) * p.chunks, p.d_ksplit);
    const int n_it = (c_end - c_lo + KG - 1) / KG, c_first = c_lo + kg * n_it, c_hi = min(c_end, c_first + n_it);
    const int n0 = block * ROWS, blocks = p.K / kMxBlock;
    unsigned char* xbuf = lds + kg * GROUP;
    unsigned char* wbuf = xbuf + XBUFS * XBUF;
    // where a thread's loads come from and go to
    const int w_first = wv * WT * 32, w_row = n0 + w_first;
    const unsigned char* w_base = p.codes + (long long)min(w_row, p.N - 1) * p.ld_codes;
    const int w_r = lane / 8, w_q = lane % 8;
    // rows behind the last one read it again: they are not stored
    auto w_offset = [&](int i) { return (unsigned)(min(w_row + i * 8 + w_r, p.N - 1) - min(w_row, p.N - 1)) * (unsigned)p.ld_codes + w_q * 16; };
    unsigned w_off[PARTS ? 1 : 4];
#pragma unroll
    for (int i = 0; i < (PARTS ? 0 : 4); ++i) w_off[i] = w_offset(i);
    const int w_to = (w_first + w_r) * 128 + (w_q ^ spread4<128>(w_r)) * 16;  // of the first rows; the others' differ in the bits that spread4() takes from the row's upper part
    const unsigned char* x_base = p.X + (long long)m0 * p.ldx;
    unsigned x_off[XP];
    int x_to[XP];
#pragma unroll
    for (int i = 0; i < XP; ++i) {
        const int t = i * XRP + gt / XL, q = gt % XL;
        x_off[i] = (unsigned)min(t, M - 1) * (unsigned)p.ldx + q * 16;  // (nor are tokens behind the last one)
        x_to[i] = t * XROW + (q ^ spread4<XROW>(t)) * 16;
    }
    const int s_first = n0 + (wv / TG) * RT * 32;
    const unsigned char* s_base = p.scales + (long long)min(s_first, p.N - 1) * p.ld_scales;
    unsigned s_off[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) s_off[t] = (unsigned)(min(s_first + t * 32 + ln, p.N - 1) - min(s_first, p.N - 1)) * (unsigned)p.ld_scales;
    mx_u32x4 wr[WD][WT * 4], xr[XD][XP];
    mx_u32x4 sr[RT];  // scales as loaded: the lane's row's 16 of the next two chunks, or blocks hh, 2 + hh, 4 + hh and 6 + hh of the next one
    auto left = [&](int it) {  // blocks of the group's it-th chunk
        const int c = c_first + it;
        return c < c_hi ? min(8, blocks - c * 8) : 0;
    };
    auto load_w = [&](int it, int i, mx_u32x4& w) {  // rows i * 8 .. i * 8 + 7 of the wavefront's
        const int n = left(it);
        unsigned at = PARTS ? w_offset(i) : w_off[PARTS ? 0 : i];
        if (n & 7) at = w_q < n ? at : kNowhere;  // K's last chunk
        w = __builtin_amdgcn_raw_buffer_load_b128(buffer4(w_base + (long long)(c_first + it) * 128, n > 0), (int)at, 0, PARTS ? 0 : 2);
    };
    auto put_w = [&](int it, int i, const mx_u32x4& w) {
        *reinterpret_cast<mx_u32x4*>(wbuf + (WBUFS > 1 ? (it & 1) * WBUF : 0) + i * 1024 + (w_to ^ (spread4<128>(i * 8) * 16))) = w;
    };
    auto load_x = [&](int it, int sub, mx_u32x4 (&x)[XP]) {
        const int n = left(it) * 4 - sub * (XK / 8);  // pieces of 8 values
        const __amdgpu_buffer_rsrc_t r = buffer4(x_base + (long long)(c_first + it) * (2 * kChunk4) + sub * XROW, n > 0);
#pragma unroll
        for (int i = 0; i < XP; ++i) {
            unsigned at = x_off[i];
            if (n < XL) at = gt % XL < n ? at : kNowhere;
            x[i] = __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0);
        }
    };
    auto put_x = [&](int buf, const mx_u32x4 (&x)[XP]) {
#pragma unroll
        for (int i = 0; i < XP; ++i)
            if (MT * 32 % XRP == 0 || i * XRP + gt / XL < MT * 32) *reinterpret_cast<mx_u32x4*>(xbuf + buf * XBUF + x_to[i]) = x[i];
    };
    auto load_s = [&](int it) {
        const int n = WORDS ? left(it) + left(it + 1) : left(it);
        const __amdgpu_buffer_rsrc_t r = buffer4(s_base + (c_first + it) * 8, n > 0);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (WORDS && n == 16) {
                sr[t] = __builtin_amdgcn_raw_buffer_load_b128(r, (int)s_off[t], 0, 0);
            } else if (WORDS) {  // (n a multiple of 4)
#pragma unroll
                for (int j = 0; j < 4; ++j) sr[t][j] = __builtin_amdgcn_raw_buffer_load_b32(r, (int)(j * 4 < n ? s_off[t] + j * 4 : kNowhere), 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) sr[t][j] = __builtin_amdgcn_raw_buffer_load_b8(r, (int)(j * 2 + hh < n ? s_off[t] + j * 2 + hh : kNowhere), 0, 0);
            }
        }
    };
    x_f32x16 acc[RT][TT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[r][t][i] = 0.f;
    // addresses of a lane's pieces, 2 sub + hh of the codes and hh * 4 + k of X, which differ in bits that the row does not touch (PARTS forms them where they are used)
    constexpr int PIECES = PARTS ? 1 : 4;
    int w_lane[PIECES], x_lane[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        w_lane[i] = kg * GROUP + XBUFS * XBUF + ((wv / TG) * RT * 32 + ln) * 128 + ((2 * i + hh) ^ spread4<128>(ln)) * 16;
        x_lane[i] = kg * GROUP + (th * TT * 32 + ln) * XROW + ((hh * 4 + i) ^ spread4<XROW>(ln)) * 16;
    }
    auto w_piece = [&](int sub) { return PARTS ? w_lane[0] ^ (sub * 32) : w_lane[sub % PIECES]; };
    auto x_piece = [&](int k) { return PARTS ? x_lane[0] ^ (k * 16) : x_lane[k % PIECES]; };
    constexpr int QS = PARTS ? 1 : 2;  // (PARTS has no registers for the next step's codes beside this one's)
    mx_u32x4 q[QS][RT];
    constexpr int AHEAD = TT == 1 ? 3 : 1;  // products' steps of 16 k between a read of X and its use
    x_bf16x8 b[AHEAD + 1][TT];
    auto codes = [&](int parity, int sub) {  // of an even or odd chunk
#pragma unroll
        for (int r = 0; r < RT; ++r) q[sub & (QS - 1)][r] = *reinterpret_cast<const mx_u32x4*>(lds + w_piece(sub) + (WBUFS > 1 ? parity * WBUF : 0) + r * 32 * 128);
    };
    auto tokens = [&](int buf, int k) {
#pragma unroll
        for (int t = 0; t < TT; ++t) b[k & AHEAD][t] = *reinterpret_cast<const x_bf16x8*>(lds + x_piece(k) + buf * XBUF + t * 32 * XROW);
    };
    // (in the order in which they are needed)
#pragma unroll
    for (int i = 0; i < WT * 4; ++i) load_w(0, i, wr[0][i]);
    load_s(0);
#pragma unroll
    for (int i = 0; i < XD; ++i) {
        load_x(i / NS, i % NS, xr[i]);
        if (WD > 1 && i < 4) load_w(1, i, wr[1][i]);
    }
    static_assert(WD == 1 || (XD >= 4 && WT == 1), "a chunk's codes are four loads, one with each of X");
#pragma unroll
    for (int i = 0; i < WT * 4; ++i) {
        put_w(0, i, wr[0][i]);
        load_w(WD, i, wr[0][i]);
    }
    put_x(0, xr[0]);
    load_x(XD / NS, XD % NS, xr[0]);
    put_x(1, xr[1 % XD]);
    load_x((1 + XD) / NS, (1 + XD) % NS, xr[1 % XD]);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    codes(0, 0);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) tokens(0, k);
    int buf = 0;  // of step g
    // A chunk's steps g = it * NS + sub: X of steps g + 3 .. g + 2 + XD is on its way.
    auto chunk = [&](int it, auto odd) {
        constexpr bool ODD = decltype(odd)::value;
        unsigned s[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < 2; ++j)  // blocks hh and 2 + hh in bytes 0 and 2 of the first, 4 + hh and 6 + hh of the second
                s[r][j] = WORDS ? sr[r][(ODD ? 2 : 0) + j] >> (hh * 8) : sr[r][2 * j] | sr[r][2 * j + 1] << 16;
        if (!WORDS || ODD) load_s(it + 1);
#pragma unroll
        for (int sub = 0; sub < NS; ++sub) {
            if (XBUFS == 4) buf = sub;
            const int next = XBUFS == 4 ? (sub + 1) % 4 : buf == 2 ? 0 : buf + 1, free = XBUFS == 4 ? (sub + 2) % 4 : next == 2 ? 0 : next + 1;
            constexpr int BASE = ODD ? NS : 0;
            put_x(free, xr[(BASE + sub + 2) % XD]);
            load_x(it + (sub + 2 + XD) / NS, (sub + 2 + XD) % NS, xr[(BASE + sub + 2) % XD]);
            if (!PARTS && sub < 3) {  // the next chunk's codes, all of them before the last step reads the first
                constexpr int W = ODD ? 0 : WD - 1;
#pragma unroll
                for (int i = sub == 0 ? 0 : sub + 1; i < sub + 2; ++i) {
                    put_w(it + 1, i, wr[W][i]);
                    load_w(it + 1 + WD, i, wr[W][i]);
                }
            }
            if (PARTS && sub == NS - 1) {  // (a wavefront's LDS operations keep their order: the chunk's codes have been read)
#pragma unroll
                for (int i = 0; i < WT * 4; ++i) {
                    put_w(it + 1, i, wr[0][i]);
                    load_w(it + 2, i, wr[0][i]);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (QS == 2 && k == 0) codes((ODD ? 1 : 0) ^ (sub + 1) / NS, (sub + 1) % NS);
                if (k + AHEAD < 4) tokens(buf, k + AHEAD);
                else tokens(next, k + AHEAD - 4);
                x_bf16x8 a[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) a[r] = mx_of_e2m1(q[sub & (QS - 1)][r][k], s[r][sub >> 1] >> ((sub & 1) * 16) & 0xff);
                if (QS == 1 && k == 3) codes((ODD ? 1 : 0) ^ (sub + 1) / NS, (sub + 1) % NS);
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int t = 0; t < TT; ++t) acc[r][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[r], b[k & AHEAD][t], acc[r][t], 0, 0, 0);
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            buf = next;
        }
    };
    int it = 0;
    for (; it + 1 < n_it; it += 2) {  // (a chunk that may be left out would have the compiler wait for what it does not request)
        chunk(it, std::false_type());
        chunk(it + 1, std::true_type());
    }
    if (it < n_it) chunk(it, std::false_type());
    // Out, a token tile at a time: the groups' sums meet in LDS and leave as rows of Y, or of the split's partials.  Register i of accumulator (r, t): token
    // m0 + (th * TT + t) * 32 + ln, row r * 32 + (i / 4) * 8 + hh * 4 + i % 4 of the wavefront's.
    float* park = reinterpret_cast<float*>(lds);
    const bool parts = p.ksplit > 1;
#pragma unroll
    for (int tile = 0; tile < MT; ++tile) {
        if (tile * 32 >= M) break;
        if (tile > 0) __syncthreads();
        if (tile / TT == th) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const x_f32x16& a = acc[r][tile % TT];
                    *reinterpret_cast<float4*>(park + (kg * 32 + ln) * PITCH + (wv / TG * RT + r) * 32 + q * 8 + hh * 4) = make_float4(a[q * 4], a[q * 4 + 1], a[q * 4 + 2], a[q * 4 + 3]);
                }
        }
        __syncthreads();
        for (int e = tid; e < 32 * ROWS / 4; e += kWaves4 * kWave) {
            const int t = e / (ROWS / 4), c = e % (ROWS / 4) * 4, m = m0 + tile * 32 + t, n = n0 + c;
            if (tile * 32 + t >= M || n >= p.N) continue;
            float4 v = *reinterpret_cast<const float4*>(park + t * PITCH + c);
#pragma unroll
            for (int g = 1; g < KG; ++g) {
                const float4 u = *reinterpret_cast<const float4*>(park + (g * 32 + t) * PITCH + c);
                v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
            }
            if (parts) {
                *reinterpret_cast<float4*>(p.part + ((long long)split * p.M + m) * p.ldp + n) = v;
            } else if (p.quads && n + 3 < p.N) {
                *reinterpret_cast<x_bf16x4*>(p.Y + m * p.ldy + n) = x_bf16x4{(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
            } else {
                const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n + i < p.N) p.Y[m * p.ldy + n + i] = (__bf16)f[i];
            }
        }
    }
}

__global__ __launch_bounds__(256) void skinny_gemm_mxfp4_reduce_kernel(const Gemm4Params p) {
    constexpr int AT = 4;  // partials requested at a time (one: 64 tokens x 2048 x 11008 19.0 us in all, here 17.7; 256 x 5120 x 27648 81.5 and 79.9)
    const int e = blockIdx.x * 256 + threadIdx.x, quads = p.ldp / 4;
    const int m = quot(e, p.d_nblocks), n = (e - m * quads) * 4;  // (d_nblocks: by quads here)
    if (m >= p.M) return;
    const float* from = p.part + (long long)m * p.ldp + n;
    const long long step = (long long)p.M * p.ldp;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < p.ksplit; s0 += AT) {
        float4 u[AT];
#pragma unroll
        for (int j = 0; j < AT; ++j) u[j] = s0 + j < p.ksplit ? *reinterpret_cast<const float4*>(from + (s0 + j) * step) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            v.x += u[j].x; v.y += u[j].y; v.z += u[j].z; v.w += u[j].w;
        }
    }
    if (p.quads && n + 3 < p.N) {
        *reinterpret_cast<x_bf16x4*>(p.Y + m * p.ldy + n) = x_bf16x4{(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
    } else {
        const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) p.Y[m * p.ldy + n + i] = (__bf16)f[i];
    }
}

// The wavefronts take every eighth 64 k each, straight from memory, the next ones on their way under the products, and add up in LDS.
__global__ __launch_bounds__(kWaves4 * kWave) void skinny_gemm_mxfp4_direct_kernel(const Gemm4Params p) {
    constexpr int WAVES = kWaves4;
    __shared__ float part[WAVES][32][33];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1), ln = lane & 31, hh = lane >> 5;
    const int n0 = blockIdx.x * 32, m0 = blockIdx.y * 32;
    const int n = min(n0 + ln, p.N - 1), m = min(m0 + ln, p.M - 1);  // rows and tokens behind the last ones are not stored
    const unsigned char *w = p.codes + n * p.ld_codes, *s = p.scales + n * p.ld_scales, *x = p.X + m * p.ldx;
    const int blocks = p.K / kMxBlock;
    struct Block {
        mx_u32x4 q;
        unsigned s;
        x_bf16x8 x[4];
    };
    auto load = [&](Block& t, int c) {
        const int b = min(2 * c + hh, blocks - 1);  // (behind an odd last block, and the last one of all, the last one again)
        t.q = *reinterpret_cast<const mx_u32x4*>(w + b * 16);
        t.s = s[b];
#pragma unroll
        for (int k = 0; k < 4; ++k) t.x[k] = *reinterpret_cast<const x_bf16x8*>(x + b * 64 + k * 16);
    };
    x_f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    auto multiply = [&](Block t, int c) {
        if (2 * c + 1 >= blocks && hh == 1) {  // zeros on both sides
            t.q = mx_u32x4{0, 0, 0, 0};
            t.s = 127;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) t.x[k][i] = (__bf16)0.f;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(mx_of_e2m1(t.q[k], t.s), t.x[k], acc, 0, 0, 0);
    };
    if (2 * wave < blocks) {
        Block cur, next;
        load(cur, wave);
        for (int c = wave; 2 * c < blocks; c += WAVES) {
            load(next, c + WAVES);
            multiply(cur, c);
            cur = next;
        }
    }
    // register i of a lane: token ln, row (i / 4) * 8 + hh * 4 + i % 4
#pragma unroll
    for (int i = 0; i < 16; ++i) part[wave][ln][(i >> 2) * 8 + hh * 4 + (i & 3)] = acc[i];
    __syncthreads();
    for (int e = threadIdx.x; e < 32 * 32; e += WAVES * kWave) {
        const int t = e / 32, r = e % 32;
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += part[i][t][r];
        if (m0 + t < p.M && n0 + r < p.N) p.Y[(m0 + t) * p.ldy + n0 + r] = (__bf16)v;
    }
}

// How the tokens are cut: token tiles of a workgroup, parts (1 or 2), tokens of a part.
struct Gemm4Tokens {
    int mt, parts, tokens;
};
static Gemm4Tokens gemm4_tokens(int M) {
    const int parts = M > 128 ? 2 : 1, tokens = (M + parts - 1) / parts;
    return {(tokens + 31) / 32, parts, tokens};
}

// The stream form's groups and splits for so many token tiles, and the time that they are expected to take, us.  Fitted to 14 matrices between 1000 x 512 and
// 152064 x 896, 1 .. 256 tokens, calls over rotated weights.  Of those 112 what is picked is within 11 % of the best of all that were tried (most within 5), but
// for 8 tokens x 896 x 4864, 10.8 us for 8.6.
//   A round of workgroups has its start and its end, by token tiles, and a chunk's time in a group: 64 tokens x 55296 x 5120 in 216 workgroups 47 us, 128 77, 256 in
//   two parts 137; 64 x 152064 x 896 in 594 workgroups 47 us, in 1188 of two groups 57.  A chunk's X for every group and its codes, 60 KB/us a unit, where that
//   is more: 7168 x 5120 at 64 tokens in 4 groups x 2 splits 19.7 us, 2 x 3 21.1.
//   A second launch and the fp32 partials, 9 TB/s: 256 tokens x 5120 x 27648 in 12 splits 79 us, 8 93, 16 110.
struct Gemm4Form {
    int kg, nblocks, ksplit;
    double us;
};
static Gemm4Form gemm4_form(int mt, int parts, int N, int chunks) {
    static const double start[] = {4.5, 6.0, 6.5, 7.0, 8.5, 8.5}, chunk_us[] = {1.4, 2.14, 2.9, 3.55, 5.0, 6.5};
    static const int splits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24};
    const int kind = parts > 1 ? (mt > 3 ? 5 : 4) : mt - 1, most_kg = parts > 1 ? 1 : mt > 2 ? 2 : 4;
    Gemm4Form best = {0, 0, 0, 0.0};
    for (int kg = 1; kg <= most_kg; kg *= 2) {
        const int rows = parts > 1 ? 512 : 256 / kg, nblocks = (N + rows - 1) / rows;
        const double us = std::max(chunk_us[kind], (35.0 * parts + 16.0 * kg * mt) / 60.0);
        for (int ks : splits) {
            const long long wgs = (long long)nblocks * ks * parts;
            if (ks > chunks || (ks > 1 && wgs > kNumCU)) break;
            const int it = ((chunks + ks - 1) / ks + kg - 1) / kg;
            const double t = 1.5 + (double)((wgs + kNumCU - 1) / kNumCU) * (start[kind] + it * us) + (ks > 1 ? 3.0 + ks * 32e-6 * mt * parts * N * 8.0 / 9.0 : 0.0);
            if (best.kg == 0 || t < best.us) best = {kg, nblocks, ks, t};
        }
    }
    return best;
}
// The direct form's: the vector memory unit takes a wavefront's 64 k -- pieces of 32 rows and as many tokens -- in 0.08 us (one token) to 0.16: 1 / 64 tokens x
// 7168 x 5120 9.2 / 33 us (streamed 12.6 / 19.7), 2560 x 2048 5.3 / 8.3 (8.1 / 11.9), 200 x 2048 x 2048 15 (23).
static double gemm4_direct(int M, int N, int K) {
    const double wgs = (double)((N + 31) / 32) * ((M + 31) / 32), rounds = (double)(long long)((wgs + kNumCU - 1) / kNumCU);
    return 3.5 + rounds * (0.5 + (K / 64.0) * (0.075 + 0.085 * std::min(M, 32) / 32.0));
}

static bool gemm4_sizes(int32_t M, int32_t N, int32_t K) { return M >= 1 && M <= 256 && N >= 1 && K >= kMxBlock && K % kMxBlock == 0 && K <= (1 << 22) && N <= (1 << 22); }
static int gemm4_chunks(int K) { return (K + kChunk4 - 1) / kChunk4; }
static int gemm4_pitch(int N) { return (N + 3) / 4 * 4; }

}  // namespace lotts

// A form's partials go by the tokens that it may have at most, or those of the call: no larger call of the same matrix asks for fewer.
extern "C" size_t skinny_gemm_mxfp4_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    using namespace lotts;
    if (!gemm4_sizes(M, N, K)) return 0;
    size_t bytes = 256;
    const int limits[] = {32, 64, 96, 128, 192, 256};
    for (int i = 0; i < 6 && (i == 0 || limits[i - 1] < M); ++i) {
        const Gemm4Tokens t = gemm4_tokens(limits[i]);
        const Gemm4Form f = gemm4_form(t.mt, t.parts, N, gemm4_chunks(K));
        if (f.ksplit > 1) bytes = std::max(bytes, (size_t)f.ksplit * std::min(M, limits[i]) * gemm4_pitch(N) * 4);
    }
    return bytes;
}

extern "C" int skinny_gemm_mxfp4(int32_t M, int32_t N, int32_t K, const void* X, int64_t ldx, const void* codes, int64_t ld_codes, const void* scales,
                                 int64_t ld_scales, void* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lotts;
    if (!gemm4_sizes(M, N, K)) return LOTTS_ERR_SHAPE;
    if (!X || !codes || !scales || !Y || !workspace) return LOTTS_ERR_NULL;
    if (ldx < K || ld_codes < K / 2 || ld_scales < K / kMxBlock || ldy < N) return LOTTS_ERR_SHAPE;
    if (M == 1) ldx = K;  // of one row the pitch is nobody's: the last token of a context, a row of a matrix of any pitch
    if (N == 1) ld_codes = K / 2, ld_scales = K / kMxBlock;
    if (ldx % 8 != 0 || ld_codes % 16 != 0) return LOTTS_ERR_SHAPE;
    // a workgroup's rows of codes and scales, and all tokens, lie within 2^31 bytes of the first; 64-bit offsets hold all of Y
    if (ldx > (1 << 22) || ld_codes > (1 << 24) || ld_scales > (1 << 24) || ldy > (1LL << 48)) return LOTTS_ERR_SHAPE;
    if ((((uintptr_t)X | (uintptr_t)codes | (uintptr_t)workspace) & 15) != 0 || ((uintptr_t)Y & 1) != 0) return LOTTS_ERR_SHAPE;
    if (workspace_bytes < skinny_gemm_mxfp4_workspace_bytes(M, N, K)) return LOTTS_ERR_WORKSPACE;
    const Gemm4Tokens tk = gemm4_tokens(M);
    const Gemm4Form form = gemm4_form(tk.mt, tk.parts, N, gemm4_chunks(K));
    Gemm4Params p;
    p.X = static_cast<const unsigned char*>(X);
    p.codes = static_cast<const unsigned char*>(codes);
    p.scales = static_cast<const unsigned char*>(scales);
    p.Y = static_cast<__bf16*>(Y);
    p.part = static_cast<float*>(workspace);
    p.ldx = ldx * 2; p.ld_codes = ld_codes; p.ld_scales = ld_scales; p.ldy = ldy;
    p.M = M; p.N = N; p.K = K; p.ldp = gemm4_pitch(N); p.tokens = tk.tokens;
    p.chunks = gemm4_chunks(K); p.ksplit = form.ksplit; p.nblocks = form.nblocks; p.items = form.nblocks * form.ksplit * tk.parts;
    p.words = K % 128 == 0 && ld_scales % 4 == 0 && ((uintptr_t)scales & 3) == 0;
    p.quads = ldy % 4 == 0 && ((uintptr_t)Y & 7) == 0;
    p.d_nblocks = fast_div(form.nblocks); p.d_ksplit = fast_div(form.ksplit);
    const hipStream_t s = (hipStream_t)stream;
    if (gemm4_direct(M, N, K) <= form.us) {
        const dim3 tiles((unsigned)((N + 31) / 32), (unsigned)((M + 31) / 32));
        LOTTS_LAUNCH(skinny_gemm_mxfp4_direct_kernel, tiles, dim3(kWaves4 * kWave), s, p);
        return check_launch();
    }
    const dim3 grid((unsigned)((p.items + kNumXCD - 1) / kNumXCD * kNumXCD)), block(kWaves4 * kWave);
#define STREAM4(MT, TG, KG, XD, PARTS)                                                                             \
    do {                                                                                                           \
        if (p.words) LOTTS_LAUNCH((skinny_gemm_mxfp4_stream_kernel<MT, TG, KG, XD, true, PARTS>), grid, block, s, p); \
        else LOTTS_LAUNCH((skinny_gemm_mxfp4_stream_kernel<MT, TG, KG, XD, false, PARTS>), grid, block, s, p);     \
    } while (0)
    switch (tk.parts * 100 + tk.mt * 10 + form.kg) {
        case 111: STREAM4(1, 1, 1, 8, false); break;
        case 112: STREAM4(1, 1, 2, 8, false); break;
        case 114: STREAM4(1, 1, 4, 8, false); break;
        case 121: STREAM4(2, 2, 1, 8, false); break;
        case 122: STREAM4(2, 2, 2, 8, false); break;
        case 124: STREAM4(2, 2, 4, 4, false); break;
        case 131: STREAM4(3, 1, 1, 4, false); break;
        case 132: STREAM4(3, 1, 2, 4, false); break;
        case 141: STREAM4(4, 2, 1, 8, false); break;
        case 142: STREAM4(4, 2, 2, 4, false); break;
        case 231: STREAM4(3, 1, 1, 2, true); break;
        default: STREAM4(4, 1, 1, 1, true); break;
    }
#undef STREAM4
    if (form.ksplit > 1) {
        p.d_nblocks = fast_div(p.ldp / 4);
        LOTTS_LAUNCH(skinny_gemm_mxfp4_reduce_kernel, dim3((unsigned)(((long long)M * (p.ldp / 4) + 255) / 256)), dim3(256), s, p);
    }
    return check_launch();
}
