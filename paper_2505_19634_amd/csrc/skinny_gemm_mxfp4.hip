// skinny_gemm_mxfp4: Y[M][N] = X[M][K] W[N][K]^T for up to 256 new tokens of a verify forward against a weight matrix held in 4-bit microscaled
// numbers (mx.h): skinny_gemm with a quarter of the bytes to stream.  The elements become bf16, exactly, on their way to the matrix cores; fp32 sums,
// bf16 out.
//
// A workgroup has 32 weight rows and 32 tokens, its four wavefronts every fourth 64 k each.  Lane (row, half) of a 32 x 32 x 16 product takes 8 of 16 k; which
// ones does not matter as long as both operands agree, so a lane takes a whole block of 32 codes, 16 bytes, with its scale over four products, and the
// same 32 values of X.
#include <algorithm>

#include "mx.h"

namespace lotts {

typedef float x_f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 x_bf16x8 __attribute__((ext_vector_type(8)));

struct Gemm4Params {
    const unsigned char *X, *codes, *scales;
    __bf16* Y;
    long long ldx, ld_codes, ld_scales;  // bytes
    long long ldy;                       // elements
    int M, N, K;
};

__global__ __launch_bounds__(256) void skinny_gemm_mxfp4_kernel(const Gemm4Params p) {
    constexpr int WAVES = 4;
    __shared__ float part[WAVES][32][33];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1), ln = lane & 31, hh = lane >> 5;
    const int n0 = blockIdx.x * 32, m0 = blockIdx.y * 32;
    const int n = min(n0 + ln, p.N - 1), m = min(m0 + ln, p.M - 1);  // rows and tokens behind the last ones are not stored
    const unsigned char *w = p.codes + n * p.ld_codes, *s = p.scales + n * p.ld_scales, *x = p.X + m * p.ldx;
    const int blocks = p.K / kMxBlock;
    x_f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    for (int c = wave; 2 * c < blocks; c += WAVES) {
        const int b = 2 * c + hh;
        const bool there = b < blocks;  // an odd last block: zeros on both sides
        mx_u32x4 q = {0, 0, 0, 0};
        unsigned scale = 127;
        if (there) {
            q = *reinterpret_cast<const mx_u32x4*>(w + b * 16);
            scale = s[b];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x_bf16x8 xv;
#pragma unroll
            for (int i = 0; i < 8; ++i) xv[i] = (__bf16)0.f;
            if (there) xv = *reinterpret_cast<const x_bf16x8*>(x + b * 64 + k * 16);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(mx_of_e2m1(q[k], scale), xv, acc, 0, 0, 0);
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

static bool gemm4_sizes(int32_t M, int32_t N, int32_t K) { return M >= 1 && M <= 256 && N >= 1 && K >= kMxBlock && K % kMxBlock == 0 && K <= (1 << 26) && N <= (1 << 26); }

}  // namespace lotts

extern "C" size_t skinny_gemm_mxfp4_workspace_bytes(int32_t M, int32_t N, int32_t K) { return lotts::gemm4_sizes(M, N, K) ? 256 : 0; }

extern "C" int skinny_gemm_mxfp4(int32_t M, int32_t N, int32_t K, const void* X, int64_t ldx, const void* codes, int64_t ld_codes, const void* scales,
                                 int64_t ld_scales, void* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace lotts;
    if (!gemm4_sizes(M, N, K)) return LOTTS_ERR_SHAPE;
    if (!X || !codes || !scales || !Y || !workspace) return LOTTS_ERR_NULL;
    if (ldx < K || ld_codes < K / 2 || ld_scales < K / kMxBlock || ldy < N || ldx % 8 != 0 || ld_codes % 16 != 0) return LOTTS_ERR_SHAPE;
    if (ldx > (1LL << 48) || ldy > (1LL << 48) || ld_codes > (1LL << 58) / N || ld_scales > (1LL << 58) / N) return LOTTS_ERR_SHAPE;  // 64-bit offsets
    if ((((uintptr_t)X | (uintptr_t)codes | (uintptr_t)workspace) & 15) != 0 || ((uintptr_t)Y & 1) != 0) return LOTTS_ERR_SHAPE;
    if (workspace_bytes < skinny_gemm_mxfp4_workspace_bytes(M, N, K)) return LOTTS_ERR_WORKSPACE;
    Gemm4Params p;
    p.X = static_cast<const unsigned char*>(X);
    p.codes = static_cast<const unsigned char*>(codes);
    p.scales = static_cast<const unsigned char*>(scales);
    p.Y = static_cast<__bf16*>(Y);
    p.ldx = ldx * 2; p.ld_codes = ld_codes; p.ld_scales = ld_scales; p.ldy = ldy;
    p.M = M; p.N = N; p.K = K;
    LOTTS_LAUNCH(skinny_gemm_mxfp4_kernel, dim3((unsigned)((N + 31) / 32), (unsigned)((M + 31) / 32)), dim3(256), (hipStream_t)stream, p);
    return check_launch();
}
