// mxfp4_quantize, mxfp4_dequantize: a weight matrix to 4-bit microscaled numbers (mx.h), once, when it is loaded, and back to the values that these
// stand for.  The verify forward streams its weights once a step (paper Section 3.1: the step is bound by loading them); in this form they are
// 4.25 bits each.  A lane has eight neighbouring values, four lanes a block; every load and store of a wavefront is one piece of memory.
// Bound by HBM: 55296 x 5120 bf16, 716 MB, one call behind another 121 us (5.9 TB/s), 130 back; in turn, among each other's writes, 141 and 119; fp32 222.
// (Two, four and eight pieces a lane requested at once 121, 126, 131; stores that pass the caches by 131, fp32 212.)
#include "mx.h"

namespace lotts {

struct Mx4Params {
    const unsigned char* values_in;
    unsigned char* values_out;
    unsigned char *codes, *scales;
    long long ld, ld_codes, ld_scales;  // bytes
    int pieces, total;                  // of eight values: of a row, of all
    FastDiv d_pieces;
};

template <typename T>
__global__ __launch_bounds__(256) void mxfp4_quantize_kernel(const Mx4Params p) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= p.total) return;  // (rows are whole blocks: four lanes leave or stay together)
    const int n = quot(i, p.d_pieces), c = i - n * p.pieces;
    MxSource<T> src;
    src.load(p.values_in + n * p.ld + (long long)c * (8 * sizeof(T)));
    float x[8];
    src.values(x);
    const unsigned s = mx_scale<E2M1>(mx_largest(x));
    *reinterpret_cast<unsigned*>(p.codes + n * p.ld_codes + c * 4) = mx_to_e2m1(x, s);
    if ((c & 3) == 0) p.scales[n * p.ld_scales + (c >> 2)] = (unsigned char)s;
}

template <typename T>
__global__ __launch_bounds__(256) void mxfp4_dequantize_kernel(const Mx4Params p) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= p.total) return;
    const int n = quot(i, p.d_pieces), c = i - n * p.pieces;
    const unsigned w = *reinterpret_cast<const unsigned*>(p.codes + n * p.ld_codes + c * 4), s = p.scales[n * p.ld_scales + (c >> 2)];
    const mx_bf16x8 v = mx_of_e2m1(w, s);
    unsigned char* to = p.values_out + n * p.ld + (long long)c * (8 * sizeof(T));
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<mx_bf16x8*>(to) = v;
    } else {
        reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

static int mx4_params(Mx4Params* p, int32_t N, int32_t K, int dtype, const void* values, int64_t ld, const void* codes, int64_t ld_codes, const void* scales,
                      int64_t ld_scales) {
    if (dtype != LOTTS_BF16 && dtype != LOTTS_F32) return LOTTS_ERR_DTYPE;
    const long long es = dtype == LOTTS_BF16 ? 2 : 4;
    if (N < 1 || K < kMxBlock || K % kMxBlock != 0 || (long long)N * (K / 8) > 0x7fffffffLL - 256) return LOTTS_ERR_SHAPE;
    if (!values || !codes || !scales) return LOTTS_ERR_NULL;
    if (ld < K || ld_codes < K / 2 || ld_scales < K / kMxBlock) return LOTTS_ERR_SHAPE;
    if (N == 1) ld = K, ld_codes = K / 2, ld_scales = K / kMxBlock;  // of one row the pitches are nobody's
    if (ld % (16 / es) != 0 || ld_codes % 16 != 0) return LOTTS_ERR_SHAPE;
    if (ld > (1LL << 56) || ld_codes > (1LL << 58) / N || ld_scales > (1LL << 58) / N || ld > (1LL << 58) / N) return LOTTS_ERR_SHAPE;  // 64-bit offsets
    if ((((uintptr_t)values | (uintptr_t)codes) & 15) != 0) return LOTTS_ERR_SHAPE;
    p->codes = static_cast<unsigned char*>(const_cast<void*>(codes));
    p->scales = static_cast<unsigned char*>(const_cast<void*>(scales));
    p->ld = ld * es; p->ld_codes = ld_codes; p->ld_scales = ld_scales;
    p->pieces = K / 8; p->total = N * (K / 8);
    p->d_pieces = fast_div(p->pieces);
    return LOTTS_OK;
}

}  // namespace lotts

extern "C" int mxfp4_quantize(int32_t N, int32_t K, lotts_dtype dtype, const void* W, int64_t ldw, void* codes, int64_t ld_codes, void* scales,
                              int64_t ld_scales, void* stream) {
    using namespace lotts;
    Mx4Params p = {};
    const int rc = mx4_params(&p, N, K, dtype, W, ldw, codes, ld_codes, scales, ld_scales);
    if (rc != LOTTS_OK) return rc;
    p.values_in = static_cast<const unsigned char*>(W);
    const dim3 grid((unsigned)((p.total + 255LL) / 256));
    if (dtype == LOTTS_BF16) LOTTS_LAUNCH(mxfp4_quantize_kernel<__bf16>, grid, dim3(256), (hipStream_t)stream, p);
    else LOTTS_LAUNCH(mxfp4_quantize_kernel<float>, grid, dim3(256), (hipStream_t)stream, p);
    return check_launch();
}

extern "C" int mxfp4_dequantize(int32_t N, int32_t K, lotts_dtype dtype, const void* codes, int64_t ld_codes, const void* scales, int64_t ld_scales, void* values,
                                int64_t ld, void* stream) {
    using namespace lotts;
    Mx4Params p = {};
    const int rc = mx4_params(&p, N, K, dtype, values, ld, codes, ld_codes, scales, ld_scales);
    if (rc != LOTTS_OK) return rc;
    p.values_out = static_cast<unsigned char*>(values);
    const dim3 grid((unsigned)((p.total + 255LL) / 256));
    if (dtype == LOTTS_BF16) LOTTS_LAUNCH(mxfp4_dequantize_kernel<__bf16>, grid, dim3(256), (hipStream_t)stream, p);
    else LOTTS_LAUNCH(mxfp4_dequantize_kernel<float>, grid, dim3(256), (hipStream_t)stream, p);
    return check_launch();
}
