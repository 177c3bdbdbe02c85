// The DiT-block operations on either side of the attention core, for gfx950:
//
//   lp_qkv_projection   y = x W^T + b cut into q | k | v, with the per-head RMS normalisation
//                       and the 3-D rotary encoding of q and k done in the product's epilogue
//   lp_linear           y = x W^T + b (the block's output projection)
//   lp_qk_norm_rope     the normalisation + rotation alone, in place, for q / k that were
//                       projected elsewhere
//
// The paper leaves the block's internals open (Sec. 5.1: 30 DiT blocks whose atomic units are
// the patches of Sec. 3.1); the form taken is stated in include/lp.h.
//
// The product itself is in lp_gemm.h.
#include <hip/hip_runtime.h>

#include "lp_gemm.h"

namespace {

// Normalisation + rotation alone, in place: one thread per 8 consecutive features of a
// (token, head) row, HD / 8 threads per row.
template <int HD>
__global__ __launch_bounds__(256) void norm_rope_kernel(__bf16 *x, const float *gain, int64_t n, int32_t heads,
                                                        int64_t stride_tok, int64_t stride_head, const RopeArgs r) {
    __shared__ float4 table[kMaxPairs];
    if (threadIdx.x < kMaxPairs)
        table[threadIdx.x] = make_float4(r.turns[threadIdx.x][0], r.turns[threadIdx.x][1], r.turns[threadIdx.x][2], 0.0f);
    __syncthreads();
    constexpr int kPer = HD / 8;                          // threads per row
    const int64_t row = (int64_t(blockIdx.x) * 256 + threadIdx.x) / kPer;
    const int part = threadIdx.x % kPer;
    const bool live = row < n * heads;
    const int64_t rc = live ? row : 0;
    const int64_t tk = rc / heads;
    const int head = int(rc - tk * heads);
    __bf16 *p = x + tk * stride_tok + int64_t(head) * stride_head + part * 8;
    union { uint4 u; bf16x2 p[4]; } in;
    in.u = *reinterpret_cast<const uint4 *>(p);
    float v[8];
    const uint32_t wds[4] = {in.u.x, in.u.y, in.u.z, in.u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {      // a bf16 is the upper half of the binary32 with the same value
        v[2 * e] = __uint_as_float(wds[e] << 16);
        v[2 * e + 1] = __uint_as_float(wds[e] & 0xffff0000u);
    }
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += v[e] * v[e];
#pragma unroll
    for (int m = 1; m < kPer; m *= 2) ss += __shfl_xor(ss, m, 64);
    const float inv = 1.0f / sqrtf(ss * (1.0f / float(HD)) + r.eps);
    const uint32_t t = fastdiv(uint32_t(tk), r.hw);
    const uint32_t rem = uint32_t(tk) - t * r.hw.d;
    const uint32_t h = fastdiv(rem, r.w);
    const float pt = float(int32_t(t) + r.off[0]), ph = float(int32_t(h) + r.off[1]), pw = float(int32_t(rem - h * r.w.d) + r.off[2]);
    const float *gr = gain + head * HD + part * 8;
    const float4 g0 = *reinterpret_cast<const float4 *>(gr), g1 = *reinterpret_cast<const float4 *>(gr + 4);
    const float gv[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
    union { uint4 u; bf16x2 p[4]; } out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float4 tb = table[part * 4 + e];
        float turns = pt * tb.x + ph * tb.y + pw * tb.z;
        turns = turns - floorf(turns);
        const float c = __builtin_amdgcn_cosf(turns), s = __builtin_amdgcn_sinf(turns);
        const float a = v[2 * e] * inv * gv[2 * e], b = v[2 * e + 1] * inv * gv[2 * e + 1];
        out.p[e] = to_bf16x2(a * c - b * s, a * s + b * c);
    }
    if (live) *reinterpret_cast<uint4 *>(p) = out.u;
}

}  // namespace

extern "C" int lp_internal_gemm_way(int64_t n, int32_t d_in, int32_t d_out, int32_t head_dim, int32_t cus, int64_t way[6]) {
    const Plan p = pick_plan(n, d_in, d_out, small_tilings(head_dim), cus);
    plan_way(p, n, d_out, head_dim == 0 && four_waves(p, d_in), way);
    return LP_OK;
}

extern "C" int lp_linear(const void *x, const void *w, const float *bias, void *y, int64_t n, int32_t d_in, int32_t d_out,
                         void *stream) {
    const int chk = check_gemm_shape(n, d_in, d_out);
    if (chk != LP_OK) return chk;
    if (n == 0) return LP_OK;
    if (x == nullptr || w == nullptr || y == nullptr) return LP_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(w) || !aligned16(y) || !aligned16(bias) || y == x || y == w) return LP_ERR_INVALID_ARG;
    GemmArgs a{};
    a.x = static_cast<const __bf16 *>(x);
    a.w = static_cast<const __bf16 *>(w);
    a.bias = bias;
    a.out[0] = static_cast<__bf16 *>(y);
    a.n = int32_t(n);
    a.d_in = d_in;
    a.d_out = d_out;
    return launch_gemm<false, 128>(a, static_cast<hipStream_t>(stream));
}

extern "C" int lp_qkv_projection(const void *x, const void *w_qkv, const float *bias, const float *gain_q, const float *gain_k,
                                 float eps, const lp_rope *rope, void *q, void *k, void *v, int64_t n_tokens, int32_t heads,
                                 int32_t head_dim, void *stream) {
    if (heads < 1) return LP_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return LP_ERR_UNSUPPORTED;
    const int64_t dm64 = int64_t(heads) * head_dim;
    if (3 * dm64 >= (int64_t(1) << 31)) return LP_ERR_UNSUPPORTED;
    const int32_t dm = int32_t(dm64);
    if (dm % 128 != 0) return LP_ERR_UNSUPPORTED;          // a wave's features (up to 128) must not straddle q | k | v
    const int chk = check_gemm_shape(n_tokens, dm, 3 * dm);
    if (chk != LP_OK) return chk;
    if (n_tokens == 0) return LP_OK;
    if (x == nullptr || w_qkv == nullptr || gain_q == nullptr || gain_k == nullptr || q == nullptr || k == nullptr || v == nullptr)
        return LP_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(w_qkv) || !aligned16(bias) || !aligned16(gain_q) || !aligned16(gain_k) || !aligned16(q) ||
        !aligned16(k) || !aligned16(v))
        return LP_ERR_INVALID_ARG;
    if (q == k || q == v || k == v || q == x || k == x || v == x) return LP_ERR_INVALID_ARG;
    GemmArgs a{};
    const int rc = make_rope_args(rope, n_tokens, head_dim, eps, &a.rope);
    if (rc != LP_OK) return rc;
    a.x = static_cast<const __bf16 *>(x);
    a.w = static_cast<const __bf16 *>(w_qkv);
    a.bias = bias;
    a.out[0] = static_cast<__bf16 *>(q);
    a.out[1] = static_cast<__bf16 *>(k);
    a.out[2] = static_cast<__bf16 *>(v);
    a.gain[0] = gain_q;
    a.gain[1] = gain_k;
    a.n = int32_t(n_tokens);
    a.d_in = dm;
    a.d_out = 3 * dm;
    a.heads = heads;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return head_dim == 128 ? launch_gemm<true, 128>(a, st) : launch_gemm<true, 64>(a, st);
}

extern "C" int lp_qk_norm_rope(void *x, const float *gain, float eps, const lp_rope *rope, int64_t n_tokens, int32_t heads,
                               int32_t head_dim, int64_t stride_tok, int64_t stride_head, void *stream) {
    if (heads < 1 || n_tokens < 0) return LP_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return LP_ERR_UNSUPPORTED;
    if (n_tokens == 0) return LP_OK;
    if (x == nullptr || gain == nullptr || !aligned16(x) || !aligned16(gain)) return LP_ERR_INVALID_ARG;
    if (stride_head < head_dim || stride_head % 8 != 0 || stride_tok % 8 != 0) return LP_ERR_INVALID_ARG;
    const bool token_major = stride_tok >= int64_t(heads) * stride_head;
    const bool head_major = stride_head >= n_tokens * stride_tok && stride_tok >= head_dim;
    if (!token_major && !head_major) return LP_ERR_INVALID_ARG;
    RopeArgs r;
    const int rc = make_rope_args(rope, n_tokens, head_dim, eps, &r);
    if (rc != LP_OK) return rc;
    const int64_t threads = n_tokens * heads * (head_dim / 8);
    const int64_t blocks = (threads + 255) / 256;
    if (blocks >= (int64_t(1) << 31)) return LP_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const void *fn = head_dim == 128 ? reinterpret_cast<const void *>(&norm_rope_kernel<128>)
                                     : reinterpret_cast<const void *>(&norm_rope_kernel<64>);
    return lp::launch_kernel(fn, dim3(uint32_t(blocks)), dim3(256), 0, st, static_cast<__bf16 *>(x), gain, n_tokens, heads,
                             stride_tok, stride_head, r);
}
