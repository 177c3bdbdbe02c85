// Normalisation with the modulation of several requests, and the gated residual in front of it, for gfx950:
//
//   lp_norm_modulate          y = norm(x) (1 + scale_r) + shift_r
//   lp_gated_residual_norm    h' = h + gate_r post(u);  y = norm(h') (1 + scale_r) + shift_r
//
// with r the request that a row belongs to.  One pass: a row's elements stay in registers between the sums over them and
// the results, so that every element of x (h and u) is read once and every result written once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "lp_device.h"
#include "lp_requests.h"

namespace {

using namespace lp;

constexpr int kMaxWidth = 16384;
constexpr int kNone = -1;                // no normalisation

struct NormArgs {
    const void *x;                       // x, or h of the residual
    const __bf16 *u;
    void *h_out;
    __bf16 *y;                           // nullptr: nothing is normalised behind the residual
    int64_t stride_x, stride_u, stride_h_out, stride_y, stride_mod;
    const float *post_weight, *post_bias, *weight, *bias, *gate, *scale, *shift;
    float post_eps, eps, inv_d;
    int32_t post, norm;                  // LP_NORM_*, or kNone
    int32_t d, n;
    RequestTable requests;
};

// Sum over the 64 lanes, in every one of them: exchanges inside rows of 16 lanes, then between the rows.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp<0xb1>(x);                   // lane ^ 1
    x += dpp<0x4e>(x);                   // lane ^ 2
    x += dpp<0x141>(x);                  // 7 - lane within 8
    x += dpp<0x140>(x);                  // 15 - lane within 16
    return over_quads(x, [](float a, float b) { return a + b; });
}

// Sums over the G threads that share a row.  Wavefronts meet through LDS; two places, used in turn, make one barrier a sum
// enough: a wavefront that writes a place again has passed the barrier of the sum between, behind everybody's reads of it.
template <int G>
struct RowSum {
    float (*place)[G / 64];              // [2]
    int turn;
    __device__ __forceinline__ float operator()(float x) {
        x = wave_sum(x);
        if constexpr (G > 64) {
            if (threadIdx.x % 64 == 0) place[turn][threadIdx.x / 64] = x;
            __syncthreads();
            x = 0.0f;
#pragma unroll
            for (int w = 0; w < G / 64; ++w) x += place[turn][w];
            turn ^= 1;
        }
        return x;
    }
};

// A thread's elements: CH pieces of 8.  VEC 8: piece c is the 8 elements from 8 (c G + t) on, moved 16 bytes at a time; VEC 1: element j
// of all of them is j G + t.  Rows are raw buffers of d elements: what lies past the end is read as 0 and not written, so that
// no address is computed and no lane masked for an element, which in single elements took all registers there are (one
// wavefront to a SIMD: 1111 x 1153 in 21.7 us).
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const T *row, int d) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(row), 0, d * int(sizeof(T)), 0x00020000);
}
template <int G, int CH, int VEC, typename T>
struct Row {
    T v[8 * CH];
    static constexpr int kPieces = 8 * sizeof(T) / 16, kPer = 16 / sizeof(T);
    typedef __attribute__((ext_vector_type(kPer))) T Piece;
    __device__ __forceinline__ void load(const T *row, int t, int d) {
        const __amdgpu_buffer_rsrc_t r = row_buffer(row, d);
        if constexpr (VEC == 8) {
#pragma unroll
            for (int c = 0; c < CH * kPieces; ++c) {
                const int first = 8 * (c / kPieces) * G + (c % kPieces) * kPer;
                const Piece p = __builtin_bit_cast(Piece, __builtin_amdgcn_raw_buffer_load_b128(r, t * 8 * sizeof(T), first * sizeof(T), 0));
#pragma unroll
                for (int i = 0; i < kPer; ++i) v[c * kPer + i] = p[i];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8 * CH; ++j) {
                if constexpr (sizeof(T) == 2) v[j] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(r, t * 2, j * G * 2, 0));
                else v[j] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(r, t * 4, j * G * 4, 0));
            }
        }
    }
    __device__ __forceinline__ void store(T *row, int t, int d) const {
        const __amdgpu_buffer_rsrc_t r = row_buffer(row, d);
        if constexpr (VEC == 8) {
#pragma unroll
            for (int c = 0; c < CH * kPieces; ++c) {
                const int first = 8 * (c / kPieces) * G + (c % kPieces) * kPer;
                Piece p;
#pragma unroll
                for (int i = 0; i < kPer; ++i) p[i] = v[c * kPer + i];
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, p), r, t * 8 * sizeof(T), first * sizeof(T), 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8 * CH; ++j) {
                if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v[j]), r, t * 2, j * G * 2, 0);
                else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v[j]), r, t * 4, j * G * 4, 0);
            }
        }
    }
};

// v <- (v - mean) / sqrt(var + eps) or v / sqrt(mean square + eps); live(j): whether element j exists (those that do not are 0).
template <int N, typename SUM, typename LIVE>
__device__ __forceinline__ void normalise(float (&v)[N], int kind, float eps, float inv_d, SUM &sum, LIVE &&live) {
    if (kind == LP_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) s += v[j];
        const float mean = sum(s) * inv_d;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = live(j) ? v[j] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) s += v[j] * v[j];
    const float inv = 1.0f / sqrtf(sum(s) * inv_d + eps);
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] *= inv;
}

// G threads to a row, every group of them a contiguous stretch of rows.
//
// What bounds it: HBM.  13230 x 5120 in bf16 (271 MB) 53.6 us, 5.05 TB/s; the residual of 24570 x 5120 (1.01 GB) 179 us, 5.6 TB/s; 22380 x 1536 in
// binary32 with norms on both sides (413 MB) 81 us, 5.1 TB/s; a binary32 row normalised 13230 x 5120 77 us, 5.3 TB/s; single elements 12000 x 1153
// 21 us in either type (2.6 and 4.0 TB/s), by their instructions; where a plain copy of 4 GiB reaches 4.7 TB/s.  The vectors of a
// request, up to four times d in binary32, would be two to four times a row's own bytes from L2 for every row: a thread keeps its part of them in
// registers, products of the weights and the modulation, and fetches them again when its stretch enters another request.
template <int G, int CH, int VEC, typename X, bool RESIDUAL>
__global__ __launch_bounds__(G > 256 ? G : 256) void norm_kernel(const NormArgs a) {
    constexpr int kThreads = G > 256 ? G : 256, kGroups = kThreads / G, N = 8 * CH;
    __shared__ float place[2][G / 64];
    const int t = threadIdx.x % G;
    const int group = __builtin_amdgcn_readfirstlane(int(blockIdx.x) * kGroups + int(threadIdx.x) / G);
    const int groups = int(gridDim.x) * kGroups, q = a.n / groups, rem = a.n % groups;
    int row = group * q + min(group, rem);
    const int last = row + q + (group < rem ? 1 : 0);
    const int32_t ends = a.requests.start[threadIdx.x % 64 + 1];
    RowSum<G> sum{place, 0};
    auto live = [&](int j) { return (VEC == 8 ? 8 * ((j / 8) * G + t) : j * G + t) < a.d; };

    // weight (1 + scale), bias (1 + scale) + shift; gate x post's weight and bias
    float mul[N], add[N], gate[N], gate_bias[N];
    int32_t request_end = 0;
    auto vectors = [&](int request) {
        Row<G, CH, VEC, float> s, w;
        const int64_t at = int64_t(request) * a.stride_mod;
        auto fetch = [&](Row<G, CH, VEC, float> &r, const float *p, int64_t off, float otherwise) {
            if (p != nullptr) {
                r.load(p + off, t, a.d);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) r.v[j] = otherwise;
            }
        };
        // bias times factor; a bias that is not there is no term, also where the factor is infinite
        auto product = [&](float (&out)[N], const float *bias, const Row<G, CH, VEC, float> &factor) {
            if (bias != nullptr) {
                w.load(bias, t, a.d);
#pragma unroll
                for (int j = 0; j < N; ++j) out[j] = w.v[j] * factor.v[j];
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) out[j] = 0.0f;
            }
        };
        if (a.norm != kNone) {
            fetch(s, a.scale, at, 0.0f);
            fetch(w, a.weight, 0, 1.0f);
#pragma unroll
            for (int j = 0; j < N; ++j) { s.v[j] += 1.0f; mul[j] = w.v[j] * s.v[j]; }
            product(add, a.bias, s);
            fetch(s, a.shift, at, 0.0f);
#pragma unroll
            for (int j = 0; j < N; ++j) add[j] += s.v[j];
        }
        if constexpr (RESIDUAL) {
            fetch(s, a.gate, at, 1.0f);
            fetch(w, a.post_weight, 0, 1.0f);
#pragma unroll
            for (int j = 0; j < N; ++j) gate[j] = s.v[j] * w.v[j];
            product(gate_bias, a.post_bias, s);
        }
    };

    // The next row is sent for before this one's sums, whose exchanges it then arrives under; not with 1024 threads to a row, which
    // have 128 registers each (three of their four residual forms keep 5 or 6 values in scratch memory as it is).  HBM binds there too: 9000 x 16384
    // 123 us in bf16 (4.8 TB/s), the residual in binary32 with norms on both sides 348 (5.1 TB/s); in single elements 181 us for 9000 x 16383.
    constexpr bool kAhead = G < 1024;
    const X *xs = static_cast<const X *>(a.x);
    Row<G, CH, VEC, X> x;
    Row<G, CH, VEC, __bf16> u;
    auto send = [&](int r) {
        x.load(xs + int64_t(r) * a.stride_x, t, a.d);
        if constexpr (RESIDUAL) u.load(a.u + int64_t(r) * a.stride_u, t, a.d);
    };
    if (kAhead && row < last) send(row);
    for (; row < last; ++row) {
        if (!kAhead) send(row);
        if (row >= request_end) {
            const int request = request_of(ends, row);
            request_end = __builtin_amdgcn_readlane(ends, request);
            vectors(request);
        }
        float v[N];
        if constexpr (RESIDUAL) {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = float(u.v[j]);
            Row<G, CH, VEC, X> h = x;
            if (kAhead && row + 1 < last) send(row + 1);
            if (a.post != kNone) normalise(v, a.post, a.post_eps, a.inv_d, sum, live);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[j] = float(h.v[j]) + (gate[j] * v[j] + gate_bias[j]);
                h.v[j] = X(v[j]);
            }
            h.store(static_cast<X *>(a.h_out) + int64_t(row) * a.stride_h_out, t, a.d);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = live(j) ? v[j] : 0.0f;
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = float(x.v[j]);
            if (kAhead && row + 1 < last) send(row + 1);
        }
        if (a.norm == kNone) continue;
        normalise(v, a.norm, a.eps, a.inv_d, sum, live);
        Row<G, CH, VEC, __bf16> y;
#pragma unroll
        for (int j = 0; j < N; ++j) y.v[j] = __bf16(v[j] * mul[j] + add[j]);
        y.store(a.y + int64_t(row) * a.stride_y, t, a.d);
    }
}

// Workgroups of `groups` rows at a time.  Few rows: one each.  Beyond two workgroups to a compute unit every group takes two rows at least
// and fetches its request's vectors once for them, and all compute units have as many (1111 x 1153 with norms on both sides 8.2 us, 10.5 with a row each; 4000 x 1536
// 6.4 and 6.7).  At most 4096 threads to a compute unit, twice what can run at a time, which evens out their ends: 13230 x 5120 53.6 us,
// 57.0 with 2048, 59.4 with 1024.  8192 for the residual in whole pieces, whose rows are four streams instead of two: 24570 x 5120 179.4
// us, 190.5 with 4096, 199 with 2048 (20000 x 3584 158 and 165; 13230 x 5120 without the residual 54.0 and 53.6; 12000 x 1153 in single elements
// 46 and 43; 9000 x 16384, 1024 threads to a row, 366 and 358).
uint32_t workgroups(int64_t n, int groups, int threads, int most_threads, int cus) {
    const int64_t one_each = (n + groups - 1) / groups, few = 2 * int64_t(cus), most = int64_t(cus) * (most_threads / threads);
    if (one_each <= few) return uint32_t(one_each);
    const int64_t two_each = n / (2 * groups) / cus * cus;
    return uint32_t(std::min(most, std::max(few, two_each)));
}

template <int G, int CH, int VEC>
int launch(const NormArgs &a, bool f32, bool residual, hipStream_t stream) {
    const int cus = lp::device_compute_units();
    if (cus <= 0) return LP_ERR_HIP;
    constexpr int kThreads = G > 256 ? G : 256, kGroups = kThreads / G;
    const void *fn = residual ? (f32 ? reinterpret_cast<const void *>(&norm_kernel<G, CH, VEC, float, true>)
                                     : reinterpret_cast<const void *>(&norm_kernel<G, CH, VEC, __bf16, true>))
                              : (f32 ? reinterpret_cast<const void *>(&norm_kernel<G, CH, VEC, float, false>)
                                     : reinterpret_cast<const void *>(&norm_kernel<G, CH, VEC, __bf16, false>));
    const int most_threads = residual && VEC == 8 && G < 1024 ? 8192 : 4096;
    return lp::launch_kernel(fn, dim3(workgroups(a.n, kGroups, kThreads, most_threads, cus)), dim3(kThreads), 0, stream, a);
}

int run(const NormArgs &a, bool vec, bool f32, bool residual, hipStream_t stream) {
    if (vec) {
        if (a.d <= 512) return launch<64, 1, 8>(a, f32, residual, stream);
        if (a.d <= 1024) return launch<64, 2, 8>(a, f32, residual, stream);
        if (a.d <= 1536) return launch<64, 3, 8>(a, f32, residual, stream);
        if (a.d <= 2048) return launch<256, 1, 8>(a, f32, residual, stream);
        if (a.d <= 4096) return launch<256, 2, 8>(a, f32, residual, stream);
        if (a.d <= 6144) return launch<256, 3, 8>(a, f32, residual, stream);
        if (a.d <= 8192) return launch<512, 2, 8>(a, f32, residual, stream);
        return launch<1024, 2, 8>(a, f32, residual, stream);
    }
    // single elements: what lies past the row's end costs an instruction each, so that the steps are finer (12000 x 1153 residual 43 us,
    // 71 with 16 elements to a thread)
    if (a.d <= 512) return launch<64, 1, 1>(a, f32, residual, stream);
    if (a.d <= 1024) return launch<64, 2, 1>(a, f32, residual, stream);
    if (a.d <= 2048) return launch<256, 1, 1>(a, f32, residual, stream);
    if (a.d <= 4096) return launch<256, 2, 1>(a, f32, residual, stream);
    if (a.d <= 8192) return launch<512, 2, 1>(a, f32, residual, stream);
    return launch<1024, 2, 1>(a, f32, residual, stream);
}

// ---- checks

bool aligned(const void *p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

int check_norm(const lp_norm *n, int32_t *kind, float *eps, const float **weight, const float **bias) {
    if (n->kind != LP_NORM_LAYER && n->kind != LP_NORM_RMS) return LP_ERR_INVALID_ARG;
    if (!(n->eps >= 0.0f) || !std::isfinite(n->eps) || !aligned(n->weight, 4) || !aligned(n->bias, 4)) return LP_ERR_INVALID_ARG;
    *kind = n->kind;
    *eps = n->eps;
    *weight = n->weight;
    *bias = n->bias;
    return LP_OK;
}

// Types, width, requests and the vectors that the call uses: the others are not looked at, nor the stride where it uses none.
int check_common(int32_t type, const lp_requests *requests, int32_t d, const lp_modulation *m, bool residual, bool norm, NormArgs *a) {
    if (type != LP_BF16 && type != LP_F32) return LP_ERR_INVALID_ARG;
    if (d < 1) return LP_ERR_INVALID_ARG;
    if (d > kMaxWidth) return LP_ERR_UNSUPPORTED;
    const int rc = make_request_table(requests, &a->requests);
    if (rc != LP_OK) return rc;
    a->d = d;
    a->inv_d = 1.0f / float(d);
    a->n = int32_t(a->requests.rows());
    if (m != nullptr) {
        if (residual) a->gate = m->gate;
        if (norm) {
            a->scale = m->scale;
            a->shift = m->shift;
        }
        if (a->gate != nullptr || a->scale != nullptr || a->shift != nullptr) {
            if (m->stride != 0 && m->stride < d) return LP_ERR_INVALID_ARG;
            if (!aligned(a->gate, 4) || !aligned(a->scale, 4) || !aligned(a->shift, 4)) return LP_ERR_INVALID_ARG;
            a->stride_mod = m->stride;
        }
    }
    return LP_OK;
}

bool vectors_aligned(const NormArgs &a) {
    return a.d % 8 == 0 && a.stride_mod % 4 == 0 && aligned16(a.gate) && aligned16(a.scale) && aligned16(a.shift) && aligned16(a.weight) &&
           aligned16(a.bias) && aligned16(a.post_weight) && aligned16(a.post_bias);
}

}  // namespace

extern "C" int lp_norm_modulate(const void *x, int32_t x_type, void *y, const lp_requests *requests, int32_t d, int64_t stride_x,
                                int64_t stride_y, const lp_norm *norm, const lp_modulation *modulation, void *stream) {
    NormArgs a{};
    int rc = check_common(x_type, requests, d, modulation, false, true, &a);
    if (rc != LP_OK) return rc;
    if (norm == nullptr || stride_x < d || stride_y < d) return LP_ERR_INVALID_ARG;
    if ((rc = check_norm(norm, &a.norm, &a.eps, &a.weight, &a.bias)) != LP_OK) return rc;
    if (a.n == 0) return LP_OK;
    if (x == nullptr || y == nullptr || !aligned(x, x_type == LP_F32 ? 4 : 2) || !aligned(y, 2)) return LP_ERR_INVALID_ARG;
    if (y == x && (x_type != LP_BF16 || stride_x != stride_y)) return LP_ERR_INVALID_ARG;
    a.x = x;
    a.y = static_cast<__bf16 *>(y);
    a.stride_x = stride_x;
    a.stride_y = stride_y;
    a.post = kNone;
    const bool vec = vectors_aligned(a) && aligned16(x) && aligned16(y) && stride_x % 8 == 0 && stride_y % 8 == 0;
    return run(a, vec, x_type == LP_F32, false, static_cast<hipStream_t>(stream));
}

extern "C" int lp_gated_residual_norm(const void *h, int32_t h_type, const void *u, void *h_out, void *y, const lp_requests *requests,
                                      int32_t d, int64_t stride_h, int64_t stride_u, int64_t stride_h_out, int64_t stride_y,
                                      const lp_norm *post, const lp_norm *norm, const lp_modulation *modulation, void *stream) {
    NormArgs a{};
    int rc = check_common(h_type, requests, d, modulation, true, norm != nullptr, &a);
    if (rc != LP_OK) return rc;
    if (stride_h < d || stride_u < d || stride_h_out < d || (norm != nullptr && stride_y < d)) return LP_ERR_INVALID_ARG;
    a.post = a.norm = kNone;
    if (post != nullptr && (rc = check_norm(post, &a.post, &a.post_eps, &a.post_weight, &a.post_bias)) != LP_OK) return rc;
    if (norm != nullptr && (rc = check_norm(norm, &a.norm, &a.eps, &a.weight, &a.bias)) != LP_OK) return rc;
    if ((norm == nullptr) != (y == nullptr) && a.n > 0) return LP_ERR_INVALID_ARG;
    if (a.n == 0) return LP_OK;
    const int size = h_type == LP_F32 ? 4 : 2;
    if (h == nullptr || u == nullptr || h_out == nullptr || !aligned(h, size) || !aligned(h_out, size) || !aligned(u, 2) || !aligned(y, 2))
        return LP_ERR_INVALID_ARG;
    if ((h_out == h && stride_h_out != stride_h) || h_out == u || (y != nullptr && (y == h || y == u || y == h_out))) return LP_ERR_INVALID_ARG;
    a.x = h;
    a.u = static_cast<const __bf16 *>(u);
    a.h_out = h_out;
    a.y = static_cast<__bf16 *>(y);
    a.stride_x = stride_h;
    a.stride_u = stride_u;
    a.stride_h_out = stride_h_out;
    a.stride_y = norm != nullptr ? stride_y : 0;
    const bool vec = vectors_aligned(a) && aligned16(h) && aligned16(u) && aligned16(h_out) && aligned16(y) && stride_h % 8 == 0 &&
                     stride_u % 8 == 0 && stride_h_out % 8 == 0 && a.stride_y % 8 == 0;
    return run(a, vec, h_type == LP_F32, true, static_cast<hipStream_t>(stream));
}
