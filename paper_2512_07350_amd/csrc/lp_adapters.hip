// Projections of several requests' tokens with a low-rank adapter of each beside the shared weights, for gfx950:
//
//   lp_linear_adapters           y = x W^T + b + s_r (x D_r^T) U_r^T
//   lp_qkv_projection_adapters   the same in the sections q | k | v, q and k normalised and rotated
//
// with r the request that a row belongs to.  Two launches (one for few rows, product_few of lp_gemm.h): adapter_down_kernel forms t = s_r x D_r^T of the rows that have an
// adapter (and looks over every U_r), and the product of lp_gemm.h takes t and U_r as further k-tiles.  The second thus costs a k-tile of 64 for every
// 32 ranks beside d_in / 64 of them, and no pass over y.
//
// What bounds it.  Large calls: the shared product; 24570 x 5120 -> 5120 with ranks 64 and 16 966 us, 900 without adapters, 64 of the
// difference for t, which reads x once more (3.9 TB/s).  q | k | v of 13230 x 5120, rank 32, 1557 and 1506, 41 for t.  Few rows and ranks: one
// launch (product_few); with more ranks two, 6 rows of d_in 1536 and rank 128 13.3 us, 5.4 without adapters.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "lp_gemm.h"

namespace {

// ---- the down products

struct DownRun {
    int32_t start, rank;                 // rows from start on, to the next run's; rank 0: no adapter
    int32_t first, first_look;           // the run's first workgroup, that of those that look over U
    float scale;
    const __bf16 *down, *up;             // D [sections * rank, d_in], U [d_out, rank]
};
struct DownArgs {
    const __bf16 *x;
    __bf16 *t;                           // see AdaptedArgs
    AdapterControl *control;
    int32_t t_row, t_blocks, d_in, d_out, sections, looks;
    DownRun run[LP_MAX_REQUESTS + 1];
};

// Workgroups that look over a U of `pieces` 16 bytes: one for 64 KB, at most kLooks.
__host__ __device__ int32_t look_parts(int64_t pieces) {
    const int64_t by_size = (pieces + 4095) / 4096;
    return int32_t(by_size < kLooks ? by_size : kLooks);
}

// Rows of D x tokens.  The four wavefronts share k where there are few tokens, and otherwise the tokens.
using DownFew = Tiling<2, 2, 2, 1, 8, kSplitK>;          // 64 x 32
using DownMany = Tiling<1, 4, 4, 2, 6>;                  // 64 x 128
using DownTall = Tiling<1, 4, 8, 1, 3>;                  // 128 x 64
constexpr int kDownThreads = 256;
static_assert(DownFew::kThreads == kDownThreads && DownMany::kThreads == kDownThreads && DownTall::kThreads == kDownThreads, "look_over's too");

// Whether part of a run's U holds an infinity or a NaN, to its word of the control block; the first workgroup writes the rest of the block.
__device__ void look_over(const DownArgs &a, int wg) {
    const int r = __builtin_amdgcn_readfirstlane(__popcll(__ballot(a.run[threadIdx.x % 64].first_look <= wg))) - 1;
    const int part = wg - a.run[r].first_look;
    const int64_t pieces = int64_t(a.d_out) * a.run[r].rank / 8;
    const int parts = look_parts(pieces);
    const uint4 *u = reinterpret_cast<const uint4 *>(a.run[r].up);
    const int64_t last = pieces * (part + 1) / parts;
    uint32_t bad = 0;
    auto look = [&](uint32_t two) { bad |= uint32_t((two & 0x7f80u) == 0x7f80u) | uint32_t((two & 0x7f800000u) == 0x7f800000u); };
#pragma unroll 8
    for (int64_t i = pieces * part / parts + threadIdx.x; i < last; i += kDownThreads) {
        const uint4 p = u[i];
        look(p.x);
        look(p.y);
        look(p.z);
        look(p.w);
    }
    const int any = __syncthreads_or(int(bad));
    const int i = int(threadIdx.x);
    if (i == 0) a.control->looks[r][part] = uint32_t(any);
    if (part == 0 && i >= parts && i < kLooks) a.control->looks[r][i] = 0;
    if (wg == 0 && i < LP_MAX_REQUESTS) {
        a.control->run[i] = AdapterRun{a.run[i].start, a.run[i + 1].start, a.run[i].rank, 0, a.run[i].up, 0};
        if (i < 32) a.control->nan[i] = 0x7fc07fc0u;
        if (a.run[i].rank == 0)
            for (int k = 0; k < kLooks; ++k) a.control->looks[i][k] = 0;
    }
}

template <typename C>
__global__ __launch_bounds__(kDownThreads, 1) void adapter_down_kernel(const DownArgs a) {
    if (int(blockIdx.x) < a.looks) return look_over(a, int(blockIdx.x));
    const int wg = int(blockIdx.x) - a.looks;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const uint32_t lds0 = uint32_t(uintptr_t(LP_LDS_PTR(unsigned char, smem)));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, col = lane % 16, quad = lane / 16;
    // the run of this workgroup: the last one that starts with it or before
    const int r = __builtin_amdgcn_readfirstlane(__popcll(__ballot(a.run[lane].first <= wg))) - 1;
    const int rank = a.run[r].rank, rows = a.sections * rank, f_tiles = (rows + C::kF - 1) / C::kF, j = wg - a.run[r].first;
    const int f0 = j % f_tiles * C::kF, t0 = a.run[r].start + j / f_tiles * C::kT;
    GemmArgs g{};
    g.x = a.x;
    g.w = a.run[r].down;
    g.n = a.run[r + 1].start;
    g.d_in = a.d_in;
    g.d_out = rows;
    f32x4 acc[C::FB][C::TB];
    if constexpr (C::SPLIT) product_split_k<C>(lds0, g, f0, t0, wave, lane, acc, 0);
    else product<C>(lds0, g, f0, t0, wave, lane, acc, 0);
    const float scale = a.run[r].scale;
#pragma unroll
    for (int f = 0; f < C::FB; ++f) {
        const int row = f0 + (wave / C::WT * C::FB + f) * 16 + 4 * quad;   // of D; four of them, of one section
        if (row >= rows) break;
        const int section = row / rank, at = row - section * rank;
        __bf16 *to = a.t + (section * a.t_blocks + at / kRanks) * (2 * kRanks) + at % kRanks;
#pragma unroll
        for (int t = 0; t < C::TB; ++t) {
            const int tok = t0 + (wave % C::WT * C::TB + t) * 16 + col;
            if (tok >= g.n) break;
            const f32x4 v = acc[f][t] * scale;
            const bf16x4 hi = __builtin_convertvector(v, bf16x4), lo = __builtin_convertvector(v - __builtin_convertvector(hi, f32x4), bf16x4);
            *reinterpret_cast<bf16x4 *>(to + int64_t(tok) * (a.t_row / 2)) = hi;
            *reinterpret_cast<bf16x4 *>(to + int64_t(tok) * (a.t_row / 2) + kRanks) = lo;
        }
    }
}

// ---- the requests' adapters

int64_t t_row_bytes(int32_t rank, int32_t sections) { return int64_t(sections) * ((rank + kRanks - 1) / kRanks) * (4 * kRanks); }

// Neighbouring requests with one adapter as runs, with the down products' launch.
struct Runs {
    RequestTable requests;
    int32_t runs = 0, largest = 0;       // runs; the largest rank
    DownArgs down{};
};

int make_runs(const lp_requests *requests, const lp_adapter *adapters, int32_t d_in, int32_t d_out, int32_t sections, Runs *out) {
    const int rc = make_request_table(requests, &out->requests);
    if (rc != LP_OK) return rc;
    const RequestTable &q = out->requests;
    if (q.count > 0 && adapters == nullptr) return LP_ERR_INVALID_ARG;
    for (int r = 0; r < q.count; ++r) {
        const lp_adapter &ad = adapters[r];
        if (ad.rank < 0) return LP_ERR_INVALID_ARG;
        if (ad.rank > LP_MAX_ADAPTER_RANK || ad.rank % 8 != 0) return LP_ERR_UNSUPPORTED;
        if (ad.rank > 0 && (ad.down == nullptr || ad.up == nullptr || !aligned16(ad.down) || !aligned16(ad.up) || !std::isfinite(ad.scale)))
            return LP_ERR_INVALID_ARG;
    }
    const lp_adapter *last = nullptr;
    for (int r = 0; r < q.count; ++r) {
        const lp_adapter &ad = adapters[r];
        if (q.start[r + 1] == q.start[r]) continue;
        const bool same = last != nullptr && last->rank == ad.rank &&
                          (ad.rank == 0 || (last->down == ad.down && last->up == ad.up && last->scale == ad.scale));
        last = &ad;
        if (same) continue;
        const int i = out->runs++;
        out->down.run[i] = DownRun{q.start[r], ad.rank, 0, 0, ad.scale, static_cast<const __bf16 *>(ad.down), static_cast<const __bf16 *>(ad.up)};
        if (ad.rank > out->largest) out->largest = ad.rank;
    }
    const int32_t n = int32_t(q.rows());
    for (int i = out->runs; i <= LP_MAX_REQUESTS; ++i)
        out->down.run[i] = DownRun{i == out->runs ? n : INT32_MAX, 0, INT32_MAX, INT32_MAX, 0.0f, nullptr, nullptr};
    out->down.d_in = d_in;
    out->down.d_out = d_out;
    out->down.sections = sections;
    return LP_OK;
}

// The tiling of a call: pick_plan's, with the k-tiles of the adapters that a tile of t tokens takes on average.  A tile that many short runs
// crowd takes more, every one of them a k-tile for 32 ranks: 48 requests of one row beside 20000 rows, all of rank 128, 1536 -> 1536, take 333 us in
// 256 x 256 tiles (199 to 283 by where the 48 lie in 128 x 128, the rest of them in 128 x 64), 62 of rank 256 710 (283 to 577).  With the longest tile in
// the price these took 206 to 290 and 431 to 665, and 20 of 1500 ordinary calls, whose tiling it changed, 0.78 to 1.14 of their time, 1.03 on average.
Plan pick_adapted(int32_t n, int32_t d_in, int32_t d_out, int32_t head_dim, int cus, int32_t runs, const DownRun *run) {
    return pick_plan(n, d_out, small_tilings(head_dim), cus, [&](int t) {
        int64_t extra = 0;
        for (int i = 0; i < runs; ++i) {
            const int64_t first = run[i].start / t, last = (run[i + 1].start - 1) / t;
            extra += (last - first + 1) * ((run[i].rank + kRanks - 1) / kRanks);
        }
        const int64_t tiles = (int64_t(n) + t - 1) / t;
        return d_in / kBK + int((extra + tiles - 1) / tiles);
    });
}

// Workgroups of C that the down products take: the tiles, every one of a single run, behind those that look over U.
template <typename C>
int64_t down_tiles(DownArgs &d, int32_t runs) {
    int64_t tiles = 0;
    for (int i = 0; i < runs; ++i) {
        d.run[i].first = int32_t(tiles);
        tiles += (int64_t(d.run[i + 1].start) - d.run[i].start + C::kT - 1) / C::kT * ((int64_t(d.sections) * d.run[i].rank + C::kF - 1) / C::kF);
    }
    return tiles;
}
template <typename C>
int launch_down(DownArgs &d, int32_t runs, int dev, hipStream_t stream) {
    const int64_t workgroups = d.looks + down_tiles<C>(d, runs);
    if (workgroups * kDownThreads > lp::kMaxLaunchThreads) return LP_ERR_UNSUPPORTED;
    static std::atomic<uint64_t> attr_set{0};
    const void *kern = reinterpret_cast<const void *>(&adapter_down_kernel<C>);
    const int rc = allow_lds(kern, C::kLds, dev, attr_set);
    if (rc != LP_OK) return rc;
    return lp::launch_kernel(kern, dim3(uint32_t(workgroups)), dim3(kDownThreads), C::kLds, stream, d);
}

// The tile of the down products.  Up to one of 64 x 32 for every compute unit the wavefronts share k: 6 rows of d_in 1536 6.0 us, 977 of 4096 in
// twelve runs 10.9, with 64 x 128 9.6 and 20.0.  Beyond, x is what binds, and tiles of more tokens read D less often: 22380 x 1536
// 20.8 us in 64 x 32, 15.7 in 64 x 128 (4.4 TB/s of x), 24570 x 5120 72 and 64 (3.9).  A run with more than 64 rows of D reads x twice there; with more
// than three quarters of the tokens in such runs 128 x 64 is faster: 13230 x 5120, 96 rows, 41 us, 45 in 64 x 128; 19052 x 1536, 40 % of
// them with 96 rows and the others with 48, 27.6 and 23.2.
enum Down { kDownFew, kDownMany, kDownTall };
Down pick_down(DownArgs &d, int32_t runs, int cus) {
    int64_t tokens = 0, passes = 0;
    for (int i = 0; i < runs; ++i) {
        if (d.run[i].rank == 0) continue;
        const int64_t n = int64_t(d.run[i + 1].start) - d.run[i].start;
        tokens += n;
        passes += n * ((d.sections * d.run[i].rank + 63) / 64);
    }
    return down_tiles<DownFew>(d, runs) <= cus ? kDownFew : 4 * passes > 7 * tokens ? kDownTall : kDownMany;
}
int run_down(DownArgs &d, int32_t runs, int dev, int cus, hipStream_t stream) {
    d.looks = 0;
    for (int i = 0; i < runs; ++i) {
        d.run[i].first_look = d.looks;
        d.looks += look_parts(int64_t(d.d_out) * d.run[i].rank / 8);
    }
    switch (pick_down(d, runs, cus)) {
        case kDownFew: return launch_down<DownFew>(d, runs, dev, stream);
        case kDownTall: return launch_down<DownTall>(d, runs, dev, stream);
        default: return launch_down<DownMany>(d, runs, dev, stream);
    }
}

// Whether a call is taken in one launch (product_few): one round of 64 x 32 tiles at most, in each of them ranks for one product of 64 rows, as many
// runs as the arguments hold; heads of 64 features (a tile's).
// us of one launch / of two: 320 x 1536 -> 1536 10.0 / 13.9, 4000 x 4096 -> 128 17.6 / 25.8, 96 x 6144 -> 5120 26.5 / 30.3, 2000 x 256 -> 256 6.4 / 9.5; in
// two rounds 400 x 1536 -> 1536 18.9 / 14.1, 1000 x 512 -> 1536 11.9 / 11.3, 6000 x 4096 -> 128 33.3 / 28.6.
bool takes_few(int64_t n, int32_t d_out, int32_t head_dim, int cus, int32_t runs, const DownRun *run) {
    if (!small_tilings(head_dim) || (n + Split64x32::kT - 1) / Split64x32::kT * ((d_out + Split64x32::kF - 1) / Split64x32::kF) > cus) return false;
    int adapters = 0, ranks = 0, tile = -1;              // ranks in the last tile so far
    for (int i = 0; i < runs; ++i) {
        if (run[i].rank == 0) continue;
        const int first = run[i].start / Split64x32::kT, last = (run[i + 1].start - 1) / Split64x32::kT;
        ranks = run[i].rank + (first == tile ? ranks : 0);
        if (ranks > kFewRanks) return false;
        if (last > first) ranks = run[i].rank;
        tile = last;
        ++adapters;
    }
    return adapters > 0 && adapters <= kFewRuns;
}
template <bool QKV, int HD>
int launch_few(const AdaptedArgs<QKV> &a, const DownArgs &d, int32_t runs, hipStream_t stream) {
    FewArgs<QKV> few{};
    static_cast<AdaptedArgs<QKV> &>(few) = a;
    int adapters = 0;
    for (int i = 0; i < runs; ++i)
        if (d.run[i].rank > 0)
            few.few[adapters++] = FewRun{d.run[i].down, d.run[i].up, d.run[i].start, d.run[i + 1].start, d.run[i].rank, d.run[i].scale};
    const int64_t tiles = (int64_t(a.n) + Split64x32::kT - 1) / Split64x32::kT * ((a.d_out + Split64x32::kF - 1) / Split64x32::kF);
    return launch_tiles<QKV, HD, Split64x32, Split64x32>(few, tiles, stream);
}

// What the calls share from here on: the workspace, the down products, the tilings.
template <bool QKV, int HD>
int project(AdaptedArgs<QKV> &a, Runs &runs, void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    const int64_t t_row = t_row_bytes(runs.largest, QKV ? 3 : 1);
    if (runs.largest > 0 && (workspace == nullptr || !aligned16(workspace) || workspace_bytes < kControlBytes + t_row * a.n)) return LP_ERR_INVALID_ARG;
    int dev = 0;
    const int cus = lp::device_compute_units(&dev);
    if (cus <= 0) return LP_ERR_HIP;
    DownArgs &d = runs.down;
    if constexpr (small_tilings(QKV ? HD : 0))
        if (takes_few(a.n, a.d_out, QKV ? HD : 0, cus, runs.runs, d.run)) return launch_few<QKV, HD>(a, d, runs.runs, stream);
    if (runs.largest > 0) {
        d.x = a.x;
        d.control = static_cast<AdapterControl *>(workspace);
        d.t = static_cast<__bf16 *>(workspace) + kControlBytes / 2;
        d.t_row = int32_t(t_row);
        d.t_blocks = (runs.largest + kRanks - 1) / kRanks;
        const int rc = run_down(d, runs.runs, dev, cus, stream);
        if (rc != LP_OK) return rc;
        a.control = d.control;
        a.t = d.t;
        a.t_row = d.t_row;
        a.t_blocks = d.t_blocks;
    }
    return launch_plan<QKV, HD>(pick_adapted(a.n, a.d_in, a.d_out, QKV ? HD : 0, cus, runs.runs, d.run), a, stream);
}

}  // namespace

extern "C" int lp_internal_adapted_call_way(const lp_requests *requests, const lp_adapter *adapters, int32_t d_in, int32_t d_out, int32_t head_dim,
                                            int32_t cus, int64_t way[8]) {
    Runs runs;
    const int rc = make_runs(requests, adapters, d_in, d_out, head_dim == 0 ? 1 : 3, &runs);
    if (rc != LP_OK) return rc;
    const int64_t n = runs.requests.rows();
    DownArgs &d = runs.down;
    if (takes_few(n, d_out, head_dim, cus, runs.runs, d.run)) {
        way[0] = Split64x32::kF;
        way[1] = Split64x32::kT;
        way[2] = way[3] = way[6] = way[7] = 0;
        way[4] = (n + Split64x32::kT - 1) / Split64x32::kT * ((d_out + Split64x32::kF - 1) / Split64x32::kF);
        way[5] = Split64x32::kThreads;
        return LP_OK;
    }
    const Plan p = pick_adapted(int32_t(n), d_in, d_out, head_dim, cus, runs.runs, d.run);
    plan_way(p, n, d_out, head_dim == 0 && four_waves(p, d_in), way);
    const Down down = pick_down(d, runs.runs, cus);
    way[6] = down == kDownFew ? DownFew::kF : down == kDownMany ? DownMany::kF : DownTall::kF;
    way[7] = down == kDownFew ? DownFew::kT : down == kDownMany ? DownMany::kT : DownTall::kT;
    return LP_OK;
}

extern "C" int lp_internal_adapted_way(const int64_t *start, const int32_t *rank, int32_t count, int32_t d_in, int32_t d_out, int32_t head_dim,
                                       int32_t cus, int64_t way[8]) {
    lp_adapter adapters[LP_MAX_REQUESTS];
    for (int r = 0; r < std::min(count, LP_MAX_REQUESTS); ++r)           // addresses that nothing reads, no two alike
        adapters[r] = lp_adapter{reinterpret_cast<const void *>(uintptr_t(32 * r + 16)), reinterpret_cast<const void *>(uintptr_t(32 * r + 32)), rank[r], 1.0f};
    const lp_requests requests{count, start};
    return lp_internal_adapted_call_way(&requests, adapters, d_in, d_out, head_dim, cus, way);
}

extern "C" int64_t lp_adapter_workspace_size(int64_t n_tokens, int32_t rank, int32_t sections) {
    if (n_tokens < 0 || rank < 0 || (sections != 1 && sections != 3)) return LP_ERR_INVALID_ARG;
    if (n_tokens >= INT32_MAX || rank > LP_MAX_ADAPTER_RANK) return LP_ERR_UNSUPPORTED;
    return n_tokens > 0 && rank > 0 ? kControlBytes + n_tokens * t_row_bytes(rank, sections) : 0;
}

extern "C" int lp_linear_adapters(const void *x, const void *w, const float *bias, void *y, const lp_requests *requests, int32_t d_in,
                                  int32_t d_out, const lp_adapter *adapters, void *workspace, int64_t workspace_bytes, void *stream) {
    Runs runs;
    int rc = make_runs(requests, adapters, d_in, d_out, 1, &runs);
    if (rc != LP_OK) return rc;
    const int64_t n = runs.requests.rows();
    if ((rc = check_gemm_shape(n, d_in, d_out)) != LP_OK) return rc;
    if (n == 0) return LP_OK;
    if (runs.largest == 0) return lp_linear(x, w, bias, y, n, d_in, d_out, stream);
    if (x == nullptr || w == nullptr || y == nullptr) return LP_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(w) || !aligned16(y) || !aligned16(bias) || y == x || y == w) return LP_ERR_INVALID_ARG;
    if (workspace == x || workspace == w || workspace == y) return LP_ERR_INVALID_ARG;
    AdaptedArgs<false> a{};
    a.x = static_cast<const __bf16 *>(x);
    a.w = static_cast<const __bf16 *>(w);
    a.bias = bias;
    a.out[0] = static_cast<__bf16 *>(y);
    a.n = int32_t(n);
    a.d_in = d_in;
    a.d_out = d_out;
    return project<false, 128>(a, runs, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int lp_qkv_projection_adapters(const void *x, const void *w_qkv, const float *bias, const float *gain_q, const float *gain_k,
                                          float eps, const lp_rope *ropes, void *q, void *k, void *v, const lp_requests *requests,
                                          int32_t heads, int32_t head_dim, const lp_adapter *adapters, void *workspace,
                                          int64_t workspace_bytes, void *stream) {
    if (heads < 1) return LP_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return LP_ERR_UNSUPPORTED;
    const int64_t dm64 = int64_t(heads) * head_dim;
    if (3 * dm64 >= (int64_t(1) << 31)) return LP_ERR_UNSUPPORTED;
    const int32_t dm = int32_t(dm64);
    if (dm % 128 != 0) return LP_ERR_UNSUPPORTED;
    Runs runs;
    int rc = make_runs(requests, adapters, dm, 3 * dm, 3, &runs);
    if (rc != LP_OK) return rc;
    const int64_t n = runs.requests.rows();
    if ((rc = check_gemm_shape(n, dm, 3 * dm)) != LP_OK) return rc;
    if (n == 0) return LP_OK;
    if (x == nullptr || w_qkv == nullptr || gain_q == nullptr || gain_k == nullptr || q == nullptr || k == nullptr || v == nullptr ||
        ropes == nullptr)
        return LP_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(w_qkv) || !aligned16(bias) || !aligned16(gain_q) || !aligned16(gain_k) || !aligned16(q) ||
        !aligned16(k) || !aligned16(v))
        return LP_ERR_INVALID_ARG;
    if (q == k || q == v || k == v || q == x || k == x || v == x) return LP_ERR_INVALID_ARG;
    if (runs.largest > 0 && (workspace == x || workspace == w_qkv || workspace == q || workspace == k || workspace == v)) return LP_ERR_INVALID_ARG;
    AdaptedArgs<true> a{};
    a.requests = runs.requests.count;
    int first = -1;
    for (int r = 0; r < a.requests; ++r) {
        const int32_t start = runs.requests.start[r], rows = runs.requests.start[r + 1] - start;
        a.grid[r] = RequestGrid{start, 1, 1, {0, 0, 0}};
        if (rows == 0) continue;
        if (first < 0) {
            first = r;
            if ((rc = make_rope_args(&ropes[r], rows, head_dim, eps, &a.rope)) != LP_OK) return rc;
        }
        const lp_rope &o = ropes[r];
        if ((rc = check_rope(&o, rows, head_dim, eps)) != LP_OK) return rc;
        if (o.base != ropes[first].base) return LP_ERR_INVALID_ARG;
        for (int ax = 0; ax < 3; ++ax)
            if (o.split[ax] != ropes[first].split[ax]) return LP_ERR_INVALID_ARG;
        a.grid[r] = RequestGrid{start, o.grid[1] * o.grid[2], o.grid[2], {o.offset[0], o.offset[1], o.offset[2]}};
    }
    a.x = static_cast<const __bf16 *>(x);
    a.w = static_cast<const __bf16 *>(w_qkv);
    a.bias = bias;
    a.out[0] = static_cast<__bf16 *>(q);
    a.out[1] = static_cast<__bf16 *>(k);
    a.out[2] = static_cast<__bf16 *>(v);
    a.gain[0] = gain_q;
    a.gain[1] = gain_k;
    a.n = int32_t(n);
    a.d_in = dm;
    a.d_out = 3 * dm;
    a.heads = heads;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return head_dim == 128 ? project<true, 128>(a, runs, workspace, workspace_bytes, st)
                           : project<true, 64>(a, runs, workspace, workspace_bytes, st);
}
