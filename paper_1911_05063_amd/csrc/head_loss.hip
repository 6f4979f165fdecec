// Log-probabilities and entropy of given tokens straight from hidden states h [T, D] and the
// vocabulary matrix w [V, D] (16-bit), without the logits x = h w^T in memory.
//
// Forward: the product's tiles stay in registers; each gives its rows' (maximum, sum, sum of
// w t) over its columns (token_common.h) and the given token's logit, and a second kernel
// joins a row's parts.  2 T D V operations; the parts are 12 bytes per row and tile.
//
// Backward: with dx = d/dx of token_loss.hip,
//     d/dh = dx w,   d/dw = dx^T h.
// The logits are computed again (the same products; over few rows in another order), so 6 T D V
// operations become 8.  dx is rounded to the operands' type for the matrix cores, like the
// operands themselves; in float16 it is scaled by a power of 2 first, so that the largest possible
// element is about 2^14 and small ones do not vanish.  The rounding adds as much to the results'
// error as their own rounding does (relative: 0.0024 instead of 0.0017 in bfloat16, 3.0e-4 instead
// of 2.1e-4 in float16).  Over few rows the errors do not average: up to kSplitRows rows, dx is
// held as a rounded part and a second row with the rest, which both go through the products.  It
// is held for a range of the vocabulary at a time (kChunkBytes): d/dw of the range is finished
// with it, d/dh is summed over ranges, and over parts of a long sum where few tiles would leave
// CUs idle, in float32 and in a fixed order.
//
// Bound by the matrix cores' clock under load and the tiles' ends.  8192 rows of 2048 against
// 65536, bfloat16, 2.2e12 operations a product (TFLOP/s): stats_kernel 1285, dx_kernel 1165,
// mul_kernel 1390 (d/dh) and 1210 (d/dw), 7.1 ms in all, where a plain library product reaches
// 1320; the matrix cores are busy in 63, 55, 63 and 57% of all cycles.  16 rows of 2048 against
// 65536 are the weights' 268 MB in 53 us, 5.1 TB/s.
#include <algorithm>
#include <type_traits>

#include "cd_internal.h"
#include "tile_product.h"
#include "token_common.h"

namespace cdk {
namespace {

constexpr int kRowThreads = 256;
constexpr int kBig = 256, kSmall = 128;         // tiles: 8 waves (2 x 4), 4 waves (2 x 2)
// Fewer large tiles than this leave too many of the 256 CUs without one (us, large -> small tiles,
// forward: 128 large tiles 2048 x 1024 against 4096 34 -> 25, 160 against 5120 even, but 192 2048
// x 2048 against 6144 54 -> 58, 256 against 8192 59 -> 66).  Large tiles read less from LDS for
// each product: 12 fragments for 32 products instead of 8 for 16.
constexpr int64_t kFewTiles = 160;
constexpr unsigned kCus = 256;                  // a workgroup of a large tile each
constexpr int64_t kWantTiles = 512;             // small tiles wanted, two for each CU
constexpr int64_t kPartK = 512;                 // k of a part of a sum, at least
// What dx takes at a time: two ranges for 8192 x 65536 (one of 1 GB is no faster), and still wide
// enough for full products.
constexpr int64_t kChunkBytes = int64_t(512) << 20;
// Rows that are split.  Up to here the weights' 2 D V elements are most of the work: 40 rows of
// 2048 against 40000 take 224 us instead of 201.
constexpr int64_t kSplitRows = 256;
// A product of so few k is bound by its result, which is written past the caches where they would
// not keep it (gradients of 16 rows of 2048 against 100000 345 -> 292 us, of 100 rows, k = 200,
// 496 -> 462; 200 rows of 1024 against 65536, k = 400, are even, 1000 rows of 1000 against 50000
// lose: 424 -> 441).  Up to 128 MB it may be read from the caches next (gradient of 16 rows of
// 1024 against 65536 106 us in the caches and 109 past them, of 100 rows of 2048 against 16384 113
// and 115; the update that reads them next is even).
constexpr int64_t kStreamK = 256;

// Rows of a workgroup that looks for the scale of float16, and the most workgroups (131072 rows 12
// us in two launches, by one workgroup 110; 3001 rows 3 us by one).
constexpr int64_t kScaleRows = 4096;
constexpr int kScaleParts = 62;

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
size_t up256(size_t a) { return (a + 255) / 256 * 256; }

template <int kTile>
struct Waves {
    static constexpr int kM = 2, kN = kTile == kBig ? 4 : 2;
};
// How the weights of all rows' one row of tiles are read.
enum FewRows { kMany, kFewRows, kFewRowsOnce };
template <typename E, int kTile, bool kAcrossA, bool kAcrossB, FewRows kFew = kMany>
using Product = TileProduct<E, kTile, kTile, Waves<kTile>::kM, Waves<kTile>::kN, kAcrossA, kAcrossB,
                            kFew != kMany, kFew == kFewRowsOnce>;

// Rows of 16-bit elements into rows of ld_out, zeros behind the first D and in rows without
// a token; all rows `copies` times.
template <typename E>
__global__ __launch_bounds__(kRowThreads) void pack_kernel(const E *in, int64_t sb, int64_t st,
                                                           uint32_t T, int64_t rows, int copies,
                                                           int32_t D, const int32_t *tokens, E *out,
                                                           int32_t ld_out)
{
    const int32_t chunks = ld_out / 8;
    const int64_t n = rows * copies * chunks;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kRowThreads) {
        const int64_t to = i / chunks, row = to % rows;
        const int32_t c = static_cast<int32_t>(i - to * chunks) * 8;
        const uint32_t b = static_cast<uint32_t>(row) / T;
        const E *src = in + b * sb + (static_cast<uint32_t>(row) - b * T) * st;
        const bool used = !tokens || tokens[row] >= 0;
        typename Half<E>::v8 v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = static_cast<E>(used && c + j < D ? src[c + j] : E(0));
        *reinterpret_cast<typename Half<E>::v8 *>(out + to * ld_out + c) = v;
    }
}

// ---- forward

struct StatsArgs {
    int32_t T, V;
    uint32_t tiles_m, tiles_n;
    int64_t D;
    float c;
    const int32_t *tokens;
    Softmax *parts;     // [T, tiles_n]
    float *given;       // [T] logit of the given token
};

// Workgroups of large tiles, one for each CU, go on to further tiles: these begin to load before
// the statistics of the last are formed (16384 x 1024 against 16384 477 -> 463 us, the step of
// 3001 x 1000 against 10007 in float16 323 -> 316 us).
template <typename E, int kTile, FewRows kFew>
__global__ __launch_bounds__(Waves<kTile>::kM *Waves<kTile>::kN * 64, 2) void stats_kernel(
    Operand<E> h, Operand<E> w, StatsArgs a)
{
    typedef Product<E, kTile, false, false, kFew> P;
    constexpr int kParts = Waves<kTile>::kN;        // of a row within the tile
    __shared__ __attribute__((aligned(1024))) char lds_a[P::A::kBuffers * P::A::kBytes],
        lds_b[P::B::kBuffers * P::B::kBytes];
    __shared__ float meet[3 * kParts * kTile];                          // [m, s, e][kParts][kTile]
    __shared__ int32_t tokens[kTile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Waves<kTile>::kN * P::kWaveM, wn = wave % Waves<kTile>::kN * P::kWaveN;
    const uint32_t tiles = a.tiles_m * a.tiles_n;
    uint32_t tm, tn;
    int32_t token;      // of row threadIdx.x
    typename P::Loads loads;
    const auto begin = [&](uint32_t tile) {
        tile_of(tile, a.tiles_m, a.tiles_n, &tm, &tn);
        const int64_t row = static_cast<int64_t>(tm) * kTile + threadIdx.x;
        token = threadIdx.x < kTile && row < a.T ? a.tokens[row] : -1;
        P::begin(loads, h, w, static_cast<int64_t>(tm) * kTile, static_cast<int64_t>(tn) * kTile, 0,
                 a.D, lds_a, lds_b, tn);
    };
    begin(blockIdx.x);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t m0 = static_cast<int64_t>(tm) * kTile;
        const uint32_t column = tn;
        const int first = static_cast<int>(tn * kTile) + wn + (lane >> 4) * 4;  // of this lane
        const bool edge = static_cast<int64_t>(tn + 1) * kTile > a.V;
        f32x4 acc[P::kM][P::kN];
        P::finish(loads, lds_a, lds_b, acc);
        if (threadIdx.x < kTile) tokens[threadIdx.x] = token;
        __syncthreads();
        // The next tile's first loads arrive during this one's statistics.
        if (tile + gridDim.x < tiles) begin(tile + gridDim.x);
        auto rows = [&](auto edge) {
#pragma unroll
            for (int i = 0; i < P::kM; ++i) {
                const int at = wm + i * 16 + (lane & 15);
                float x[P::kN * 4];
                float bm = -INFINITY;
#pragma unroll
                for (int j = 0; j < P::kN; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v = acc[i][j][r];
                        if (edge && first + j * 16 + r >= a.V) v = -INFINITY;
                        x[j * 4 + r] = v;
                        bm = fmaxf(bm, v);
                    }
                // (The four lanes of a row take one maximum, so that their sums are only added.)
                Softmax s = softmax_empty();
                softmax_add<edge>(s, x, rows_max(bm), a.c);
                s.s = rows_sum(s.s);
                s.e = rows_sum(s.e);
                if (lane < 16) {
                    float *to = meet + wn / P::kWaveN * kTile + at;
                    to[0] = s.m;
                    to[kParts * kTile] = s.s;
                    to[2 * kParts * kTile] = s.e;
                }
                // The lane that holds the given token's logit keeps it.
                const int off = tokens[at] - first;
                if (off >= 0 && off < P::kWaveN && (off & 12) == 0) {
                    float v = 0.0f;
#pragma unroll
                    for (int j = 0; j < P::kN; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) v = off == j * 16 + r ? acc[i][j][r] : v;
                    a.given[m0 + at] = v;
                }
            }
        };
        if (edge) rows(std::true_type{});
        else rows(std::false_type{});
        __syncthreads();
        if (threadIdx.x < kTile && m0 + threadIdx.x < a.T) {
            const auto part = [&](int i) {
                const float *from = meet + i * kTile + threadIdx.x;
                return Softmax{from[0], from[kParts * kTile], from[2 * kParts * kTile]};
            };
            Softmax r = part(0);
#pragma unroll
            for (int i = 1; i < kParts; ++i) {
                Softmax s = part(i);
                const float m = fmaxf(r.m, s.m);
                softmax_rescale(r, m, a.c);
                softmax_rescale(s, m, a.c);
                r.s += s.s;
                r.e += s.e;
            }
            a.parts[(m0 + threadIdx.x) * a.tiles_n + column] = r;
        }
    }
}

// Joins a row's parts; a wave per row.
__global__ __launch_bounds__(kRowThreads) void finish_kernel(int32_t T, int32_t V, uint32_t nparts,
                                                             float c, const int32_t *tokens,
                                                             const Softmax *parts,
                                                             const float *given, float *logprob,
                                                             float *entropy, ScoreRow *saved)
{
    const int lane = threadIdx.x & 63;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * (kRowThreads / 64) + threadIdx.x / 64; row < T;
         row += static_cast<int64_t>(gridDim.x) * (kRowThreads / 64)) {
        const int32_t t = tokens[row];
        float lp = 0.0f, h2 = 0.0f, l2s = 0.0f, m = -INFINITY;
        if (t >= 0) {
            Softmax r = softmax_empty();
            for (uint32_t i = lane; i < nparts; i += 64) {
                Softmax s = parts[row * nparts + i];
                const float bm = fmaxf(r.m, s.m);
                softmax_rescale(r, bm, c);
                softmax_rescale(s, bm, c);
                r.s += s.s;
                r.e += s.e;
            }
            softmax_group<64>(r, c);
            const bool empty = r.s == 0.0f;
            l2s = empty ? 0.0f : log2f(r.s);
            h2 = empty ? 0.0f : l2s - r.e / r.s;
            m = empty ? -INFINITY : softmax_ref(r.m);
            if (t >= V) lp = __builtin_nanf("");
            else lp = empty ? -INFINITY : ((given[row] - r.m) * c - l2s) * kTokLn2;
        }
        if (lane == 0) {
            logprob[row] = lp;
            entropy[row] = h2 * kTokLn2;
            if (saved) saved[row] = {m, l2s, h2, 0};
        }
    }
}

// ---- backward

// dx = w (gp + gh t), w = 2^t, and gt more at the token.  t = fma(x, c, -R), or (x - m) c where
// |R| is at least kFarExponent; R = +inf and m = +inf where the gradient is 0.
struct HeadRow {
    float m, R, gp, gh;
    float gt;
    int32_t token;
    int32_t rest;   // 1: the row holds what rounding leaves of dx
    int32_t pad;
};

// The power of 2 that takes the largest possible |dx|, `most`, to about 2^14 (float16).
__device__ __forceinline__ void set_scale(float most, float *scale)
{
    int e = 0;
    if (most > 0.0f) e = 14 - ilogbf(most);
    e = e > 100 ? 100 : e < -100 ? -100 : e;
    scale[0] = ldexpf(1.0f, e);
    scale[1] = ldexpf(1.0f, -e);
}

// That of all rows by one workgroup, or (several) the largest possible |dx| of each workgroup's.
// Rows count as head_rows_kernel takes them: one without a token or a gradient may come with any
// g. Nor do rows count whose g is not finite: their d/d hidden is not at any scale, the other
// rows' is.
__global__ __launch_bounds__(1024) void scale_kernel(int32_t T, int32_t V, float lnv,
                                                     float inv_temperature, const int32_t *tokens,
                                                     const ScoreRow *saved, const float *g_logprob,
                                                     const float *g_entropy, float *parts,
                                                     float *scale)
{
    __shared__ float part[16];
    float most = 0.0f;
    for (int64_t i = blockIdx.x * 1024 + threadIdx.x; i < T; i += gridDim.x * 1024) {
        // (all asked for at once, used or not)
        const int32_t t = tokens[i];
        const float m = saved[i].m;
        const float gl = g_logprob ? fabsf(g_logprob[i]) : 0.0f;
        const float ge = g_entropy ? fabsf(g_entropy[i]) : 0.0f;
        const float g = ((t < V ? gl : 0.0f) + ge * (lnv + 1.0f)) * inv_temperature;
        if (t >= 0 && m != -INFINITY && g < INFINITY) most = fmaxf(most, g);
    }
    most = group_max<64>(most);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int i = 1; i < 16; ++i) most = fmaxf(most, part[i]);
    if (gridDim.x == 1) set_scale(most, scale);
    else parts[blockIdx.x] = most;
}
__global__ __launch_bounds__(64) void join_scale_kernel(int n, const float *parts, float *scale)
{
    const float most = group_max<64>(static_cast<int>(threadIdx.x) < n ? parts[threadIdx.x] : 0.0f);
    if (threadIdx.x == 0) set_scale(most, scale);
}

__global__ __launch_bounds__(kRowThreads) void head_rows_kernel(
    int32_t T, int copies, int64_t rows, int32_t V, float temperature, const int32_t *tokens,
    const ScoreRow *saved, const float *g_logprob, const float *g_entropy, const float *scale,
    HeadRow *out)
{
    const int64_t to = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x;
    if (to >= rows) return;
    const int32_t rest = to >= T, row = static_cast<int32_t>(to % T);
    HeadRow r{INFINITY, INFINITY, 0.0f, 0.0f, 0.0f, -1, 0, 0};
    if (to < static_cast<int64_t>(copies) * T) {
        const ScoreRow s = saved[row];
        const int32_t t = tokens[row];
        if (t >= 0 && s.m != -INFINITY) {
            const float k = scale ? scale[0] : 1.0f, inv_temperature = 1.0f / temperature;
            const float gl = g_logprob && t < V ? g_logprob[row] * inv_temperature * k : 0.0f;
            const float he = g_entropy ? g_entropy[row] * inv_temperature * k : 0.0f;
            const float c = kTokLog2e / temperature, R = s.m * c;
            // By which t is off: log2 p = t - d - l2s.
            const float d = fabsf(R) < kFarExponent ? __builtin_fmaf(s.m, c, -R) : 0.0f;
            const float p = tok_exp2(-s.l2s - d), h = -he * kTokLn2 * p;
            r = {s.m, R, __builtin_fmaf(h, s.h2 - s.l2s - d, -gl * p), h, gl, t < V ? t : -1,
                 rest, 0};
        }
    }
    out[to] = r;
}

struct DxArgs {
    int32_t V;
    uint32_t tiles_m, tiles_n;
    int64_t D, v0;
    float c;
    bool split;             // some rows hold the rest
    const HeadRow *rows;    // [tiles_m * kTile]
    void *dx;               // [tiles_m * kTile, ld]
    int64_t ld;
};

template <typename E, int kTile, FewRows kFew>
__global__ __launch_bounds__(Waves<kTile>::kM *Waves<kTile>::kN * 64, 2) void dx_kernel(Operand<E> h,
                                                                                       Operand<E> w,
                                                                                       DxArgs a)
{
    typedef Product<E, kTile, false, false, kFew> P;
    __shared__ __attribute__((aligned(1024))) char lds_a[P::A::kBuffers * P::A::kBytes],
        lds_b[P::B::kBuffers * P::B::kBytes];
    uint32_t tm, tn;
    tile_of(blockIdx.x, a.tiles_m, a.tiles_n, &tm, &tn);
    const int64_t m0 = static_cast<int64_t>(tm) * kTile, n0 = static_cast<int64_t>(tn) * kTile;
    f32x4 acc[P::kM][P::kN];
    P::run(h, w, m0, n0, 0, a.D, lds_a, lds_b, acc, tn);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Waves<kTile>::kN * P::kWaveM, wn = wave % Waves<kTile>::kN * P::kWaveN;
    const int first = static_cast<int>(a.v0 + n0) + wn + (lane >> 4) * 4;
    char *out = P::out_lds(lds_a, lds_b);
    __syncthreads();
    const bool edge = a.v0 + n0 + kTile > a.V;
    auto rows = [&](auto edge) {
#pragma unroll
        for (int i = 0; i < P::kM; ++i) {
            const int64_t row = m0 + wm + i * 16 + (lane & 15);
            const HeadRow p = a.rows[row];
            float d[P::kN * 4];
            float R = p.R;
            if (__builtin_expect(!(fabsf(R) < kFarExponent), 0)) {
#pragma unroll
                for (int j = 0; j < P::kN; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] -= p.m;
                R = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < P::kN * 4; ++j) {
                const float t = __builtin_fmaf(acc[i][j / 4][j % 4], a.c, -R);
                d[j] = tok_exp2(t) * __builtin_fmaf(p.gh, fmaxf(t, -200.0f), p.gp);
            }
            const int off = p.token - first;
            if (off >= 0 && off < P::kWaveN && (off & 12) == 0) {
#pragma unroll
                for (int j = 0; j < P::kN * 4; ++j) d[j] += off == j / 4 * 16 + j % 4 ? p.gt : 0.0f;
            }
            if (a.split) {
#pragma unroll
                for (int j = 0; j < P::kN * 4; ++j)
                    d[j] -= p.rest ? static_cast<float>(static_cast<E>(d[j])) : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < P::kN; ++j) {
                typename Half<E>::v4 v;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (edge && first + j * 16 + r >= a.V) d[j * 4 + r] = 0.0f;
                    v[r] = static_cast<E>(d[j * 4 + r]);
                }
                P::out_put(out, i, j, v);
            }
        }
    };
    if (edge) rows(std::true_type{});
    else rows(std::false_type{});
    wave_fence();
    E *dx = static_cast<E *>(a.dx) + (m0 + wm + (lane >> 3)) * a.ld + n0 + wn + (lane & 7) * 8;
#pragma unroll
    for (int t = 0; t < P::kWaveM / 8; ++t)
        *reinterpret_cast<typename Half<E>::v8 *>(dx + t * 8 * a.ld) = P::out_get(out, t);
}

struct MulArgs {
    int64_t M, N;           // extents that are written
    int64_t K, part_k;      // part z sums k in [z part_k, (z + 1) part_k)
    uint32_t tiles_m, tiles_n;
    void *out;              // [M, ld] 16-bit, or null
    int64_t ld;
    bool stream;            // `out` is written past the caches
    const float *scale;     // scale[1] multiplies what is written to `out`, or null
    float *part;            // [parts, M, N] float32
};

template <typename E, int kTile, bool kAcrossA>
__global__ __launch_bounds__(Waves<kTile>::kM *Waves<kTile>::kN * 64, 2) void mul_kernel(Operand<E> x,
                                                                                        Operand<E> y,
                                                                                        MulArgs a)
{
    typedef Product<E, kTile, kAcrossA, true> P;
    __shared__ __attribute__((aligned(1024))) char lds_a[P::A::kBuffers * P::A::kBytes],
        lds_b[P::B::kBuffers * P::B::kBytes];
    uint32_t tm, tn;
    tile_of(blockIdx.x, a.tiles_m, a.tiles_n, &tm, &tn);
    const int64_t m0 = static_cast<int64_t>(tm) * kTile, n0 = static_cast<int64_t>(tn) * kTile;
    const int64_t k0 = blockIdx.y * a.part_k, k1 = min(a.K, k0 + a.part_k);
    f32x4 acc[P::kM][P::kN];
    P::run(x, y, m0, n0, k0, k1, lds_a, lds_b, acc);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Waves<kTile>::kN * P::kWaveM, wn = wave % Waves<kTile>::kN * P::kWaveN;
    if (a.out) {
        const float k = a.scale ? a.scale[1] : 1.0f;
        char *out = P::out_lds(lds_a, lds_b);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < P::kM; ++i)
#pragma unroll
            for (int j = 0; j < P::kN; ++j) {
                typename Half<E>::v4 v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = static_cast<E>(acc[i][j][r] * k);
                P::out_put(out, i, j, v);
            }
        wave_fence();
        const int64_t col = n0 + wn + (lane & 7) * 8;
        const bool whole = a.N % 8 == 0;    // then rows start at multiples of 8 elements
        const auto store = [&](auto past) {
#pragma unroll
            for (int t = 0; t < P::kWaveM / 8; ++t) {
                const int64_t row = m0 + wm + t * 8 + (lane >> 3);
                const typename Half<E>::v8 v = P::out_get(out, t);
                E *to = static_cast<E *>(a.out) + row * a.ld + col;
                if (row >= a.M) continue;
                if (whole && col < a.N) {
                    if constexpr (decltype(past)::value)
                        __builtin_nontemporal_store(v, reinterpret_cast<typename Half<E>::v8 *>(to));
                    else
                        *reinterpret_cast<typename Half<E>::v8 *>(to) = v;
                } else {
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        if (col + r < a.N) to[r] = v[r];
                }
            }
        };
        // (Two loops: were they one, the compiler would make the two kinds of stores one.)
        if (a.stream) store(std::true_type{});
        else store(std::false_type{});
        return;
    }
    const bool whole = a.N % 4 == 0;        // then rows start at multiples of 4 elements
#pragma unroll
    for (int i = 0; i < P::kM; ++i) {
        const int64_t row = m0 + wm + i * 16 + (lane & 15);
        if (row >= a.M) continue;
#pragma unroll
        for (int j = 0; j < P::kN; ++j) {
            const int64_t col = n0 + wn + j * 16 + (lane >> 4) * 4;
            float *out = a.part + (blockIdx.y * a.M + row) * a.N + col;
            if (whole && col < a.N) {
                *reinterpret_cast<f32x4 *>(out) = acc[i][j];
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (col + r < a.N) out[r] = acc[i][j][r];
            }
        }
    }
}

// sum = (carry ? sum : 0) + the parts in order, each of `copies` times n; written to `out` if
// given, else kept.
template <typename E>
__global__ __launch_bounds__(kRowThreads) void sum_kernel(int64_t n, int copies, int parts,
                                                          const float *part, float *sum, bool carry,
                                                          E *out, const float *scale)
{
    const float k = scale ? scale[1] : 1.0f;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x; i < n;
         i += static_cast<int64_t>(gridDim.x) * kRowThreads) {
        float s = carry ? sum[i] : 0.0f;
        int p = 0;
        for (; p + 16 <= parts * copies; p += 16) {     // (asked for together, added in order)
            float v[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = part[(p + q) * n + i];
#pragma unroll
            for (int q = 0; q < 16; ++q) s += v[q];
        }
        for (; p < parts * copies; ++p) s += part[p * n + i];
        if (out) out[i] = static_cast<E>(s * k);
        else sum[i] = s;
    }
}

// ---- plans

struct MulPlan {
    bool big;
    uint32_t tiles_m, tiles_n;
    int parts;
    int64_t part_k;
};

MulPlan plan_mul(int64_t M, int64_t N, int64_t K)
{
    MulPlan p{};
    // (With up to 128 rows half of a large tile would be idle.)
    p.big = std::min(M, N) > kSmall && (up(M, kBig) / kBig) * (up(N, kBig) / kBig) >= kFewTiles;
    const int64_t tile = p.big ? kBig : kSmall;
    p.tiles_m = static_cast<uint32_t>(up(M, tile) / tile);
    p.tiles_n = static_cast<uint32_t>(up(N, tile) / tile);
    int64_t parts = 1;
    if (!p.big) {
        const int64_t tiles = static_cast<int64_t>(p.tiles_m) * p.tiles_n;
        parts = std::max<int64_t>(1, std::min(kWantTiles / tiles, K / kPartK));
    }
    p.part_k = up((K + parts - 1) / parts, kStepK);
    p.parts = static_cast<int>((K + p.part_k - 1) / p.part_k);
    return p;
}

bool stream_out(int64_t M, int64_t N, int64_t K)
{
    return K <= kStreamK && M * N * 2 > kCacheBytes / 2;
}

bool pack_hidden(const Head &x)
{
    return x.D % kStepK != 0 || x.stride_t % 8 != 0 || x.stride_t > kMostLd ||
           (x.B > 1 && x.stride_b != x.T * x.stride_t);
}
bool pack_weight(const Head &x)
{
    return x.D % 8 != 0 || x.ld_weight % 8 != 0 || x.ld_weight > kMostLd;
}

// Rows of dx with those that are filled up with zeros.
int64_t dx_rows(int64_t n) { return n <= kSmall ? kSmall : up(n, kBig); }

// Where one row of tiles takes all rows, the weights come from memory and not from the L2, and
// all workgroups at once: each starts at another k, or all would ask for the same few hundred
// bytes of every 4 KB row, which few of the memory's channels hold.  (16 rows of 2048 against
// 65536, cold: 71 -> 59 us.)  Weights that the last cache does not keep go past the caches: these
// 62.7 -> 57.2 us, against 100000 93 -> 87.5; 128 MB, 65536 of 1024, rather stay: 36 against 38.8.
FewRows few_rows(int64_t tiles_m, const Head &x)
{
    if (tiles_m != 1 || x.D % kStepK != 0) return kMany;
    return x.V * x.D * 2 > kCacheBytes / 2 ? kFewRowsOnce : kFewRows;
}

// Calls f with one of these as a constant.
template <typename F>
void with_few_rows(FewRows few, F &&f)
{
    if (few == kFewRowsOnce) f(std::integral_constant<FewRows, kFewRowsOnce>{});
    else if (few == kFewRows) f(std::integral_constant<FewRows, kFewRows>{});
    else f(std::integral_constant<FewRows, kMany>{});
}

// Byte offsets into the workspace.
struct HeadLayout {
    int64_t rows;               // B * T
    int copies;                 // rows of dx for each: 2 where it is split
    size_t hidden, weight, parts, given, scale, head_rows, dx, mul, sum, total;
    bool pack_h, pack_w;
    bool big;                   // tile of the logits
    uint32_t tiles_m, tiles_n;  // of the whole vocabulary (forward)
    int64_t chunk;              // columns of dx
};

HeadLayout layout_of(const Head &x, bool backward)
{
    HeadLayout l{};
    l.rows = x.B * x.T;
    l.copies = backward && l.rows <= kSplitRows ? 2 : 1;
    l.pack_h = backward || pack_hidden(x);
    l.pack_w = pack_weight(x);
    size_t at = 0;
    auto take = [&at](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    l.hidden = take(l.pack_h ? static_cast<size_t>(l.rows) * l.copies * up(x.D, kStepK) * 2 : 0);
    l.weight = take(l.pack_w ? static_cast<size_t>(x.V) * up(x.D, 8) * 2 : 0);
    const MulPlan p = plan_mul(l.rows, x.V, 1);
    l.big = p.big;
    l.tiles_m = p.tiles_m;
    l.tiles_n = p.tiles_n;
    if (!backward) {
        l.parts = take(static_cast<size_t>(l.rows) * l.tiles_n * sizeof(Softmax));
        l.given = take(static_cast<size_t>(l.rows) * sizeof(float));
        l.total = at;
        return l;
    }
    const int64_t all = l.rows * l.copies, rows = dx_rows(all);
    const int64_t most = std::max<int64_t>(kChunkBytes / (rows * 2), 1024);
    l.chunk = std::min(up(x.V, kBig), most / kBig * kBig);
    l.scale = take((2 + kScaleParts) * sizeof(float));
    l.head_rows = take(static_cast<size_t>(rows) * sizeof(HeadRow));
    l.dx = take(static_cast<size_t>(rows) * l.chunk * 2);
    // Parts of d/dh and of d/dw share their place: one is summed up before the other starts.
    const bool chunks = l.chunk < x.V;
    size_t mul = 0;
    // All ranges but the last are alike.
    for (const int64_t cols : {std::min(l.chunk, x.V), x.V - (x.V - 1) / l.chunk * l.chunk}) {
        const MulPlan ph = plan_mul(all, x.D, up(cols, kStepK)), pw = plan_mul(cols, x.D, all);
        if (ph.parts > 1 || chunks || l.copies > 1)
            mul = std::max(mul, static_cast<size_t>(ph.parts) * all * x.D * sizeof(float));
        if (pw.parts > 1)
            mul = std::max(mul, static_cast<size_t>(pw.parts) * cols * x.D * sizeof(float));
    }
    l.mul = take(mul);
    l.sum = take(chunks ? static_cast<size_t>(l.rows) * x.D * sizeof(float) : 0);
    l.total = at;
    return l;
}

template <typename T>
T *at(void *ws, size_t offset)
{
    return reinterpret_cast<T *>(static_cast<char *>(ws) + offset);
}

template <typename E>
void operands(const Head &x, const HeadLayout &l, const int32_t *tokens, void *ws, Operand<E> *h,
              Operand<E> *w, hipStream_t stream)
{
    const auto grid = [](int64_t n) {
        return static_cast<unsigned>(std::min<int64_t>((n + kRowThreads - 1) / kRowThreads, 1 << 16));
    };
    *h = {static_cast<const E *>(x.hidden), x.B > 1 || x.T > 1 ? x.stride_t : x.D,
          static_cast<int32_t>(l.rows), static_cast<int32_t>(x.D)};
    if (l.pack_h) {
        const int32_t ld = static_cast<int32_t>(up(x.D, kStepK));
        pack_kernel<E><<<grid(l.rows * l.copies * ld / 8), kRowThreads, 0, stream>>>(
            h->data, x.stride_b, x.stride_t, static_cast<uint32_t>(x.T), l.rows, l.copies,
            static_cast<int32_t>(x.D), tokens, at<E>(ws, l.hidden), ld);
        *h = {at<E>(ws, l.hidden), ld, static_cast<int32_t>(l.rows * l.copies), ld};
    }
    *w = {static_cast<const E *>(x.weight), x.ld_weight, static_cast<int32_t>(x.V),
          static_cast<int32_t>(x.D)};
    if (l.pack_w) {
        const int32_t ld = static_cast<int32_t>(up(x.D, 8));
        pack_kernel<E><<<grid(x.V * ld / 8), kRowThreads, 0, stream>>>(
            w->data, 0, x.ld_weight, static_cast<uint32_t>(x.V), x.V, 1, static_cast<int32_t>(x.D),
            nullptr, at<E>(ws, l.weight), ld);
        *w = {at<E>(ws, l.weight), ld, static_cast<int32_t>(x.V), ld};
    }
}

template <typename E>
hipError_t forward(const Head &x, const int32_t *tokens, float temperature, float *logprob,
                   float *entropy, ScoreRow *saved, void *ws, hipStream_t stream)
{
    const HeadLayout l = layout_of(x, false);
    Operand<E> h, w;
    operands(x, l, tokens, ws, &h, &w, stream);
    const StatsArgs a{static_cast<int32_t>(l.rows), static_cast<int32_t>(x.V), l.tiles_m, l.tiles_n,
                      x.D, kTokLog2e / temperature, tokens, at<Softmax>(ws, l.parts),
                      at<float>(ws, l.given)};
    const unsigned tiles = l.tiles_m * l.tiles_n;
    if (l.big)
        stats_kernel<E, kBig, kMany><<<std::min(tiles, kCus), 512, 0, stream>>>(h, w, a);
    else
        with_few_rows(few_rows(l.tiles_m, x), [&](auto few) {
            stats_kernel<E, kSmall, decltype(few)::value><<<tiles, 256, 0, stream>>>(h, w, a);
        });
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(up(l.rows, 4) / 4, 1 << 16));
    finish_kernel<<<grid, kRowThreads, 0, stream>>>(a.T, a.V, l.tiles_n, a.c, tokens, a.parts, a.given,
                                                    logprob, entropy, saved);
    return hipGetLastError();
}

template <typename E, bool kAcrossA>
void multiply(const Operand<E> &x, const Operand<E> &y, const MulPlan &p, const MulArgs &a,
              hipStream_t stream)
{
    const dim3 grid(p.tiles_m * p.tiles_n, p.parts);
    if (p.big) mul_kernel<E, kBig, kAcrossA><<<grid, 512, 0, stream>>>(x, y, a);
    else mul_kernel<E, kSmall, kAcrossA><<<grid, 256, 0, stream>>>(x, y, a);
}

template <typename E>
void add_parts(int64_t n, int copies, int parts, const float *part, float *sum, bool carry, E *out,
               const float *scale, hipStream_t stream)
{
    const unsigned grid =
        static_cast<unsigned>(std::min<int64_t>((n + kRowThreads - 1) / kRowThreads, 1 << 16));
    sum_kernel<E><<<grid, kRowThreads, 0, stream>>>(n, copies, parts, part, sum, carry, out, scale);
}

template <typename E>
hipError_t backward(const Head &x, const int32_t *tokens, float temperature, const ScoreRow *saved,
                    const float *g_logprob, const float *g_entropy, E *g_hidden, E *g_weight,
                    void *ws, hipStream_t stream)
{
    const HeadLayout l = layout_of(x, true);
    Operand<E> h, w;
    operands(x, l, tokens, ws, &h, &w, stream);
    const int64_t all = l.rows * l.copies, rows = dx_rows(all);
    const float inv = 1.0f / temperature;
    float *scale = nullptr;
    if (x.dtype == CD_F16) {
        scale = at<float>(ws, l.scale);
        const int parts = static_cast<int>(
            std::min<int64_t>((l.rows + kScaleRows - 1) / kScaleRows, kScaleParts));
        scale_kernel<<<parts, 1024, 0, stream>>>(static_cast<int32_t>(l.rows),
                                                 static_cast<int32_t>(x.V),
                                                 logf(static_cast<float>(x.V)), inv, tokens, saved,
                                                 g_logprob, g_entropy, scale + 2, scale);
        if (parts > 1) join_scale_kernel<<<1, 64, 0, stream>>>(parts, scale + 2, scale);
    }
    HeadRow *head_rows = at<HeadRow>(ws, l.head_rows);
    head_rows_kernel<<<static_cast<unsigned>(up(rows, kRowThreads) / kRowThreads), kRowThreads, 0,
                       stream>>>(
        static_cast<int32_t>(l.rows), l.copies, rows, static_cast<int32_t>(x.V), temperature, tokens, saved, g_logprob,
        g_entropy, scale, head_rows);
    E *dx = at<E>(ws, l.dx);
    float *part = at<float>(ws, l.mul), *sum = at<float>(ws, l.sum);
    const bool chunks = l.chunk < x.V;
    for (int64_t v0 = 0; v0 < x.V; v0 += l.chunk) {
        const int64_t cols = std::min(l.chunk, x.V - v0), wide = up(cols, kBig);
        const Operand<E> wc{w.data + v0 * w.ld, w.ld, static_cast<int32_t>(cols), w.cols};
        const bool big = rows > kSmall && (rows / kBig) * (wide / kBig) >= kFewTiles;
        const int tile = big ? kBig : kSmall;
        const DxArgs d{static_cast<int32_t>(x.V), static_cast<uint32_t>(rows / tile),
                       static_cast<uint32_t>(wide / tile), x.D, v0, kTokLog2e / temperature, l.copies > 1,
                       head_rows, dx, l.chunk};
        const unsigned tiles = d.tiles_m * d.tiles_n;
        if (big)
            dx_kernel<E, kBig, kMany><<<tiles, 512, 0, stream>>>(h, wc, d);
        else
            with_few_rows(few_rows(d.tiles_m, x), [&](auto few) {
                dx_kernel<E, kSmall, decltype(few)::value><<<tiles, 256, 0, stream>>>(h, wc, d);
            });
        const Operand<E> dxo{dx, l.chunk, static_cast<int32_t>(rows), static_cast<int32_t>(wide)};
        if (g_hidden) {
            const int64_t k = up(cols, kStepK);
            const MulPlan p = plan_mul(all, x.D, k);
            const bool one = p.parts == 1 && l.copies == 1;
            const bool direct = one && !chunks, first = one && chunks && v0 == 0;
            multiply<E, false>(dxo, wc, p,
                               {all, x.D, k, p.part_k, p.tiles_m, p.tiles_n,
                                direct ? g_hidden : nullptr, x.D, stream_out(all, x.D, k), scale,
                                first ? sum : part},
                               stream);
            if (!direct && !first)
                add_parts<E>(l.rows * x.D, l.copies, p.parts, part, sum, v0 > 0,
                             v0 + l.chunk >= x.V ? g_hidden : nullptr, scale, stream);
        }
        if (g_weight) {
            const MulPlan p = plan_mul(cols, x.D, all);
            E *out = g_weight + v0 * x.D;
            multiply<E, true>(dxo, h, p,
                              {cols, x.D, all, p.part_k, p.tiles_m, p.tiles_n,
                               p.parts == 1 ? out : nullptr, x.D, stream_out(cols, x.D, all),
                               scale, part},
                              stream);
            if (p.parts > 1)
                add_parts<E>(cols * x.D, 1, p.parts, part, nullptr, false, out, scale, stream);
        }
    }
    return hipGetLastError();
}

}  // namespace

size_t head_workspace_bytes(const Head &x, bool backward) { return layout_of(x, backward).total; }

hipError_t launch_head_forward(const Head &x, const int32_t *tokens, float temperature,
                               float *logprob, float *entropy, ScoreRow *saved, void *ws,
                               hipStream_t stream)
{
    if (x.dtype == CD_BF16)
        return forward<__bf16>(x, tokens, temperature, logprob, entropy, saved, ws, stream);
    return forward<_Float16>(x, tokens, temperature, logprob, entropy, saved, ws, stream);
}

hipError_t launch_head_backward(const Head &x, const int32_t *tokens, float temperature,
                                const ScoreRow *saved, const float *g_logprob,
                                const float *g_entropy, void *g_hidden, void *g_weight, void *ws,
                                hipStream_t stream)
{
    if (x.dtype == CD_BF16)
        return backward<__bf16>(x, tokens, temperature, saved, g_logprob, g_entropy,
                                static_cast<__bf16 *>(g_hidden), static_cast<__bf16 *>(g_weight), ws,
                                stream);
    return backward<_Float16>(x, tokens, temperature, saved, g_logprob, g_entropy,
                              static_cast<_Float16 *>(g_hidden), static_cast<_Float16 *>(g_weight), ws,
                              stream);
}

}  // namespace cdk
