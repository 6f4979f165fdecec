// Losses and metrics of networks that answer with tokens, from the logits:
// log-probabilities of given tokens with entropy and top alternatives, and
// distillation from a teacher's top logits, forward and backward.
//
// With z = x / temperature, m = max x, c = log2(e) / temperature and the sums s, e
// of token_common.h:
//     log p_j = ((x_j - m) c - log2 s) ln 2,   entropy = (log2 s - e / s) ln 2,
// where both terms of the entropy are >= 0, so that nothing cancels;
//     d/dx_j (g log p_t + h entropy) = (g (delta_jt - p_j) - h p_j (log p_j + entropy)) / temperature
//     distillation: q = softmax of the teacher's logits over the given entries,
//     loss = temperature^2 sum_k q_k (log q_k - log p_k),
//     d loss / d x_j = temperature (p_j - sum of the q_k with token j).
//
//  * rows_kernel: one pass over the logits.  A unit is a row, taken by a wave (64 lanes) or,
//    for short rows, by 16 lanes; its running maximum and sums stay in registers, blocks of 4
//    vectors rescaling them once.  Where rows are few or long, 4 or 16 waves of a workgroup
//    share a row and meet in LDS; the longest of few rows are cut over workgroups too, and
//    join_kernel joins the cuts.  Bound by memory in large calls (bfloat16: 8192 x 65536 in 177 us,
//    6.1 TB/s; 262144 x 1024 in 87 us, 6.2 TB/s) with the vector units close behind: 16-bit
//    logits take about a conversion, a maximum, two fused multiply-adds, an addition and an
//    exponential each.  A single row of 65536 takes 6 us without alternatives and 12 with its
//    20 best: the selection's dependent steps are half.
//  * The k best entries: every lane keeps the largest entry of each of its groups of vectors,
//    with the vector it first appeared in.  The lanes' best are sorted; the k-th of them bounds
//    the k-th entry of the row, and the few groups that reach it are read again (from the cache)
//    for the entries that do, which are sorted 64 at a time.  Keys of (value, lowest index
//    first) make every order strict, so ties need nothing of their own, and the cost hardly
//    depends on the data.  Sorting goes through registers (DPP and row swaps), not LDS.
//    4096 x 32768 bfloat16: 40 us without, 77 us with the 64 best.  Many short rows are bound by
//    instructions (262144 x 500: 87 us, 521 with the 5 best): two sorts of 64 keys for each row (three
//    and a merge above 16 best), and blocks of 4 vectors a lane where a row has one.
//  * grad_kernel: one pass, element by element; the given token's term is added by the lane that
//    owns it, and the teacher's tokens are written once more by the wave that wrote their
//    neighbours, so no atomics are needed.  Bound by memory: 8192 x 65536 bfloat16 takes 489 us
//    with its forward, 3.2 GB at 6.6 TB/s.
#include <algorithm>
#include <type_traits>

#include "cd_internal.h"
#include "token_common.h"

namespace cdk {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kBlock = 4;            // vectors per lane between two rescalings
// Groups of vectors per lane of which the largest is kept, where a row has few waves and many.
constexpr int kGroupsFew = 16, kGroupsMany = 8;
constexpr int kMostWaves = 16;       // waves that a row is given where rows are few
constexpr int kBestOnly = 16;        // alternatives up to which the lanes' best are bound enough
constexpr int kPending = 128;        // candidates a wave gathers before it sorts them
constexpr int kShortVecs = 128;      // vectors of a row that 16 lanes take
constexpr int64_t kMaxGrid = 1 << 20;   // workgroups of a launch; they loop over their units
constexpr int64_t kFillWaves = 2048;    // waves wanted: rows get several where they are few
constexpr int64_t kLongVecs = 4096;     // vectors of a row that 4 waves share in any case
constexpr int64_t kWaveVecs = 128;      // vectors for each of a row's waves, at least
// Vectors (512 KB) up to which a row is one workgroup's.  Cuts of 32 KB and their join take less on
// the GPU (32 rows of 100000 float32 with 8 best: 12 + 4 us instead of 19; one row of 65536 with 20
// best 10 + 4 instead of 12), but a second launch and a workspace on the host, which bounds
// such calls: 23.5 us instead of 19.5, and 23.6 instead of 19.2.
constexpr int64_t kCutVecs = 32768;
constexpr int kMaxCuts = 64;
// Gradients that do not fit in the last cache together with their logits go past the
// caches (us, forward and backward, through them -> past them: 8192 x 65536 bfloat16 558 -> 518,
// 131072 x 1024 155 -> 134; 3001 x 50021 float32 351 -> 312, its backward alone 221 -> 235;
// 262144 x 200 bfloat16, 105 MB, the backward 50 -> 58).  Logits of that size are read past
// them where no backward will read them again (4096 x 32768 bfloat16 48 -> 44, 3000 x 50000
// float32 101 -> 93; with a backward 3001 x 50021 306 -> 332).
bool past_caches(int64_t R, int64_t V, int dtype)
{
    return R * V * (dtype == CD_F32 ? 4 : 2) > kCacheBytes / 2;
}

// What rows_kernel and join_kernel are given.
struct RowsArgs {
    const void *x;          // logits
    int64_t sb, st;         // strides (elements) of row b * T + t
    int64_t R;
    uint32_t T;
    int32_t V;
    int32_t cuts, cut_vecs;
    float c;                // log2(e) / temperature
    float temperature;
    const int32_t *tokens;  // score: [R] or null; < 0: no token, the row is not read
    int32_t k;              // score: alternatives; distillation: entries
    float *logprob, *entropy, *top_logprob;
    int32_t *top_token;
    ScoreRow *saved;
    const int32_t *ids;     // distillation: [R, k]
    const void *teacher;    // [R, k]
    int32_t teacher_dtype;
    float *loss;
    DistillRow *distilled;
    Softmax *cut_stats;     // [R, cuts]
    uint64_t *cut_keys;     // [R, cuts, k]
    bool once;              // the logits are read once, past the caches
};

template <typename E>
__device__ __forceinline__ const E *row_ptr(const RowsArgs &a, int64_t row)
{
    const uint32_t b = static_cast<uint32_t>(row) / a.T;
    const uint32_t t = static_cast<uint32_t>(row) - b * a.T;
    return static_cast<const E *>(a.x) + b * a.sb + t * a.st;
}

// Vector v of a row that is read up to vector v1, -inf for what it does not have.  The row's last
// vector is loaded so that it ends with the row, and keeps only what no other vector has: the
// values stand at other places in it then.
template <typename E>
__device__ __forceinline__ void load_part(const E *x, int32_t V, int v, int v1,
                                          float (&e)[Vec<E>::kN])
{
    constexpr int N = Vec<E>::kN;
    const int64_t at = static_cast<int64_t>(v) * N;
    if (V < N) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            e[j] = v < v1 && at + j < V ? static_cast<float>(x[at + j]) : -INFINITY;
        return;
    }
    const int64_t first = at + N <= V ? at : V - N;
    const int skip = v < v1 ? static_cast<int>(at - first) : N;
    load_vec(x + first, e);
#pragma unroll
    for (int j = 0; j < N; ++j) e[j] = j < skip ? -INFINITY : e[j];
}

// ---- ordered keys: larger key = larger value, then lower index; 0 = none.

__device__ __forceinline__ uint64_t make_key(float x, uint32_t index)
{
    const uint32_t b = __float_as_uint(x + 0.0f);   // -0 equals 0
    const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
    return static_cast<uint64_t>(o) << 32 | ~index;
}
__device__ __forceinline__ float key_value(uint64_t key)
{
    const uint32_t o = static_cast<uint32_t>(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return ~static_cast<uint32_t>(key); }

__device__ __forceinline__ uint64_t key_lane(uint64_t key, int lane)
{
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(key), lane);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(key >> 32), lane);
    return static_cast<uint64_t>(hi) << 32 | lo;
}

// The value of lane `lane ^ kMask`, without a way through LDS: within 16 lanes by DPP
// (4 = 7 ^ 3, 8 is a rotation), across by row swaps.
template <int kMask>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x)
{
    if constexpr (kMask >= 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        const uint32_t y = threadIdx.x & 32 ? r[0] : r[1];
        if constexpr (kMask == 32) return y;
        else return lane_xor<kMask - 32>(y);
    } else if constexpr (kMask >= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        const uint32_t y = threadIdx.x & 16 ? r[0] : r[1];
        if constexpr (kMask == 16) return y;
        else return lane_xor<kMask - 16>(y);
    } else if constexpr (kMask == 4) {
        return lane_xor<7>(lane_xor<3>(x));
    } else {
        static_assert(kMask == 1 || kMask == 2 || kMask == 3 || kMask == 7 || kMask == 8 || kMask == 15,
                      "one DPP move");
        constexpr int kCtrl = kMask == 1   ? kDppXor1
                              : kMask == 2 ? kDppXor2
                              : kMask == 3 ? 0x1B
                              : kMask == 7 ? kDppHalfMirror
                              : kMask == 8 ? 0x128
                                           : kDppMirror;
        return __builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, 0xf, 0xf, true);
    }
}
template <int kMask>
__device__ __forceinline__ uint64_t key_xor(uint64_t key)
{
    return static_cast<uint64_t>(lane_xor<kMask>(static_cast<uint32_t>(key >> 32))) << 32 |
           lane_xor<kMask>(static_cast<uint32_t>(key));
}

// The lane with bit kBit clear keeps the larger of its own and its partner's key.
template <int kMask, int kBit>
__device__ __forceinline__ uint64_t exchange(uint64_t key, int lane)
{
    const uint64_t other = key_xor<kMask>(key);
    return (key > other) == ((lane & kBit) == 0) ? key : other;
}

// Descending runs of 2 kBit lanes from a bitonic sequence in each.
template <int kBit>
__device__ __forceinline__ uint64_t bitonic(uint64_t key, int lane)
{
    if constexpr (kBit > 0) return bitonic<kBit / 2>(exchange<kBit, kBit>(key, lane), lane);
    else return key;
}

// 64 keys, one per lane, into descending order: descending runs of kRun lanes meet their
// neighbour's mirror image.
template <int kRun = 1>
__device__ __forceinline__ uint64_t sort_keys(uint64_t key, int lane)
{
    if constexpr (kRun == 64) {
        return key;
    } else {
        key = exchange<2 * kRun - 1, kRun>(key, lane);
        return sort_keys<2 * kRun>(bitonic<kRun / 2>(key, lane), lane);
    }
}

// The 64 largest of two descending lists, in descending order.
__device__ __forceinline__ uint64_t merge_keys(uint64_t a, uint64_t b, int lane)
{
    const uint64_t r = key_xor<63>(b);
    return bitonic<32>(a > r ? a : r, lane);
}

// The k best keys that a wave has seen, and the candidates waiting in LDS.
struct Best {
    uint64_t list;      // descending over the lanes
    uint64_t bound;     // at least k keys are no smaller
    uint64_t *pending;  // [kPending]
    int k, n, seen;

    __device__ void flush(int lane)
    {
        wave_fence();
        const uint64_t key = lane < n ? pending[lane] : 0;
        const uint64_t rest = lane + 64 < n ? pending[lane + 64] : 0;
        wave_fence();
        const uint64_t sorted = sort_keys(key, lane);
        list = seen > 0 ? merge_keys(list, sorted, lane) : sorted;
        seen += n < 64 ? n : 64;
        if (seen >= k) {
            const uint64_t last = key_lane(list, k - 1);
            bound = last > bound ? last : bound;
        }
        pending[lane] = rest;
        n = n > 64 ? n - 64 : 0;
        wave_fence();
    }
    __device__ void push(bool want, uint64_t key, int lane)
    {
        const uint64_t mask = __ballot(want && key >= bound);
        if (mask == 0) return;
        if (want && key >= bound)
            pending[n + __builtin_amdgcn_mbcnt_hi(
                            static_cast<uint32_t>(mask >> 32),
                            __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0))] = key;
        n += __popcll(mask);
        if (n >= 64) flush(lane);
    }
};

// The k (<= 64) best of n keys, descending over the lanes.  The keys may be a row of
// descending lists: a lane takes keys of different ranks, so that the k-th of the lanes' best
// bounds well.
__device__ __forceinline__ uint64_t join_best(const uint64_t *keys, int n, int k, uint64_t *pending,
                                              int lane)
{
    const int per_lane = (n + 63) / 64;
    const auto get = [&](int i) {
        const int at = i * 64 + ((lane + 4 * i) & 63);
        return at < n ? keys[at] : uint64_t(0);
    };
    uint64_t mine = 0;
    for (int i = 0; i < per_lane; ++i) {
        const uint64_t key = get(i);
        mine = key > mine ? key : mine;
    }
    const uint64_t sorted = sort_keys(mine, lane);
    if (per_lane <= 1) return sorted;
    Best best{0, key_lane(sorted, k - 1), pending, k, 0, 0};
    for (int i = 0; i < per_lane; ++i) {
        const uint64_t key = get(i);
        best.push(key != 0, key, lane);
    }
    if (best.n > 0) best.flush(lane);
    return best.list;
}

// ---- what a finished row gives.

// The row's token and its logit, asked for before the row is read.
struct Given {
    int32_t token;
    float x;
};
template <typename E>
__device__ __forceinline__ Given given_of(const RowsArgs &a, int64_t row, const E *x)
{
    if (!a.tokens) return {0, 0.0f};
    const int32_t t = a.tokens[row];
    return {t, t >= 0 && t < a.V ? static_cast<float>(x[t]) : __builtin_nanf("")};
}

__device__ __forceinline__ void finish_score(const RowsArgs &a, int64_t row, const Given &given,
                                             const Softmax &r)
{
    const bool empty = r.s == 0.0f;
    const float l2s = empty ? 0.0f : log2f(r.s);
    const float h2 = empty ? 0.0f : l2s - r.e / r.s;
    if (a.tokens) {
        float lp = ((given.x - r.m) * a.c - l2s) * kTokLn2;
        if (empty && given.token < a.V) lp = -INFINITY;
        a.logprob[row] = lp;
    }
    a.entropy[row] = h2 * kTokLn2;
    if (a.saved) a.saved[row] = {empty ? -INFINITY : softmax_ref(r.m), l2s, h2, 0};
}

__device__ __forceinline__ void finish_top(const RowsArgs &a, int64_t row, const Softmax &r,
                                           uint64_t key, int lane)
{
    if (lane >= a.k) return;
    float lp = __builtin_nanf("");
    if (r.s == 0.0f) lp = -INFINITY;
    else if (key != 0) lp = ((key_value(key) - r.m) * a.c - log2f(r.s)) * kTokLn2;
    a.top_logprob[row * a.k + lane] = lp;
    a.top_token[row * a.k + lane] = key != 0 ? static_cast<int32_t>(key_index(key)) : -1;
}

// A row without a token: nothing of it is read.
template <int L>
__device__ __forceinline__ void skip_score(const RowsArgs &a, int64_t row, int sub, int k)
{
    if (sub == 0) {
        a.logprob[row] = 0.0f;
        a.entropy[row] = 0.0f;
        if (a.saved) a.saved[row] = {-INFINITY, 0.0f, 0.0f, 0};
    }
    for (int i = sub; i < k; i += L) {
        a.top_logprob[row * k + i] = -INFINITY;
        a.top_token[row * k + i] = -1;
    }
}

__device__ __forceinline__ float teacher_logit(const void *t, int dtype, int64_t i)
{
    if (dtype == CD_F32) return static_cast<const float *>(t)[i];
    if (dtype == CD_BF16) return static_cast<float>(static_cast<const __bf16 *>(t)[i]);
    return static_cast<float>(static_cast<const _Float16 *>(t)[i]);
}

// Words of LDS by which the L lanes that finish a row see whether a token comes twice: a table
// twice the size of the most entries, or a bit for each token of a short row.  (256 entries,
// 4096 x 16384 bfloat16: 40 us, with a comparison of each with each 65 us.)
template <int L>
constexpr int kSeen = L == 64 ? 2 * CD_DISTILL_MAX_K : kShortVecs * 8 / 32;

template <int L>
__device__ __forceinline__ bool given_twice(const int32_t *ids, int k, uint32_t *seen, int sub)
{
    constexpr uint32_t kFree = L == 64 ? ~0u : 0u;
    bool twice = false;
    for (int i = sub; i < kSeen<L>; i += L) seen[i] = kFree;
    wave_fence();
    for (int i = sub; i < k; i += L) {
        const int32_t id = ids[i];
        if (id < 0) continue;
        if constexpr (L == 64) {
            // (a multiplicative hash; at least half of the table stays free, so a place is found)
            uint32_t at = static_cast<uint32_t>(id) * 2654435769u / (0xffffffffu / kSeen<L> + 1);
            for (;;) {
                const uint32_t was = atomicCAS(&seen[at], kFree, static_cast<uint32_t>(id));
                twice |= was == static_cast<uint32_t>(id);
                if (was == kFree || was == static_cast<uint32_t>(id)) break;
                at = (at + 1) % kSeen<L>;
            }
        } else {
            const uint32_t bit = 1u << (id & 31);
            twice |= (atomicOr(&seen[id >> 5], bit) & bit) != 0;
        }
    }
    return twice;
}

template <typename E, int L>
__device__ __forceinline__ void finish_distill(const RowsArgs &a, int64_t row, const E *x,
                                               const Softmax &r, uint32_t *seen, int sub)
{
    const int32_t *ids = a.ids + row * a.k;
    float tm = -INFINITY, outside = 0.0f, nan = 0.0f;
    for (int i = sub; i < a.k; i += L) {
        const int32_t id = ids[i];
        if (id < 0) continue;
        const float t = teacher_logit(a.teacher, a.teacher_dtype, row * a.k + i);
        if (id >= a.V) outside = 1.0f;
        if (t != t) nan = 1.0f;
        tm = fmaxf(tm, t);
    }
    tm = group_max<L>(tm);
    outside = group_max<L>(outside);
    nan = group_max<L>(nan);
    // Weights e_i = 2^((t_i - tm) c), their sum, and their sum with log2 e_i - log2 of p's weight.
    float ts = 0.0f, term = 0.0f, twice = 0.0f;
    if (outside == 0.0f && tm != -INFINITY) {
        for (int i = sub; i < a.k; i += L) {
            const int32_t id = ids[i];
            if (id < 0) continue;
            const float d = (teacher_logit(a.teacher, a.teacher_dtype, row * a.k + i) - tm) * a.c;
            const float w = tok_exp2(d);
            ts += w;
            const float xi = static_cast<float>(x[id]);
            if (w > 0.0f) term = __builtin_fmaf(w, d - (xi - softmax_ref(r.m)) * a.c, term);
        }
        if (a.distilled && given_twice<L>(ids, a.k, seen, sub)) twice = 1.0f;
    }
    ts = group_sum<L>(ts);
    term = group_sum<L>(term);
    twice = group_max<L>(twice);
    if (sub != 0) return;
    DistillRow d{softmax_ref(r.m), 0.0f, tm, 0.0f, kDistillNone};
    float loss;
    if (outside != 0.0f) {
        loss = __builtin_nanf("");
    } else if (nan != 0.0f) {       // and NaN in the gradient at the given tokens
        loss = __builtin_nanf("");
        d.l2s = r.s == 0.0f ? 0.0f : log2f(r.s);
        d.l2ts = loss;
        d.kind = kDistillDistinct;
    } else if (tm == -INFINITY) {
        loss = 0.0f;
    } else if (r.s == 0.0f) {
        loss = INFINITY;
    } else {
        d.l2s = log2f(r.s);
        d.l2ts = log2f(ts);
        loss = (term / ts - d.l2ts + d.l2s) * (kTokLn2 * a.temperature * a.temperature);
        d.kind = twice != 0.0f ? kDistillRepeated : kDistillDistinct;
    }
    a.loss[row] = loss;
    if (a.distilled) a.distilled[row] = d;
}

// The k best entries of a wave's share, by way of its lanes' groups of per_group vectors each:
// groups[i * 64] is this lane's largest entry of its i-th, at its vector's first index.
//
// lane_best: the lanes' best groups (and second best: `more`), descending.
__device__ __forceinline__ uint64_t lane_best(const uint64_t *groups, int ngroups, bool more, int lane)
{
    uint64_t mine = 0, second = 0;
    for (int i = 0; i < ngroups; ++i) {
        const uint64_t key = groups[i * 64];
        second = key > mine ? mine : key > second ? key : second;
        mine = key > mine ? key : mine;
    }
    const uint64_t sorted = sort_keys(mine, lane);
    return more ? merge_keys(sorted, sort_keys(second, lane), lane) : sorted;
}

// The entries that may be among the k best of the row where k groups are no worse than
// `last`: those of the groups that reach it, each lane reading one of its own at a time.
template <typename E>
__device__ __forceinline__ Best candidates(const E *x, int32_t V, int v0, int v1, int per_group,
                           const uint64_t *groups, int ngroups, uint64_t last, int k,
                           uint64_t *pending, int lane)
{
    constexpr int N = Vec<E>::kN;
    // An entry of last's value lies in the vector that starts at its index.
    Best best{0, last == 0 ? 1 : last - (N - 1), pending, k, 0, 0};
    uint32_t todo = 0;
    for (int i = 0; i < ngroups; ++i)
        todo |= groups[i * 64] != 0 && groups[i * 64] >= last ? 1u << i : 0u;
    while (__ballot(todo != 0) != 0) {
        const int first = todo != 0 ? (__ffs(todo) - 1) * per_group : (v1 - v0);
        todo &= todo - 1;
        for (int i = 0; i < per_group; i += kBlock) {
            float e[kBlock][N];
            const int n = min(kBlock, per_group - i);
#pragma unroll
            for (int b = 0; b < kBlock; ++b) {
                if (b >= n) break;
                const int v = v0 + (first + i + b) * 64 + lane;
                const bool in = first < v1 - v0 && v < v1;
                const int64_t at = static_cast<int64_t>(v) * N;
                if (in && at + N <= V) {
                    load_vec(x + at, e[b]);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        e[b][j] = in && at + j < V ? static_cast<float>(x[at + j])
                                                   : __builtin_nanf("");
                }
            }
#pragma unroll
            for (int b = 0; b < kBlock; ++b) {
                if (b >= n) break;
                const uint32_t at = static_cast<uint32_t>(v0 + (first + i + b) * 64 + lane) * N;
                // NaN is none of the best.
                const float floor = best.bound == 1 ? -INFINITY : key_value(best.bound);
                uint32_t above = 0;
#pragma unroll
                for (int j = 0; j < N; ++j) above |= e[b][j] >= floor ? 1u << j : 0u;
                while (__ballot(above != 0) != 0) {
                    const int j = __ffs(above) - 1;
                    float value = 0.0f;
#pragma unroll
                    for (int l = 0; l < N; ++l) value = j == l ? e[b][l] : value;
                    best.push(above != 0, make_key(value, at + j), lane);
                    above &= above - 1;
                }
            }
        }
    }
    return best;
}

// What the waves of a row tell each other.
struct Meet {
    Softmax stats[kMostWaves];
    uint64_t keys[kMostWaves * 64];
    uint64_t last;
    int n;
};

enum RowsMode { kScore, kScoreTop, kDistill };

// kPer waves take a row (or a cut of one); 0: 16 lanes do.
template <typename E, int kPer, RowsMode kMode>
__global__ __launch_bounds__(kPer > kWaves ? kPer * 64 : kThreads) void rows_kernel(RowsArgs a)
{
    constexpr int N = Vec<E>::kN;
    constexpr bool kTop = kMode == kScoreTop;
    constexpr bool kParts = !kTop && sizeof(E) == 2;
    constexpr int L = kPer == 0 ? 16 : 64;
    constexpr int kAll = kPer > kWaves ? kPer : kWaves;             // waves of the workgroup
    constexpr int kShares = kPer > 1 ? kPer : 1;
    constexpr int kUnits = kPer == 0 ? kThreads / 16 : kAll / kShares;  // rows at a time
    constexpr int kGroups = kPer > kWaves ? kGroupsMany : kGroupsFew;
    __shared__ uint64_t groups_lds[kTop ? kAll : 1][kTop ? kGroups * 64 : 1];
    __shared__ uint64_t pending_lds[kTop ? kAll : 1][kTop ? kPending : 1];
    __shared__ uint32_t seen_lds[kMode == kDistill ? kUnits : 1][kMode == kDistill ? kSeen<L> : 1];
    __shared__ Meet meet;       // (kPer > 1: then a workgroup takes one row at a time)
    const int lane = threadIdx.x & 63, sub = threadIdx.x & (L - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = kPer == 0 ? threadIdx.x / 16 : wave / kShares;
    const int share = kPer > 1 ? wave : 0;
    uint64_t *groups = groups_lds[kTop ? wave : 0] + (kTop ? lane : 0);
    uint64_t *pending = pending_lds[kTop ? wave : 0];
    const int64_t units = a.R * a.cuts;
    const int nvec = (a.V + N - 1) / N;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kUnits;
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * kUnits + unit; u < units; u += step) {
        const int64_t row = a.cuts == 1 ? u : u / a.cuts;
        const int cut = a.cuts == 1 ? 0 : static_cast<int>(u - row * a.cuts);
        const E *x = row_ptr<E>(a, row);
        Given given{0, 0.0f};
        if (kMode != kDistill) {
            given = given_of(a, row, x);
            if (given.token < 0) {
                if (a.cuts == 1 && share == 0) skip_score<L>(a, row, sub, kTop ? a.k : 0);
                continue;
            }
        }
        const int c0 = cut * a.cut_vecs, c1 = min(nvec, c0 + a.cut_vecs);
        const int per_wave = (a.cut_vecs + kShares - 1) / kShares;
        const int v0 = min(c1, c0 + share * per_wave), v1 = min(c1, v0 + per_wave);
        const int iters = (v1 - v0 + L - 1) / L;
        // A group is a vector, or a whole number of blocks.
        const int blocks = (iters + kBlock - 1) / kBlock;
        const int per_group = iters <= kGroups ? 1 : (blocks + kGroups - 1) / kGroups * kBlock;
        Softmax r = softmax_empty();
        float gm = -INFINITY;
        int gv = 0, ngroups = 0, in_group = 0;
        for (int it = 0; it < iters; it += kBlock) {
            float e[kBlock * N];
            const int vb = v0 + it * L + sub;
            // One vector left of 16-bit elements is not made up to a block (us, as a block -> alone:
            // 262144 x 64 52 -> 32, 53687 x 2500 86 -> 63; float32 as often loses: 262144 x 64
            // 31 -> 22, but x 200 42 -> 49 and 134217 x 1000 90 -> 102).
            if (kParts && iters - it == 1) {
                float last[N];
                load_part(x, a.V, vb, v1, last);
                float vm = last[0];
#pragma unroll
                for (int j = 1; j < N; ++j) vm = fmaxf(vm, last[j]);
                softmax_add<true>(r, last, vm, a.c);
                break;
            }
            // Vectors that end inside the row and before v1 need no checks.
            const bool whole = v0 + (it + kBlock) * L <= v1 &&
                               static_cast<int64_t>(v0 + (it + kBlock) * L) * N <= a.V;
            if (!kTop && whole && a.once) {
#pragma unroll
                for (int b = 0; b < kBlock; ++b)
                    load_vec<true>(x + static_cast<int64_t>(vb + b * L) * N,
                                   reinterpret_cast<float(&)[N]>(e[b * N]));
            } else if (whole) {
#pragma unroll
                for (int b = 0; b < kBlock; ++b)
                    load_vec(x + static_cast<int64_t>(vb + b * L) * N,
                             reinterpret_cast<float(&)[N]>(e[b * N]));
            } else {
#pragma unroll
                for (int b = 0; b < kBlock; ++b) {
                    const int v = vb + b * L;
                    const int64_t at = static_cast<int64_t>(v) * N;
                    if (kParts) {
                        load_part(x, a.V, v, v1, reinterpret_cast<float(&)[N]>(e[b * N]));
                    } else if (v < v1 && at + N <= a.V) {
                        load_vec(x + at, reinterpret_cast<float(&)[N]>(e[b * N]));
                    } else {
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            e[b * N + j] = v < v1 && at + j < a.V ? static_cast<float>(x[at + j])
                                                                 : -INFINITY;
                    }
                }
            }
            float bm = -INFINITY;
#pragma unroll
            for (int b = 0; b < kBlock; ++b) {
                float vm = e[b * N];
#pragma unroll
                for (int j = 1; j < N; ++j) vm = fmaxf(vm, e[b * N + j]);
                if (kTop) {
                    const int v = vb + b * L;
                    if (per_group == 1) {
                        if (it + b < iters)
                            groups[ngroups++ * 64] =
                                v < v1 ? make_key(vm, static_cast<uint32_t>(v) * N) : 0;
                    } else {    // (what lies behind v1 is -inf)
                        if (b == 0 && in_group == 0) gv = v;
                        gv = vm > gm ? v : gv;
                        gm = fmaxf(gm, vm);
                    }
                }
                bm = fmaxf(bm, vm);
            }
            softmax_add<true>(r, e, bm, a.c);
            in_group += kBlock;
            if (kTop && per_group > 1 && (in_group == per_group || it + kBlock >= iters)) {
                groups[ngroups * 64] = gv < v1 ? make_key(gm, static_cast<uint32_t>(gv) * N) : 0;
                ++ngroups;
                in_group = 0;
                gm = -INFINITY;
            }
        }
        softmax_group<L>(r, a.c);
        uint64_t key = 0;
        if (kTop && kPer == 1) {
            // Of many entries some lanes hold several: with the lanes' best alone, 64 of 32768
            // random entries leave 270 above the bound, with their second best 80.
            const uint64_t best = lane_best(groups, ngroups, a.k > kBestOnly, lane);
            Best found = candidates(x, a.V, v0, v1, per_group, groups, ngroups,
                                    key_lane(best, a.k - 1), a.k, pending, lane);
            if (found.n > 0) found.flush(lane);
            key = found.list;
        }
        if (kPer > 1) {
            if (lane == 0) meet.stats[wave] = r;
            if (kTop) {
                // 64 (or 128) of the row's lanes' best bound the row's k-th, and what all waves
                // find above is little more than k entries.
                constexpr int kEach = 64 / kShares;
                const uint64_t best = lane_best(groups, ngroups, false, lane);
                if (lane < 2 * kEach)
                    meet.keys[lane / kEach * 64 + wave * kEach + lane % kEach] = best;
                if (threadIdx.x == 0) meet.n = 0;
                __syncthreads();
                if (wave == 0) {
                    uint64_t some = sort_keys(meet.keys[lane], lane);
                    if (a.k > 32) some = merge_keys(some, sort_keys(meet.keys[64 + lane], lane), lane);
                    const uint64_t last = key_lane(some, a.k - 1);     // (by all lanes, as it is of one)
                    if (lane == 0) meet.last = last;
                }
                __syncthreads();
                Best found = candidates(x, a.V, v0, v1, per_group, groups, ngroups, meet.last, a.k,
                                        pending, lane);
                if (found.seen > 0 && found.n > 0) found.flush(lane);
                wave_fence();
                const uint64_t mine = found.seen > 0 ? found.list
                                      : lane < found.n ? pending[lane]
                                                       : 0;
                const int n = found.seen > 0 ? 64 : found.n;
                int at = 0;
                if (lane == 0 && n > 0) at = atomicAdd(&meet.n, n);     // (their order is sorted out)
                at = __builtin_amdgcn_readfirstlane(at);
                if (lane < n) meet.keys[at + lane] = mine;
            }
            __syncthreads();
            if (wave == 0) {
                r = lane < kPer ? meet.stats[lane] : softmax_empty();
                softmax_group<64>(r, a.c);
                if (kTop) key = join_best(meet.keys, meet.n, a.k, pending, lane);
            }
            __syncthreads();
            if (wave != 0) continue;
        }
        if (a.cuts > 1) {
            if (sub == 0) a.cut_stats[u] = r;
            if (kTop && lane < a.k) a.cut_keys[u * a.k + lane] = key;
        } else if (kMode == kDistill) {
            finish_distill<E, L>(a, row, x, r, seen_lds[kMode == kDistill ? unit : 0], sub);
        } else {
            if (sub == 0) finish_score(a, row, given, r);
            if (kTop) finish_top(a, row, r, key, lane);
        }
    }
}

// Joins the cuts of a row; a wave per row.
template <typename E, RowsMode kMode>
__global__ __launch_bounds__(kThreads) void join_kernel(RowsArgs a)
{
    constexpr bool kTop = kMode == kScoreTop;
    __shared__ uint64_t pending_lds[kTop ? kWaves : 1][kTop ? kPending : 1];
    __shared__ uint32_t seen_lds[kMode == kDistill ? kWaves : 1][kMode == kDistill ? kSeen<64> : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWaves;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * kWaves + wave; row < a.R; row += step) {
        Softmax r = lane < a.cuts ? a.cut_stats[row * a.cuts + lane] : softmax_empty();
        const E *x = row_ptr<E>(a, row);
        Given given{0, 0.0f};
        if (kMode != kDistill) {
            given = given_of(a, row, x);
            if (given.token < 0) {
                skip_score<64>(a, row, lane, kTop ? a.k : 0);
                continue;
            }
        }
        softmax_group<64>(r, a.c);
        if (kMode == kDistill) {
            finish_distill<E, 64>(a, row, x, r, seen_lds[kMode == kDistill ? wave : 0], lane);
            continue;
        }
        if (lane == 0) finish_score(a, row, given, r);
        if (kTop) {
            const int n = a.cuts * a.k;
            finish_top(a, row, r, join_best(a.cut_keys + row * n, n, a.k, pending_lds[wave], lane),
                       lane);
        }
    }
}

// ---- gradients.

struct GradArgs {
    const void *x;
    int64_t sb, st;
    int64_t R;
    uint32_t T;
    int32_t V;
    int32_t chunks;         // units per row
    float c, temperature;
    const int32_t *tokens;
    const ScoreRow *saved;
    const float *g_logprob, *g_entropy;   // [R], either may be null
    int32_t k;
    const int32_t *ids;
    const void *teacher;
    int32_t teacher_dtype;
    const DistillRow *distilled;
    const float *g_loss;
    void *gx;               // [R, V]
};

// A unit is kBlock vectors per lane of one row: units of all rows run in any order, so a few long
// rows fill the chip like many short ones.
template <typename E, int L, bool kDistillGrad, bool kStream>
__global__ __launch_bounds__(kThreads) void grad_kernel(GradArgs a)
{
    constexpr int N = Vec<E>::kN;
    const int sub = threadIdx.x & (L - 1);
    const int unit = L == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x / L;
    const int64_t units = a.R * a.chunks;
    const int64_t step = static_cast<int64_t>(gridDim.x) * (kThreads / L);
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kThreads / L) + unit; u < units;
         u += step) {
        const int64_t row = a.chunks == 1 ? u : u / a.chunks;
        const int chunk = a.chunks == 1 ? 0 : static_cast<int>(u - row * a.chunks);
        const uint32_t b = static_cast<uint32_t>(row) / a.T;
        const E *x = static_cast<const E *>(a.x) + b * a.sb +
                     (static_cast<uint32_t>(row) - b * a.T) * a.st;
        E *gx = static_cast<E *>(a.gx) + row * a.V;
        // dx = w (gp + gh (t - tref)), w = 2^t, t = (x - m) c, and gt more at the token.
        float m, gp, gh = 0.0f, gt = 0.0f, tref = 0.0f;
        int32_t token = -1;
        bool live;
        DistillRow d;
        if (kDistillGrad) {
            d = a.distilled[row];
            live = d.kind != kDistillNone;
            m = d.m;
            gp = a.g_loss[row] * a.temperature;
            gt = gp;
            gp *= tok_exp2(-d.l2s);
        } else {
            const ScoreRow s = a.saved[row];
            token = a.tokens ? a.tokens[row] : -1;
            live = s.m != -INFINITY && !(a.tokens && token < 0);
            m = s.m;
            const float inv = 1.0f / a.temperature;
            const float gl = a.g_logprob && token >= 0 && token < a.V ? a.g_logprob[row] * inv : 0.0f;
            const float he = a.g_entropy ? a.g_entropy[row] * inv : 0.0f;
            const float scale = tok_exp2(-s.l2s);
            gt = gl;
            gp = -gl * scale;
            gh = -he * kTokLn2 * scale;
            tref = s.l2s - s.h2;    // log2 p + entropy = t - tref
        }
        const int first = (chunk * kBlock) * L + sub;
#pragma unroll
        for (int i = 0; i < kBlock; ++i) {
            const int64_t at = static_cast<int64_t>(first + i * L) * N;
            if (at >= a.V) break;
            const bool whole = at + N <= a.V;
            float e[N];
            if (!live) {
#pragma unroll
                for (int j = 0; j < N; ++j) e[j] = 0.0f;
            } else {
                if (whole) {
                    load_vec<kStream>(x + at, e);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        e[j] = at + j < a.V ? static_cast<float>(x[at + j]) : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float t = (e[j] - m) * a.c;
                    const float w = tok_exp2(t);
                    float f = gp;
                    if (!kDistillGrad) f = __builtin_fmaf(gh, fmaxf(t, -200.0f) - tref, gp);
                    e[j] = w * f;
                }
                if (!kDistillGrad && token >= at && token < at + N) {
#pragma unroll
                    for (int j = 0; j < N; ++j) e[j] += token == at + j ? gt : 0.0f;
                }
            }
            if (whole) {
                store_vec<kStream>(gx + at, e);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (at + j < a.V) gx[at + j] = static_cast<E>(e[j]);
            }
        }
        if (kDistillGrad && live) {
            // The teacher's tokens of this unit: their elements are written again,
            // behind the group's own stores.
            const int64_t lo = static_cast<int64_t>(chunk * kBlock) * L * N;
            const int64_t hi = lo + static_cast<int64_t>(kBlock) * L * N;
            const int32_t *ids = a.ids + row * a.k;
            wave_fence();
            // (kMost at once: lanes beyond k and tokens of other units hold -1)
            constexpr int kMost = CD_DISTILL_MAX_K / L;
            int32_t id[kMost];
            float q[kMost];
            const auto weight = [&](int i) {
                return tok_exp2((teacher_logit(a.teacher, a.teacher_dtype, row * a.k + i) - d.tm) *
                                    a.c -
                                d.l2ts);
            };
            const auto write = [&](int32_t at, float sum) {
                const float w = tok_exp2((static_cast<float>(x[at]) - m) * a.c);
                gx[at] = static_cast<E>(__builtin_fmaf(w, gp, -sum * gt));
            };
            if (d.kind != kDistillRepeated) {
                for (int i = sub; i < a.k; i += L)
                    if (ids[i] >= lo && ids[i] < hi) write(ids[i], weight(i));
                continue;
            }
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                id[i] = -1;
                q[i] = 0.0f;
                if (i * L + sub < a.k) {
                    const int32_t one = ids[i * L + sub];
                    if (one >= lo && one < hi) {
                        id[i] = one;
                        q[i] = weight(i * L + sub);
                    }
                }
            }
            // An entry at a time: where more than it have its token, all lanes add what they hold
            // of that, in a fixed order.
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                float sum = q[i];
                uint64_t todo = __ballot(id[i] >= 0);
                if (L == 16) todo = todo >> (threadIdx.x & 48) & 0xffff;
                for (; todo != 0; todo &= todo - 1) {
                    const int l = __builtin_ctzll(todo);
                    const int32_t one = L == 64 ? __builtin_amdgcn_readlane(id[i], l)
                                                : __shfl(id[i], l, L);
                    int n = sub == l ? -1 : 0;
                    float s = 0.0f;
#pragma unroll
                    for (int j = 0; j < kMost; ++j) {
                        n += id[j] == one ? 1 : 0;
                        s += id[j] == one ? q[j] : 0.0f;
                    }
                    if (__ballot(n > 0) == 0) continue;
                    s = group_sum<L>(s);
                    sum = sub == l ? s : sum;
                }
                if (id[i] >= 0) write(id[i], sum);
            }
        }
    }
}

// ---- launches.

int64_t vectors(int64_t V, int dtype)
{
    const int n = dtype == CD_F32 ? 4 : 8;
    return (V + n - 1) / n;
}

// How a row is shared out: waves (0: 16 lanes) and cuts.
struct Share {
    int waves, cuts;
};

// Long rows without alternatives go to 4 waves however many there are (us, 1 wave -> 4 waves a
// row, bfloat16): 4096 x 32768 45 -> 40, 8192 x 65536 193 -> 177, but 4096 x 26000 35 -> 40,
// 8192 x 9000 29 -> 42, and with 64 alternatives 4096 x 32768 79 -> 103.
Share share_of(int64_t R, int64_t V, int dtype, RowsMode mode)
{
    const int64_t n = vectors(V, dtype);
    if (n <= kShortVecs && mode != kScoreTop) return {0, 1};
    if (R * kWaves < kFillWaves && n >= kMostWaves * kWaveVecs) {
        const int64_t cuts = std::min((n + kCutVecs - 1) / kCutVecs, (kFillWaves / kMostWaves + R) / R);
        return {kMostWaves, static_cast<int>(std::min<int64_t>(cuts, kMaxCuts))};
    }
    const bool few = R < kFillWaves && n >= kWaves * kWaveVecs;
    return {few || (mode == kScore && n >= kLongVecs) ? kWaves : 1, 1};
}

unsigned grid_of(int64_t units, int per_group)
{
    return static_cast<unsigned>(std::min<int64_t>((units + per_group - 1) / per_group, kMaxGrid));
}

template <typename E, RowsMode kMode>
void start_rows(const RowsArgs &a, int waves, hipStream_t stream)
{
    if (waves == kMostWaves)
        rows_kernel<E, kMostWaves, kMode>
            <<<grid_of(a.R * a.cuts, 1), kMostWaves * 64, 0, stream>>>(a);
    else if (waves == kWaves)
        rows_kernel<E, kWaves, kMode><<<grid_of(a.R, 1), kThreads, 0, stream>>>(a);
    else if (waves == 1)
        rows_kernel<E, 1, kMode><<<grid_of(a.R, kWaves), kThreads, 0, stream>>>(a);
    else if constexpr (kMode != kScoreTop)
        rows_kernel<E, 0, kMode><<<grid_of(a.R, kThreads / 16), kThreads, 0, stream>>>(a);
    if (a.cuts > 1) join_kernel<E, kMode><<<grid_of(a.R, kWaves), kThreads, 0, stream>>>(a);
}

template <RowsMode kMode>
void start_rows(const RowsArgs &a, int dtype, int waves, hipStream_t stream)
{
    if (dtype == CD_F32) start_rows<float, kMode>(a, waves, stream);
    else if (dtype == CD_BF16) start_rows<__bf16, kMode>(a, waves, stream);
    else start_rows<_Float16, kMode>(a, waves, stream);
}

template <typename E, bool kDistillGrad>
void start_grad(GradArgs a, int dtype, hipStream_t stream)
{
    const int64_t nvec = vectors(a.V, dtype);
    const bool narrow = nvec <= kShortVecs;
    const int lanes = narrow ? 16 : 64;
    a.chunks = static_cast<int>((nvec + lanes * kBlock - 1) / (lanes * kBlock));
    const unsigned grid = grid_of(a.R * a.chunks, kThreads / lanes);
    const auto run = [&](auto past) {
        constexpr bool kStream = decltype(past)::value;
        if (narrow) grad_kernel<E, 16, kDistillGrad, kStream><<<grid, kThreads, 0, stream>>>(a);
        else grad_kernel<E, 64, kDistillGrad, kStream><<<grid, kThreads, 0, stream>>>(a);
    };
    if (past_caches(a.R, a.V, dtype)) run(std::true_type{});
    else run(std::false_type{});
}

template <bool kDistillGrad>
hipError_t start_grad_of(const GradArgs &a, int dtype, hipStream_t stream)
{
    if (dtype == CD_F32) start_grad<float, kDistillGrad>(a, dtype, stream);
    else if (dtype == CD_BF16) start_grad<__bf16, kDistillGrad>(a, dtype, stream);
    else start_grad<_Float16, kDistillGrad>(a, dtype, stream);
    return hipGetLastError();
}

size_t stats_bytes(int64_t R, int cuts)
{
    return (static_cast<size_t>(R) * cuts * sizeof(Softmax) + 255) / 256 * 256;
}

RowsArgs rows_args(const Logits &x, float temperature, const Share &share, void *ws)
{
    RowsArgs a{};
    a.x = x.data;
    a.sb = x.stride_b;
    a.st = x.stride_t;
    a.R = x.B * x.T;
    a.T = static_cast<uint32_t>(x.T);
    a.V = static_cast<int32_t>(x.V);
    a.c = kTokLog2e / temperature;
    a.temperature = temperature;
    a.cuts = share.cuts;
    a.cut_vecs = static_cast<int32_t>((vectors(x.V, x.dtype) + a.cuts - 1) / a.cuts);
    a.cut_stats = static_cast<Softmax *>(ws);
    a.cut_keys = reinterpret_cast<uint64_t *>(static_cast<char *>(ws) + stats_bytes(a.R, a.cuts));
    return a;
}

GradArgs grad_args(const Logits &x, float temperature, void *gx)
{
    GradArgs a{};
    a.x = x.data;
    a.sb = x.stride_b;
    a.st = x.stride_t;
    a.R = x.B * x.T;
    a.T = static_cast<uint32_t>(x.T);
    a.V = static_cast<int32_t>(x.V);
    a.c = kTokLog2e / temperature;
    a.temperature = temperature;
    a.gx = gx;
    return a;
}

}  // namespace

size_t rows_workspace_bytes(int64_t R, int64_t V, int dtype, int top)
{
    const int cuts = share_of(R, V, dtype, top > 0 ? kScoreTop : kScore).cuts;
    if (cuts == 1) return 0;
    return stats_bytes(R, cuts) + static_cast<size_t>(R) * cuts * top * sizeof(uint64_t);
}

hipError_t launch_score_forward(const Logits &x, const int32_t *tokens, float temperature, int top,
                                float *logprob, float *entropy, float *top_logprob,
                                int32_t *top_token, ScoreRow *saved, void *ws, hipStream_t stream)
{
    const Share share = share_of(x.B * x.T, x.V, x.dtype, top > 0 ? kScoreTop : kScore);
    RowsArgs a = rows_args(x, temperature, share, ws);
    a.tokens = tokens;
    a.k = top;
    a.logprob = logprob;
    a.entropy = entropy;
    a.top_logprob = top_logprob;
    a.top_token = top_token;
    a.saved = saved;
    a.once = !saved && past_caches(a.R, a.V, x.dtype);
    if (top > 0) start_rows<kScoreTop>(a, x.dtype, share.waves, stream);
    else start_rows<kScore>(a, x.dtype, share.waves, stream);
    return hipGetLastError();
}

hipError_t launch_score_backward(const Logits &x, const int32_t *tokens, float temperature,
                                 const ScoreRow *saved, const float *g_logprob,
                                 const float *g_entropy, void *g_logits, hipStream_t stream)
{
    GradArgs a = grad_args(x, temperature, g_logits);
    a.tokens = tokens;
    a.saved = saved;
    a.g_logprob = g_logprob;
    a.g_entropy = g_entropy;
    return start_grad_of<false>(a, x.dtype, stream);
}

hipError_t launch_distill_forward(const Logits &x, int K, const int32_t *ids, const void *teacher,
                                  int teacher_dtype, float temperature, float *loss,
                                  DistillRow *saved, void *ws, hipStream_t stream)
{
    const Share share = share_of(x.B * x.T, x.V, x.dtype, kDistill);
    RowsArgs a = rows_args(x, temperature, share, ws);
    a.k = K;
    a.ids = ids;
    a.teacher = teacher;
    a.teacher_dtype = teacher_dtype;
    a.loss = loss;
    a.distilled = saved;
    a.once = !saved && past_caches(a.R, a.V, x.dtype);
    start_rows<kDistill>(a, x.dtype, share.waves, stream);
    return hipGetLastError();
}

hipError_t launch_distill_backward(const Logits &x, int K, const int32_t *ids, const void *teacher,
                                   int teacher_dtype, float temperature, const DistillRow *saved,
                                   const float *g_loss, void *g_logits, hipStream_t stream)
{
    GradArgs a = grad_args(x, temperature, g_logits);
    a.k = K;
    a.ids = ids;
    a.teacher = teacher;
    a.teacher_dtype = teacher_dtype;
    a.distilled = saved;
    a.g_loss = g_loss;
    return start_grad_of<true>(a, x.dtype, stream);
}

}  // namespace cdk
