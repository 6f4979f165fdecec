// What the token-loss kernels use of HIP, for a CPU: every lane of a workgroup is a context of its own,
// and an operation between lanes is where they meet.  The kernels' memory accesses are then the
// process's own, and one that leaves its buffer meets an unmapped page beside it.
//
// Loads straight to LDS arrive as late as a wait allows (or, lanes::early, at once), and waves run one
// after another from barrier to barrier, in either order (lanes::backwards): a missing wait or
// barrier gives wrong results.
//
// Lanes that wait at the same operation take part in it, as if the others were masked off: right
// where the lanes that read each other (a wave, or 16 lanes) go the same way.
#pragma once

#include <setjmp.h>
#include <ucontext.h>

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <vector>

typedef int hipError_t;
typedef struct ihipStream_t *hipStream_t;
constexpr hipError_t hipSuccess = 0;
inline hipError_t hipGetLastError() { return hipSuccess; }

#define __global__
#define __device__
#define __host__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define address_space(n)

struct dim3 {
    unsigned x = 1, y = 1, z = 1;
    dim3(unsigned x, unsigned y = 1, unsigned z = 1) : x(x), y(y), z(z) {}
};

namespace lanes {

// The kernel does what this file does not provide for.
[[noreturn]] inline void stop(const char *what)
{
    fprintf(stderr, "lanes: %s\n", what);
    abort();
}

enum Kind { kFence, kBallot, kDpp, kSwap16, kSwap32, kReadLane, kReadFirst, kShuffle, kTranspose, kMatrix, kBarrier, kDone, kRun };

struct Lane {
    ucontext_t context;     // its start
    jmp_buf here;           // where it waits
    bool started;
    unsigned id;
    Kind kind;
    int control;        // of which lanes that meet have the same
    unsigned from;      // lane that is read
    uint32_t in, in2, out, out2;
    int16_t part[4];    // kTranspose: read, and result
    float a[8], b[8];   // kMatrix: a row of each operand
    float c[4];
    struct Load {
        char *to;
        char bytes[16];
    };
    std::vector<Load> loads;    // on their way to LDS
};
inline bool early, backwards;

struct Index {
    unsigned x, y, z;
};
inline Index block, grid, dim;
inline Lane *lane_now;
inline jmp_buf scheduler;
inline std::function<void()> body;

__attribute__((noinline)) inline void resume(Lane *l)
{
    lane_now = l;
    if (_setjmp(scheduler) != 0) return;
    if (l->started) _longjmp(l->here, 1);
    l->started = true;
    setcontext(&l->context);
}

__attribute__((noinline)) inline void pause()
{
    if (_setjmp(lane_now->here) == 0) _longjmp(scheduler, 1);
}

inline void wait(Kind kind, int control = 0)
{
    lane_now->kind = kind;
    lane_now->control = control;
    pause();
}

inline void enter()
{
    body();
    wait(kDone);
}

// The operation that the lanes `some` of a wave wait at.
inline void join(Lane *wave, uint64_t some)
{
    const auto has = [&](unsigned l) { return l < 64 && (some >> l & 1) != 0; };
    const auto read = [&](unsigned l) { return has(l) ? wave[l].in : 0u; };
    for (unsigned l = 0; l < 64; ++l) {
        if (!has(l)) continue;
        Lane &me = wave[l];
        const unsigned row = l & ~15u, i = l & 15;
        switch (me.kind) {
        case kDpp:
            switch (me.control) {
            case 0xB1: me.out = read(l ^ 1); break;
            case 0x4E: me.out = read(l ^ 2); break;
            case 0x1B: me.out = read(l ^ 3); break;
            case 0x141: me.out = read(l ^ 7); break;
            case 0x140: me.out = read(l ^ 15); break;
            case 0x128: me.out = read(row + ((i + 8) & 15)); break;
            default: stop("an unknown move within 16 lanes");
            }
            break;
        case kSwap16:
            me.out = l & 16 ? (has(l - 16) ? wave[l - 16].in2 : 0) : me.in;
            me.out2 = l & 16 ? me.in2 : read(l + 16);
            break;
        case kSwap32:
            me.out = l & 32 ? (has(l - 32) ? wave[l - 32].in2 : 0) : me.in;
            me.out2 = l & 32 ? me.in2 : read(l + 32);
            break;
        case kBallot: {
            uint64_t mask = 0;
            for (unsigned k = 0; k < 64; ++k) mask |= has(k) && wave[k].in ? uint64_t(1) << k : 0;
            me.out = static_cast<uint32_t>(mask);
            me.out2 = static_cast<uint32_t>(mask >> 32);
            break;
        }
        case kReadLane:
            if (!has(me.from)) stop("a value is read of a lane that is elsewhere");
            me.out = read(me.from);
            break;
        case kTranspose:
        case kMatrix: break;
        case kShuffle: me.out = read(row + me.from); break;
        case kReadFirst: me.out = read(static_cast<unsigned>(__builtin_ctzll(some))); break;
        default: break;
        }
    }
    // 16 lanes' 4 elements each, 4 rows of 16: a lane gets a column.
    const Kind kind = wave[__builtin_ctzll(some)].kind;
    if (kind == kTranspose) {
        int16_t got[64][4];
        for (unsigned l = 0; l < 64; ++l)
            for (unsigned j = 0; j < 4; ++j) got[l][j] = wave[(l & ~15u) + j * 4 + (l & 15) / 4].part[l & 3];
        for (unsigned l = 0; l < 64; ++l) memcpy(wave[l].part, got[l], 8);
    }
    // Lane l has row l & 15 of each operand at k = (l >> 4) * 8 .., and result rows (l >> 4) * 4 ..
    // of column l & 15.
    if (kind == kMatrix) {
        float a[16][32], b[32][16];
        for (unsigned l = 0; l < 64; ++l)
            for (unsigned k = 0; k < 8; ++k) {
                a[l & 15][l / 16 * 8 + k] = wave[l].a[k];
                b[l / 16 * 8 + k][l & 15] = wave[l].b[k];
            }
        for (unsigned row = 0; row < 16; ++row) {
            float c[16] = {};
            for (unsigned k = 0; k < 32; ++k)
                for (unsigned n = 0; n < 16; ++n) c[n] += a[row][k] * b[k][n];
            for (unsigned n = 0; n < 16; ++n) wave[row / 4 * 16 + n].c[row % 4] += c[n];
        }
    }
    if ((kind == kTranspose || kind == kMatrix) && some != ~uint64_t(0)) stop("part of a wave at a matrix");
    for (unsigned l = 0; l < 64; ++l)
        if (has(l)) wave[l].kind = kRun;
}

inline void arrive(Lane &l, size_t pending)
{
    const size_t n = l.loads.size() > pending ? l.loads.size() - pending : 0;
    for (size_t i = 0; i < n; ++i) memcpy(l.loads[i].to, l.loads[i].bytes, 16);
    l.loads.erase(l.loads.begin(), l.loads.begin() + n);
}

template <typename F>
void launch(dim3 blocks, unsigned threads, F &&f)
{
    static std::vector<Lane> lanes(1024);
    static std::vector<char> stacks(size_t(1024) << 16);
    if (threads % 64 != 0 || threads > 1024) stop("a workgroup of part of a wave, or of more than 1024");
    body = f;
    grid = {blocks.x, blocks.y, 1};
    dim = {threads, 1, 1};
    for (unsigned b = 0; b < blocks.x * blocks.y; ++b) {
        block = {b % blocks.x, b / blocks.x, 0};
        for (unsigned i = 0; i < threads; ++i) {
            Lane &l = lanes[i];
            l.id = i;
            l.kind = kRun;
            l.started = false;
            l.loads.clear();
            getcontext(&l.context);
            l.context.uc_stack.ss_sp = stacks.data() + (size_t(i) << 16);
            l.context.uc_stack.ss_size = size_t(1) << 16;
            l.context.uc_link = nullptr;
            makecontext(&l.context, enter, 0);
        }
        for (;;) {
            unsigned done = 0, waiting = 0;
            for (unsigned w = 0; w < threads; w += 64) {
                Lane *wave = &lanes[backwards ? threads - 64 - w : w];
                for (;;) {
                    int first = -1;
                    for (int i = 0; i < 64; ++i) {
                        if (wave[i].kind == kRun) resume(&wave[i]);
                        if (first < 0 && wave[i].kind < kBarrier) first = i;
                    }
                    if (first < 0) break;
                    uint64_t some = 0;
                    for (int i = 0; i < 64; ++i)
                        if (wave[i].kind == wave[first].kind && wave[i].control == wave[first].control)
                            some |= uint64_t(1) << i;
                    join(wave, some);
                }
                for (int i = 0; i < 64; ++i) (wave[i].kind == kDone ? done : waiting) += 1;
            }
            if (waiting == 0) break;
            if (done != 0) stop("a barrier that some lanes do not reach");
            for (unsigned i = 0; i < threads; ++i) lanes[i].kind = kRun;
        }
    }
    body = nullptr;
}

struct Pair {
    uint32_t v[2];
    uint32_t operator[](int i) const { return v[i]; }
};
inline Pair swap(Kind kind, uint32_t a, uint32_t b)
{
    lane_now->in = a;
    lane_now->in2 = b;
    wait(kind);
    return {{lane_now->out, lane_now->out2}};
}
inline uint32_t move(Kind kind, uint32_t x, int control = 0, unsigned from = 0)
{
    lane_now->in = x;
    lane_now->from = from;
    wait(kind, control);
    return lane_now->out;
}
inline uint64_t ballot(bool x, int line)
{
    lane_now->in = x;
    wait(kBallot, line);
    return static_cast<uint64_t>(lane_now->out2) << 32 | lane_now->out;
}
inline uint32_t below(uint64_t mask) { return __builtin_popcountll(mask & ((uint64_t(1) << (lane_now->id & 63)) - 1)); }
template <typename V>
V transpose(const V *p)
{
    memcpy(lane_now->part, p, 8);
    wait(kTranspose);
    V v;
    memcpy(&v, lane_now->part, 8);
    return v;
}
template <typename V, typename C>
C matrix(const V &a, const V &b, const C &c)
{
    for (int i = 0; i < 8; ++i) {
        lane_now->a[i] = static_cast<float>(a[i]);
        lane_now->b[i] = static_cast<float>(b[i]);
    }
    memcpy(lane_now->c, &c, 16);
    wait(kMatrix);
    C out;
    memcpy(&out, lane_now->c, 16);
    return out;
}
inline void load(const void *from, void *lds, unsigned offset)
{
    Lane::Load l;
    l.to = static_cast<char *>(lds) + (lane_now->id & 63) * 16;
    memcpy(l.bytes, static_cast<const char *>(from) + offset, 16);
    lane_now->loads.push_back(l);
    if (early) arrive(*lane_now, 0);
}
inline void waitcnt(unsigned n) { arrive(*lane_now, (n & 15) | (n >> 14 & 3) << 4); }

inline Index thread() { return {lane_now->id, 0, 0}; }

template <typename T>
T fetch(T *p, T v, T (*f)(T, T))
{
    const T was = *p;
    *p = f(was, v);
    return was;
}

}  // namespace lanes

#define threadIdx lanes::thread()
#define blockIdx lanes::block
#define gridDim lanes::grid
#define blockDim lanes::dim
#define __syncthreads() lanes::wait(lanes::kBarrier)
#define __ballot(x) lanes::ballot(x, __LINE__)
#define __shfl(x, l, width) static_cast<int>(lanes::move(lanes::kShuffle, x, __LINE__, l))
#define __builtin_amdgcn_fence(...) lanes::wait(lanes::kFence, __LINE__)
#define __builtin_amdgcn_wave_barrier() (void)0
#define __builtin_amdgcn_update_dpp(old, x, control, rows, banks, bound) \
    static_cast<int>(lanes::move(lanes::kDpp, static_cast<uint32_t>(x), control))
#define __builtin_amdgcn_permlane16_swap(a, b, x, y) lanes::swap(lanes::kSwap16, a, b)
#define __builtin_amdgcn_permlane32_swap(a, b, x, y) lanes::swap(lanes::kSwap32, a, b)
#define __builtin_amdgcn_readlane(x, l) lanes::move(lanes::kReadLane, static_cast<uint32_t>(x), __LINE__, l)
#define __builtin_amdgcn_readfirstlane(x) \
    static_cast<int>(lanes::move(lanes::kReadFirst, static_cast<uint32_t>(x), __LINE__))
#define __builtin_amdgcn_mbcnt_lo(mask, n) ((n) + lanes::below(mask))
#define __builtin_amdgcn_mbcnt_hi(mask, n) ((n) + lanes::below(static_cast<uint64_t>(mask) << 32))
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, size, flags) (p)
#define __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds, size, offset, add, at, cache) \
    lanes::load(from, lds, static_cast<unsigned>(offset))
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) lanes::transpose(p)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) lanes::matrix(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) lanes::matrix(a, b, c)
#define __builtin_amdgcn_s_waitcnt(n) lanes::waitcnt(n)
#define __builtin_amdgcn_s_barrier() lanes::wait(lanes::kBarrier)
#define __builtin_amdgcn_sched_barrier(x) (void)0
#define __builtin_amdgcn_sched_group_barrier(x, y, z) (void)0
#define __builtin_nontemporal_load(p) (*(p))
#define __builtin_nontemporal_store(v, p) (void)(*(p) = (v))

template <typename T, typename U>
T as(U x)
{
    T y;
    static_assert(sizeof x == sizeof y, "the same bits");
    memcpy(&y, &x, sizeof y);
    return y;
}
inline int __float_as_int(float x) { return as<int>(x); }
inline float __int_as_float(int x) { return as<float>(x); }
inline uint32_t __float_as_uint(float x) { return as<uint32_t>(x); }
inline float __uint_as_float(uint32_t x) { return as<float>(x); }
inline int __ffs(uint32_t x) { return __builtin_ffs(static_cast<int>(x)); }
inline int __popcll(uint64_t x) { return __builtin_popcountll(x); }
inline uint32_t atomicCAS(uint32_t *p, uint32_t was, uint32_t now)
{
    const uint32_t v = *p;
    if (v == was) *p = now;
    return v;
}
inline uint32_t atomicOr(uint32_t *p, uint32_t v) { return lanes::fetch<uint32_t>(p, v, [](uint32_t a, uint32_t b) { return a | b; }); }
inline int atomicAdd(int *p, int v) { return lanes::fetch<int>(p, v, [](int a, int b) { return a + b; }); }
using std::max;
using std::min;

// float to bfloat16, to nearest even: the compiler calls it where the processor cannot.  (The result
// is the low half of the register that a float comes back in.)
extern "C" inline __attribute__((used)) float to_bf16(float x) __asm__("__truncsfbf2");
extern "C" inline float to_bf16(float x)
{
    const uint32_t b = __float_as_uint(x);
    return __uint_as_float(x != x ? 0x7fc0 : (b + 0x7fff + (b >> 16 & 1)) >> 16);
}
