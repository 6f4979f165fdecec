// A matrix product of 16-bit operands on the matrix cores, one tile of the result
// per workgroup, left in registers for the caller to use.
//
//     C[m][n] = sum_k A(m, k) B(n, k),   float32 accumulation
//
// An operand lies either with k adjacent (rows m or n of k) or with m or n adjacent
// (rows k).  It is staged straight into LDS (16 bytes per lane).
//  * k adjacent: 64 k at a time, whole cache lines, into two buffers in turn.  LDS rows of 64 k
//    = 8 chunks of 16 bytes; chunk c of row r lies at place c ^ (r & 7), so that 8 rows read
//    at one c touch all banks once.
//  * m or n adjacent: 32 k at a time, into four buffers in turn.  LDS rows (k) of kSize
//    elements; fragments are read transposed (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16
//    elements and each lane gets a column), and pairs of chunks are permuted by the row
//    bits that such a read spans.
// Rows of m or n beyond an operand's end are read at its last row, and are the caller's to
// ignore.  At k beyond its end an operand gives other elements of its own (with k adjacent the
// last ones of the same row: what lies between its rows is not its own, and may be anything);
// the caller makes the other operand 0 there.
//
// The products run as 16 x 16 x 32 with the operands exchanged, so that a lane holds, for
// one m (lane & 15), four adjacent n ((lane >> 4) * 4 ..): a row's values meet in few
// lanes, and stores are 8 or 16 bytes.
//
// What bounds it: a step of 32 k is 32 products of 16 cycles for a wave of a large tile, in between
// its 12 fragments are read from LDS, and every load has two steps' time.  The kernels reach 1165
// to 1390 TFLOP/s at the 1.8 to 2.0 GHz that the card holds under this load (8192 x 65536 x
// 2048, bfloat16; 256 x 256 tiles of 8 waves, one workgroup a CU); bank conflicts are at most
// 1% of the LDS cycles (3.7% in dx_kernel, at the tile's end).  A tile's first loads and its end,
// 4 to 10 us, overlap with no products.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace cdk {

template <typename E>
struct Half;
template <>
struct Half<__bf16> {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    typedef __bf16 v4 __attribute__((ext_vector_type(4)));
};
template <>
struct Half<_Float16> {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    typedef _Float16 v4 __attribute__((ext_vector_type(4)));
};
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 product(Half<__bf16>::v8 a, Half<__bf16>::v8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(Half<_Float16>::v8 a, Half<_Float16>::v8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

constexpr int64_t kMostLd = int64_t(1) << 21;   // 256 rows stay within 2^30 bytes

template <typename E>
struct Operand {
    const E *data;      // 16-byte aligned
    int64_t ld;         // elements between rows, a multiple of 8, at most kMostLd
    int32_t rows;       // >= 1
    int32_t cols;       // a multiple of 8, >= 8
};

constexpr int kStepK = 64;       // k of two halves

// Staging and reading of one operand: kSize rows of m (or n) per tile, kWaves waves.  kTurn: k
// may start anywhere and goes round.  kOnce: the operand is read past the caches.  kWhole: with k
// adjacent, rows are whole steps of k.
// A lane's places relative to the tile and the step are 32-bit offsets that stay the same from
// step to step; the step moves a uniform pointer.
template <typename E, int kSize, bool kAcross, int kWaves, bool kTurn, bool kOnce, bool kWhole>
struct Stage {
    static constexpr int kK = kAcross ? kStepK / 2 : kStepK; // k at a time
    static constexpr int kBuffers = kAcross ? 4 : 2;
    static constexpr int kChunks = kSize * kK / 8;          // 16-byte chunks of them
    static constexpr int kLoads = kChunks / (kWaves * 64);  // per lane
    static constexpr int kRowChunks = kAcross ? kSize / 8 : kK / 8;
    static constexpr int kRowsPerLoad = 64 / kRowChunks;    // rows that a wave's load fills
    static constexpr int kBytes = kChunks * 16;

    const char *at;             // of the tile at the next load's k
    const char *final;          // m or n adjacent: the operand's last 16 bytes
    uint32_t tail;              // k adjacent: bytes of a row in the load that its end cuts
    int64_t stride;             // bytes between loads
    int64_t round;              // kTurn: bytes of all loads
    int32_t until;              // kTurn: loads until the last k; then the first comes
    int32_t whole;              // loads to come that lie within the operand
    uint32_t off[kLoads];       // bytes

    // Bits of a row (m or n adjacent) that permute its pairs of chunks.
    static __device__ __forceinline__ int permute(int r) { return (r & 3) | (r >> 1 & 4); }

    __device__ __forceinline__ void init(const Operand<E> &op, int64_t first, int64_t k0, int wave,
                                         int lane)
    {
        whole = static_cast<int32_t>(((kAcross ? op.rows : op.cols) - k0) / kK);
        stride = kK * (kAcross ? op.ld * 2 : 2);
        const int in_load = lane / kRowChunks, chunk = lane % kRowChunks;
        const uint32_t ld = static_cast<uint32_t>(op.ld) * 2;
        if (kAcross) {
            final = reinterpret_cast<const char *>(op.data + (op.rows - 1) * op.ld + op.cols - 8);
            at = reinterpret_cast<const char *>(op.data + k0 * op.ld);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = (i * kWaves + wave) * kRowsPerLoad + in_load;
                const int64_t c = first + ((chunk ^ (permute(r) << 1)) * 8);
                off[i] = r * ld + static_cast<uint32_t>(c < op.cols ? c : op.cols - 8) * 2;
            }
        } else {
            tail = static_cast<uint32_t>(op.cols % kK) * 2;
            const int64_t from = first < op.rows ? first : op.rows - 1;
            at = reinterpret_cast<const char *>(op.data + from * op.ld + k0);
            // Row bits 0..2 are in_load's: a load fills 8 rows.
            const uint32_t place = (chunk ^ (in_load & 7)) * 16;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int64_t r = first + (i * kWaves + wave) * kRowsPerLoad + in_load;
                off[i] = static_cast<uint32_t>((r < op.rows ? r : op.rows - 1) - from) * ld + place;
            }
        }
    }

    // The next k, kK of them.  A raw buffer: a uniform address and the lanes' 32-bit offsets.
    __device__ __forceinline__ void load(char *lds, int wave)
    {
        const auto put = [&](const char *from, int i, uint32_t o) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from), 0, -1, 0x00020000),
                (__attribute__((address_space(3))) void *)(lds + (i * kWaves + wave) * 1024), 16,
                static_cast<int>(o), 0, 0, kOnce ? 2 : 0);     // (2: non-temporal)
        };
        if ((!kAcross && kWhole) || __builtin_expect(whole > 0, 1)) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) put(at, i, off[i]);
        } else if (!kAcross) {      // past a row's end its last 16 bytes
            const uint32_t lane = threadIdx.x & 63;
            const uint32_t place = (lane % kRowChunks ^ (lane / kRowChunks & 7)) * 16;
            const uint32_t back = place < tail ? 0 : place - (tail - 16);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) put(at, i, off[i] - back);
        } else {    // past the operand's end its last 16 bytes
            const char *from = min(at, final);
            const uint32_t last = static_cast<uint32_t>(min(final - from, int64_t(1) << 31));
#pragma unroll
            for (int i = 0; i < kLoads; ++i) put(from, i, min(off[i], last));
        }
        --whole;
        at += stride;
        if (kTurn && --until == 0) at -= round;
    }
    // kTurn: begin with load number `first` of the n (whole) ones.
    __device__ __forceinline__ void start(int first, int n)
    {
        at += first * stride;
        round = n * stride;
        until = n - first;
    }

    // This lane's places in a staged tile for its fragments of the wave's rows, first the
    // tile's row: one for each fragment, or (k adjacent) one for each half.
    static constexpr int kPlaces(int frags) { return kAcross ? frags : 2; }
    static constexpr int kReads = kAcross ? 2 : 1;          // LDS reads of a fragment
    static __device__ __forceinline__ int place_of(int first, int i, int lane)
    {
        if (kAcross) {
            const int r = (lane >> 4) * 8 + (lane >> 2 & 3);
            return r * (kSize * 2) + ((first / 16 + i) ^ permute(r)) * 32 + (lane & 3) * 8;
        }
        return (first + (lane & 15)) * (kK * 2) + ((i * 4 + (lane >> 4)) ^ (lane & 7)) * 16;
    }
    // The 8 values of k = half * 32 + (lane >> 4) * 8 .. of its row of fragment i.
    static __device__ __forceinline__ typename Half<E>::v8 read(const char *lds, const int *places,
                                                                int i, int half)
    {
        union {
            typename Half<E>::v8 v;
            s16x4 h[2];
        } f;
        if (kAcross) {
            const char *p = lds + places[i];
            f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)p);
            f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)(p + 4 * kSize * 2));
        } else {
            f.v = *reinterpret_cast<const typename Half<E>::v8 *>(lds + places[half] +
                                                                  i * 16 * (kK * 2));
        }
        return f.v;
    }
    // Where the step s (of 32 k) lies.
    static __device__ __forceinline__ int buffer(int s)
    {
        return (kAcross ? s & 3 : s >> 1 & 1) * kBytes;
    }
};

// kTileM x kTileN per workgroup of kWavesM x kWavesN waves.  A's columns are a multiple of kStepK
// where its k is adjacent; so are B's with kTurn.
template <typename E, int kTileM, int kTileN, int kWavesM, int kWavesN, bool kAcrossA, bool kAcrossB,
          bool kTurn = false, bool kOnceB = false>
struct TileProduct {
    static constexpr int kWaves = kWavesM * kWavesN;
    static constexpr int kThreads = kWaves * 64;
    static constexpr int kWaveM = kTileM / kWavesM, kWaveN = kTileN / kWavesN;
    static constexpr int kM = kWaveM / 16, kN = kWaveN / 16;
    typedef Stage<E, kTileM, kAcrossA, kWaves, kTurn, false, true> A;
    typedef Stage<E, kTileN, kAcrossB, kWaves, kTurn, kOnceB, kTurn> B;

    // Loads of a wave with every step (of 32 k) and with every other one.
    static constexpr int kEach = (kAcrossA ? A::kLoads : 0) + (kAcrossB ? B::kLoads : 0);
    static constexpr int kOther = (kAcrossA ? 0 : A::kLoads) + (kAcrossB ? 0 : B::kLoads);

    struct Frags {
        typename Half<E>::v8 a[2][kM], b[2][kN];
    };

    // The products of one step, and in between the reads of the next step's fragments.
    static __device__ __forceinline__ void half_step(int half, const char *next_a,
                                                     const char *next_b, const int *places_a,
                                                     const int *places_b, Frags &f,
                                                     f32x4 (&acc)[kM][kN])
    {
#pragma unroll
        for (int j = 0; j < kN; ++j) f.b[half ^ 1][j] = B::read(next_b, places_b, j, half ^ 1);
#pragma unroll
        for (int i = 0; i < kM; ++i) f.a[half ^ 1][i] = A::read(next_a, places_a, i, half ^ 1);
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j)
                acc[i][j] = product(f.b[half][j], f.a[half][i], acc[i][j]);
        constexpr int kReads = kM * A::kReads + kN * B::kReads;
        constexpr int kPer = kM * kN / kReads > 0 ? kM * kN / kReads : 1;
#pragma unroll
        for (int r = 0; r < kReads; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // a read from LDS
            __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);   // products
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    // All waves are here, and of a wave's loads at most the last kPending are under way; kReads:
    // nor any of its LDS reads.
    template <int kPending, bool kReads>
    static __device__ __forceinline__ void meet()
    {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt((kReads ? 0x0070 : 0x0f70) | kPending);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }

    // Steps s and s + 1 (s even).  Each begins when the next step's loads have arrived
    // everywhere.  At step s the buffers of s - 1 (m or n adjacent) are read no more and take
    // the loads of s + 3; at step s + 1 those of s take s + 4's, and what is staged 64 k at a
    // time, all read by then, takes s + 4's and s + 5's.  So every load has two steps' time.
    static __device__ __forceinline__ void two_steps(A &sa, B &sb, int s, int steps, int wave,
                                                     char *a_s3, char *a_s4, char *b_s3,
                                                     char *b_s4, const char *a_s1,
                                                     const char *a_s2, const char *b_s1,
                                                     const char *b_s2, const int *places_a,
                                                     const int *places_b, Frags &f,
                                                     f32x4 (&acc)[kM][kN])
    {
        if (kEach > 0) {
            if (s + 2 < steps) meet<kEach + kOther, false>();
            else meet<0, false>();
            if (s + 3 < steps) {
                if (kAcrossA) sa.load(a_s3, wave);
                if (kAcrossB) sb.load(b_s3, wave);
            }
        }
        half_step(0, a_s1, b_s1, places_a, places_b, f, acc);
        if (s + 3 < steps) meet<kEach, (kOther > 0)>();
        else meet<0, (kOther > 0)>();
        if (s + 4 < steps) {
            if (!kAcrossA) sa.load(a_s4, wave);
            if (!kAcrossB) sb.load(b_s4, wave);
            if (kAcrossA) sa.load(a_s4, wave);
            if (kAcrossB) sb.load(b_s4, wave);
        }
        half_step(1, a_s2, b_s2, places_a, places_b, f, acc);   // (at the end: of what is not used)
    }

    // Different buffers are told apart by `restrict`: otherwise the compiler has every read wait
    // for all loads to LDS.  Where both k are adjacent, each buffer is in its place again after
    // four steps (s a multiple of 4); else the four of m or n adjacent are all different within
    // two.
    static __device__ __forceinline__ void four_steps(A &sa, B &sb, int s, int steps, int wave,
                                                      char *__restrict__ a0, char *__restrict__ a1,
                                                      char *__restrict__ b0, char *__restrict__ b1,
                                                      const int *places_a, const int *places_b,
                                                      Frags &f, f32x4 (&acc)[kM][kN])
    {
        two_steps(sa, sb, s, steps, wave, a1, a0, b1, b0, a0, a1, b0, b1, places_a, places_b, f, acc);
        if (s + 2 < steps)
            two_steps(sa, sb, s + 2, steps, wave, a0, a1, b0, b1, a1, a0, b1, b0, places_a, places_b, f,
                      acc);
    }
    // (With k adjacent the buffer of step s + 1 is that of s + 4.)
    static __device__ __forceinline__ void two_steps_across(
        A &sa, B &sb, int s, int steps, int wave, char *__restrict__ a_s3, char *__restrict__ a_s4,
        char *__restrict__ b_s3, char *__restrict__ b_s4, const char *__restrict__ a_s1,
        const char *__restrict__ a_s2, const char *__restrict__ b_s1,
        const char *__restrict__ b_s2, const int *places_a, const int *places_b, Frags &f,
        f32x4 (&acc)[kM][kN])
    {
        two_steps(sa, sb, s, steps, wave, a_s3, a_s4, b_s3, b_s4, kAcrossA ? a_s1 : a_s4, a_s2,
                  kAcrossB ? b_s1 : b_s4, b_s2, places_a, places_b, f, acc);
    }

    // acc[i][j][r] = C[m0 + wm + i * 16 + (lane & 15)][n0 + wn + j * 16 + (lane >> 4) * 4 + r]
    // for k in [k0, k1), k0 a multiple of kStepK; every wave of the workgroup calls it.  k runs
    // on to a multiple of kStepK: up to there one operand is 0, or has no elements but the other is.
    // lds_a, lds_b: kBuffers buffers of each operand; free once all waves are past a barrier.
    // kTurn (k adjacent, a multiple of kStepK): the step to begin with is first % steps.
    static __device__ __forceinline__ void run(const Operand<E> &a, const Operand<E> &b, int64_t m0,
                                               int64_t n0, int64_t k0, int64_t k1, char *lds_a,
                                               char *lds_b, f32x4 (&acc)[kM][kN], uint32_t first = 0)
    {
        Loads l;
        begin(l, a, b, m0, n0, k0, k1, lds_a, lds_b, first);
        finish(l, lds_a, lds_b, acc);
    }

    // run() in two: begin() asks for the first loads, finish() does the rest.
    struct Loads {
        A sa;
        B sb;
        int steps;
    };
    static __device__ __forceinline__ void begin(Loads &l, const Operand<E> &a, const Operand<E> &b,
                                                 int64_t m0, int64_t n0, int64_t k0, int64_t k1,
                                                 char *lds_a, char *lds_b, uint32_t first = 0)
    {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        l.sa.init(a, m0, k0, wave, lane);
        l.sb.init(b, n0, k0, wave, lane);
        const int steps = l.steps = static_cast<int>((k1 - k0 + kStepK - 1) / kStepK) * 2;
        if (steps <= 0) return;
        if (kTurn) {
            static_assert(!kTurn || (!kAcrossA && !kAcrossB), "k adjacent");
            l.sa.start(static_cast<int>(first % (steps / 2)), steps / 2);
            l.sb.start(static_cast<int>(first % (steps / 2)), steps / 2);
        }
        for (int s = 0; s < 4 && s < steps; ++s) {
            if (kAcrossA ? s < 3 : s % 2 == 0) l.sa.load(lds_a + A::buffer(s), wave);
            if (kAcrossB ? s < 3 : s % 2 == 0) l.sb.load(lds_b + B::buffer(s), wave);
        }
    }
    static __device__ __forceinline__ void finish(Loads &l, char *lds_a, char *lds_b,
                                                  f32x4 (&acc)[kM][kN])
    {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave / kWavesN * kWaveM, wn = wave % kWavesN * kWaveN;
        const int steps = l.steps;
        A &sa = l.sa;
        B &sb = l.sb;
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (steps <= 0) return;
        int places_a[A::kPlaces(kM)], places_b[B::kPlaces(kN)];
#pragma unroll
        for (int i = 0; i < A::kPlaces(kM); ++i) places_a[i] = A::place_of(wm, i, lane);
#pragma unroll
        for (int i = 0; i < B::kPlaces(kN); ++i) places_b[i] = B::place_of(wn, i, lane);
        meet<0, false>();
        Frags f;
#pragma unroll
        for (int j = 0; j < kN; ++j) f.b[0][j] = B::read(lds_b, places_b, j, 0);
#pragma unroll
        for (int i = 0; i < kM; ++i) f.a[0][i] = A::read(lds_a, places_a, i, 0);
        if constexpr (kEach == 0) {
            for (int s = 0; s < steps; s += 4)
                four_steps(sa, sb, s, steps, wave, lds_a, lds_a + A::kBytes, lds_b, lds_b + B::kBytes,
                           places_a, places_b, f, acc);
        } else {
            for (int s = 0; s < steps; s += 2)
                two_steps_across(sa, sb, s, steps, wave, lds_a + A::buffer(s + 3),
                                 lds_a + A::buffer(s + 4), lds_b + B::buffer(s + 3),
                                 lds_b + B::buffer(s + 4), lds_a + A::buffer(s + 1),
                                 lds_a + A::buffer(s + 2), lds_b + B::buffer(s + 1),
                                 lds_b + B::buffer(s + 2), places_a, places_b, f, acc);
        }
    }

    // A wave's results as 16-bit rows of 64 columns, by way of LDS: from four columns of 16 rows
    // a register to 16 bytes a lane, whole cache lines.  After a barrier behind run().
    static_assert(kWaveN == 64, "a row is 128 bytes");
    static constexpr int kOutBytes = kWaveM * 128;
    static __device__ __forceinline__ char *out_lds(char *lds_a, char *lds_b)
    {
        constexpr int kInA = A::kBuffers * A::kBytes / kOutBytes;
        static_assert(kWaves <= kInA + B::kBuffers * B::kBytes / kOutBytes, "the waves' rows fit");
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        return wave < kInA ? lds_a + wave * kOutBytes : lds_b + (wave - kInA) * kOutBytes;
    }
    // Columns j * 16 + (lane >> 4) * 4 .. of row i * 16 + (lane & 15).
    static __device__ __forceinline__ void out_put(char *lds, int i, int j, typename Half<E>::v4 v)
    {
        const int lane = threadIdx.x & 63, r = i * 16 + (lane & 15), c = j * 2 + (lane >> 5);
        *reinterpret_cast<typename Half<E>::v4 *>(lds + r * 128 + (c ^ (r & 7)) * 16 +
                                                  (lane >> 4 & 1) * 8) = v;
    }
    // Columns (lane & 7) * 8 .. of row t * 8 + (lane >> 3), t < kWaveM / 8.
    static __device__ __forceinline__ typename Half<E>::v8 out_get(const char *lds, int t)
    {
        const int lane = threadIdx.x & 63, r = t * 8 + (lane >> 3);
        return *reinterpret_cast<const typename Half<E>::v8 *>(lds + r * 128 +
                                                               ((lane & 7) ^ (r & 7)) * 16);
    }
};

// Tile (tm, tn) of workgroup `id` of tiles_m x tiles_n.  Workgroups go to the 8 XCDs in
// turn; each XCD gets a range of tiles, walked in bands of 8 tiles of m, so that the
// workgroups that run together on it share rows of both operands in its L2.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t *tm,
                                        uint32_t *tn)
{
    const uint32_t n = tiles_m * tiles_n, xcd = id % 8, q = n / 8, rest = n % 8;
    const uint32_t at = xcd * q + (xcd < rest ? xcd : rest) + id / 8;
    const uint32_t band = at / (8 * tiles_n), in_band = at - band * 8 * tiles_n;
    const uint32_t height = min(8u, tiles_m - band * 8);
    *tm = band * 8 + in_band % height;
    *tn = in_band / height;
}

}  // namespace cdk
