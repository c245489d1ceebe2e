// Gated feed-forward block on gfx950: y = (act(x Wg^T) o (x Wu^T)) Wd^T and its
// gradients, as matrix products with the activation in their epilogues.
//
// One tiled product serves every part: a workgroup forms a BM x BN tile of C,
// its operands streamed through LDS 128 bytes of k at a time by loads that go
// straight there, two stages deep, and multiplied on the matrix cores (bf16:
// 16x16x32, fp32: 16x16x4, accumulated in fp32).  The two gates are one
// product whose B tile holds rows of Wg and of Wu in turn, so that a lane
// holds g and u of the same elements.  Operands whose k runs down the rows
// (the gradients') are read out of LDS with the transposing read.
//
// Tiles: 256 x 256 in bf16 (eight waves of 128 x 64, a compute unit to itself)
// where there are enough of them, 128 x 128 (four of 64 x 64, two workgroups a
// unit) elsewhere; 128 and 64 in fp32.  The larger a wave's tile, the fewer bytes
// of LDS a product: a step of the large one reads 192 KB and writes 64 KB for
// 2048 cycles of the matrix units.  8192 tokens, 2048 -> 8192 in bf16: 650 us, 442
// the gates and 204 the way back (1240 and 1350 TFLOP/s; a library's products of
// these sizes 1450 and 1580).  The matrix units are busy 57 and 62% of the cycles
// (44% in the gates' backward) at a clock of 2.07 GHz, without LDS conflicts: the
// clock, 2.4 with little at work, costs a seventh, and for two cycles of five
// the units wait, for a stage's loads (all of them, once a step: a step takes 1.1
// us with 32 compute units at work and 1.54 with all 256) and in the epilogues,
// which nothing else hides (5 us a round of tiles, 22 in the backward, whose gates
// read dh and write three arrays).  fp32: the matrix units, 140 TFLOP/s of the
// library's 154 (2048 tokens, 2048 -> 8192); small products lose a third of it to
// the last round of tiles.
//
// Roundings: sums, g, u, the activation and dh stay in fp32.  In bf16 h, dg and du
// are rounded to bf16 once, as operands of the next product: the matrix units take
// bf16 pairs, and keeping the cut-off part as a second operand would double
// those products.  A result is then off by 0.0023 of its size (root mean square)
// where its own rounding alone would leave 0.0017.
//
// Edges: buffer loads return zero past the end of an operand, so rows past M,
// N or (turned) K need no masks; k past K within a row is sent out of range.
#include <algorithm>
#include <cmath>

#include "m3_device.h"
#include "m3_ffn.h"
#include "m3_scan_common.h"

namespace m3 {
namespace ffn {
namespace {

using scan::Rsrc;
using scan::make_rsrc;

constexpr int kRowBytes = 128;              // bytes of k a stage
constexpr uint32_t kOut = 0x80000000u;      // an offset past every operand's end

// Where a 16-byte piece of an LDS row is stored: pieces are moved within their
// row so that the rows one read takes lie on different banks.
// [row][k] tiles: rows of eight pieces, piece g of row r at g ^ spread(r).
template <bool kPair> __device__ __forceinline__ int spread(int row) {
    return kPair ? (row & 3) | (row >> 1 & 4) : row & 7;
}
// [k][row] tiles: blocks of 16 elements, block b of k-row r at b ^ turn(r).
template <typename T> __device__ __forceinline__ int turn(int k) {
    return sizeof(T) == 2 ? (k & 3) | (k >> 1 & 4) : k >> 2 & 3;
}

// A buffer resource's words, in scalar registers
typedef int Words __attribute__((ext_vector_type(4)));
__device__ __forceinline__ Words make_words(const void *base, uint32_t bytes) {
    const uint64_t p = (uint64_t)(uintptr_t)base;
    return Words{(int)(uint32_t)p, (int)(uint32_t)(p >> 32), (int)bytes, 0x00020000};
}

// One 16-byte piece a lane from `off` bytes into a buffer to LDS: lane l's goes
// to `to` + 16 l.  In assembly, so that the compiler, which cannot tell the two
// stages apart, does not wait for these loads before it reads the other stage:
// the kernel waits for them itself (vmcnt 0 and a barrier) before it reads
// theirs.  (The loads write no register.)
__device__ __forceinline__ void load_lds(Words r, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(r)
                 : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const char *p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}

// An operand tile's loads: ROWS rows of the operand by 128 bytes of k.
template <typename T, int ROWS, int NW, bool kTurned, bool kPair> struct Tile {
    static constexpr int EL = 16 / sizeof(T), BK = kRowBytes / sizeof(T);
    static constexpr int PR = ROWS * sizeof(T) / 16;               // pieces of a turned row
    static constexpr int RPI = kTurned ? 64 / (PR < 64 ? PR : 64) : 8;   // LDS rows an instruction
    static constexpr int NI = ROWS * kRowBytes / 1024 / NW;        // instructions a wave
    static_assert(ROWS * kRowBytes % (1024 * NW) == 0 && PR <= 64, "whole instructions");
    uint32_t off[NI];
    // k (turned: the row's place in the tile) of the lane's piece, and its offset
    __device__ __forceinline__ void init(int64_t ld, int wave, int lane) {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int row0 = (j * NW + wave) * RPI;
            if constexpr (kTurned) {
                const int row = row0 + lane / PR, pos = lane % PR;
                constexpr int PB = 16 * sizeof(T) / 16;            // pieces a block of 16 elements
                const int src = (pos / PB ^ turn<T>(row)) * PB + pos % PB;
                off[j] = (uint32_t)(row * (int)(ld * sizeof(T)) + src * 16);
            } else {
                const int row = row0 + lane / 8, src = (lane % 8) ^ spread<kPair>(row);
                off[j] = (uint32_t)(row * (int)(ld * sizeof(T)) + src * 16);
            }
        }
    }
    // k of instruction j's piece in a [row][k] tile
    __device__ __forceinline__ int k_of(int j, int wave, int lane) const {
        const int row = (j * NW + wave) * 8 + lane / 8;
        return ((lane % 8) ^ spread<kPair>(row)) * EL;
    }
};

// Bytes that up to `most` of `rows` rows take whose last ends with the 16-byte
// piece that holds its element cols - 1 (rows are padded to whole pieces).
template <typename T> __device__ __forceinline__ uint32_t span(int rows, int64_t ld, int cols, int most) {
    constexpr int EL = 16 / (int)sizeof(T);
    const int r = min(rows, most);
    return r <= 0 ? 0u : (uint32_t)(r - 1) * (uint32_t)(ld * sizeof(T)) + (uint32_t)((cols + EL - 1) / EL * 16);
}

// Operand fragments of 16 rows by 64 bytes of k (kk = 0, 1): lane (q, l16) holds
// 16 bytes of k of row l16.  `at` is where the lane's piece of the fragment is
// at kk = 0 in a [row][k] tile, and in a turned one at kk = 0 and for its first
// four (bf16) or one (fp32) of k.
template <typename T, int ROWS, bool kTurned, bool kPair>
__device__ __forceinline__ uint32_t frag_at(int row0, int i, int q, int l16) {
    if constexpr (!kTurned) {
        // (pairs of tiles: the tile's row r is column 8 (r / 4) + r % 4, + 4 in odd tiles, of 32)
        const int row = row0 + (kPair ? i / 2 * 32 + l16 / 4 * 8 + l16 % 4 + i % 2 * 4 : 16 * i + l16);
        return (uint32_t)(row * kRowBytes + (q ^ spread<kPair>(row)) * 16);
    } else {
        constexpr int W = ROWS * (int)sizeof(T);
        const int k = sizeof(T) == 2 ? 8 * q + l16 / 4 : 4 * q, blk = (row0 / 16 + i) ^ turn<T>(k);
        return (uint32_t)(k * W + blk * (16 * (int)sizeof(T)) + (sizeof(T) == 2 ? l16 % 4 * 8 : l16 * 4));
    }
}
template <typename T, int ROWS, bool kTurned>
__device__ __forceinline__ f32x4 frag(const char *tile, uint32_t at, int kk) {
    constexpr int W = ROWS * (int)sizeof(T);
    if constexpr (!kTurned) {
        return *reinterpret_cast<const f32x4 *>(tile + (at ^ (uint32_t)(kk * 64)));
    } else if constexpr (sizeof(T) == 2) {   // (rows k and k + 4, and k + 32, turn alike)
        const bf16x4 lo = scan::lds_tr4(reinterpret_cast<const bf16 *>(tile + at + kk * 32 * W));
        const bf16x4 hi = scan::lds_tr4(reinterpret_cast<const bf16 *>(tile + at + (kk * 32 + 4) * W));
        return __builtin_bit_cast(f32x4, scan::cat4(lo, hi));
    } else {                                 // (rows k .. k + 3, and k + 16, turn alike)
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float *>(tile + at + (kk * 16 + j) * W);
        return v;
    }
}
template <typename T> __device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c) {
    if constexpr (sizeof(T) == 2) {
        return Mma<bf16>::mma(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = Mma<float>::mma(a[j], b[j], c);
        return c;
    }
}

// Up to N values of a row (`cols` are left in it), in vectors that start on any
// element: the hardware takes them so, and rows of odd lengths need them
// (2730 columns of bf16, 777 tokens: 29.6 us the weights' gradients, 42.7
// in single elements).
template <typename O, int N> __device__ __forceinline__ void store_run(O *o, const float (&v)[N], int cols) {
    constexpr int W = sizeof(O) == 4 ? 4 : N;
    typedef O piece __attribute__((ext_vector_type(W), aligned(sizeof(O))));
    if (cols >= N) {
#pragma unroll
        for (int k = 0; k < N; k += W) {
            piece w;
#pragma unroll
            for (int e = 0; e < W; ++e) w[e] = (O)v[k + e];
            *reinterpret_cast<piece *>(o + k) = w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < cols) o[e] = (O)v[e];
    }
}

// act(g) = g sigmoid(p) and its derivative sigmoid(p) + g sigmoid(p) (1 - sigmoid(p)) p':
// SiLU with p = g, GELU's tanh form with p = 2 sqrt(2 / pi) (g + 0.044715 g^3)
__device__ __forceinline__ float act(float g, bool gelu, float &slope) {
    constexpr float kS = 1.59576912160573071176f, kC = 0.044715f;
    const float p = gelu ? kS * g * fmaf(kC, g * g, 1.f) : g;
    const float dp = gelu ? kS * fmaf(3.f * kC, g * g, 1.f) : 1.f;
    const float s = __builtin_amdgcn_rcpf(1.f + __expf(-p));
    const float f = g * s;
    // (where s (1 - s) has gone to zero, g p' may have overflowed: their product is zero)
    const float t = 1.f - s;
    slope = fmaf(t > 0.f && s > 0.f ? f * dp : 0.f, t, s);
    return s > 0.f ? f : 0.f * s;
}

// The waves a SIMD that the compiler schedules for.  Two in bf16, as many as
// shared memory lets in (8192 x 2048 x 8192 in tiles of 128: 227 us, 276 when it
// is left to choose).  In fp32 the gates and the products with B alone turned are
// better left to it (777 tokens, 1000 -> 2730: 71 us a product, 78 with two), the
// others not (68 us of a weight's gradient, 72).
template <typename T, bool kAT, bool kBT, Kind KIND> constexpr int waves() {
    return sizeof(T) == 4 && (KIND != kStore || (kBT && !kAT)) ? 1 : 2;
}

template <typename T, int BM, int BN, int NWM, int NWN, bool kAT, bool kBT, Kind KIND>
__global__ __launch_bounds__(NWM * NWN * 64, (waves<T, kAT, kBT, KIND>())) void k_gemm(GemmArgs g) {
    constexpr int NW = NWM * NWN, BK = kRowBytes / sizeof(T);
    constexpr int WM = BM / NWM, WN = BN / NWN, MT = WM / 16, NT = WN / 16;
    constexpr bool kGates = KIND == kGate || KIND == kGateBwd;
    constexpr bool kPair = !kBT;                 // n in the order that gives a lane eight in a row
    constexpr int NB = kGates ? BN / 2 : BN;     // columns of C a tile
    static_assert(!kGates || (WN == 64 && !kAT && !kBT), "a wave's 32 columns of g, then of u");
    __shared__ __attribute__((aligned(1024))) char lds[2][(BM + BN) * kRowBytes];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wm = wave / NWN, wn = wave % NWN, l16 = lane & 15, q = lane / 16;

    // (divisions leave their results in vector registers: back to scalar ones,
    // where addresses and resources are formed)
    auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int z = scalar((int)blockIdx.z / g.splits), split = scalar((int)blockIdx.z % g.splits);
    const bool third = kAT && z == 2;
    const int64_t M = third ? g.N : g.M, N = third ? g.M : g.N;
    const int64_t a_ld = third ? g.lda3 : g.lda, b_ld = third ? g.ldb3 : g.ldb, c_ld = third ? g.ldc3 : g.ldc;
    const int tiles_m = third ? g.tiles_n : g.tiles_m, tiles_n = third ? g.tiles_m : g.tiles_n;

    // Workgroups go to the XCDs in turn: each XCD gets a run of tiles, eight
    // rows of tiles at a time, column by column, so that what runs together
    // on an XCD shares operand rows in its L2.
    const int total = tiles_m * tiles_n, id = (int)blockIdx.x;
    const int xcd = id % 8, per = total / 8, rem = total % 8;
    const int t = xcd * per + min(xcd, rem) + id / 8;
    constexpr int GM = 8;
    const int grp = t / (GM * tiles_n), in = t % (GM * tiles_n);
    const int gm = min(GM, tiles_m - grp * GM);
    const int64_t m0 = (int64_t)scalar(grp * GM + in % gm) * BM, n0 = (int64_t)scalar(in / gm) * NB;

    Tile<T, BM, NW, kAT, false> ta;
    Tile<T, BN, NW, kBT, kPair> tb;
    ta.init(a_ld, wave, lane);
    if constexpr (kGates) {
        // LDS row r: column r % 32 of wave r / 64's part of Wg (r % 64 < 32) or Wu
#pragma unroll
        for (int j = 0; j < tb.NI; ++j) {
            const int row = (j * NW + wave) * 8 + lane / 8;
            tb.off[j] = (uint32_t)((row / 64 * 32 + row % 32) * (int)(b_ld * sizeof(T)) + ((lane % 8) ^ spread<kPair>(row)) * 16);
        }
    } else {
        tb.init(b_ld, wave, lane);
    }

    const int K = (int)g.K, nk = (K + BK - 1) / BK, steps = nk * g.nseg;
    const int it0 = scalar((int)((int64_t)steps * split / g.splits)), it1 = scalar((int)((int64_t)steps * (split + 1) / g.splits));
    // The tile's operands at k = 0 of the first and of the second product summed
    auto at0 = [](const void *p, bool turned, int64_t ld, int64_t r0) { return static_cast<const T *>(p) + (turned ? r0 : r0 * ld); };
    const T *pa0 = at0(g.a[kGates ? 0 : z], kAT, a_ld, m0), *pa1 = kGates ? pa0 : at0(g.a[(z + 1) & 1], kAT, a_ld, m0);
    const T *pb0 = at0(g.b[kGates ? 0 : z], kBT, b_ld, n0), *pb1 = at0(g.b[kGates ? 1 : (z + 1) & 1], kBT, b_ld, n0);
    if constexpr (kGates && NW == 8) {   // (a wave's rows are all of Wg, or all of Wu)
        if (wave >= 4) pb0 = pb1;
    }
    // A stage's resource: zero past the rows, past k, and after the last step.
    // No branches: the scalar work and the loads go in between the products.
    const uint32_t lda = (uint32_t)(a_ld * sizeof(T)), ldb = (uint32_t)(b_ld * sizeof(T));
    const uint32_t sa0 = kAT ? span<T>(1, 0, (int)(M - m0), 1) : span<T>((int)(M - m0), a_ld, K, BM);
    const uint32_t sb0 = kBT ? span<T>(1, 0, (int)(N - n0), 1) : span<T>((int)(N - n0), b_ld, K, NB);
    auto stage_rsrc = [&](const T *p, bool turned, uint32_t ld, uint32_t span0, int k0, bool in) {
        const int rows = min(K - k0, BK);
        const uint32_t n = turned ? (uint32_t)(rows - 1) * ld + span0 : span0 - (uint32_t)k0 * (uint32_t)sizeof(T);
        const char *base = reinterpret_cast<const char *>(p) + (turned ? (int64_t)k0 * ld : (int64_t)k0 * (int64_t)sizeof(T));
        return make_words(base, in ? n : 0u);
    };
    struct Stage {
        Words ra, rb, ru;
        int left;       // of k
        uint32_t to;
    };
    auto stage = [&](int it) {
        const bool in = it < it1, second = it >= nk;
        const int k0 = (second && g.nseg > 1 ? it - nk : it) * BK;
        Stage s;
        s.ra = stage_rsrc(second ? pa1 : pa0, kAT, lda, sa0, k0, in);
        s.rb = stage_rsrc(!kGates && second ? pb1 : pb0, kBT, ldb, sb0, k0, in);
        s.ru = kGates && NW != 8 ? stage_rsrc(pb1, kBT, ldb, sb0, k0, in) : s.rb;
        s.left = K - k0;
        s.to = lds_address(lds[0]) + (uint32_t)(it & 1) * (uint32_t)sizeof lds[0];
        return s;
    };
    auto load = [&](const Stage &s) {
#pragma unroll
        for (int j = 0; j < ta.NI; ++j) {
            uint32_t off = ta.off[j];
            if constexpr (!kAT) off = ta.k_of(j, wave, lane) >= s.left ? kOut : off;
            load_lds(s.ra, off, s.to + (j * NW + wave) * 1024);
        }
#pragma unroll
        for (int j = 0; j < tb.NI; ++j) {
            uint32_t off = tb.off[j];
            if constexpr (!kBT) off = tb.k_of(j, wave, lane) >= s.left ? kOut : off;
            load_lds(kGates && NW != 8 && j % 2 ? s.ru : s.rb, off, s.to + BM * kRowBytes + (j * NW + wave) * 1024);
        }
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // Where the lane's fragments are in a stage
    uint32_t fa_at[MT], fb_at[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) fa_at[i] = frag_at<T, BM, kAT, false>(wm * WM, i, q, l16);
#pragma unroll
    for (int j = 0; j < NT; ++j) fb_at[j] = BM * kRowBytes + frag_at<T, BN, kBT, kPair>(wn * WN, j, q, l16);
    auto read = [&](int it, int kk, f32x4 (&fa)[MT], f32x4 (&fb)[NT]) {
        const char *stage = lds[it & 1];
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[j] = frag<T, BN, kBT>(stage, fb_at[j], kk);
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[i] = frag<T, BM, kAT>(stage, fa_at[i], kk);
    };
    auto multiply = [&](const f32x4 (&fa)[MT], const f32x4 (&fb)[NT]) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mma<T>(fb[j], fa[i], acc[i][j]);
    };
    // One half of a stage is multiplied while the next half is read: the
    // matrix units never wait for LDS, and a stage's loads have a whole step
    // to land.  The schedule spreads the reads over the products.
    constexpr int kReads = MT * (kAT ? (sizeof(T) == 2 ? 2 : 4) : 1) + NT * (kBT ? (sizeof(T) == 2 ? 2 : 4) : 1);
    constexpr int kMmas = MT * NT * (sizeof(T) == 2 ? 1 : 4), kEach = kMmas / kReads > 0 ? kMmas / kReads : 1;
    auto interleave = [&]() {
#pragma unroll
        for (int k = 0; k < kReads; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);  // products
        }
    };
    f32x4 a0[MT], b0[NT], a1[MT], b1[NT];
    if (it0 < it1) {
        load(stage(it0));
        __builtin_amdgcn_s_waitcnt(0x0F70);   // (vmcnt 0: this wave's pieces have landed)
        __syncthreads();
        load(stage(it0 + 1));
        read(it0, 0, a0, b0);
    }
    for (int it = it0; it < it1; ++it) {
        read(it, 1, a1, b1);
        const Stage next = stage(it + 2);
        multiply(a0, b0);
        interleave();
        __builtin_amdgcn_s_waitcnt(0x0070);   // the next stage has landed, this one has been read
        __syncthreads();                      // by every wave
        load(next);
        __builtin_amdgcn_sched_barrier(0);    // (as early as can be)
        read(it + 1, 0, a0, b0);              // (past the last stage: zeros, never used)
        multiply(a1, b1);
        interleave();
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);       // (nothing may land in LDS after the workgroup's end)

    // A lane holds row m = l16 of each 16-row tile, and four columns of each of
    // the NT column tiles: 4 q .. 4 q + 3, or (pairs of tiles) 8 q .. 8 q + 7.
    const int64_t mw = m0 + wm * WM;
    if constexpr (kGates) {
        const int64_t n = n0 + wn * 32 + 8 * q;      // (ldc is a multiple of eight, bf16, or four)
        if (n >= c_ld) return;
        const bool gelu = g.gelu != 0;
        // (dh's rows are asked for at once, before the first is used: rows past the
        // last, and columns past a row's four in fp32, as zeros)
        const int w = min(8, (int)(c_ld - n));   // 8, or 4 in fp32
        f32x4 rows[KIND == kGateBwd ? MT : 1][2];
        if constexpr (KIND == kGateBwd) {
            const int left = __builtin_amdgcn_readfirstlane(min((int)(M - mw), WM)), row = (int)c_ld * 4;
            const Rsrc rs = make_rsrc(g.dh + mw * c_ld, left > 0 ? (uint32_t)(left * row) : 0u);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    rows[i][p] = scan::buf_load<f32x4>(rs, 4 * p < w ? (uint32_t)((16 * i + l16) * row + ((int)n + 4 * p) * 4) : kOut);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = mw + 16 * i + l16;
            if (m >= M) continue;
            float h[8], dg[8], du[8];
            const int64_t at = m * c_ld + n;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float gv = acc[i][e / 4][e % 4], uv = acc[i][2 + e / 4][e % 4];
                float slope;
                const float f = act(gv, gelu, slope);
                h[e] = f * uv;
                if constexpr (KIND == kGateBwd) {
                    const float dh = rows[i][e / 4][e % 4];
                    du[e] = dh * f;
                    dg[e] = dh * uv * slope;
                }
            }
            auto put = [&](void *dst, const float (&v)[8]) {
                T *p = static_cast<T *>(dst) + at;
                if constexpr (sizeof(T) == 2) {
                    bf16x8 o;
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = (bf16)v[e];
                    *reinterpret_cast<bf16x8 *>(p) = o;
                } else {
                    *reinterpret_cast<f32x4 *>(p) = f32x4{v[0], v[1], v[2], v[3]};
                    if (w == 8) *reinterpret_cast<f32x4 *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
                }
            };
            put(g.c[0], h);
            if constexpr (KIND == kGateBwd) {
                put(g.dg, dg);
                put(g.du, du);
            }
        }
    } else {
        constexpr int RUN = kPair ? 8 : 4;         // columns in a row a lane
        // (c or a part, in fp32 or the io dtype)
        auto store = [&](auto *c, int64_t ldc, int64_t cols) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int64_t m = mw + 16 * i + l16;
                if (m >= M) continue;
#pragma unroll
                for (int p = 0; p < NT; p += RUN / 4) {
                    const int64_t n = n0 + wn * WN + (kPair ? p / 2 * 32 + 8 * q : 16 * p + 4 * q);
                    float v[RUN];
#pragma unroll
                    for (int e = 0; e < RUN; ++e) v[e] = acc[i][p + e / 4][e % 4];
                    store_run(c + m * ldc + n, v, (int)(cols - n));
                }
            }
        };
        const int64_t part_ld = (N + 3) / 4 * 4;
        if (g.splits > 1) store(g.part + (int64_t)blockIdx.z * g.part_each, part_ld, part_ld);
        else if (g.f32_out) store(static_cast<float *>(g.c[z]), c_ld, N);
        else store(static_cast<T *>(g.c[z]), c_ld, N);
    }
}

// Sums of a product's parts, in order, to the io dtype or fp32: four columns a thread.
struct JoinArgs {
    const float *part;
    int64_t each;              // elements of a part
    int splits;
    int64_t M, N;              // (a third product is N x M)
    void *c[3];
    int64_t ldc, ldc3;
};
template <typename O> __global__ __launch_bounds__(256) void k_join(JoinArgs g) {
    const bool third = blockIdx.y == 2;
    const int64_t M = third ? g.N : g.M, N = third ? g.M : g.N, ldc = third ? g.ldc3 : g.ldc;
    const int64_t per = (N + 3) / 4, k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (k >= M * per) return;
    const int64_t m = k / per, n = k % per * 4;
    const float *p = g.part + (int64_t)blockIdx.y * g.splits * g.each + m * per * 4 + n;
    f32x4 v = *reinterpret_cast<const f32x4 *>(p);
    for (int s = 1; s < g.splits; ++s) v += *reinterpret_cast<const f32x4 *>(p + s * g.each);
    const float o[4] = {v[0], v[1], v[2], v[3]};
    store_run(static_cast<O *>(g.c[blockIdx.y]) + m * ldc + n, o, (int)(N - n));
}
hipError_t join(const JoinArgs &g, int batch, bool f32, hipStream_t s) {
    const dim3 grid((unsigned)((g.each / 4 + 255) / 256), (unsigned)batch), block(256);
    if (f32) k_join<float><<<grid, block, 0, s>>>(g);
    else k_join<bf16><<<grid, block, 0, s>>>(g);
    return hipGetLastError();
}

// Few rows of x: bound by reading the weights once.  A workgroup takes up to 16 RT
// rows of weights (of both gates), its waves interleaved pieces of k, U runs of
// 64 bytes of every row at a time; the weights are the MFMA's row operand straight from
// global memory (rows past the workgroup's out of range), x (read again by every
// workgroup, from the caches) its columns, 16 a tile.  The waves' sums meet in LDS.
// Without gates k may be split over workgroups too (the parts joined after).
// Loading x a unit ahead as well cost more in registers than it gave (5% more time
// at 48 tokens).  2048 -> 8192 in bf16: one token 12.1 us the gates (5.5 TB/s of
// weights), 9.2 the way back (3.6); 48 tokens 18 and 13, and 4 to join.
template <typename T, int TT, int RT, bool kGates>
__global__ __launch_bounds__(512) void k_few(FewArgs a) {
    constexpr int NW = 8, NM = kGates ? 2 : 1, U = NM * RT * TT >= 8 ? 2 : 4;
    constexpr int EL = 16 / sizeof(T), KS = 4 * EL;
    __shared__ f32x4 s_acc[NW][NM * TT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int l16 = lane & 15, q = lane / 16;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows;
    const Rsrc rx = make_rsrc(a.x, span<T>((int)a.T, a.ldx, (int)a.K, kFewRows));
    Rsrc rw[NM];
#pragma unroll
    for (int m = 0; m < NM; ++m)
        rw[m] = make_rsrc(static_cast<const T *>(a.w[m]) + r0 * a.ldw, span<T>((int)(a.R - r0), a.ldw, (int)a.K, a.rows));
    const uint32_t wo = (uint32_t)(l16 * (int)(a.ldw * sizeof(T)) + q * 16), wt = (uint32_t)(16 * (int)(a.ldw * sizeof(T)));
    const uint32_t xo = (uint32_t)(l16 * (int)(a.ldx * sizeof(T)) + q * 16), xt = (uint32_t)(16 * (int)(a.ldx * sizeof(T)));
    const int K = (int)a.K, all = (K + U * KS - 1) / (U * KS), split = (int)blockIdx.y;
    const int u0 = (int)((int64_t)all * split / a.splits), u1 = (int)((int64_t)all * (split + 1) / a.splits);

    f32x4 acc[RT][NM][TT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[i][m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 w[U][RT][NM];
    auto load_w = [&](int unit) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (unit * U + u) * KS;
            const bool in = k + q * EL < K;
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int m = 0; m < NM; ++m)
                    w[u][i][m] = scan::buf_load<f32x4>(rw[m], in ? wo + i * wt + (uint32_t)(k * (int)sizeof(T)) : kOut);
        }
    };
    // The wave's units of k, each workgroup from another one on: not all of them
    // ask for the same part of every row at once.
    const int count = max(0, (u1 - u0 - wave + NW - 1) / NW), turn = count ? (int)(blockIdx.x % (unsigned)count) : 0;
    auto unit_of = [&](int c) { return u0 + wave + (c + turn >= count ? c + turn - count : c + turn) * NW; };
    if (count) load_w(unit_of(0));
    for (int c = 0; c < count; ++c) {
        const int unit = unit_of(c);
        f32x4 x[U][TT], v[U][RT][NM];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (unit * U + u) * KS;
            const bool in = k + q * EL < K;
#pragma unroll
            for (int t = 0; t < TT; ++t)
                x[u][t] = scan::buf_load<f32x4>(rx, in ? xo + t * xt + (uint32_t)(k * (int)sizeof(T)) : kOut);
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int m = 0; m < NM; ++m) v[u][i][m] = w[u][i][m];
        }
        if (c + 1 < count) load_w(unit_of(c + 1));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int m = 0; m < NM; ++m) acc[i][m][t] = mma<T>(v[u][i][m], x[u][t], acc[i][m][t]);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int t = 0; t < TT; ++t) s_acc[wave][m * TT + t][lane] = acc[i][m][t];
        __syncthreads();
        // rows 4 q .. 4 q + 3 of the weights' tile, row l16 of x's
        for (int k = threadIdx.x; k < TT * 64; k += NW * 64) {
            const int t = k / 64, ln = k % 64;
            f32x4 sum[NM];
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                sum[m] = s_acc[0][m * TT + t][ln];
                for (int v = 1; v < NW; ++v) sum[m] += s_acc[v][m * TT + t][ln];
            }
            const int64_t col = t * 16 + ln % 16, r = r0 + 16 * i + ln / 16 * 4;
            if (col >= a.T || r >= a.Ro || 16 * i + ln / 16 * 4 >= a.rows) continue;
            if (!kGates && a.splits > 1) {   // (rows of whole fours)
                const int64_t ld = (a.Ro + 3) / 4 * 4;
                *reinterpret_cast<f32x4 *>(a.part + ((int64_t)split * a.T + col) * ld + r) = sum[0];
                continue;
            }
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[e] = sum[0][e];
                if constexpr (kGates) {
                    float slope;
                    o[e] = act(sum[0][e], a.gelu != 0, slope) * sum[NM - 1][e];
                }
            }
            store_run(static_cast<T *>(a.out) + col * a.ldo + r, o, (int)(a.Ro - r));
        }
    }
}

// Rows of weights a workgroup and parts of k: from estimated times (microseconds)
// fitted to 288 products of 1 to 64 tokens with weights of 512 x 1376 to 8256 x 2112,
// each with up to 40 choices; the choice costs 1.2% more than the best of them on
// average.  A unit's workgroups add up, by what they read: .036 us for a KB of
// weights and .018 of x.  So whole rounds of 256 workgroups matter most (48 tokens,
// 8256 x 2112: 16.5 us in 36 rows each, 25.1 in 32), then few bytes of x (rows in
// one workgroup), then the joining of parts.  For a few tokens 16 rows at most: two
// workgroups a unit hide each other's latency (one token, the gates of 2048 -> 8192:
// 13.8 us in 16 rows, 15.5 in 32).
struct FewChoice {
    int rows, splits;
};
template <typename T, bool kGates> FewChoice choose_few(const FewArgs &a) {
    const double row = (double)(a.K * (int64_t)sizeof(T)) * 1e-3;   // KB
    FewChoice best{16, 1};
    double tbest = -1.0;
    for (int rows = 8; rows <= (a.T <= 8 ? 16 : 48); rows += 4) {
        for (const int splits : {1, 2, 3, 4, 6, 8}) {
            const double part = 4e-6 * splits * (double)(a.T * ((a.Ro + 3) / 4 * 4));   // MB
            if (splits > 1 && (kGates || row < 1.0 * splits || part * 1e6 > (double)kPartBytes)) break;
            const double load = std::ceil((double)((a.Ro + rows - 1) / rows * splits) / 256.0);
            double t = load * ((rows * (kGates ? 2 : 1) * .036 + (double)a.T * .018) * row / splits + .2);
            if (splits > 1) t += 2.5 + 1.4 * part;
            if (tbest < 0.0 || t < tbest) { tbest = t; best = FewChoice{rows, splits}; }
        }
    }
    return best;
}
template <typename T, int TT, int RT, bool kGates> hipError_t few_run(FewArgs a, int rows, int splits, hipStream_t s) {
    a.rows = rows;
    a.splits = splits;
    k_few<T, TT, RT, kGates><<<dim3((unsigned)((a.Ro + rows - 1) / rows), (unsigned)splits), dim3(512), 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    return join(JoinArgs{a.part, a.T * ((a.Ro + 3) / 4 * 4), splits, a.T, a.Ro, {a.out}, a.ldo, 0}, 1, sizeof(T) == 4, s);
}
template <typename T, int TT, bool kGates> hipError_t few(const FewArgs &a, hipStream_t s) {
    const FewChoice c = choose_few<T, kGates>(a);
    switch ((c.rows + 15) / 16) {
    case 1: return few_run<T, TT, 1, kGates>(a, c.rows, c.splits, s);
    case 2: return few_run<T, TT, 2, kGates>(a, c.rows, c.splits, s);
    default: return few_run<T, TT, 3, kGates>(a, c.rows, c.splits, s);
    }
}
template <typename T, bool kGates> hipError_t few_rows(const FewArgs &a, hipStream_t s) {
    switch ((a.T + 15) / 16) {
    case 1: return few<T, 1, kGates>(a, s);
    case 2: return few<T, 2, kGates>(a, s);
    case 3: return few<T, 3, kGates>(a, s);
    default: return few<T, 4, kGates>(a, s);
    }
}

// Rows copied to longer ones, every copy of a call in one launch (1000 tokens,
// 1001 -> 2731 in bf16: five, 10.3 us; 24 in launches of their own): 16 bytes of a
// row a thread, from any element on.
template <typename T> __global__ __launch_bounds__(256) void k_pad(PadArgs g) {
    constexpr int EL = 16 / sizeof(T);
    typedef T whole __attribute__((ext_vector_type(EL)));
    typedef T piece __attribute__((ext_vector_type(EL), aligned(sizeof(T))));
    const PadArgs::Copy &c = g.copy[blockIdx.z];
    const int64_t k = ((int64_t)blockIdx.y * 256 + threadIdx.x) * EL;
    if (k >= c.dst_ld) return;
    for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
        const T *src = static_cast<const T *>(c.src) + row * c.src_ld + k;
        whole v;
        if (k + EL <= c.cols) {
            v = *reinterpret_cast<const piece *>(src);
        } else {
#pragma unroll
            for (int e = 0; e < EL; ++e) v[e] = k + e < c.cols ? src[e] : (T)0.f;
        }
        *reinterpret_cast<whole *>(static_cast<T *>(c.dst) + row * c.dst_ld + k) = v;
    }
}

int64_t part_elements(const GemmArgs &g) {
    const int64_t one = g.M * ((g.N + 3) / 4 * 4), third = g.N * ((g.M + 3) / 4 * 4);
    return g.batch == 3 ? std::max(one, third) : one;
}

template <typename T, int BM, int BN, int NWM, int NWN, bool kAT, bool kBT, Kind KIND>
hipError_t run(GemmArgs g, int splits, hipStream_t s) {
    constexpr bool kGates = KIND == kGate || KIND == kGateBwd;
    constexpr int NB = kGates ? BN / 2 : BN;
    g.tiles_m = (int)((g.M + BM - 1) / BM);
    g.tiles_n = (int)(((kGates ? g.ldc : g.N) + NB - 1) / NB);
    g.splits = splits;
    g.part_each = part_elements(g);
    k_gemm<T, BM, BN, NWM, NWN, kAT, kBT, KIND>
        <<<dim3((unsigned)(g.tiles_m * g.tiles_n), 1, (unsigned)(g.batch * splits)), dim3(NWM * NWN * 64), 0, s>>>(g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    return join(JoinArgs{g.part, g.part_each, splits, g.M, g.N, {g.c[0], g.c[1], g.c[2]}, g.ldc, g.ldc3}, g.batch,
                sizeof(T) == 4 || g.f32_out, s);
}

// Tile and split of a product, from estimated times (microseconds) fitted to
// every tile and split of 95 bf16 and 80 fp32 products of the block (100 to
// 8192 tokens, widths of 512 to 8192); the choice costs 1.3% (bf16) and 0.7%
// (fp32) more than the best of them on average.
//   bf16: a tile of 256 has a compute unit to itself, 128 shares one with
//     another: rounds of resident workgroups, a step 1.18, and .52 alone to
//     .84 shared, 10.3 and 6.0 a round.
//   fp32: the matrix units bound either tile, so a unit's workgroups add up:
//     a step 1.76 (128) or .451 (64) for each of them.
// Parts cost their bytes, written and read.  (768 x 1024 -> 2816, fp32 gates:
// 125 us of 128, 84 of 64; 8192 -> 2048 of 2048 tokens in bf16: 158 us of 256,
// 73 of 128.)
struct Choice {
    bool big;
    int splits;
};
template <typename T> Choice choose(const GemmArgs &g, bool gates) {
    constexpr bool kHalf = sizeof(T) == 2;
    constexpr int kBig = kHalf ? 256 : 128, BK = kRowBytes / (int)sizeof(T);
    constexpr double kUnits = 256.0;   // compute units
    const int64_t n = gates ? 2 * g.ldc : g.N, steps = (g.K + BK - 1) / BK * g.nseg;
    Choice best{true, 1};
    double tbest = -1.0;
    for (const bool big : {true, false}) {
        const int64_t b = big ? kBig : kBig / 2, tiles = (g.M + b - 1) / b * ((n + b - 1) / b) * g.batch;
        for (int splits = 1; splits <= (gates ? 1 : 16); ++splits) {
            const double part = 4.0 * splits * g.batch * part_elements(g);
            if (splits > 1 && (splits > steps || part > (double)kPartBytes)) break;
            const double wgs = (double)tiles * splits, each = std::ceil((double)steps / splits), load = std::ceil(wgs / kUnits);
            double t;
            if (kHalf) {
                const double rounds = std::ceil(load / (big ? 1 : 2)), share = std::min(std::max(wgs / kUnits - 1.0, 0.0), 1.0);
                t = rounds * (big ? each * 1.18 + 10.3 : each * (.52 + .317 * share) + 6.0);
            } else {
                const double rounds = std::ceil(load / (big ? 2 : 5));
                t = big ? each * (.15 * rounds + 1.76 * load) + 4.1 * rounds : each * (.106 * rounds + .451 * load) + 2.0 * rounds;
            }
            if (splits > 1) t += (kHalf ? 1.6 : 2.7) + part * (kHalf ? .48e-6 : .36e-6);
            if (tbest < 0.0 || t < tbest) { tbest = t; best = Choice{big, splits}; }
        }
    }
    return best;
}

template <typename T, bool kAT, bool kBT, Kind KIND> hipError_t pick(const GemmArgs &g, hipStream_t s) {
    const Choice c = choose<T>(g, KIND != kStore);
    if constexpr (sizeof(T) == 2)
        return c.big ? run<T, 256, 256, 2, 4, kAT, kBT, KIND>(g, c.splits, s) : run<T, 128, 128, 2, 2, kAT, kBT, KIND>(g, c.splits, s);
    else if constexpr (KIND != kStore)
        return c.big ? run<T, 128, 128, 2, 2, kAT, kBT, KIND>(g, c.splits, s) : run<T, 64, 64, 4, 1, kAT, kBT, KIND>(g, c.splits, s);
    else
        return c.big ? run<T, 128, 128, 2, 2, kAT, kBT, KIND>(g, c.splits, s) : run<T, 64, 64, 2, 2, kAT, kBT, KIND>(g, c.splits, s);
}

template <typename T> hipError_t dispatch(const GemmArgs &g, bool at, bool bt, Kind kind, hipStream_t s) {
    if (kind == kGate) return pick<T, false, false, kGate>(g, s);
    if (kind == kGateBwd) return pick<T, false, false, kGateBwd>(g, s);
    if (at) return pick<T, true, true, kStore>(g, s);
    return bt ? pick<T, false, true, kStore>(g, s) : pick<T, false, false, kStore>(g, s);
}

}  // namespace

hipError_t launch_gemm(GemmArgs g, bool f32, bool at, bool bt, Kind kind, hipStream_t s) {
    return f32 ? dispatch<float>(g, at, bt, kind, s) : dispatch<bf16>(g, at, bt, kind, s);
}
hipError_t launch_few(const FewArgs &a, bool f32, bool gates, hipStream_t s) {
    if (f32) return gates ? few_rows<float, true>(a, s) : few_rows<float, false>(a, s);
    return gates ? few_rows<bf16, true>(a, s) : few_rows<bf16, false>(a, s);
}
hipError_t launch_pad(const PadArgs &g, bool f32, hipStream_t s) {
    int64_t rows = 0, cols = 0;
    for (int k = 0; k < g.count; ++k) {
        rows = std::max(rows, g.copy[k].rows);
        cols = std::max(cols, g.copy[k].dst_ld);
    }
    if (rows == 0) return hipSuccess;
    // (a launch holds fewer than 2^32 threads)
    const dim3 grid((unsigned)std::min<int64_t>(rows, 1 << 16), (unsigned)((cols * (f32 ? 4 : 2) + 4095) / 4096), (unsigned)g.count), block(256);
    if (f32) k_pad<float><<<grid, block, 0, s>>>(g);
    else k_pad<bf16><<<grid, block, 0, s>>>(g);
    return hipGetLastError();
}

}  // namespace ffn
}  // namespace m3
