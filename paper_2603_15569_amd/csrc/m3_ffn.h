// Kernel arguments of the gated feed-forward block (m3_ffn.hip), already
// validated and laid out by the front end (m3_layers.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace m3 {
namespace ffn {

// C[m][n] = sum over k of A(m, k) B(n, k).  An operand lies either with k
// next to each other ([m][k]) or with its own axis so ([k][m], "turned").
// Rows start on 16 bytes.
struct GemmArgs {
    // two: two products summed (nseg), two products (batch), or the two gates (b);
    // a third product (batch) is N x M, with its own lda, ldb and ldc
    const void *a[3], *b[3];
    int64_t lda, ldb;          // elements
    int64_t M, N, K;
    int nseg, batch;
    void *c[3];
    int64_t ldc;
    int64_t lda3, ldb3, ldc3;
    int f32_out;               // c is fp32 whatever the io dtype
    // gates: h, dg, du with rows of ldc elements (columns N .. ldc - 1 are written as zeros), dh in fp32
    void *dg, *du;
    const float *dh;
    int gelu;
    // set at launch: tiles, and the parts that k is split into (their sums go
    // to `part`, [product][split], each of part_each elements and in rows of N
    // rounded up to four, and are joined there)
    int tiles_m, tiles_n, splits;
    float *part;
    int64_t part_each;
};

enum Kind {
    kStore,      // C
    kGate,       // h = act(g) u
    kGateBwd,    // h, dg, du from g, u and dh
};

// Room for the parts of split products, and the few rows' (below).
constexpr size_t kPartBytes = (size_t)32 << 20;

// C = A B (both as [row][k], or B or both turned), the two gates
hipError_t launch_gemm(GemmArgs g, bool f32, bool at, bool bt, Kind kind, hipStream_t s);

// Rows of `cols` elements copied to rows of dst_ld, zeros after
struct PadArgs {
    struct Copy {
        const void *src;
        void *dst;
        int64_t src_ld, dst_ld, rows, cols;
    } copy[5];
    int count;
};
hipError_t launch_pad(const PadArgs &g, bool f32, hipStream_t s);

// A few rows of x (T of them) times many rows of weights: out[t][r] = sum over
// k of x(t, k) w(r, k), or the two gates with w[0] = Wg and w[1] = Wu.
constexpr int kFewRows = 64;
struct FewArgs {
    const void *x, *w[2];
    int64_t ldx, ldw;      // elements; rows start on 16 bytes
    int64_t T, R, K;       // K: whole 16-byte pieces
    int64_t Ro;            // columns of out: R and any padding, written as zeros
    void *out;
    int64_t ldo;
    int gelu;
    float *part;           // kPartBytes
    int rows, splits;      // set at launch: rows of w a workgroup, parts of k
};
hipError_t launch_few(const FewArgs &a, bool f32, bool gates, hipStream_t s);

}  // namespace ffn
}  // namespace m3
