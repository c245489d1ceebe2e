// Gated linear recurrence with one decay per channel and token on gfx950:
//     rho = sigmoid(r_t), iota = sigmoid(i_t), log a_t = A_d rho
//     h_t = a_t h_{t-1} + sqrt(1 - a_t^2) iota x_t,   y_t = h_t [SiLU(z_t)]
// forward over long sequences, backward, and one decode step.
//
// Every channel is a scalar recurrence, so a run of tokens is an affine map
// h -> (prod a) h + c of the state entering it, and maps compose.  A workgroup
// takes one tile of kChunk tokens by 64 V channels; each of its waves holds S
// consecutive tokens of the tile in registers, every lane V channels.  The
// waves' maps meet in LDS, the tiles' maps in the workspace: a tile publishes
// its map, finds the nearest earlier tile of its channels whose state is
// known, folds the maps between, and publishes the state after itself.  So
// every input is read once and every output written once; the tile's tokens
// wait in registers meanwhile.  The backward runs the same way from the last
// tile to the first on q_t = a_t (dh_t + q_{t+1}), with the states entering
// the tiles as the forward saved them.
//
// Bound by HBM, and by the look-back where a sequence has few tiles: 16 tokens a
// wave are what its registers hold with the gate (123 of them), so a compute unit
// keeps 200 KB of loads on their way.  65536 tokens of 2048 channels in bf16:
// forward 247 us (4.3 TB/s of the operator's bytes), backward 398 (4.7); 4 x 2048 of
// 4096 with the gate and inputs as slices: 75 us (4.5).  A streaming kernel reaches
// 6.1; 10 to 20% more bytes move than the operator has (the maps and states of
// the look-back, and their polling).  3 x 1001 tokens of 1000 channels in fp32, one
// and a half workgroups a unit: 18 us forward, 32 backward.
#include <type_traits>

#include "m3_device.h"
#include "m3_glr.h"

namespace m3 {
namespace glr {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// V neighbouring channels of one row as loaded, unpacked one by one
template <typename T, int V> struct Raw;
template <> struct Raw<bf16, 1> { typedef uint16_t type; };
template <> struct Raw<bf16, 2> { typedef uint32_t type; };
template <> struct Raw<float, 1> { typedef float type; };

__device__ __forceinline__ float get(uint16_t v, int) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float get(uint32_t v, int e) { return __uint_as_float(e ? v & 0xffff0000u : v << 16); }
__device__ __forceinline__ float get(float v, int) { return v; }

// Up to `n` rows of an array from a uniform address on, as a buffer: a lane's
// offset in the row in a vector register, the row's in a scalar one, so that
// an access takes no address arithmetic.  Past the rows and past the width
// (kOut) loads return zero and stores do nothing.  (A scalar offset past the
// buffer's end would not be caught: rows from n on go to the first one with
// kOut as the lane's offset.)
constexpr uint32_t kOut = 0x80000000u;
struct Rows {
    __amdgpu_buffer_rsrc_t r;
    uint32_t stride;
    int n;
};
template <typename T> __device__ __forceinline__ Rows rows(const void *p, int64_t at, int64_t stride, int n, int64_t width) {
    const uint32_t st = (uint32_t)(stride * sizeof(T));
    const int bytes = n > 0 ? (int)((uint32_t)(n - 1) * st + (uint32_t)(width * sizeof(T))) : 0;
    return Rows{__builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(static_cast<const T *>(p) + at), (short)0, bytes, 0x00020000), st, n};
}
// Outputs go past the caches (kOnce): nothing here reads them again, and the
// inputs keep the room (a tenth of the time of 4 x 2048 of 4096 forward).  The
// backward's loads too, the last use of its inputs (a twentieth of 65536 x 2048);
// the forward's not (they cost it a sixteenth), the backward reads them again.
// (W: the buffer is known to hold the row)
constexpr int kOnce = 2;
template <typename R, int kAux = 0, typename W> __device__ __forceinline__ R row_load(const Rows &w, int s, uint32_t off, W) {
    const bool in = W::value || s < w.n;
    const int lane = (int)(in ? off : kOut), row = in ? (int)(s * w.stride) : 0;
    if constexpr (sizeof(R) == 2) return __builtin_bit_cast(R, __builtin_amdgcn_raw_buffer_load_b16(w.r, lane, row, kAux));
    else return __builtin_bit_cast(R, __builtin_amdgcn_raw_buffer_load_b32(w.r, lane, row, kAux));
}
template <typename R, typename W> __device__ __forceinline__ void row_store(const Rows &w, int s, uint32_t off, R v, W) {
    const bool in = W::value || s < w.n;
    const int lane = (int)(in ? off : kOut), row = in ? (int)(s * w.stride) : 0;
    if constexpr (sizeof(R) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), w.r, lane, row, kOnce);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), w.r, lane, row, kOnce);
}
// Keeps the compiler from overlapping more tokens than registers are for.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// Makes a value unknown to the compiler, so that what is formed from it a
// second time is formed again and not held in registers meanwhile.
template <typename R> __device__ __forceinline__ void forget(R &v) { asm volatile("" : "+v"(v)); }

template <typename T, int V> __device__ __forceinline__ typename Raw<T, V>::type put(const float (&v)[V]) {
    if constexpr (sizeof(T) == 2) {
        typename Raw<T, V>::type w = __builtin_bit_cast(uint16_t, (bf16)v[0]);
        if constexpr (V == 2) w |= (uint32_t)__builtin_bit_cast(uint16_t, (bf16)v[1]) << 16;
        return w;
    } else {
        static_assert(V == 1, "fp32: one channel a lane");
        return v[0];
    }
}

__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.f + exp2_fast(-kLog2e * v));
}
// 1 - a^2 of a decay a = 2^l, l <= 0: -2 a sinh(l ln 2) near l = 0, where the
// plain form would keep few digits (by its series: relative error below 7e-8
// up to |l ln 2| = 0.25).
__device__ __forceinline__ float one_minus_square(float a, float l) {
    constexpr float kLn2 = 0.693147180559945309417f, k3 = kLn2 * kLn2 * kLn2;
    constexpr float c0 = -2.f * kLn2, c1 = -2.f * k3 / 6.f, c2 = -2.f * k3 * kLn2 * kLn2 / 120.f;
    const float q = l * l;
    const float near = a * l * fmaf(q, fmaf(q, c2, c1), c0);
    return l > -0.25f / kLn2 ? near : fmaf(-a, a, 1.f);
}
// The state after a map (A, c) from the state h before it: one rounding order
// everywhere, so that a fold of published maps and their owner's own state
// have the same bits whatever the timing.
__device__ __forceinline__ float after(float A, float h, float c) { return __fmaf_rn(A, h, c); }

// A published number with the call that wrote it, in one 8-byte access, so
// that a reader needs no flag and no fence: it is there once its tag is the
// call's.
__device__ __forceinline__ void put_word(uint64_t *p, float v, uint32_t tag) {
    __hip_atomic_store(p, (uint64_t)__float_as_uint(v) | (uint64_t)tag << 32, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t get_word(const uint64_t *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float word_value(uint64_t w) { return __uint_as_float((uint32_t)w); }

struct Item {
    bool none;      // no item: the workgroup leaves
    int tile;       // index of the tile in the order of its recurrence
    int b, grp;     // batch row, channel group
    uint32_t tag;
};

// Work items in ticket order, tile-major: every tile that an item waits for
// has an earlier ticket, so it is running or done.  The counter's upper half
// is the count of calls on the workspace (plus one: the tag); whoever takes
// the last ticket sets it up for the next call.  A workspace that was not
// cleared may hold any ticket: one past the items takes none, and is counted as
// a wait that gave up (in both calls' words: the count of calls means nothing).
__device__ __forceinline__ Item take_item(uint64_t *ctl, uint32_t B, uint32_t tiles, uint32_t G, uint64_t *s_ticket) {
    // (divisions leave their results in vector registers: back to scalar ones)
    auto scalar = [](uint32_t v) { return __builtin_amdgcn_readfirstlane((int)v); };
    uint32_t k = blockIdx.x, tag = 0;
    if (tiles > 1) {
        if (threadIdx.x == 0) {
            const uint64_t w = __hip_atomic_fetch_add(ctl, (uint64_t)1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if ((uint32_t)w == B * G * tiles - 1) {
                const uint32_t epoch = (uint32_t)(w >> 32);
                __hip_atomic_store(reinterpret_cast<uint32_t *>(ctl) + 2 + ((epoch + 1) & 1), 0u, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(ctl, (uint64_t)(epoch + 1) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            if ((uint32_t)w >= B * G * tiles)
                for (int e = 0; e < 2; ++e)
                    __hip_atomic_fetch_add(reinterpret_cast<uint32_t *>(ctl) + 2 + e, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *s_ticket = w;
        }
        __syncthreads();
        const uint64_t w = *s_ticket;
        k = (uint32_t)scalar((uint32_t)w);
        tag = (uint32_t)(w >> 32) + 1u;
    }
    const uint32_t tile = k / (B * G), in = k - tile * (B * G), b = in / G;
    return Item{k >= B * G * tiles, scalar(tile), scalar(b), scalar(in - b * G), (uint32_t)scalar(tag)};
}

// Published words of a tile and channel: the state after the tile, and the
// tile's map
struct Words {
    uint64_t *inc, *mapA, *mapC;
};

// The state that enters a tile (tile > 0, all threads of the workgroup).  Each
// wave polls one of the NW tiles before this one; when that was not enough and
// the sequence's start is in reach, kReach of them, back to `first`, the state
// there (4096 tokens of 512 channels: 13.8 us against 15.7 without; further into
// a sequence the wider polling mostly costs more than it saves, 247 us -> 278 at
// 65536 tokens of 2048 channels, 54 -> 59 at 2 x 16384 of 768, though not where
// the channels are few, 72 -> 45 at 32768 of 256).  The nearest tile whose state is
// known, with the maps of all after it, gives the state, folded in token order.
// `enter` is the state of the lane's channels, NaN when the wait gave up.
constexpr int kReach = 4;
template <int V, int NW> struct Polled {
    float v[kReach * NW][2][64 * V];   // the state after the tile, or its map
    uint32_t kind[64];                 // 2: state, 1: map, 0: nothing yet
};
template <int V, int NW>
__device__ __forceinline__ void look_back(const Words &wd, int64_t slot0, int tile, int64_t D, int64_t d0, bool live,
                                          uint32_t tag, uint64_t *ctl, uint32_t spin_max, int wave, int lane,
                                          const float (&first)[V], Polled<V, NW> &s, float (&enter)[V]) {
    static_assert(kReach * NW <= 64, "a lane for each polled tile");
    for (uint32_t spin = 0;; ++spin) {
        const int reach = spin == 0 || tile > kReach * NW ? 1 : kReach;
#pragma unroll 1
        for (int r = 0; r < reach; ++r) {
            const int p = r * NW + wave, j = tile - 1 - p;
            uint32_t kind = 0;
            float v[2][V];
            if (j >= 0) {
                const int64_t at = slot0 + j * D + d0;
                uint64_t wi[V], wa[V], wc[V];
                bool inc = true, map = true;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    wi[e] = live ? get_word(wd.inc + at + e) : (uint64_t)tag << 32;
                    wa[e] = live ? get_word(wd.mapA + at + e) : (uint64_t)tag << 32;
                    wc[e] = live ? get_word(wd.mapC + at + e) : (uint64_t)tag << 32;
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    inc = inc && (uint32_t)(wi[e] >> 32) == tag;
                    map = map && (uint32_t)(wa[e] >> 32) == tag && (uint32_t)(wc[e] >> 32) == tag;
                }
                kind = __all(inc) ? 2u : __all(map) ? 1u : 0u;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    v[0][e] = word_value(kind == 2u ? wi[e] : wa[e]);
                    v[1][e] = word_value(wc[e]);
                }
            } else if (j == -1) {
                kind = 2u;
#pragma unroll
                for (int e = 0; e < V; ++e) { v[0][e] = first[e]; v[1][e] = 0.f; }
            }
            if (kind)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    s.v[p][0][lane * V + e] = v[0][e];
                    s.v[p][1][lane * V + e] = v[1][e];
                }
            if (lane == 0) s.kind[p] = kind;
        }
        __syncthreads();
        const uint32_t kind = lane < reach * NW ? s.kind[lane] : 0u;
        const uint64_t known = __ballot(kind == 2u), none = __ballot(kind == 0u);
        const int at = known ? __builtin_ctzll(known) : 64;
        if (at < (none ? __builtin_ctzll(none) : 64)) {
#pragma unroll
            for (int e = 0; e < V; ++e) enter[e] = s.v[at][0][lane * V + e];
#pragma unroll 2
            for (int k = at - 1; k >= 0; --k)
#pragma unroll
                for (int e = 0; e < V; ++e) enter[e] = after(s.v[k][0][lane * V + e], enter[e], s.v[k][1][lane * V + e]);
            return;
        }
        if (spin + 1 >= spin_max) {
            if (threadIdx.x == 0)
                __hip_atomic_fetch_add(reinterpret_cast<uint32_t *>(ctl) + 2 + ((tag - 1) & 1), 1u, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int e = 0; e < V; ++e) enter[e] = __builtin_nanf("");
            return;
        }
        __syncthreads();
        __builtin_amdgcn_s_sleep(1);
    }
}

template <typename T, int V, bool kGate>
__global__ __launch_bounds__(kFwdWaves * 64, 4) void k_fwd(FwdArgs a) {
    typedef typename Raw<T, V>::type R;
    constexpr int NW = kFwdWaves, S = kChunk / NW, C = 64 * V;
    __shared__ uint64_t s_ticket;
    __shared__ float s_A[NW][C], s_c[NW][C];
    __shared__ Polled<V, NW> s_polled;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Item it = take_item(a.ctl, (uint32_t)a.B, (uint32_t)a.tiles, (uint32_t)a.G, &s_ticket);
    if (it.none) return;
    const int64_t d0 = (int64_t)it.grp * C + lane * V;
    const bool live = d0 < a.D;      // (V divides D)
    const int64_t dl = live ? d0 : 0;
    const int64_t t0 = (int64_t)it.tile * kChunk + wave * S;
    const int n = max(0, min(S, (int)a.L - (int)t0));   // tokens of this wave (L is below 2^31)

    const uint32_t lo = live ? (uint32_t)(d0 * sizeof(T)) : kOut;
    const Rows rx = rows<T>(a.x, it.b * a.x_sb + t0 * a.x_st, a.x_st, n, a.D), rr = rows<T>(a.r, it.b * a.r_sb + t0 * a.r_st, a.r_st, n, a.D),
               ri = rows<T>(a.i, it.b * a.i_sb + t0 * a.i_st, a.i_st, n, a.D);
    R vx[S], vr[S], vi[S], vz[kGate ? S : 1];
    float A[V];   // of powers of two
#pragma unroll
    for (int e = 0; e < V; ++e) A[e] = a.A[dl + e] * kLog2e;

    float pa[S][V], ph[S][V];   // the map of the wave's tokens up to and with s
    float ca[V], ch[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { ca[e] = 1.f; ch[e] = 0.f; }
    auto maps = [&](auto whole) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            vr[s] = row_load<R>(rr, s, lo, whole);
            vi[s] = row_load<R>(ri, s, lo, whole);
            vx[s] = row_load<R>(rx, s, lo, whole);
        }
        fence();
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (decltype(whole)::value || s < n) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float l = A[e] * sigmoid(get(vr[s], e)), at = exp2_fast(l);
                    const float wt = __builtin_amdgcn_sqrtf(one_minus_square(at, l));
                    ca[e] *= at;
                    ch[e] = fmaf(at, ch[e], wt * sigmoid(get(vi[s], e)) * get(vx[s], e));
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) { pa[s][e] = ca[e]; ph[s][e] = ch[e]; }
            fence();
        }
        if constexpr (kGate) {
            const Rows rz = rows<T>(a.z, it.b * a.z_sb + t0 * a.z_st, a.z_st, n, a.D);
#pragma unroll
            for (int s = 0; s < S; ++s) vz[s] = row_load<R>(rz, s, lo, whole);
        }
    };
    if (n >= S) maps(std::true_type{});
    else maps(std::false_type{});
#pragma unroll
    for (int e = 0; e < V; ++e) {
        s_A[wave][lane * V + e] = ca[e];
        s_c[wave][lane * V + e] = ch[e];
    }
    __syncthreads();
    // the maps of the waves before this one, and of the tile
    float wA[V], wc[V], tA[V], tc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { wA[e] = 1.f; wc[e] = 0.f; tA[e] = 1.f; tc[e] = 0.f; }
#pragma unroll 4
    for (int k = 0; k < NW; ++k) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (k == wave) { wA[e] = tA[e]; wc[e] = tc[e]; }
            const float mA = s_A[k][lane * V + e], mc = s_c[k][lane * V + e];
            tc[e] = fmaf(mA, tc[e], mc);
            tA[e] *= mA;
        }
    }
    const int64_t slot0 = it.b * a.tiles * a.D, slot = slot0 + it.tile * a.D + d0;
    const bool last = it.tile == a.tiles - 1;
    float first[V], enter[V];
#pragma unroll
    for (int e = 0; e < V; ++e) enter[e] = first[e] = a.init ? a.init[it.b * a.D + dl + e] : 0.f;
    if (it.tile > 0) {
        if (!last && wave == 0 && live) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                put_word(a.mapA + slot + e, tA[e], it.tag);
                put_word(a.mapC + slot + e, tc[e], it.tag);
            }
        }
        look_back<V, NW>(Words{a.inc, a.mapA, a.mapC}, slot0, it.tile, a.D, d0, live, it.tag, a.ctl, a.spin_max, wave, lane,
                         first, s_polled, enter);
    }
    if (wave == 0 && live) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float leave = after(tA[e], enter[e], tc[e]);
            if (!last) put_word(a.inc + slot + e, leave, it.tag);
            else a.final_state[it.b * a.D + d0 + e] = leave;
            if (a.states) a.states[slot + e] = enter[e];
        }
    }
    float hw[V];
#pragma unroll
    for (int e = 0; e < V; ++e) hw[e] = after(wA[e], enter[e], wc[e]);
    const Rows ry = rows<T>(a.y, (it.b * a.L + t0) * a.D, a.D, n, a.D);
    auto out = [&](auto whole) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                o[e] = fmaf(pa[s][e], hw[e], ph[s][e]);
                if constexpr (kGate) o[e] *= silu(get(vz[s], e));
            }
            row_store<R>(ry, s, lo, put<T, V>(o), whole);
        }
    };
    if (n >= S) out(std::true_type{});
    else out(std::false_type{});
}

// Gradients.  With dh_t = dy_t [SiLU(z_t)], q_t = a_t (dh_t + q_{t+1}) (q_L =
// dfinal) is the gradient of h_{t-1}, and g_t = dh_t + q_{t+1} that of h_t:
//     dx = g w iota,  di = g w x iota (1 - iota),  dz = dy h SiLU'(z)
//     dlog a = a g h_{t-1} - (a^2 / w) g iota x
//     dr = A dlog a rho (1 - rho),  dA = sum rho dlog a
// Where 1 - a^2 is below fp32's smallest normal number, 2^-126 (rho has all but
// underflowed), w and the second term of dlog a are taken as zero: w is at most
// 1.1e-19 there, and the term, multiplied by rho as in dr and dA, goes to zero with
// it.  (The hardware's root and its reciprocal read a subnormal number as zero.)
template <typename T, int V, bool kGate>
__global__ __launch_bounds__(kBwdWaves * 64) void k_bwd(BwdArgs a) {
    typedef typename Raw<T, V>::type R;
    constexpr int NW = kBwdWaves, S = kChunk / NW, C = 64 * V;
    __shared__ uint64_t s_ticket;
    __shared__ float s_A[NW][C], s_c[NW][C], s_q[NW][C];
    __shared__ Polled<V, NW> s_polled;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Item it = take_item(a.ctl, (uint32_t)a.B, (uint32_t)a.tiles, (uint32_t)a.G, &s_ticket);
    if (it.none) return;
    const int tile = (int)a.tiles - 1 - it.tile;    // in token order; it.tile counts from the end
    const int64_t d0 = (int64_t)it.grp * C + lane * V;
    const bool live = d0 < a.D;
    const int64_t dl = live ? d0 : 0;
    const int64_t t0 = (int64_t)tile * kChunk + wave * S;
    const int n = max(0, min(S, (int)a.L - (int)t0));

    const uint32_t lo = live ? (uint32_t)(d0 * sizeof(T)) : kOut;
    const int64_t orow = (it.b * a.L + t0) * a.D;
    const Rows rx = rows<T>(a.x, it.b * a.x_sb + t0 * a.x_st, a.x_st, n, a.D), rr = rows<T>(a.r, it.b * a.r_sb + t0 * a.r_st, a.r_st, n, a.D),
               ri = rows<T>(a.i, it.b * a.i_sb + t0 * a.i_st, a.i_st, n, a.D), rd = rows<T>(a.dy, orow, a.D, n, a.D);
    R vx[S], vr[S], vi[S], vd[S], vz[kGate ? S : 1];
    float A[V], A2[V], enter[V];   // (A2: of powers of two)
    const int64_t srow = (it.b * a.tiles + tile) * a.D;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        A[e] = a.A[dl + e];
        A2[e] = A[e] * kLog2e;
        enter[e] = a.states[srow + dl + e];
    }
    // the wave's maps: of the state (A, c) from its first token to its last, of
    // the gradient (A, q) from its last to its first
    float at[S][V], bt[S][V], rho[S][V], iota[S][V];
    float cA[V], cc[V], cq[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { cA[e] = 1.f; cc[e] = 0.f; cq[e] = 0.f; }
    auto maps = [&](auto whole) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            vr[s] = row_load<R, kOnce>(rr, s, lo, whole);
            vi[s] = row_load<R, kOnce>(ri, s, lo, whole);
            vx[s] = row_load<R, kOnce>(rx, s, lo, whole);
            vd[s] = row_load<R, kOnce>(rd, s, lo, whole);
        }
        if constexpr (kGate) {
            const Rows rz = rows<T>(a.z, it.b * a.z_sb + t0 * a.z_st, a.z_st, n, a.D);
#pragma unroll
            for (int s = 0; s < S; ++s) vz[s] = row_load<R, kOnce>(rz, s, lo, whole);
        }
        fence();
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                rho[s][e] = sigmoid(get(vr[s], e));
                iota[s][e] = sigmoid(get(vi[s], e));
                const float l = A2[e] * rho[s][e];
                at[s][e] = exp2_fast(l);
                bt[s][e] = __builtin_amdgcn_sqrtf(one_minus_square(at[s][e], l)) * iota[s][e] * get(vx[s], e);
                if (!decltype(whole)::value && s >= n) { at[s][e] = 1.f; bt[s][e] = 0.f; }
                cA[e] *= at[s][e];
                cc[e] = fmaf(at[s][e], cc[e], bt[s][e]);
            }
            fence();
        }
#pragma unroll
        for (int s = S - 1; s >= 0; --s) {
            if (!decltype(whole)::value && s >= n) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float dh = get(vd[s], e);
                if constexpr (kGate) dh *= silu(get(vz[s], e));
                cq[e] = at[s][e] * (dh + cq[e]);
            }
            fence();
        }
    };
    if (n >= S) maps(std::true_type{});
    else maps(std::false_type{});
#pragma unroll
    for (int e = 0; e < V; ++e) {
        s_A[wave][lane * V + e] = cA[e];
        s_c[wave][lane * V + e] = cc[e];
        s_q[wave][lane * V + e] = cq[e];
    }
    __syncthreads();
    float h[V], tA[V], tq[V], wA[V], wq[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { h[e] = enter[e]; tA[e] = 1.f; tq[e] = 0.f; wA[e] = 1.f; wq[e] = 0.f; }
#pragma unroll 1
    for (int k = 0; k < wave; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = fmaf(s_A[k][lane * V + e], h[e], s_c[k][lane * V + e]);
#pragma unroll 4
    for (int k = NW - 1; k >= 0; --k) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (k == wave) { wA[e] = tA[e]; wq[e] = tq[e]; }
            const float mA = s_A[k][lane * V + e], mq = s_q[k][lane * V + e];
            tq[e] = fmaf(mA, tq[e], mq);
            tA[e] *= mA;
        }
    }
    // h becomes the state before each token
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float nh = fmaf(at[s][e], h[e], bt[s][e]);
            bt[s][e] = h[e];
            h[e] = nh;
        }

    const int64_t slot0 = it.b * a.tiles * a.D, slot = slot0 + it.tile * a.D + d0;
    const bool last = it.tile == a.tiles - 1;
    float first[V], q[V];
#pragma unroll
    for (int e = 0; e < V; ++e) q[e] = first[e] = a.dfinal ? a.dfinal[it.b * a.D + dl + e] : 0.f;
    if (it.tile > 0) {
        if (!last && wave == 0 && live) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                put_word(a.mapA + slot + e, tA[e], it.tag);
                put_word(a.mapC + slot + e, tq[e], it.tag);
            }
        }
        look_back<V, NW>(Words{a.inc, a.mapA, a.mapC}, slot0, it.tile, a.D, d0, live, it.tag, a.ctl, a.spin_max, wave, lane,
                         first, s_polled, q);
    }
    if (wave == 0 && live) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float leave = after(tA[e], q[e], tq[e]);
            if (!last) put_word(a.inc + slot + e, leave, it.tag);
            else if (a.dinit) a.dinit[it.b * a.D + d0 + e] = leave;
        }
    }
    float dA[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { q[e] = after(wA[e], q[e], wq[e]); dA[e] = 0.f; }
    const Rows wx = rows<T>(a.dx, orow, a.D, n, a.D), wr = rows<T>(a.dr, orow, a.D, n, a.D), wi = rows<T>(a.di, orow, a.D, n, a.D);
    const Rows wz = rows<T>(kGate ? a.dz : a.dx, orow, a.D, n, a.D);
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
        if (s >= n) continue;
        forget(vx[s]);
        forget(vd[s]);
        float ox[V], orr[V], oi[V], oz[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float x = get(vx[s], e), dy = get(vd[s], e), av = at[s][e], ig = iota[s][e];
            forget(rho[s][e]);   // (w is formed again)
            const float om = one_minus_square(av, A2[e] * rho[s][e]);
            const float iw = om >= 0x1p-126f ? __builtin_amdgcn_rsqf(om) : 0.f, w = om * iw;
            float dh = dy;
            if constexpr (kGate) {
                const float z = get(vz[s], e), sz = sigmoid(z), gz = z * sz;
                dh = dy * gz;
                const float hv = fmaf(av, bt[s][e], w * ig * x);
                oz[e] = dy * hv * fmaf(gz, 1.f - sz, sz);
            }
            const float g = dh + q[e], gi = g * ig;
            q[e] = av * g;
            ox[e] = gi * w;
            oi[e] = ox[e] * x * (1.f - ig);
            const float dl_ = fmaf(q[e], bt[s][e], -(av * av * iw) * (gi * x));
            const float rl = rho[s][e] * dl_;
            orr[e] = A[e] * rl * (1.f - rho[s][e]);
            dA[e] += rl;
        }
        row_store<R>(wx, s, lo, put<T, V>(ox), std::true_type{});
        row_store<R>(wr, s, lo, put<T, V>(orr), std::true_type{});
        row_store<R>(wi, s, lo, put<T, V>(oi), std::true_type{});
        if constexpr (kGate) row_store<R>(wz, s, lo, put<T, V>(oz), std::true_type{});
        fence();
    }
    // the tile's part of dA (tagged like every word of the workspace)
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) s_c[wave][lane * V + e] = dA[e];
    __syncthreads();
    if (wave == 0 && live) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float sum = 0.f;
#pragma unroll 4
            for (int k = 0; k < NW; ++k) sum += s_c[k][lane * V + e];
            a.part[(it.b * a.tiles + tile) * a.D + d0 + e] = (uint64_t)__float_as_uint(sum);
        }
    }
}

// dA: the tiles' parts of a channel summed in fp64, in one order (512 of 2048
// channels: 6.7 us with eight of a thread's loads at once, 11 one by one).
constexpr int kSumRows = 16;
__global__ __launch_bounds__(64 * kSumRows) void k_sum(const uint64_t *part, int64_t rows, int64_t D, float *dA) {
    __shared__ double s[kSumRows][64];
    const int lane = threadIdx.x % 64, row = threadIdx.x / 64;
    const int64_t d = (int64_t)blockIdx.x * 64 + lane;
    double v = 0.0;
    if (d < D)
#pragma unroll 8
        for (int64_t k = row; k < rows; k += kSumRows) v += (double)word_value(part[k * D + d]);
    s[row][lane] = v;
    __syncthreads();
    if (row == 0 && d < D) {
        for (int k = 1; k < kSumRows; ++k) v += s[k][lane];
        dA[d] = (float)v;
    }
}

// An empty sequence: the state passes through (dA may be null).
__global__ __launch_bounds__(256) void k_empty(const float *in, float *out, int64_t n, float *dA, int64_t D) {
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (out && k < n) out[k] = in ? in[k] : 0.f;
    if (dA && k < D) dA[k] = 0.f;
}

// One token: the state is read and written once (64 rows of 4096 channels with
// the gate: 4.7 MB, 2.8 us, a launch's own time).
template <typename T, int V, bool kGate>
__global__ __launch_bounds__(256) void k_step(StepArgs a) {
    typedef typename Raw<T, V>::type R;
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x, per = a.D / V;
    if (k >= a.B * per) return;
    const int64_t b = k / per, d = (k % per) * V;
    const R vx = *reinterpret_cast<const R *>(static_cast<const T *>(a.x) + b * a.x_sb + d);
    const R vr = *reinterpret_cast<const R *>(static_cast<const T *>(a.r) + b * a.r_sb + d);
    const R vi = *reinterpret_cast<const R *>(static_cast<const T *>(a.i) + b * a.i_sb + d);
    R vz = {};
    if constexpr (kGate) vz = *reinterpret_cast<const R *>(static_cast<const T *>(a.z) + b * a.z_sb + d);
    float *ps = a.state + b * a.D + d;
    float h[V], o[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float l = a.A[d + e] * kLog2e * sigmoid(get(vr, e)), at = exp2_fast(l);
        const float w = __builtin_amdgcn_sqrtf(one_minus_square(at, l));
        h[e] = fmaf(at, ps[e], w * sigmoid(get(vi, e)) * get(vx, e));
        o[e] = h[e];
        if constexpr (kGate) o[e] *= silu(get(vz, e));
    }
#pragma unroll
    for (int e = 0; e < V; ++e) ps[e] = h[e];
    *reinterpret_cast<R *>(static_cast<T *>(a.y) + b * a.D + d) = put<T, V>(o);
}

template <typename T, int V> hipError_t fwd(const FwdArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)(a.B * a.G * a.tiles)), block(kFwdWaves * 64);
    if (a.z) k_fwd<T, V, true><<<grid, block, 0, s>>>(a);
    else k_fwd<T, V, false><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, int V> hipError_t bwd(const BwdArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)(a.B * a.G * a.tiles)), block(kBwdWaves * 64);
    if (a.z) k_bwd<T, V, true><<<grid, block, 0, s>>>(a);
    else if constexpr (V == 1) k_bwd<T, V, false><<<grid, block, 0, s>>>(a);   // (bwd_channels)
    else return hipErrorInvalidValue;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_sum<<<dim3((unsigned)((a.D + 63) / 64)), dim3(64 * kSumRows), 0, s>>>(a.part, a.B * a.tiles, a.D, a.dA);
    return hipGetLastError();
}
template <typename T, int V> hipError_t step(const StepArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((a.B * (a.D / V) + 255) / 256)), block(256);
    if (a.z) k_step<T, V, true><<<grid, block, 0, s>>>(a);
    else k_step<T, V, false><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_fwd(const FwdArgs &a, bool f32, int V, hipStream_t s) {
    if (a.tiles == 0) {
        const int64_t n = a.B * a.D;
        k_empty<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(a.init, a.final_state, n, nullptr, 0);
        return hipGetLastError();
    }
    return f32 ? fwd<float, 1>(a, s) : V == 2 ? fwd<bf16, 2>(a, s) : fwd<bf16, 1>(a, s);
}
hipError_t launch_bwd(const BwdArgs &a, bool f32, int V, hipStream_t s) {
    if (a.tiles == 0) {
        const int64_t n = a.B * a.D;
        k_empty<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(a.dfinal, a.dinit, n, a.dA, a.D);
        return hipGetLastError();
    }
    return f32 ? bwd<float, 1>(a, s) : V == 2 ? bwd<bf16, 2>(a, s) : bwd<bf16, 1>(a, s);
}
hipError_t launch_step(const StepArgs &a, bool f32, int V, hipStream_t s) {
    return f32 ? step<float, 1>(a, s) : V == 2 ? step<bf16, 2>(a, s) : step<bf16, 1>(a, s);
}

}  // namespace glr
}  // namespace m3
