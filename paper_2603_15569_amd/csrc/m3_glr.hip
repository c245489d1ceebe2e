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

// Row access: a uniform pointer to the row and the lane's byte offset in it
template <typename R> __device__ __forceinline__ R row_load(const void *row, uint32_t off) {
    return *reinterpret_cast<const R *>(static_cast<const char *>(row) + off);
}
template <typename R> __device__ __forceinline__ void row_store(void *row, uint32_t off, R v) {
    *reinterpret_cast<R *>(static_cast<char *>(row) + off) = v;
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
// a = e^l and w = sqrt(1 - a^2) of a log-decay l <= 0.  1 - a^2 = -2 a sinh(l):
// near l = 0, where 1 - a^2 would keep few digits, by the series of sinh
// (relative error below 2e-8 up to |l| = 0.5).
__device__ __forceinline__ void decay(float l, float &a, float &w) {
    a = exp2_fast(kLog2e * l);
    const float q = l * l;
    const float sh = fmaf(l * q, fmaf(q, fmaf(q, 1.f / 5040.f, 1.f / 120.f), 1.f / 6.f), l);
    const float om = l > -0.5f ? -2.f * a * sh : fmaf(-a, a, 1.f);
    w = __builtin_amdgcn_sqrtf(om);
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
    int64_t tile;       // index of the tile in the order of its recurrence
    int64_t b, grp;     // batch row, channel group
    uint32_t tag;
};

// Work items in ticket order, tile-major: every tile that an item waits for
// has an earlier ticket, so it is running or done.  The counter's upper half
// is the count of calls on the workspace (the tag, never zero in use); whoever
// takes the last ticket sets it up for the next call.
__device__ __forceinline__ Item take_item(uint64_t *ctl, int64_t per_tile, int64_t tiles, int64_t G, uint64_t *s_ticket) {
    if (tiles == 1) {
        const int64_t k = blockIdx.x;
        return Item{0, k / G, k % G, 0};
    }
    if (threadIdx.x == 0) {
        const uint64_t w = __hip_atomic_fetch_add(ctl, (uint64_t)1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if ((uint32_t)w == (uint32_t)(per_tile * tiles - 1)) {
            const uint32_t epoch = (uint32_t)(w >> 32);
            __hip_atomic_store(reinterpret_cast<uint32_t *>(ctl) + 2 + ((epoch + 1) & 1), 0u, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(ctl, (uint64_t)(epoch + 1) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        *s_ticket = w;
    }
    __syncthreads();
    const uint64_t w = *s_ticket;
    const int64_t k = (int64_t)(uint32_t)w;
    const int64_t in = k % per_tile;
    return Item{k / per_tile, in / G, in % G, (uint32_t)(w >> 32) + 1u};
}

// Published words of a tile and channel: the state after the tile, and the
// tile's map
struct Words {
    uint64_t *inc, *mapA, *mapC;
};

// The state that enters a tile (tile > 0, all threads of the workgroup).  Each
// wave polls one of the NW tiles before this one; the nearest whose state is
// known, with the maps of all after it, gives the state, folded in token
// order.  `enter` is the state of the lane's channels, NaN when the wait gave up.
template <int V, int NW>
__device__ __forceinline__ void look_back(const Words &wd, int64_t slot0, int64_t tile, int64_t D, int64_t d0, bool live,
                                          uint32_t tag, uint64_t *ctl, uint32_t spin_max, int wave, int lane,
                                          float (*s_val)[3][64 * V], uint32_t *s_kind, float (&enter)[V]) {
    for (uint32_t spin = 0;; ++spin) {
        const int64_t j = tile - 1 - wave;
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
                s_val[wave][0][lane * V + e] = word_value(wi[e]);
                s_val[wave][1][lane * V + e] = word_value(wa[e]);
                s_val[wave][2][lane * V + e] = word_value(wc[e]);
            }
            const bool all_inc = __all(inc), all_map = __all(map);
            if (lane == 0) s_kind[wave] = all_inc ? 2u : all_map ? 1u : 0u;
        } else if (lane == 0) {
            s_kind[wave] = 0u;
        }
        __syncthreads();
        int at = -1;
#pragma unroll 1
        for (int k = 0; k < NW; ++k) {
            const uint32_t kind = s_kind[k];
            if (kind == 2u) { at = k; break; }
            if (kind == 0u) break;
        }
        if (at >= 0) {
#pragma unroll
            for (int e = 0; e < V; ++e) enter[e] = s_val[at][0][lane * V + e];
#pragma unroll 1
            for (int k = at - 1; k >= 0; --k)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    enter[e] = after(s_val[k][1][lane * V + e], enter[e], s_val[k][2][lane * V + e]);
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
__global__ __launch_bounds__(kFwdWaves * 64) void k_fwd(FwdArgs a) {
    typedef typename Raw<T, V>::type R;
    constexpr int NW = kFwdWaves, S = kChunk / NW, C = 64 * V;
    __shared__ uint64_t s_ticket;
    __shared__ float s_A[NW][C], s_c[NW][C];
    __shared__ float s_val[NW][3][C];
    __shared__ uint32_t s_kind[NW];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Item it = take_item(a.ctl, a.B * a.G, a.tiles, a.G, &s_ticket);
    const int64_t d0 = it.grp * C + lane * V;
    const bool live = d0 < a.D;      // (V divides D)
    const int64_t dl = live ? d0 : 0;
    const int64_t t0 = it.tile * kChunk + wave * S;
    const int n = (int)min((int64_t)S, a.L - t0);   // tokens of this wave, possibly none

    // rows past the end read the last token's (their maps are the identity)
    const uint32_t lo = (uint32_t)(dl * sizeof(T));
    const T *px = static_cast<const T *>(a.x) + it.b * a.x_sb;
    const T *pr = static_cast<const T *>(a.r) + it.b * a.r_sb;
    const T *pi = static_cast<const T *>(a.i) + it.b * a.i_sb;
    R vx[S], vr[S], vi[S], vz[kGate ? S : 1];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t t = min(t0 + s, a.L - 1);
        vr[s] = row_load<R>(pr + t * a.r_st, lo);
        vi[s] = row_load<R>(pi + t * a.i_st, lo);
        vx[s] = row_load<R>(px + t * a.x_st, lo);
    }
    float A[V];
#pragma unroll
    for (int e = 0; e < V; ++e) A[e] = a.A[dl + e];

    float pa[S][V], ph[S][V];   // the map of the wave's tokens up to and with s
    float ca[V], ch[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { ca[e] = 1.f; ch[e] = 0.f; }
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float at, wt;
            decay(A[e] * sigmoid(get(vr[s], e)), at, wt);
            const float bt = wt * sigmoid(get(vi[s], e)) * get(vx[s], e);
            const float na = ca[e] * at, nh = fmaf(at, ch[e], bt);
            ca[e] = s < n ? na : ca[e];
            ch[e] = s < n ? nh : ch[e];
            pa[s][e] = ca[e];
            ph[s][e] = ch[e];
        }
        fence();
    }
    if constexpr (kGate) {
        const T *pz = static_cast<const T *>(a.z) + it.b * a.z_sb;
#pragma unroll
        for (int s = 0; s < S; ++s) vz[s] = row_load<R>(pz + min(t0 + s, a.L - 1) * a.z_st, lo);
    }
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
    float enter[V];
    if (it.tile == 0) {
#pragma unroll
        for (int e = 0; e < V; ++e) enter[e] = a.init ? a.init[it.b * a.D + dl + e] : 0.f;
    } else {
        if (!last && wave == 0 && live) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                put_word(a.mapA + slot + e, tA[e], it.tag);
                put_word(a.mapC + slot + e, tc[e], it.tag);
            }
        }
        look_back<V, NW>(Words{a.inc, a.mapA, a.mapC}, slot0, it.tile, a.D, d0, live, it.tag, a.ctl, a.spin_max, wave, lane,
                         s_val, s_kind, enter);
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
    if (!live) return;
    float hw[V];
#pragma unroll
    for (int e = 0; e < V; ++e) hw[e] = after(wA[e], enter[e], wc[e]);
    T *py = static_cast<T *>(a.y) + (it.b * a.L + t0) * a.D;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (s >= n) continue;
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            o[e] = fmaf(pa[s][e], hw[e], ph[s][e]);
            if constexpr (kGate) o[e] *= silu(get(vz[s], e));
        }
        row_store<R>(py + s * a.D, lo, put<T, V>(o));
    }
}

// Gradients.  With dh_t = dy_t [SiLU(z_t)], q_t = a_t (dh_t + q_{t+1}) (q_L =
// dfinal) is the gradient of h_{t-1}, and g_t = dh_t + q_{t+1} that of h_t:
//     dx = g w iota,  di = g w x iota (1 - iota),  dz = dy h SiLU'(z)
//     dlog a = a g h_{t-1} - (a^2 / w) g iota x
//     dr = A dlog a rho (1 - rho),  dA = sum rho dlog a
// At w = 0 (a = 1: rho has underflowed) the second term of dlog a is taken as
// zero: multiplied by rho, as in dr and dA, it goes to zero there.
template <typename T, int V, bool kGate>
__global__ __launch_bounds__(kBwdWaves * 64) void k_bwd(BwdArgs a) {
    typedef typename Raw<T, V>::type R;
    constexpr int NW = kBwdWaves, S = kChunk / NW, C = 64 * V;
    __shared__ uint64_t s_ticket;
    __shared__ float s_A[NW][C], s_c[NW][C], s_q[NW][C];
    __shared__ float s_val[NW][3][C];
    __shared__ uint32_t s_kind[NW];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Item it = take_item(a.ctl, a.B * a.G, a.tiles, a.G, &s_ticket);
    const int64_t tile = a.tiles - 1 - it.tile;    // in token order; it.tile counts from the end
    const int64_t d0 = it.grp * C + lane * V;
    const bool live = d0 < a.D;
    const int64_t dl = live ? d0 : 0;
    const int64_t t0 = tile * kChunk + wave * S;
    const int n = (int)min((int64_t)S, a.L - t0);

    const uint32_t lo = (uint32_t)(dl * sizeof(T));
    const T *px = static_cast<const T *>(a.x) + it.b * a.x_sb;
    const T *pr = static_cast<const T *>(a.r) + it.b * a.r_sb;
    const T *pi = static_cast<const T *>(a.i) + it.b * a.i_sb;
    const T *pd = static_cast<const T *>(a.dy) + it.b * a.L * a.D;
    R vx[S], vr[S], vi[S], vd[S], vz[kGate ? S : 1];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t t = min(t0 + s, a.L - 1);
        vr[s] = row_load<R>(pr + t * a.r_st, lo);
        vi[s] = row_load<R>(pi + t * a.i_st, lo);
        vx[s] = row_load<R>(px + t * a.x_st, lo);
        vd[s] = row_load<R>(pd + t * a.D, lo);
        if constexpr (kGate) vz[s] = row_load<R>(static_cast<const T *>(a.z) + it.b * a.z_sb + t * a.z_st, lo);
    }
    float A[V], enter[V];
    const int64_t srow = (it.b * a.tiles + tile) * a.D;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        A[e] = a.A[dl + e];
        enter[e] = a.states[srow + dl + e];
    }
    // the wave's maps: of the state (A, c) from its first token to its last, of
    // the gradient (A, q) from its last to its first
    float at[S][V], bt[S][V];
    float cA[V], cc[V], cq[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { cA[e] = 1.f; cc[e] = 0.f; cq[e] = 0.f; }
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float wt;
            decay(A[e] * sigmoid(get(vr[s], e)), at[s][e], wt);
            bt[s][e] = wt * sigmoid(get(vi[s], e)) * get(vx[s], e);
            if (s >= n) { at[s][e] = 1.f; bt[s][e] = 0.f; }
            cA[e] *= at[s][e];
            cc[e] = fmaf(at[s][e], cc[e], bt[s][e]);
        }
        fence();
    }
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float dh = get(vd[s], e);
            if constexpr (kGate) dh *= silu(get(vz[s], e));
            cq[e] = s < n ? at[s][e] * (dh + cq[e]) : cq[e];
        }
        fence();
    }
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
    float q[V];
    if (it.tile == 0) {
#pragma unroll
        for (int e = 0; e < V; ++e) q[e] = a.dfinal ? a.dfinal[it.b * a.D + dl + e] : 0.f;
    } else {
        if (!last && wave == 0 && live) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                put_word(a.mapA + slot + e, tA[e], it.tag);
                put_word(a.mapC + slot + e, tq[e], it.tag);
            }
        }
        look_back<V, NW>(Words{a.inc, a.mapA, a.mapC}, slot0, it.tile, a.D, d0, live, it.tag, a.ctl, a.spin_max, wave, lane,
                         s_val, s_kind, q);
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
    const int64_t orow = (it.b * a.L + t0) * a.D;
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
        if (s >= n) continue;
        forget(vr[s]);
        forget(vi[s]);
        forget(vx[s]);
        forget(vd[s]);
        float ox[V], orr[V], oi[V], oz[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float x = get(vx[s], e), dy = get(vd[s], e);
            const float rho = sigmoid(get(vr[s], e)), iota = sigmoid(get(vi[s], e));
            float av, w;
            decay(A[e] * rho, av, w);
            float dh = dy;
            if constexpr (kGate) {
                const float z = get(vz[s], e), sz = sigmoid(z), gz = z * sz;
                dh = dy * gz;
                const float hv = fmaf(av, bt[s][e], w * iota * x);
                oz[e] = dy * hv * fmaf(gz, 1.f - sz, sz);
            }
            const float g = dh + q[e], gi = g * iota;
            q[e] = av * g;
            ox[e] = gi * w;
            oi[e] = ox[e] * x * (1.f - iota);
            const float ratio = w > 0.f ? av * av * __builtin_amdgcn_rcpf(w) : 0.f;
            const float dl_ = fmaf(q[e], bt[s][e], -ratio * (gi * x));
            const float rd = rho * dl_;
            orr[e] = A[e] * rd * (1.f - rho);
            dA[e] += rd;
        }
        if (live) {
            row_store<R>(static_cast<T *>(a.dx) + orow + s * a.D, lo, put<T, V>(ox));
            row_store<R>(static_cast<T *>(a.dr) + orow + s * a.D, lo, put<T, V>(orr));
            row_store<R>(static_cast<T *>(a.di) + orow + s * a.D, lo, put<T, V>(oi));
            if constexpr (kGate) row_store<R>(static_cast<T *>(a.dz) + orow + s * a.D, lo, put<T, V>(oz));
        }
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

// dA: the tiles' parts of a channel summed in fp64, in one order.
constexpr int kSumRows = 16;
__global__ __launch_bounds__(64 * kSumRows) void k_sum(const uint64_t *part, int64_t rows, int64_t D, float *dA) {
    __shared__ double s[kSumRows][64];
    const int lane = threadIdx.x % 64, row = threadIdx.x / 64;
    const int64_t d = (int64_t)blockIdx.x * 64 + lane;
    double v = 0.0;
    if (d < D)
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

// One token: the state is read and written once.
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
        float at, w;
        decay(a.A[d + e] * sigmoid(get(vr, e)), at, w);
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
    else k_bwd<T, V, false><<<grid, block, 0, s>>>(a);
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
