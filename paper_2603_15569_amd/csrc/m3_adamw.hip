// AdamW over many tensors in one launch, by a table of them on the device:
//     g' = grad_scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2
//     p = (1 - lr wd) p - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// with m and v in fp32, or in 8 bits: m and sqrt(v) as e4m3 with one fp32
// scale each for 256 elements (their largest magnitude / 448).  The 8-bit
// states are rounded stochastically: a moving average with a decay near one
// moves by less than a rounding step a time, and to nearest it would stand
// still; up or down with the probabilities of the part cut off, it moves as it
// should on average.  (sqrt(v), not v: half the range in powers of two.)  The
// random numbers are a hash of the element's index and the tensor's seed.
//
// Streaming: every byte is read and written once, past the caches (they hold
// nothing of it that is used again: 268 million parameters in fp32, 5.5 TB/s
// through them, 6.1 past them).  A wave takes one block of 256 consecutive
// elements, four a lane, so an 8-bit block's largest magnitude is one wave
// reduction; more blocks a wave were slower (four: 5.9 TB/s).  132 small tensors
// of 2.4 million elements in all: 13.5 us, 11 of them the bytes'.  Operations are
// rounded to fp32 one by one.  The 8-bit step has enough of them to wait for
// the vector units: 770 us for 268 million parameters (bf16 gradients and copy; 5.6
// TB/s) with the hardware's root and reciprocal, the ones that the codes depend on
// refined; a tenth more with the library's, a tenth less without the refinement,
// but an ulp there turns codes over.
#include "m3_adamw.h"
#include "m3_device.h"

namespace m3 {
namespace adamw {
namespace {

constexpr int kWaves = kChunkElems / kBlockElems;

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
    return v;
}
// Odd parts of the golden ratio and of sqrt 2; `first` is (index ^ seed) kGolden.
constexpr uint32_t kGolden = 0x9E3779B1u, kRoot2 = 0x6A09E667u;
__device__ __forceinline__ uint32_t noise(uint32_t first) {
    uint32_t h = (first ^ (first >> 15)) * kRoot2;
    h = (h ^ (h >> 13)) * kGolden;
    return h ^ (h >> 16);
}
// |w| <= 448 (a rounding more at most) to an e4m3 number, up with the
// probability of the part cut off; u is 16 uniform bits.
__device__ __forceinline__ float round8(float w, uint32_t u) {
    const float a = fabsf(w);
    const float big = __uint_as_float((__float_as_uint(a) + (u << 4)) & ~0xfffffu);
    const float small = floorf(__fadd_rn(__fmul_rn(a, 512.f), (float)u * 0x1p-16f)) * 0x1p-9f;
    const float q = a >= 0x1p-6f ? big : small;
    // (NaN stays NaN: it is neither below nor above)
    const float c = q > 448.f ? 448.f : q;
    return w < 0.f ? -c : c;
}

// Four elements of a tensor, which may start on any element: the vector
// accesses of global memory need no more alignment than that.
template <typename G> struct Four;
template <> struct Four<float> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Four<bf16> { typedef __bf16 type __attribute__((ext_vector_type(4), aligned(2))); };
typedef uint32_t Codes __attribute__((aligned(1)));

// Element e of lane `lane` in a block: four in a row, or one of each 64 in the
// block that a tensor ends in.
template <bool kVec> __device__ __forceinline__ int place(int lane, int e) { return kVec ? lane * 4 + e : lane + 64 * e; }

template <typename X, bool kVec>
__device__ __forceinline__ void load4(const X *p, int lane, int left, float (&o)[4]) {
    if constexpr (kVec) {
        const typename Four<X>::type w = __builtin_nontemporal_load(reinterpret_cast<const typename Four<X>::type *>(p + lane * 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (float)w[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = place<false>(lane, e) < left ? (float)p[place<false>(lane, e)] : 0.f;
    }
}
template <typename X, bool kVec>
__device__ __forceinline__ void store4(X *p, int lane, int left, const float (&v)[4]) {
    if constexpr (kVec) {
        typename Four<X>::type w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (X)v[e];
        __builtin_nontemporal_store(w, reinterpret_cast<typename Four<X>::type *>(p + lane * 4));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (place<false>(lane, e) < left) p[place<false>(lane, e)] = (X)v[e];
    }
}
// Four e4m3 codes
template <bool kVec> __device__ __forceinline__ void load8(const uint8_t *p, int lane, int left, float (&o)[4]) {
    if constexpr (kVec) {
        const uint32_t w = __builtin_nontemporal_load(reinterpret_cast<const Codes *>(p + lane * 4));
        o[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
        o[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
        o[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
        o[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[e] = place<false>(lane, e) < left ? __builtin_amdgcn_cvt_f32_fp8((int)p[place<false>(lane, e)], 0) : 0.f;
    }
}
template <bool kVec> __device__ __forceinline__ void store8(uint8_t *p, int lane, int left, const float (&q)[4]) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
    if constexpr (kVec) {
        __builtin_nontemporal_store((uint32_t)w, reinterpret_cast<Codes *>(p + lane * 4));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (place<false>(lane, e) < left) p[place<false>(lane, e)] = (uint8_t)((uint32_t)w >> (8 * e));
    }
}

// The hardware's root reads a subnormal number as zero, which without eps would
// make the step of a small gradient infinite: such a v is scaled (by 2^64, and
// the root back).  A branch that waves seldom take: with the scaling for all the
// 8-bit step of 268 million parameters took 790 us, 763 so.
__device__ __forceinline__ float root_of_subnormal(float v, float root) {
    const bool tiny = __builtin_amdgcn_classf(v, 0x80);   // (positive, subnormal)
    if (__builtin_expect(__any(tiny), 0)) root = tiny ? __builtin_amdgcn_sqrtf(v * 0x1p64f) * 0x1p-32f : root;
    return root;
}
// The root and the reciprocal a rounding step refined: to the nearest but for
// about one number in a million.  (What the 8-bit codes and scales are formed
// from: an ulp there can turn a code over, a step of 6% or more.)
__device__ __forceinline__ float root_near(float v) {
    const float s = __builtin_amdgcn_rsqf(v), g = v * s;
    const float r = __fmaf_rn(__fmaf_rn(-g, g, v), 0.5f * s, g);
    return v > 0x1p-100f && v < __builtin_inff() ? r : __builtin_amdgcn_sqrtf(v);   // (and NaN)
}
__device__ __forceinline__ float reciprocal_near(float v) {
    const float r = __builtin_amdgcn_rcpf(v);
    return __fmaf_rn(__fmaf_rn(-v, r, 1.f), r, r);
}

struct Step {
    float b1, c1, b2, c2, rate, root, eps, gs;
    bool scaled;
};

// One element: m and v, the root of v, and the new p.
template <bool kNear>
__device__ __forceinline__ void update(const Step &k, float shrink, float g, float &p, float &m, float &v, float &rv) {
#pragma clang fp contract(off)
    if (k.scaled) g = g * k.gs;
    m = m * k.b1 + g * k.c1;
    v = v * k.b2 + (g * g) * k.c2;
    rv = root_of_subnormal(v, kNear ? root_near(v) : __builtin_amdgcn_sqrtf(v));
    // (the whole change first: p itself is rounded once)
    p = p - (p * shrink + m * k.rate * __builtin_amdgcn_rcpf(rv * k.root + k.eps));
}

template <typename G, bool kEight, bool kVec>
__device__ __forceinline__ void block(const Tensor &t, const Step &k, float shrink, uint32_t seed, int64_t base, int left, int lane) {
    float g[4], p[4], m[4], v[4], rv[4];
    load4<G, kVec>(static_cast<const G *>(t.g) + base, lane, left, g);
    load4<float, kVec>(t.p + base, lane, left, p);
    float *sc = t.scales + base / kBlockElems * 2;
    if constexpr (kEight) {
        load8<kVec>(static_cast<const uint8_t *>(t.m) + base, lane, left, m);
        load8<kVec>(static_cast<const uint8_t *>(t.v) + base, lane, left, v);
        const float sm = sc[0], sv = sc[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] = __fmul_rn(m[e], sm);
            const float r = __fmul_rn(v[e], sv);
            v[e] = __fmul_rn(r, r);
        }
    } else {
        load4<float, kVec>(static_cast<const float *>(t.m) + base, lane, left, m);
        load4<float, kVec>(static_cast<const float *>(t.v) + base, lane, left, v);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) update<kEight>(k, shrink, g[e], p[e], m[e], v[e], rv[e]);
    store4<float, kVec>(t.p + base, lane, left, p);
    if (t.low) store4<bf16, kVec>(static_cast<bf16 *>(t.low) + base, lane, left, p);
    if constexpr (!kEight) {
        store4<float, kVec>(static_cast<float *>(t.m) + base, lane, left, m);
        store4<float, kVec>(static_cast<float *>(t.v) + base, lane, left, v);
    } else {
        float am = 0.f, av = 0.f;
        bool bad_m = false, bad_v = false;   // (fmaxf drops a NaN: it is carried beside the maximum)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!kVec && place<false>(lane, e) >= left) { m[e] = 0.f; rv[e] = 0.f; }
            am = fmaxf(am, fabsf(m[e]));
            av = fmaxf(av, rv[e]);
            bad_m = bad_m || m[e] != m[e];
            bad_v = bad_v || rv[e] != rv[e];
        }
        am = wave_max(am);
        av = wave_max(av);
        if (__any(bad_m)) am = __builtin_nanf("");
        if (__any(bad_v)) av = __builtin_nanf("");
        const float nm = __fmul_rn(am, 1.f / 448.f), nv = __fmul_rn(av, 1.f / 448.f);
        // (below 2^-100 a block is stored as zeros; NaN spoils it)
        const float im = am <= 0x1p-100f ? 0.f : reciprocal_near(nm), iv = av <= 0x1p-100f ? 0.f : reciprocal_near(nv);
        float qm[4], qv[4];
        // (four indices in a row differ in their last two bits: one product for all)
        const uint32_t row = (((uint32_t)base + 4u * (uint32_t)lane) ^ (seed & ~3u)) * kGolden;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t h = noise(kVec ? row + ((uint32_t)e ^ (seed & 3u)) * kGolden
                                          : (((uint32_t)base + (uint32_t)place<false>(lane, e)) ^ seed) * kGolden);
            qm[e] = round8(__fmul_rn(m[e], im), h & 0xffffu);
            qv[e] = round8(__fmul_rn(rv[e], iv), h >> 16);
            // a second moment that is not zero is not stored as zero: the next
            // step would divide by almost nothing
            if (rv[e] > 0.f && qv[e] < 0x1p-9f) qv[e] = 0x1p-9f;
        }
        store8<kVec>(static_cast<uint8_t *>(t.m) + base, lane, left, qm);
        store8<kVec>(static_cast<uint8_t *>(t.v) + base, lane, left, qv);
        if (lane == 0) { sc[0] = nm; sc[1] = nv; }
    }
}

template <typename G, bool kEight>
__global__ __launch_bounds__(kWaves * 64) void k_adamw(Args a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Tensor t = a.t[a.of[blockIdx.x]];
    Now now = a.now;
    if (a.from) now = *a.from;
    const float shrink = (float)(now.lr * t.decay);
    const uint32_t seed = now.seed + t.index;
    Step k{a.b1, a.c1, a.b2, a.c2, now.rate, now.root, a.eps, 1.f, a.grad_scale != nullptr};
    if (k.scaled) k.gs = *a.grad_scale;
    const int chunk = (int)blockIdx.x - t.first, first = wave * kBlockElems;
    const int left = min((chunk == t.chunks - 1 ? t.tail : kChunkElems) - first, kBlockElems);   // elements of this wave
    if (left <= 0) return;
    const int64_t base = (int64_t)chunk * kChunkElems + first;
    if (left == kBlockElems) block<G, kEight, true>(t, k, shrink, seed, base, left, lane);
    else block<G, kEight, false>(t, k, shrink, seed, base, left, lane);
}

// (one thread, 3 us before the step: the powers in fp64 for every wave would cost
// the 8-bit step, which has no vector time to spare, more)
__global__ void k_now(NowArgs a) {
    const int64_t t = a.device_step ? *a.device_step : a.step;
    const double lr = a.device_lr ? *a.device_lr : a.lr;
    Now n = now(lr, a.beta1, a.beta2, t, a.seed + (a.device_step ? (uint64_t)t : 0));
    if (t < 1) n.rate = __builtin_nanf("");
    *a.to = n;
}

}  // namespace

hipError_t launch_now(const NowArgs &a, hipStream_t s) {
    k_now<<<dim3(1), dim3(1), 0, s>>>(a);
    return hipGetLastError();
}
hipError_t launch(const Args &a, bool grad_f32, bool eight, hipStream_t s) {
    const dim3 grid((unsigned)a.groups), blk(kWaves * 64);
    if (grad_f32 && eight) k_adamw<float, true><<<grid, blk, 0, s>>>(a);
    else if (grad_f32) k_adamw<float, false><<<grid, blk, 0, s>>>(a);
    else if (eight) k_adamw<bf16, true><<<grid, blk, 0, s>>>(a);
    else k_adamw<bf16, false><<<grid, blk, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace adamw
}  // namespace m3
