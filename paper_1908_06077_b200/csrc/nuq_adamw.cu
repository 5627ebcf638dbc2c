// AdamW over lists of tensors, with moments in 32 or in 8 bits, and the norm of a list of gradients.
//
// What bounds them is memory: 28 bytes an element with fp32 moments (and fp32 gradients), 16 with 8-bit ones, 4 for the norm, each read
// or written once.  The tensors' table travels in the kernel's parameters, so that nothing is uploaded, nothing is kept and a
// captured call holds its own.  A tile is 1024 elements of one tensor, a warp's part of it 256: the block that shares the scales
// of 8-bit moments, so that its largest magnitude is one warp reduction.
//
// Measured, of a copy's 6538 GB/s (2^28 elements, passes for half a second): fp32 moments 1158 us, 106 %; the norm of bf16
// gradients 80.4 us, 102 %; 8-bit moments with bf16 gradients and copy 770 to 796 us from card to card, 83 to 86 %, in short bursts 720 to
// 750: that kernel
// issues 535 instructions for a warp's 256 elements (76 % of the issue slots, two for each of the 36 wide products of the random
// bits; ALU pipe 47 %, multiply-add pipe 53 %), which take 515 us by themselves, and the clock falls under the load.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/nuq.h"
#include "nuq_adamw.cuh"
#include "nuq_async.cuh"
#include "nuq_launch.h"

namespace nuq {

constexpr uint32_t kNormThreads = 256;
constexpr uint32_t kStepThreads = 128;
constexpr uint32_t kStepTile = kStepThreads / 32u * NUQ_STATE_BLOCK;   // elements that a CTA takes at a time
constexpr uint32_t kStepCtas32 = 6, kStepCtas8 = 7;         // CTAs of an SM
constexpr uint32_t kNormVectors = 2048;                     // 16-byte vectors of a tile of the norm
constexpr uint32_t kNormMaxGrid = (NUQ_CONTROL_BYTES - 64u) / 8u;

// A tensor of the step.  flags: the types, and which arrays are moved by whole vectors.
enum : uint32_t { kWideGrad = 1u << 24, kWideW = 2u << 24, kWideCopy = 4u << 24, kWideStates = 8u << 24, kWide = 15u << 24 };
struct StepTensor {
    const void* g;
    float* w;
    void* copy;
    void* m;
    void* v;
    float* scales;
    uint64_t n;
    float decay;             // lr weight_decay
    uint32_t flags;
    uint32_t index;          // in the caller's list
};
template <uint32_t CAP>
struct StepTable {
    uint32_t count, tiles;
    uint32_t first[CAP];     // the tensors' first tiles
    StepTensor tensor[CAP];
};
struct NormTensor {
    const void* g;
    uint64_t n;
};
template <uint32_t CAP>
struct NormTable {
    uint32_t count, tiles;
    uint32_t first[CAP];     // the tensors' first tiles
    NormTensor tensor[CAP];
    uint8_t type[CAP];       // NUQ_GRAD_*
};

// The last tensor that begins at or before `tile`, `from` or one behind it.
template <class Table>
__device__ __forceinline__ uint32_t tensor_of(const Table& T, uint32_t tile, uint32_t from) {
    uint32_t lo = from, hi = T.count;
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if (T.first[mid] <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Elements between the 16-byte boundary at or below a gradient and its first one.
__host__ __device__ inline uint32_t norm_skew(const void* g, uint32_t type) {
    return (uint32_t)(reinterpret_cast<uintptr_t>(g) & 15u) / (type == NUQ_GRAD_F32 ? 4u : 2u);
}

__device__ __forceinline__ float half_to_float(uint32_t bits, uint32_t type) {
    return type == NUQ_GRAD_BF16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half((unsigned short)bits));
}
__device__ __forceinline__ uint32_t pack_halves(float a, float b, bool bf16) {
    if (bf16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// ---- 8-bit moments ----

// Philox4x32-10 of the counter (quad (two words), t, j): 128 random bits.  Of the first two rounds' four products two are the same for
// all quads with the same upper word.
struct RandomBits {
    uint32_t c0, a0, a1, c1, t, j;
    __device__ __forceinline__ RandomBits(uint32_t high, uint32_t t_, uint32_t j_, const uint32_t (&keys)[20]) : t(t_), j(j_) {
        const uint64_t b = (uint64_t)t * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ high ^ keys[0];
        c1 = (uint32_t)b;
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u;
        a0 = (uint32_t)a;
        a1 = (uint32_t)(a >> 32);
    }
    __device__ __forceinline__ uint4 of(uint32_t quad, const uint32_t (&keys)[20]) const {
        const uint64_t a = (uint64_t)quad * 0xD2511F53u;
        const uint64_t b = (uint64_t)((uint32_t)(a >> 32) ^ j ^ keys[1]) * 0xCD9E8D57u;
        uint32_t x0 = (uint32_t)(b >> 32) ^ c1 ^ keys[2], x1 = (uint32_t)b, x2 = a1 ^ (uint32_t)a ^ keys[3], x3 = a0;
#pragma unroll
        for (int r = 2; r < 10; ++r) {
            const uint64_t p = (uint64_t)x0 * 0xD2511F53u, q = (uint64_t)x2 * 0xCD9E8D57u;
            x0 = (uint32_t)(q >> 32) ^ x1 ^ keys[2 * r];
            x2 = (uint32_t)(p >> 32) ^ x3 ^ keys[2 * r + 1];
            x1 = (uint32_t)q;
            x3 = (uint32_t)p;
        }
        return make_uint4(x0, x1, x2, x3);
    }
};

// four e4m3 codes as floats
__device__ __forceinline__ float4 code_values(uint32_t codes) {
    uint32_t a, b;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(a) : "h"((unsigned short)codes));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b) : "h"((unsigned short)(codes >> 16)));
    const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&a)), hi = __half22float2(*reinterpret_cast<const __half2*>(&b));
    return make_float4(lo.x, lo.y, hi.x, hi.y);
}

// |x| inv (at most 448) in e4m3, rounded up with the probability that keeps the mean, in the top byte.  Times 2^-120 the number has
// e4m3's exponents as fp32's own, down to the subnormals of both: the code's seven bits are bits 20 to 26, and what lies below
// them is a fraction of the code's spacing, to which 16 random bits (and a half of their last place) are added.
constexpr uint32_t kLowHalf = 0x5104u, kHighHalf = 0x5324u;     // a word's random bits: as __byte_perm takes them, above a byte 0x80
// ORDINARY: no number reaches 2^14 and no root is 0, and inv has been multiplied by 2^-120 (which would underflow from 2^15 on).  Else
// infinity and NaN become the code of NaN, 0x7f.
template <bool ORDINARY>
__device__ __forceinline__ uint32_t coded(float x, float inv, uint32_t word, uint32_t half) {
    float y = fabsf(ORDINARY ? __fmul_rn(x, inv) : __fmul_rn(__fmul_rn(x, inv), 0x1p-120f));
    if (!ORDINARY) y = fminf(y, __uint_as_float(0x07f00000u));
    return (__float_as_uint(y) << 4) + __byte_perm(word, 0x80u, half);
}
template <bool ORDINARY>
__device__ __forceinline__ uint32_t coded_moment(float m, float inv, uint32_t word) {
    return coded<ORDINARY>(m, inv, word, kLowHalf) | (__float_as_uint(m) & 0x80000000u);
}
// a root that is not 0 is at least code 1 (the smallest number's root is above 2^-75, whose bits are far above 1 << 24)
template <bool ORDINARY>
__device__ __forceinline__ uint32_t coded_root(float root, float inv, uint32_t word) {
    return max(coded<ORDINARY>(root, inv, word, kHighHalf), ORDINARY ? 1u << 24 : min(__float_as_uint(root), 1u << 24));
}
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073u), __byte_perm(c, d, 0x0073u), 0x5410u);
}

// The largest finite magnitude among a warp's elements, 2^-100 at least.
__device__ __forceinline__ float largest_finite(const float (&x)[8]) {
    float most = 0x1p-100f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (fabsf(x[i]) < __uint_as_float(0x7f800000u)) most = fmaxf(most, fabsf(x[i]));
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
}

// A lane's elements of a block: two groups of four neighbours, 128 apart, or eight that are 32 apart.
struct Elements {
    float g[8], w[8], m[8], v[8];                           // m and v: the old ones, then the new ones
};
// What the step finds out about the lane's elements that the codes need.
struct Found {
    float root[8], most_m, most_v;                          // the largest magnitudes, NaN if one is
    bool ordinary;                                          // of the warp's elements
};

// The step.  With 8-bit states m and v come as codes' values: v's that of its root.
template <bool BITS8>
__device__ __forceinline__ Found step(Elements& x, const AdamwParams& P, const AdamwFactors& f, float keep, float2 scales) {
    Found o;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float g = __fmul_rn(x.g[i], f.scale);
        float m = x.m[i], v = x.v[i];
        if (BITS8) {
            m = __fmul_rn(m, scales.x);
            v = __fmul_rn(v, scales.y);
            v = __fmul_rn(v, v);
        }
        x.m[i] = moment1(P, g, m);
        x.v[i] = moment2(P, g, v);
        o.root[i] = ordinary_root(x.v[i]);
    }
    const float inf = __uint_as_float(0x7f800000u);
    const float least = smallest3(smallest3(x.v[0], x.v[1], x.v[2]), smallest3(x.v[3], x.v[4], x.v[5]), fminf(x.v[6], x.v[7]));
    o.most_v = largest3(largest3(x.v[0], x.v[1], x.v[2]), largest3(x.v[3], x.v[4], x.v[5]), largest3(x.v[6], x.v[7], x.v[7]));
    o.most_m = !BITS8 ? 0.0f : largest3(largest3(fabsf(x.m[0]), fabsf(x.m[1]), fabsf(x.m[2])), largest3(fabsf(x.m[3]), fabsf(x.m[4]), fabsf(x.m[5])), largest3(fabsf(x.m[6]), fabsf(x.m[7]), fabsf(x.m[7])));
    o.ordinary = __all_sync(0xffffffffu, least >= kLeastRoot && (BITS8 ? o.most_v < 0x1p28f && o.most_m < 0x1p14f : o.most_v < inf));
    if (!o.ordinary) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o.root[i] = __fsqrt_rn(x.v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i] = adamw_value(f, keep, x.w[i], x.m[i], o.root[i]);
    return o;
}

// The codes of the lane's moments, four to a word (two groups of four neighbours), and the block's scales.
template <bool ORDINARY>
__device__ __forceinline__ float2 code_words(const StepTensor& t, const AdamwParams& P, uint32_t step, uint64_t e0, const float (&m)[8], const float (&root)[8],
                                             float most_m, float most_r, uint32_t (&cm)[2], uint32_t (&cv)[2]) {
    const float inv_m = ORDINARY ? __fmul_rn(448.0f * 0x1p-120f, reciprocal(most_m)) : __fmul_rn(448.0f, __frcp_rn(most_m));
    const float inv_r = ORDINARY ? __fmul_rn(448.0f * 0x1p-120f, reciprocal(most_r)) : __fmul_rn(448.0f, __frcp_rn(most_r));
    const RandomBits random((uint32_t)(e0 >> 34), step, t.index, P.round_keys);             // (a block's quads have one upper word)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const uint4 r = random.of((uint32_t)(e0 / 4u) + 32u * q + lane_id(), P.round_keys);
        const int i = 4 * q;
        cm[q] = top_bytes(coded_moment<ORDINARY>(m[i], inv_m, r.x), coded_moment<ORDINARY>(m[i + 1], inv_m, r.y), coded_moment<ORDINARY>(m[i + 2], inv_m, r.z), coded_moment<ORDINARY>(m[i + 3], inv_m, r.w));
        cv[q] = top_bytes(coded_root<ORDINARY>(root[i], inv_r, r.x), coded_root<ORDINARY>(root[i + 1], inv_r, r.y), coded_root<ORDINARY>(root[i + 2], inv_r, r.z), coded_root<ORDINARY>(root[i + 3], inv_r, r.w));
    }
    return make_float2(__fmul_rn(most_m, 1.0f / 448.0f), __fmul_rn(most_r, 1.0f / 448.0f));
}
__device__ __forceinline__ float2 make_codes(const StepTensor& t, const AdamwParams& P, uint32_t step, uint64_t e0, const Elements& x, const Found& o, uint32_t (&cm)[2], uint32_t (&cv)[2]) {
    if (o.ordinary) {
        // (bits of numbers that are not negative compare like these; the largest root is the root of the largest v)
        const float most_m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(o.most_m)));
        const float most_v = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(o.most_v)));
        return code_words<true>(t, P, step, e0, x.m, o.root, fmaxf(most_m, 0x1p-100f), ordinary_root(most_v), cm, cv);
    }
    return code_words<false>(t, P, step, e0, x.m, o.root, largest_finite(x.m), largest_finite(o.root), cm, cv);
}

__device__ __forceinline__ void put4(float (&x)[8], int q, float4 y) {
    x[4 * q] = y.x; x[4 * q + 1] = y.y; x[4 * q + 2] = y.z; x[4 * q + 3] = y.w;
}
__device__ __forceinline__ float4 get4(const float (&x)[8], int q) { return make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]); }
// four gradients of 16 bits
__device__ __forceinline__ float4 from_halves(uint2 raw, uint32_t type) {
    if (type == NUQ_GRAD_BF16) return make_float4(__uint_as_float(raw.x << 16), __uint_as_float(raw.x & 0xffff0000u), __uint_as_float(raw.y << 16), __uint_as_float(raw.y & 0xffff0000u));
    const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&raw.x)), hi = __half22float2(*reinterpret_cast<const __half2*>(&raw.y));
    return make_float4(lo.x, lo.y, hi.x, hi.y);
}
__device__ __forceinline__ uint2 to_halves(float4 x, uint32_t copy_type) {
    const bool bf16 = copy_type == NUQ_COPY_BF16;
    return make_uint2(pack_halves(x.x, x.y, bf16), pack_halves(x.z, x.w, bf16));
}

// A warp's 256 elements from e0 on, all of which exist and can be moved by whole groups of four: a lane has two groups of neighbours,
// 128 apart, so that an instruction moves up to 512 bytes in a row and one Philox block serves a group.
template <bool BITS8>
__device__ __forceinline__ void step_whole(const StepTensor& t, const AdamwParams& P, const AdamwFactors& f, float keep, uint64_t e0) {
    const uint32_t type = t.flags & 0xffu, copy_type = t.flags & 0xff00u;
    const uint64_t e = e0 + 4u * lane_id();
    Elements x;
    uint4 wide[2];
    uint2 halves[2];
    uint32_t cm[2], cv[2];
    float2 scales = make_float2(0.f, 0.f);
#pragma unroll
    for (int q = 0; q < 2; ++q) {                           // (all loads before the first use)
        if (type == NUQ_GRAD_F32) wide[q] = *reinterpret_cast<const uint4*>(static_cast<const float*>(t.g) + e + 128 * q);
        else halves[q] = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(t.g) + e + 128 * q);
        put4(x.w, q, *reinterpret_cast<const float4*>(t.w + e + 128 * q));
        if (BITS8) {
            cm[q] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.m) + e + 128 * q);
            cv[q] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.v) + e + 128 * q);
        } else {
            put4(x.m, q, *reinterpret_cast<const float4*>(static_cast<const float*>(t.m) + e + 128 * q));
            put4(x.v, q, *reinterpret_cast<const float4*>(static_cast<const float*>(t.v) + e + 128 * q));
        }
    }
    if (BITS8) scales = *reinterpret_cast<const float2*>(t.scales + 2u * (e0 / NUQ_STATE_BLOCK));
    if (type == NUQ_GRAD_F32) {
#pragma unroll
        for (int q = 0; q < 2; ++q) put4(x.g, q, make_float4(__uint_as_float(wide[q].x), __uint_as_float(wide[q].y), __uint_as_float(wide[q].z), __uint_as_float(wide[q].w)));
    } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) put4(x.g, q, from_halves(halves[q], type));
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (!BITS8) break;
        put4(x.m, q, code_values(cm[q]));
        put4(x.v, q, code_values(cv[q]));
    }
    const Found o = step<BITS8>(x, P, f, keep, scales);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        *reinterpret_cast<float4*>(t.w + e + 128 * q) = get4(x.w, q);
        if (copy_type != NUQ_COPY_NONE) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(t.copy) + e + 128 * q) = to_halves(get4(x.w, q), copy_type);
        if (!BITS8) {
            *reinterpret_cast<float4*>(static_cast<float*>(t.m) + e + 128 * q) = get4(x.m, q);
            *reinterpret_cast<float4*>(static_cast<float*>(t.v) + e + 128 * q) = get4(x.v, q);
        }
    }
    if (BITS8) {
        const float2 s = make_codes(t, P, f.t, e0, x, o, cm, cv);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.m) + e + 128 * q) = cm[q];
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + e + 128 * q) = cv[q];
        }
        if (lane_id() == 0) *reinterpret_cast<float2*>(t.scales + 2u * (e0 / NUQ_STATE_BLOCK)) = s;
    }
}

// The first `left` elements of a block, or a block that starts anywhere.  Every instruction moves 32 neighbours, one per lane, which needs
// no more than the elements' own alignment.
// With fp32 states that is also how they are computed.
__device__ __forceinline__ void step_part32(const StepTensor& t, const AdamwParams& P, const AdamwFactors& f, float keep, uint64_t e0, uint32_t left) {
    const uint32_t type = t.flags & 0xffu, copy_type = t.flags & 0xff00u, lane = lane_id();
    Elements x;
    uint32_t raw[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint64_t e = e0 + 32u * i + lane;
        const bool there = 32u * i + lane < left;
        raw[i] = !there ? 0u : type == NUQ_GRAD_F32 ? static_cast<const uint32_t*>(t.g)[e] : static_cast<const uint16_t*>(t.g)[e];
        x.w[i] = there ? t.w[e] : 0.0f;
        x.m[i] = there ? static_cast<const float*>(t.m)[e] : 0.0f;
        x.v[i] = there ? static_cast<const float*>(t.v)[e] : 1.0f;
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        x.g[i] = type == NUQ_GRAD_F32 ? __uint_as_float(raw[i]) : type == NUQ_GRAD_BF16 ? __uint_as_float(raw[i] << 16) : __half2float(__ushort_as_half((unsigned short)raw[i]));
    step<false>(x, P, f, keep, make_float2(0.f, 0.f));
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint64_t e = e0 + 32u * i + lane;
        if (32u * i + lane >= left) continue;
        t.w[e] = x.w[i];
        if (copy_type != NUQ_COPY_NONE) static_cast<uint16_t*>(t.copy)[e] = (uint16_t)pack_halves(x.w[i], 0.0f, copy_type == NUQ_COPY_BF16);
        static_cast<float*>(t.m)[e] = x.m[i];
        static_cast<float*>(t.v)[e] = x.v[i];
    }
}

// With 8-bit states a lane has groups of four neighbours, as the random bits have: the elements pass through the warp's shared memory.
struct alignas(16) Staged {
    float g[NUQ_STATE_BLOCK], w[NUQ_STATE_BLOCK];           // (16-bit gradients, later the copy, take the first half of g)
    uint8_t m[NUQ_STATE_BLOCK], v[NUQ_STATE_BLOCK];
};
// WHOLE: all 256 exist.
template <bool WHOLE, class T>
__device__ __forceinline__ void stage_in(T* shared, const T* from, uint32_t left) {
    T x[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) x[i] = WHOLE || 32u * i + lane_id() < left ? from[32u * i + lane_id()] : T(0);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) shared[32u * i + lane_id()] = x[i];
}
// (four bytes at a time past the registers; the warp waits for its copies before it meets)
template <bool WHOLE>
__device__ __forceinline__ void stage_in(float* shared, const float* from, uint32_t left) {
    const uint32_t to = smem_u32(shared) + 4u * lane_id();
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        if (WHOLE || 32u * i + lane_id() < left) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + 128u * i), "l"(from + 32u * i + lane_id()) : "memory");
        else shared[32u * i + lane_id()] = 0.0f;
    }
}
template <bool WHOLE, class T>
__device__ __forceinline__ void stage_out(T* to, const T* shared, uint32_t left) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (WHOLE || 32u * i + lane_id() < left) to[32u * i + lane_id()] = shared[32u * i + lane_id()];
}
template <bool WHOLE>
__device__ __forceinline__ void step_part8(const StepTensor& t, const AdamwParams& P, const AdamwFactors& f, float keep, uint64_t e0, uint32_t left, Staged& s) {
    const uint32_t type = t.flags & 0xffu, copy_type = t.flags & 0xff00u, lane = lane_id();
    // (of a whole block those arrays that allow it are moved by groups all the same)
    const bool codes_wide = WHOLE && (t.flags & kWideStates), w_wide = WHOLE && (t.flags & kWideW);
    uint8_t *const tm = static_cast<uint8_t*>(t.m) + e0, *const tv = static_cast<uint8_t*>(t.v) + e0;
    float* const tw = t.w + e0;
    const float2 scales = *reinterpret_cast<const float2*>(t.scales + 2u * (e0 / NUQ_STATE_BLOCK));
    Elements x;
    uint32_t cm[2], cv[2];
    __syncwarp();                                           // (what the block before left there has been read)
    if (codes_wide) {
#pragma unroll
        for (uint32_t q = 0; q < 2; ++q) {
            cm[q] = *reinterpret_cast<const uint32_t*>(tm + 128u * q + 4u * lane);
            cv[q] = *reinterpret_cast<const uint32_t*>(tv + 128u * q + 4u * lane);
        }
    }
    if (w_wide) {
#pragma unroll
        for (uint32_t q = 0; q < 2; ++q) put4(x.w, q, *reinterpret_cast<const float4*>(tw + 128u * q + 4u * lane));
    }
    if (type == NUQ_GRAD_F32) stage_in<WHOLE>(s.g, static_cast<const float*>(t.g) + e0, left);
    else stage_in<WHOLE>(reinterpret_cast<uint16_t*>(s.g), static_cast<const uint16_t*>(t.g) + e0, left);
    if (!w_wide) stage_in<WHOLE>(s.w, tw, left);
    if (!codes_wide) {
        stage_in<WHOLE>(s.m, tm, left);
        stage_in<WHOLE>(s.v, tv, left);
    }
    asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
        const uint32_t at = 128u * q + 4u * lane;
        put4(x.g, q, type == NUQ_GRAD_F32 ? *reinterpret_cast<const float4*>(s.g + at) : from_halves(*reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(s.g) + at), type));
        if (!w_wide) put4(x.w, q, *reinterpret_cast<const float4*>(s.w + at));
        if (!codes_wide) {
            cm[q] = *reinterpret_cast<const uint32_t*>(s.m + at);
            cv[q] = *reinterpret_cast<const uint32_t*>(s.v + at);
        }
        put4(x.m, q, code_values(cm[q]));
        put4(x.v, q, code_values(cv[q]));
    }
    const Found o = step<true>(x, P, f, keep, scales);
    __syncwarp();
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
        const uint32_t at = 128u * q + 4u * lane;
        if (w_wide) *reinterpret_cast<float4*>(tw + at) = get4(x.w, q);
        else *reinterpret_cast<float4*>(s.w + at) = get4(x.w, q);
        if (copy_type != NUQ_COPY_NONE) *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(s.g) + at) = to_halves(get4(x.w, q), copy_type);
    }
    __syncwarp();
    if (!w_wide) stage_out<WHOLE>(tw, s.w, left);
    if (copy_type != NUQ_COPY_NONE) stage_out<WHOLE>(static_cast<uint16_t*>(t.copy) + e0, reinterpret_cast<const uint16_t*>(s.g), left);
    const float2 made = make_codes(t, P, f.t, e0, x, o, cm, cv);
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
        const uint32_t at = 128u * q + 4u * lane;
        *reinterpret_cast<uint32_t*>((codes_wide ? tm : s.m) + at) = cm[q];
        *reinterpret_cast<uint32_t*>((codes_wide ? tv : s.v) + at) = cv[q];
    }
    if (!codes_wide) {
        __syncwarp();
        stage_out<WHOLE>(tm, s.m, left);
        stage_out<WHOLE>(tv, s.v, left);
    }
    if (lane == 0) *reinterpret_cast<float2*>(t.scales + 2u * (e0 / NUQ_STATE_BLOCK)) = made;
}

// Which line of a block's this lane asks for, of which array: where it lies in the tensor's first block, and the bytes from one
// block to the next (0: none).  21 lines: 8 of w, 8 or 4 of g, 2 each of m and v, the scales.
struct Line {
    const char* at;
    uint32_t pitch;
};
__device__ __forceinline__ Line line_of(const StepTensor& t) {
    const uint32_t lane = lane_id(), k = lane & 7u, array = lane >> 3;
    const bool halves = (t.flags & 0xffu) != NUQ_GRAD_F32;
    Line l;
    l.at = reinterpret_cast<const char*>(t.w) + 128u * k;
    l.pitch = array == 0u ? 1024u : 0u;
    if (array == 1u) {
        l.at = static_cast<const char*>(t.g) + 128u * k;
        l.pitch = !halves ? 1024u : k < 4u ? 512u : 0u;
    } else if (array == 2u && k < 4u) {
        l.at = static_cast<const char*>(k < 2u ? t.m : t.v) + 128u * (k & 1u);
        l.pitch = 256u;
    } else if (array == 2u && k == 4u) {
        l.at = reinterpret_cast<const char*>(t.scales);
        l.pitch = 8u;
    }
    return l;
}

// rounds: blocks of a warp in a tile, one behind the other
// KIND: what states the tensors have; those with 8-bit states whose arrays do not all start where groups of four may be moved have a kernel
// of their own (in one kernel the usual path has 25 registers too few).
enum : int { kStates32 = 0, kStates8 = 1, kStates8Narrow = 2 };
template <uint32_t CAP, int KIND>
__global__ void __launch_bounds__(kStepThreads, KIND != kStates32 ? kStepCtas8 : kStepCtas32) adamw_kernel(const __grid_constant__ StepTable<CAP> T, const __grid_constant__ AdamwParams P, const uint32_t rounds) {
    constexpr bool BITS8 = KIND != kStates32;
    const uint32_t tile = blockIdx.x, i = tensor_of(T, tile, 0u);
    const StepTensor t = T.tensor[i];
    asm volatile("griddepcontrol.wait;" ::: "memory");      // nothing before it reads or writes memory: see launch_overlapped
    const AdamwFactors f = adamw_factors(P);
    if (!f.taken) return;
    uint64_t e0 = (uint64_t)(tile - T.first[i]) * (kStepTile * rounds) + (threadIdx.x >> 5) * NUQ_STATE_BLOCK;
    const float keep = adamw_keep(f, t.decay);
    __shared__ Staged s_staged[BITS8 ? kStepThreads / 32u : 1u];
    Line line = {};
    if (BITS8) {
        line = line_of(t);
        line.at += (e0 + kStepTile) / NUQ_STATE_BLOCK * line.pitch;
    }
#pragma unroll 1
    for (uint32_t r = 0; r < rounds && e0 < t.n; ++r, e0 += kStepTile) {
        const uint64_t left = t.n - e0;
        if (BITS8) {                                        // the warp's next block is asked into the L1, if it is whole
            if (line.pitch != 0u && r + 1u < rounds && left >= kStepTile + NUQ_STATE_BLOCK) asm volatile("prefetch.global.L1 [%0];" ::"l"(line.at));
            line.at += kStepTile / NUQ_STATE_BLOCK * line.pitch;
        }
        const uint32_t have = left < NUQ_STATE_BLOCK ? (uint32_t)left : NUQ_STATE_BLOCK;
        if constexpr (KIND == kStates8Narrow) {
            if (have == NUQ_STATE_BLOCK) step_part8<true>(t, P, f, keep, e0, have, s_staged[threadIdx.x >> 5]);
            else step_part8<false>(t, P, f, keep, e0, have, s_staged[threadIdx.x >> 5]);
        } else if (have == NUQ_STATE_BLOCK && (BITS8 || (t.flags & kWide) == kWide)) {
            step_whole<BITS8>(t, P, f, keep, e0);
        } else if constexpr (BITS8) {
            step_part8<false>(t, P, f, keep, e0, have, s_staged[threadIdx.x >> 5]);
        } else {
            step_part32(t, P, f, keep, e0, have);
        }
    }
}

// Launches a kernel so that its CTAs may be set up while the kernel before it in the stream ends, if that one lets it in (the norm lets
// the step in; the step, whose CTAs come and go, nobody).
template <class... Params, class... Args>
static cudaError_t launch_overlapped(void (*kernel)(Params...), uint32_t grid, uint32_t threads, cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t cfg = cudaLaunchConfig_t{};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <uint32_t CAP, int KIND>
static cudaError_t launch_step(const StepTable<CAP>& T, const AdamwParams& P, uint32_t rounds, cudaStream_t stream) {
    return launch_overlapped(adamw_kernel<CAP, KIND>, T.tiles, kStepThreads, stream, T, P, rounds);
}

constexpr uint32_t kStepMany = 400;                         // tensors of a launch: what fits the parameters
constexpr uint32_t kMaxTiles = 1u << 30;                    // of a launch

template <uint32_t CAP, class Table>
static Table shortened(const StepTable<kStepMany>& all) {
    Table T;
    T.count = all.count;
    T.tiles = all.tiles;
    for (uint32_t i = 0; i < all.count; ++i) {
        T.first[i] = all.first[i];
        T.tensor[i] = all.tensor[i];
    }
    return T;
}

static uint32_t flags_of(const nuq_tensor& x) {
    auto off = [](const void* p, uintptr_t unit) { return reinterpret_cast<uintptr_t>(p) & (unit - 1u); };
    const uintptr_t state = x.types & NUQ_STATES_8BIT ? 4u : 16u;
    uint32_t flags = x.types;
    if (!off(x.g, (x.types & 0xffu) == NUQ_GRAD_F32 ? 16u : 8u)) flags |= kWideGrad;
    if (!off(x.w, 16u)) flags |= kWideW;
    if ((x.types & 0xff00u) == NUQ_COPY_NONE || !off(x.copy, 8u)) flags |= kWideCopy;
    if (!off(x.m, state) && !off(x.v, state)) flags |= kWideStates;
    return flags;
}
static int kind_of(const nuq_tensor& x) { return !(x.types & NUQ_STATES_8BIT) ? kStates32 : (flags_of(x) & kWide) == kWide ? kStates8 : kStates8Narrow; }

template <int KIND>
static cudaError_t launch_kind(const nuq_tensor* tensors, uint32_t count, const AdamwParams& P, double lr, uint64_t elements, int sms, cudaStream_t stream) {
    StepTable<kStepMany> T;
    T.count = T.tiles = 0;
    // 8-bit states: up to sixteen blocks to a warp, as long as every SM gets its CTAs four times over (2^28 elements in one tensor, passes for
    // half a second: four blocks 809 us, eight 793, sixteen 783; twice as many or half as many CTAs: no difference there,
    // 25.6 x 10^6 elements in 161 tensors 78.6 and 80.9 with twice as many).  fp32 states: one (persistent CTAs 1260 to 1330
    // us for 2^28 elements, CTAs of one block 1160).
    const uint64_t share = elements / ((uint64_t)sms * kStepCtas8 * 4u * kStepTile);
    const uint32_t rounds = KIND == kStates32 || share <= 1u ? 1u : share < 16u ? (uint32_t)share : 16u;
    auto flush = [&] {
        if (T.count == 0u) return cudaSuccess;
        // (A launch takes longer the more parameters it has, 7 ns for a tensor's place: one tensor of 256 elements 3.1 us in a table
        // of 16, 3.5 of 64, 4.9 of 256, 5.9 of 400.  So each table has four times the places of the one before.)
        const cudaError_t e = T.count <= 16u    ? launch_step<16u, KIND>(shortened<16u, StepTable<16u>>(T), P, rounds, stream)
                              : T.count <= 64u  ? launch_step<64u, KIND>(shortened<64u, StepTable<64u>>(T), P, rounds, stream)
                              : T.count <= 256u ? launch_step<256u, KIND>(shortened<256u, StepTable<256u>>(T), P, rounds, stream)
                                                : launch_step<kStepMany, KIND>(T, P, rounds, stream);
        T.count = T.tiles = 0;
        return e;
    };
    for (uint32_t i = 0; i < count; ++i) {
        const nuq_tensor& x = tensors[i];
        if (x.n == 0u || kind_of(x) != KIND) continue;
        const uint64_t tiles = (x.n + kStepTile * rounds - 1u) / (kStepTile * rounds);
        if (T.count == kStepMany || T.tiles + tiles > kMaxTiles) {
            const cudaError_t e = flush();
            if (e != cudaSuccess) return e;
        }
        StepTensor& t = T.tensor[T.count];
        t.g = x.g;
        t.w = x.w;
        t.copy = x.copy;
        t.m = x.m;
        t.v = x.v;
        t.scales = x.scales;
        t.n = x.n;
        t.decay = (float)(lr * (double)x.weight_decay);
        t.flags = flags_of(x);
        t.index = i;
        T.first[T.count++] = T.tiles;
        T.tiles += (uint32_t)tiles;
    }
    return flush();
}

cudaError_t launch_adamw(const nuq_tensor* tensors, uint32_t count, const AdamwParams& P, double lr, int sms, cudaStream_t stream) {
    uint64_t elements[3] = {0, 0, 0};
    for (uint32_t i = 0; i < count; ++i) elements[kind_of(tensors[i])] += tensors[i].n;
    cudaError_t e = cudaSuccess;
    if (elements[kStates32]) e = launch_kind<kStates32>(tensors, count, P, lr, elements[kStates32], sms, stream);
    if (e == cudaSuccess && elements[kStates8]) e = launch_kind<kStates8>(tensors, count, P, lr, elements[kStates8], sms, stream);
    if (e == cudaSuccess && elements[kStates8Narrow]) e = launch_kind<kStates8Narrow>(tensors, count, P, lr, elements[kStates8Narrow], sms, stream);
    return e;
}

// ---- the norm ----

// nuq_control and, behind its fields, the norm's scratch
struct ControlRecord {
    nuq_control c;
    double carried;          // sum of the launches before this one
    uint32_t arrived;        // CTAs whose sums are there
    uint32_t begun;          // 1: the norm has written c (its scale may be 0 all the same)
    double pad[3];
    double sums[kNormMaxGrid];
};
static_assert(sizeof(nuq_control) == 24 && offsetof(ControlRecord, begun) == 36 && offsetof(ControlRecord, sums) == 64 && sizeof(ControlRecord) <= NUQ_CONTROL_BYTES, "the record");

// The sum of eight squares.  In fp32 unless they leave its range: eight roundings of relative size 2^-24 (seven with 16-bit gradients, whose
// squares are exact) in sums that are added up in fp64.
__device__ __forceinline__ double eight_squares(const float (&x)[8]) {
    float p = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) p = __fmaf_rn(x[i], x[i], p);
    if (p >= 0x1p-60f && p < 0x1p120f) return (double)p;
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
    if (p == 0.0f && most == 0.0f) return 0.0;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) d += (double)x[i] * (double)x[i];
    return d;
}

// The 16 bytes of elements [first, first + unit) of a tensor of n, with zeros for those that are not there.
__device__ __noinline__ uint4 load_part(const void* g, uint32_t unit, uint64_t first, uint64_t n) {
    uint32_t r[4] = {0, 0, 0, 0};
    for (uint32_t j = 0; j < unit; ++j) {
        const uint64_t e = first + j;                       // (in front of the tensor: below 0, that is huge)
        if (e >= n) continue;
        const uint32_t x = unit == 4u ? static_cast<const uint32_t*>(g)[e] : (uint32_t)static_cast<const uint16_t*>(g)[e] << (16u * (j & 1u));
        const uint32_t k = unit == 4u ? j : j >> 1;
        if (k == 0u) r[0] |= x;
        else if (k == 1u) r[1] |= x;
        else if (k == 2u) r[2] |= x;
        else r[3] |= x;
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// The squares of tile `tile` of a tensor: what this thread adds of them.  Tiles are counted from the 16-byte boundary at or below the
// tensor's first element, so that all their vectors are aligned; the first and the last may reach over the tensor's ends.
__device__ __forceinline__ double squares_of(const NormTensor& t, uint32_t type, uint32_t tile) {
    const uint32_t unit = type == NUQ_GRAD_F32 ? 4u : 8u;   // elements of a vector
    const uint32_t skew = norm_skew(t.g, type);
    const uint64_t first = (uint64_t)tile * kNormVectors * unit;            // counted from the boundary
    const uint4* const vectors = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(t.g) & ~(uintptr_t)15u) + (uint64_t)tile * kNormVectors;
    uint4 raw[kNormVectors / kNormThreads];
    if (first >= skew && first + kNormVectors * unit <= t.n + skew) {
#pragma unroll
        for (uint32_t i = 0; i < kNormVectors / kNormThreads; ++i) raw[i] = __ldcs(vectors + i * kNormThreads + threadIdx.x);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < kNormVectors / kNormThreads; ++i) {
            const uint64_t at = first + (uint64_t)(i * kNormThreads + threadIdx.x) * unit;
            raw[i] = make_uint4(0, 0, 0, 0);
            if (at >= skew && at + unit <= t.n + skew) raw[i] = vectors[i * kNormThreads + threadIdx.x];
            else if (at + unit > skew && at < t.n + skew) raw[i] = load_part(t.g, unit, at - skew, t.n);
        }
    }
    double sum = 0.0;
    if (type == NUQ_GRAD_F32) {
#pragma unroll
        for (uint32_t i = 0; i < kNormVectors / kNormThreads; i += 2) {
            const uint4 a = raw[i], b = raw[i + 1];
            const float x[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                                __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
            sum += eight_squares(x);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < kNormVectors / kNormThreads; ++i) {
            const uint4 a = raw[i];
            const float x[8] = {half_to_float(a.x & 0xffffu, type), half_to_float(a.x >> 16, type), half_to_float(a.y & 0xffffu, type), half_to_float(a.y >> 16, type),
                                half_to_float(a.z & 0xffffu, type), half_to_float(a.z >> 16, type), half_to_float(a.w & 0xffffu, type), half_to_float(a.w >> 16, type)};
            sum += eight_squares(x);
        }
    }
    return sum;
}

__device__ __forceinline__ double block_sum(double x, double (&shared)[kNormThreads / 32]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if (lane_id() == 0) shared[threadIdx.x >> 5] = x;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (uint32_t i = 0; i < kNormThreads / 32; ++i) s += shared[i];
    return s;
}

// begin, end: the first and the last launch of the call
template <uint32_t CAP>
__global__ void __launch_bounds__(kNormThreads) grad_norm_kernel(const __grid_constant__ NormTable<CAP> T, ControlRecord* control, float scale, float max_norm,
                                                                  uint32_t begin, uint32_t end) {
    __shared__ double shared[kNormThreads / 32];
    __shared__ bool s_last;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double sum = 0.0;
    uint32_t at = 0, end_tile = 0;                          // the tile's tensor, the tile behind its last
    for (uint32_t tile = blockIdx.x; tile < T.tiles; tile += gridDim.x) {
        if (tile >= end_tile) {
            at = tensor_of(T, tile, at);
            end_tile = at + 1u < T.count ? T.first[at + 1u] : T.tiles;
        }
        sum += squares_of(T.tensor[at], T.type[at], tile - T.first[at]);
    }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) {
        control->sums[blockIdx.x] = sum;
        __threadfence();
        s_last = atomicAdd(&control->arrived, 1u) + 1u == gridDim.x;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    // the CTA that came last adds them up, in an order that does not depend on which it is
    double total = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kNormThreads) total += *static_cast<volatile double*>(control->sums + i);
    total = block_sum(total, shared);
    if (threadIdx.x != 0) return;
    control->arrived = 0;
    if (!begin) total += control->carried;
    control->carried = total;
    if (!end) return;
    const float norm = (float)(fabs((double)scale) * sqrt(total));
    const bool fine = norm < __uint_as_float(0x7f800000u);
    control->c.norm = norm;
    control->c.scale = norm > max_norm ? scale * __fdiv_rn(max_norm, norm) : scale;
    control->c.skip = fine ? 0u : 1u;
    control->begun = 1u;
    if (fine) control->c.step += 1u;
}

constexpr uint32_t kNormMany = 1536;                        // (31.5 KB of parameters)

template <uint32_t CAP>
static cudaError_t launch_norm(const NormTable<kNormMany>& all, ControlRecord* control, float scale, float max_norm, bool begin, bool end, int sms, cudaStream_t stream) {
    NormTable<CAP> T;
    T.count = all.count;
    T.tiles = all.tiles;
    for (uint32_t i = 0; i < all.count; ++i) {
        T.first[i] = all.first[i];
        T.tensor[i] = all.tensor[i];
        T.type[i] = all.type[i];
    }
    uint32_t grid = (uint32_t)sms * 8u;
    if (grid > kNormMaxGrid) grid = kNormMaxGrid;
    if (grid > T.tiles) grid = T.tiles ? T.tiles : 1u;
    return launch_overlapped(grad_norm_kernel<CAP>, grid, kNormThreads, stream, T, control, scale, max_norm, (uint32_t)begin, (uint32_t)end);
}

cudaError_t launch_grad_norm(const nuq_tensor* tensors, uint32_t count, float scale, float max_norm, nuq_control* control, int sms, cudaStream_t stream) {
    NormTable<kNormMany> T;
    T.count = T.tiles = 0;
    bool begin = true;
    auto flush = [&](bool end) {
        ControlRecord* const record = reinterpret_cast<ControlRecord*>(control);
        // (the largest table costs 1.1 us more than one of 256 places, that one 0.1 more than one of 32)
        const cudaError_t e = T.count <= 32u    ? launch_norm<32u>(T, record, scale, max_norm, begin, end, sms, stream)
                              : T.count <= 256u ? launch_norm<256u>(T, record, scale, max_norm, begin, end, sms, stream)
                                                : launch_norm<kNormMany>(T, record, scale, max_norm, begin, end, sms, stream);
        T.count = T.tiles = 0;
        begin = false;
        return e;
    };
    for (uint32_t i = 0; i < count; ++i) {
        const nuq_tensor& x = tensors[i];
        if (x.n == 0u) continue;
        const uint64_t tile = kNormVectors * ((x.types & 0xffu) == NUQ_GRAD_F32 ? 4u : 8u);
        const uint64_t tiles = (x.n + norm_skew(x.g, x.types & 0xffu) + tile - 1u) / tile;
        if (T.count == kNormMany || T.tiles + tiles > kMaxTiles) {
            const cudaError_t e = flush(false);
            if (e != cudaSuccess) return e;
        }
        T.tensor[T.count].g = x.g;
        T.tensor[T.count].n = x.n;
        T.type[T.count] = (uint8_t)(x.types & 0xffu);
        T.first[T.count++] = T.tiles;
        T.tiles += (uint32_t)tiles;
    }
    return flush(true);
}

}  // namespace nuq
