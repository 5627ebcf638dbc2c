// AdamW over lists of tensors, with moments in 32 or in 8 bits, and the norm of a list of gradients.
//
// All three are bound by memory: 28 bytes an element with fp32 moments, 16 with 8-bit ones, 4 for the norm (fp32 gradients).  The
// tensors' table travels in the kernel's parameters, so that nothing is uploaded, nothing is kept and a captured call holds its own.
// A tile is 2048 elements of one tensor, a warp's part of it 256: the block that shares the scales of 8-bit moments, so that its
// largest magnitude is one warp reduction and every array is read and written once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/nuq.h"
#include "nuq_adamw.cuh"
#include "nuq_launch.h"

namespace nuq {

constexpr uint32_t kStepThreads = 256;
constexpr uint32_t kStepTile = 8 * NUQ_STATE_BLOCK;
constexpr uint32_t kNormTile = 8192;
constexpr uint32_t kNormMaxGrid = (NUQ_CONTROL_BYTES - 64u) / 8u;

// A tensor of the step.  flags: the types, and which arrays are moved by whole vectors.
enum : uint32_t { kWide = 1u << 24 };
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
    uint32_t first[CAP];     // bits 0-29: the tensors' first tiles, 30-31: their types
    NormTensor tensor[CAP];
};

// The last tensor that begins at or before `tile`.
template <class Table>
__device__ __forceinline__ uint32_t tensor_of(const Table& T, uint32_t tile) {
    uint32_t lo = 0, hi = T.count;
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) >> 1;
        if (T.first[mid] <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
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

// Four gradients as they lie in memory, from element e on; `have` of them exist.
template <bool WIDE>
__device__ __forceinline__ uint4 load_grad(const void* g, uint32_t type, uint64_t e, uint32_t have) {
    uint4 r = make_uint4(0, 0, 0, 0);
    if (type == NUQ_GRAD_F32) {
        const uint32_t* p = static_cast<const uint32_t*>(g) + e;
        if (WIDE) return *reinterpret_cast<const uint4*>(p);
        if (have > 0u) r.x = p[0];
        if (have > 1u) r.y = p[1];
        if (have > 2u) r.z = p[2];
        if (have > 3u) r.w = p[3];
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(g) + e;
        if (WIDE) {
            const uint2 h = *reinterpret_cast<const uint2*>(p);
            r.x = h.x;
            r.y = h.y;
            return r;
        }
        if (have > 0u) r.x = p[0];
        if (have > 1u) r.x |= (uint32_t)p[1] << 16;
        if (have > 2u) r.y = p[2];
        if (have > 3u) r.y |= (uint32_t)p[3] << 16;
    }
    return r;
}
__device__ __forceinline__ float4 grad_values(uint4 r, uint32_t type) {
    if (type == NUQ_GRAD_F32) return make_float4(__uint_as_float(r.x), __uint_as_float(r.y), __uint_as_float(r.z), __uint_as_float(r.w));
    return make_float4(half_to_float(r.x & 0xffffu, type), half_to_float(r.x >> 16, type), half_to_float(r.y & 0xffffu, type), half_to_float(r.y >> 16, type));
}
template <bool WIDE>
__device__ __forceinline__ float4 load_floats(const float* p, uint32_t have) {
    if (WIDE) return *reinterpret_cast<const float4*>(p);
    return make_float4(have > 0u ? p[0] : 0.f, have > 1u ? p[1] : 0.f, have > 2u ? p[2] : 0.f, have > 3u ? p[3] : 0.f);
}
template <bool WIDE>
__device__ __forceinline__ void store_floats(float* p, float4 x, uint32_t have) {
    if (WIDE) {
        *reinterpret_cast<float4*>(p) = x;
        return;
    }
    if (have > 0u) p[0] = x.x;
    if (have > 1u) p[1] = x.y;
    if (have > 2u) p[2] = x.z;
    if (have > 3u) p[3] = x.w;
}
template <bool WIDE>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, uint32_t have) {
    if (WIDE) return *reinterpret_cast<const uint32_t*>(p);
    uint32_t r = 0;
    if (have > 0u) r = p[0];
    if (have > 1u) r |= (uint32_t)p[1] << 8;
    if (have > 2u) r |= (uint32_t)p[2] << 16;
    if (have > 3u) r |= (uint32_t)p[3] << 24;
    return r;
}
template <bool WIDE>
__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t x, uint32_t have) {
    if (WIDE) {
        *reinterpret_cast<uint32_t*>(p) = x;
        return;
    }
    if (have > 0u) p[0] = (uint8_t)x;
    if (have > 1u) p[1] = (uint8_t)(x >> 8);
    if (have > 2u) p[2] = (uint8_t)(x >> 16);
    if (have > 3u) p[3] = (uint8_t)(x >> 24);
}
template <bool WIDE>
__device__ __forceinline__ void store_copy(void* copy, uint64_t e, float4 x, bool bf16, uint32_t have) {
    const uint32_t lo = pack_halves(x.x, x.y, bf16), hi = pack_halves(x.z, x.w, bf16);
    uint16_t* const p = static_cast<uint16_t*>(copy) + e;
    if (WIDE) {
        *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
        return;
    }
    if (have > 0u) p[0] = (uint16_t)lo;
    if (have > 1u) p[1] = (uint16_t)(lo >> 16);
    if (have > 2u) p[2] = (uint16_t)hi;
    if (have > 3u) p[3] = (uint16_t)(hi >> 16);
}

// ---- 8-bit moments ----

// Philox4x32-10 of (c0, c1, c2, c3): 128 random bits
__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, const uint32_t (&keys)[20]) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ keys[2 * r];
        c2 = (uint32_t)(a >> 32) ^ c3 ^ keys[2 * r + 1];
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}

// four e4m3 codes as floats
__device__ __forceinline__ float4 code_values(uint32_t codes) {
    uint32_t a, b;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(a) : "h"((unsigned short)codes));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b) : "h"((unsigned short)(codes >> 16)));
    const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&a)), hi = __half22float2(*reinterpret_cast<const __half2*>(&b));
    return make_float4(lo.x, lo.y, hi.x, hi.y);
}

// |x| inv (at most 448, or not finite) in e4m3, rounded up with the probability that keeps the mean: the bits below the code's three of the
// mantissa are a fraction of its spacing, to which 16 random bits (and a half of their last place) are added.  Below 2^-6 the
// spacing stays 2^-9: adding 2^-6 brings such a number to where that is its spacing.
__device__ __forceinline__ uint32_t coded(float x, float inv, uint32_t random16) {
    const float y = __fmul_rn(fabsf(x), inv);
    const bool small = y < 0x1p-6f;
    const uint32_t code = ((__float_as_uint(small ? __fadd_rn(y, 0x1p-6f) : y) + (random16 << 4) + 8u) >> 20) - (small ? 968u : 960u);
    return fabsf(x) < __uint_as_float(0x7f800000u) ? code : 0x7fu;
}

// The largest finite magnitude of a warp's values, 2^-100 at least.
__device__ __forceinline__ float largest(const float (&x)[8]) {
    const float inf = __uint_as_float(0x7f800000u);
    float most = 0x1p-100f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));     // (NaN counts for nothing)
    most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
    if (most == inf) {
        most = 0x1p-100f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (fabsf(x[i]) < inf) most = fmaxf(most, fabsf(x[i]));
        most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
    }
    return most;
}

// A warp's 256 elements from e0 on, `left` of which exist.  A lane has two groups of four neighbours, 128 apart: what it loads
// at once from fp32 arrays are 16 bytes, and one Philox block serves a group.
template <bool BITS8, bool WIDE>
__device__ __forceinline__ void step_block(const StepTensor& t, const AdamwParams& P, const AdamwFactors& f, uint64_t e0, uint32_t left) {
    const uint32_t lane = lane_id(), type = t.flags & 0xffu, copy_type = t.flags & 0xff00u;
    const float keep = 1.0f - f.lr_factor * t.decay;
    uint4 raw[2];
    float4 w[2], m4[2], v4[2];
    uint32_t cm[2], cv[2], have[2];
    float2 scales = make_float2(0.f, 0.f);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const uint32_t at = 128u * q + 4u * lane;
        const uint64_t e = e0 + at;
        have[q] = WIDE ? 4u : left > at ? left - at : 0u;
        raw[q] = load_grad<WIDE>(t.g, type, e, have[q]);
        w[q] = load_floats<WIDE>(t.w + e, have[q]);
        if (BITS8) {
            cm[q] = load_codes<WIDE>(static_cast<const uint8_t*>(t.m) + e, have[q]);
            cv[q] = load_codes<WIDE>(static_cast<const uint8_t*>(t.v) + e, have[q]);
        } else {
            m4[q] = load_floats<WIDE>(static_cast<const float*>(t.m) + e, have[q]);
            v4[q] = load_floats<WIDE>(static_cast<const float*>(t.v) + e, have[q]);
        }
    }
    if (BITS8) scales = *reinterpret_cast<const float2*>(t.scales + 2u * (e0 / NUQ_STATE_BLOCK));
    float m[8], v[8];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const uint64_t e = e0 + 128u * q + 4u * lane;
        const float4 g4 = grad_values(raw[q], type);
        if (BITS8) {
            m4[q] = code_values(cm[q]);
            v4[q] = code_values(cv[q]);
        }
        const float g[4] = {g4.x, g4.y, g4.z, g4.w}, mo[4] = {m4[q].x, m4[q].y, m4[q].z, m4[q].w}, vo[4] = {v4[q].x, v4[q].y, v4[q].z, v4[q].w};
        float wn[4] = {w[q].x, w[q].y, w[q].z, w[q].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mi = mo[i], vi = vo[i];
            if (BITS8) {
                mi = __fmul_rn(mi, scales.x);
                vi = __fmul_rn(vi, scales.y);
                vi = __fmul_rn(vi, vi);
            }
            adamw_moments(P, __fmul_rn(g[i], f.scale), mi, vi);
            const float root = __fsqrt_rn(vi);
            wn[i] = adamw_value(P, f, keep, wn[i], mi, root);
            m[4 * q + i] = mi;
            v[4 * q + i] = BITS8 ? root : vi;
        }
        const float4 out = make_float4(wn[0], wn[1], wn[2], wn[3]);
        store_floats<WIDE>(t.w + e, out, have[q]);
        if (copy_type != NUQ_COPY_NONE) store_copy<WIDE>(t.copy, e, out, copy_type == NUQ_COPY_BF16, have[q]);
        if (!BITS8) {
            store_floats<WIDE>(static_cast<float*>(t.m) + e, make_float4(m[4 * q], m[4 * q + 1], m[4 * q + 2], m[4 * q + 3]), have[q]);
            store_floats<WIDE>(static_cast<float*>(t.v) + e, make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]), have[q]);
        }
    }
    if (BITS8) {
        const float most_m = largest(m), most_v = largest(v);
        const float inv_m = __fdiv_rn(448.0f, most_m), inv_v = __fdiv_rn(448.0f, most_v);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint64_t e = e0 + 128u * q + 4u * lane, quad = e >> 2;
            const uint4 r = philox((uint32_t)quad, (uint32_t)(quad >> 32), f.t, t.index, P.round_keys);
            const uint32_t random[4] = {r.x, r.y, r.z, r.w};
            uint32_t nm = 0, nv = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = coded(m[4 * q + i], inv_m, random[i] & 0xffffu), b = coded(v[4 * q + i], inv_v, random[i] >> 16);
                const uint32_t sign_m = __float_as_uint(m[4 * q + i]) >> 31, sign_v = __float_as_uint(v[4 * q + i]) >> 31;
                nm |= (a | sign_m << 7) << (8 * i);
                nv |= ((v[4 * q + i] > 0.0f && b == 0u ? 1u : b) | sign_v << 7) << (8 * i);
            }
            store_codes<WIDE>(static_cast<uint8_t*>(t.m) + e, nm, have[q]);
            store_codes<WIDE>(static_cast<uint8_t*>(t.v) + e, nv, have[q]);
        }
        if (lane == 0)
            *reinterpret_cast<float2*>(t.scales + 2u * (e0 / NUQ_STATE_BLOCK)) = make_float2(__fdiv_rn(most_m, 448.0f), __fdiv_rn(most_v, 448.0f));
    }
}

template <uint32_t CAP, bool BITS8>
__global__ void __launch_bounds__(kStepThreads) adamw_kernel(const __grid_constant__ StepTable<CAP> T, const __grid_constant__ AdamwParams P) {
    const AdamwFactors f = adamw_factors(P);
    if (!f.taken) return;
    for (uint32_t tile = blockIdx.x; tile < T.tiles; tile += gridDim.x) {
        const uint32_t i = tensor_of(T, tile);
        const StepTensor& t = T.tensor[i];
        const uint64_t e0 = (uint64_t)(tile - T.first[i]) * kStepTile + (threadIdx.x >> 5) * NUQ_STATE_BLOCK;
        if (e0 >= t.n) continue;
        const uint64_t left = t.n - e0;
        if (left >= NUQ_STATE_BLOCK && (t.flags & kWide)) step_block<BITS8, true>(t, P, f, e0, NUQ_STATE_BLOCK);
        else step_block<BITS8, false>(t, P, f, e0, left < NUQ_STATE_BLOCK ? (uint32_t)left : NUQ_STATE_BLOCK);
    }
}

template <uint32_t CAP, bool BITS8>
static cudaError_t launch_step(const StepTable<CAP>& T, const AdamwParams& P, int sms, cudaStream_t stream) {
    const uint32_t most = (uint32_t)sms * 16u;
    adamw_kernel<CAP, BITS8><<<T.tiles < most ? T.tiles : most, kStepThreads, 0, stream>>>(T, P);
    return cudaGetLastError();
}

constexpr uint32_t kStepMany = 400;                         // tensors of a launch: what fits the parameters
constexpr uint32_t kStepMaxTiles = 1u << 30;

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

template <bool BITS8>
static cudaError_t launch_list(const nuq_tensor* tensors, uint32_t count, const AdamwParams& P, double lr, int sms, cudaStream_t stream) {
    StepTable<kStepMany> T;
    T.count = T.tiles = 0;
    auto flush = [&] {
        if (T.count == 0u) return cudaSuccess;
        // (a launch takes longer the more parameters it has: a small table for few tensors)
        const cudaError_t e = T.count <= 16u    ? launch_step<16u, BITS8>(shortened<16u, StepTable<16u>>(T), P, sms, stream)
                              : T.count <= 176u ? launch_step<176u, BITS8>(shortened<176u, StepTable<176u>>(T), P, sms, stream)
                                                : launch_step<kStepMany, BITS8>(T, P, sms, stream);
        T.count = T.tiles = 0;
        return e;
    };
    for (uint32_t i = 0; i < count; ++i) {
        const nuq_tensor& x = tensors[i];
        if (x.n == 0u || ((x.types & NUQ_STATES_8BIT) != 0u) != BITS8) continue;
        const uint64_t tiles = (x.n + kStepTile - 1u) / kStepTile;
        if (T.count == kStepMany || T.tiles + tiles > kStepMaxTiles) {
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
        t.index = i;
        auto off = [](const void* p, uintptr_t unit) { return reinterpret_cast<uintptr_t>(p) & (unit - 1u); };
        const bool narrow = off(x.g, (x.types & 0xffu) == NUQ_GRAD_F32 ? 16u : 8u) || off(x.w, 16u) || off(x.m, BITS8 ? 4u : 16u) || off(x.v, BITS8 ? 4u : 16u) ||
                            ((x.types & 0xff00u) != NUQ_COPY_NONE && off(x.copy, 8u));
        t.flags = x.types | (narrow ? 0u : kWide);
        T.first[T.count++] = T.tiles;
        T.tiles += (uint32_t)tiles;
    }
    return flush();
}

cudaError_t launch_adamw(const nuq_tensor* tensors, uint32_t count, const AdamwParams& P, double lr, int sms, cudaStream_t stream) {
    const cudaError_t e = launch_list<false>(tensors, count, P, lr, sms, stream);
    return e != cudaSuccess ? e : launch_list<true>(tensors, count, P, lr, sms, stream);
}

// ---- the norm ----

// nuq_control and, behind its fields, the norm's scratch
struct ControlRecord {
    nuq_control c;
    double carried;          // sum of the launches before this one
    uint32_t arrived, pad;   // CTAs whose sums are there
    double pad2[3];
    double sums[kNormMaxGrid];
};
static_assert(sizeof(nuq_control) == 24 && offsetof(ControlRecord, sums) == 64 && sizeof(ControlRecord) <= NUQ_CONTROL_BYTES, "the record");

// The sum of eight squares.  In fp32 unless they leave its range: seven roundings of relative size 2^-24 in sums that are
// added up in fp64.
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

// The squares of elements [from, to) of a tensor: what this thread adds of them.
__device__ __forceinline__ double squares_of(const NormTensor& t, uint32_t type, uint64_t from, uint64_t to) {
    const uint32_t unit = type == NUQ_GRAD_F32 ? 4u : 8u;   // elements of 16 bytes
    const uintptr_t base = reinterpret_cast<uintptr_t>(t.g);
    const uint64_t skew = (base & 15u) / (16u / unit);      // elements between the 16-byte boundary below the tensor and its first
    // 16-byte vectors, counted from that boundary; the first and the last may hold elements that are not in the range
    const uint64_t v0 = (from + skew) / unit, v1 = (to + skew + unit - 1u) / unit;
    const uint4* const vectors = reinterpret_cast<const uint4*>(base & ~(uintptr_t)15u);
    auto load = [&](uint64_t i) {
        const uint64_t first = i * unit, lo = from + skew, hi = to + skew;
        if (first >= lo && first + unit <= hi) return vectors[i];
        uint32_t r[4] = {0, 0, 0, 0};
        for (uint32_t j = 0; j < unit; ++j) {
            if (first + j < lo || first + j >= hi) continue;
            const uint64_t e = first + j - skew;
            if (unit == 4u) r[j & 3u] = static_cast<const uint32_t*>(t.g)[e];
            else r[(j >> 1) & 3u] |= (uint32_t)static_cast<const uint16_t*>(t.g)[e] << (16u * (j & 1u));
        }
        return make_uint4(r[0], r[1], r[2], r[3]);
    };
    double sum = 0.0;
    const uint32_t at_once = unit == 4u ? 2u : 1u;
    for (uint64_t i = v0 + threadIdx.x * 1u; i < v1; i += kStepThreads * at_once) {
        float x[8];
        if (unit == 4u) {
            const uint64_t j = i + kStepThreads;
            const uint4 a = load(i), b = j < v1 ? load(j) : make_uint4(0, 0, 0, 0);
            x[0] = __uint_as_float(a.x); x[1] = __uint_as_float(a.y); x[2] = __uint_as_float(a.z); x[3] = __uint_as_float(a.w);
            x[4] = __uint_as_float(b.x); x[5] = __uint_as_float(b.y); x[6] = __uint_as_float(b.z); x[7] = __uint_as_float(b.w);
        } else {
            const uint4 a = load(i);
            x[0] = half_to_float(a.x & 0xffffu, type); x[1] = half_to_float(a.x >> 16, type);
            x[2] = half_to_float(a.y & 0xffffu, type); x[3] = half_to_float(a.y >> 16, type);
            x[4] = half_to_float(a.z & 0xffffu, type); x[5] = half_to_float(a.z >> 16, type);
            x[6] = half_to_float(a.w & 0xffffu, type); x[7] = half_to_float(a.w >> 16, type);
        }
        sum += eight_squares(x);
    }
    return sum;
}

__device__ __forceinline__ double block_sum(double x, double (&shared)[kStepThreads / 32]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if (lane_id() == 0) shared[threadIdx.x >> 5] = x;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (uint32_t i = 0; i < kStepThreads / 32; ++i) s += shared[i];
    return s;
}

// begin, end: the first and the last launch of the call
template <uint32_t CAP>
__global__ void __launch_bounds__(kStepThreads) grad_norm_kernel(const __grid_constant__ NormTable<CAP> T, ControlRecord* control, float scale, float max_norm,
                                                                  uint32_t begin, uint32_t end) {
    __shared__ double shared[kStepThreads / 32];
    __shared__ bool s_last;
    double sum = 0.0;
    for (uint32_t tile = blockIdx.x; tile < T.tiles; tile += gridDim.x) {
        uint32_t lo = 0, hi = T.count;
        while (hi - lo > 1u) {
            const uint32_t mid = (lo + hi) >> 1;
            if ((T.first[mid] & 0x3fffffffu) <= tile) lo = mid;
            else hi = mid;
        }
        const NormTensor& t = T.tensor[lo];
        const uint64_t from = (uint64_t)(tile - (T.first[lo] & 0x3fffffffu)) * kNormTile, to = t.n - from < kNormTile ? t.n : from + kNormTile;
        sum += squares_of(t, T.first[lo] >> 30, from, to);
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
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kStepThreads) total += *static_cast<volatile double*>(control->sums + i);
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
    if (fine) control->c.step += 1u;
}

constexpr uint32_t kNormMany = 1536;

template <uint32_t CAP>
static cudaError_t launch_norm(const NormTable<kNormMany>& all, ControlRecord* control, float scale, float max_norm, bool begin, bool end, int sms, cudaStream_t stream) {
    NormTable<CAP> T;
    T.count = all.count;
    T.tiles = all.tiles;
    for (uint32_t i = 0; i < all.count; ++i) {
        T.first[i] = all.first[i];
        T.tensor[i] = all.tensor[i];
    }
    uint32_t grid = (uint32_t)sms * 8u;
    if (grid > kNormMaxGrid) grid = kNormMaxGrid;
    if (grid > T.tiles) grid = T.tiles ? T.tiles : 1u;
    grad_norm_kernel<CAP><<<grid, kStepThreads, 0, stream>>>(T, control, scale, max_norm, begin, end);
    return cudaGetLastError();
}

cudaError_t launch_grad_norm(const nuq_tensor* tensors, uint32_t count, float scale, float max_norm, nuq_control* control, int sms, cudaStream_t stream) {
    NormTable<kNormMany> T;
    T.count = T.tiles = 0;
    bool begin = true;
    auto flush = [&](bool end) {
        ControlRecord* const record = reinterpret_cast<ControlRecord*>(control);
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
        const uint64_t tiles = (x.n + kNormTile - 1u) / kNormTile;
        if (T.count == kNormMany || T.tiles + tiles >= 1u << 30) {
            const cudaError_t e = flush(false);
            if (e != cudaSuccess) return e;
        }
        T.tensor[T.count].g = x.g;
        T.tensor[T.count].n = x.n;
        T.first[T.count++] = T.tiles | (x.types & 0xffu) << 30;
        T.tiles += (uint32_t)tiles;
    }
    return flush(true);
}

}  // namespace nuq
