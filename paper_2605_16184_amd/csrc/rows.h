// Rows of eight-element chunks, fp32 or bf16, at any alignment, and the sums and generator that the row-wise operators
// (norm, dropout) share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace asteria {

// A launch may have less than 2^32 threads.
constexpr int64_t MOST_BLOCKS = (1 << 24) - 1;     // of 256 threads

// A vector access needs only the alignment of its elements: global memory takes unaligned vectors, so rows at any offset
// and of any length are read by the same instructions, and only the chunk at a row's end goes element by element.
typedef uint16_t u16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint8_t u8x8_any __attribute__((ext_vector_type(8), aligned(1)));

struct bf16_elem { uint16_t bits; };

// to nearest, ties to even; the conversion instruction keeps what is no number
__device__ __forceinline__ uint16_t f32_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// n = 8 or fewer elements of a row as they lie in memory; the rest are zero.
template <typename T> struct Chunk;
template <> struct Chunk<float> {
    f32x4_any a, b;
    __device__ __forceinline__ void load(const float *p, int n)
    {
        if (n >= 8) {
            a = *reinterpret_cast<const f32x4_any *>(p);
            b = *reinterpret_cast<const f32x4_any *>(p + 4);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { a[e] = e < n ? p[e] : 0.0f; b[e] = e + 4 < n ? p[e + 4] : 0.0f; }
        }
    }
    __device__ __forceinline__ void zero() { a = 0.0f; b = 0.0f; }
    __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e] : b[e - 4]; }
};
template <> struct Chunk<bf16_elem> {
    u16x8_any a;
    __device__ __forceinline__ void load(const bf16_elem *p_, int n)
    {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(p_);
        if (n >= 8) {
            a = *reinterpret_cast<const u16x8_any *>(p);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = e < n ? p[e] : (uint16_t)0;
        }
    }
    __device__ __forceinline__ void zero() { a = (uint16_t)0; }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float((uint32_t)a[e] << 16); }
};

__device__ __forceinline__ void store8(float *p, const float (&v)[8], int n)
{
    if (n >= 8) {
        *reinterpret_cast<f32x4_any *>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4_any *>(p + 4) = f32x4_any{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (e < n) p[e] = v[e];
    }
}
__device__ __forceinline__ void store8(bf16_elem *p_, const float (&v)[8], int n)
{
    uint16_t *p = reinterpret_cast<uint16_t *>(p_);
    u16x8_any a;
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = f32_bf16(v[e]);
    if (n >= 8) {
        *reinterpret_cast<u16x8_any *>(p) = a;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (e < n) p[e] = a[e];
    }
}
// stores to an array whose type is known at run time only (uniform over the launch)
__device__ __forceinline__ void store8(void *base, int dtype, size_t off, const float (&v)[8], int n)
{
    if (dtype == ASTERIA_BF16) store8(reinterpret_cast<bf16_elem *>(base) + off, v, n);
    else store8(reinterpret_cast<float *>(base) + off, v, n);
}
__device__ __forceinline__ void load8(const void *base, int dtype, size_t off, float (&v)[8], int n)
{
    if (dtype == ASTERIA_BF16) {
        Chunk<bf16_elem> c;
        c.load(reinterpret_cast<const bf16_elem *>(base) + off, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c.get(e);
    } else {
        Chunk<float> c;
        c.load(reinterpret_cast<const float *>(base) + off, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c.get(e);
    }
}

// ---- dropout ------------------------------------------------------------------------------------
// What a kernel needs of an asteria_rng: keep where the 16 bits are >= threshold (0: everything is kept), times scale.
struct Dropper {
    uint64_t seed, offset;
    const uint64_t *state;
    uint32_t threshold;
    float scale;
};

// false: not a valid probability.  rng NULL or p = 0: nothing is dropped.
inline bool make_dropper(const asteria_rng *rng, Dropper &d)
{
    d = Dropper{0, 0, nullptr, 0, 1.0f};
    if (!rng) return true;
    if (!(rng->p >= 0.0f && rng->p <= 1.0f)) return false;
    const uint32_t t = (uint32_t)(65536.0 * (double)rng->p + 0.5);
    if (t > 65535u) return false;
    if (t == 0) return true;
    d.seed = rng->seed; d.offset = rng->offset; d.state = rng->state;
    d.threshold = t;
    d.scale = (float)(65536.0 / (65536.0 - t));
    return true;
}

__device__ __forceinline__ void read_state(Dropper &d)
{
    if (d.threshold && d.state) { d.seed = d.state[0]; d.offset = d.state[1]; }
}

// The eight 16-bit numbers of chunk `c` of row `r`: one block of the generator.  Sixteen bits an element, because the ten
// rounds (two 32 x 32 bit products each) would bound dropout in bf16 at 32: 35 operations an element against 18.
__device__ __forceinline__ void drop_chunk(const Dropper &d, uint32_t r, uint32_t c, float (&v)[8])
{
    uint32_t x0 = c, x1 = r, x2 = (uint32_t)d.offset, x3 = (uint32_t)(d.offset >> 32);
    uint32_t k0 = (uint32_t)d.seed, k1 = (uint32_t)(d.seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = (uint64_t)x0 * 0xD2511F53u, q = (uint64_t)x2 * 0xCD9E8D57u;
        x0 = (uint32_t)(q >> 32) ^ x1 ^ k0;
        x2 = (uint32_t)(p >> 32) ^ x3 ^ k1;
        x1 = (uint32_t)q;
        x3 = (uint32_t)p;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {x0, x1, x2, x3};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = (e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
        v[e] = u >= d.threshold ? v[e] * d.scale : 0.0f;
    }
}

// ---- sums and maxima over the threads of a row -----------------------------------------------------
template <bool MAX> __device__ __forceinline__ float join(float a, float b) { return MAX ? fmaxf(a, b) : a + b; }

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}

// Over 16 lanes side by side or the 64 of the wavefront, the result in all of them, without LDS.
template <bool MAX, int WIDTH> __device__ __forceinline__ float lanes_reduce(float v)
{
    static_assert(WIDTH == 16 || WIDTH == 64, "");
    v = join<MAX>(v, dpp<0xb1>(v));       // lanes 1 0 3 2 of a quad
    v = join<MAX>(v, dpp<0x4e>(v));       // lanes 2 3 0 1
    v = join<MAX>(v, dpp<0x141>(v));      // 7 - i of eight
    v = join<MAX>(v, dpp<0x140>(v));      // 15 - i of sixteen
    if constexpr (WIDTH == 64) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = join<MAX>(__uint_as_float(a[0]), __uint_as_float(a[1]));
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = join<MAX>(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    return v;
}

// N values over TPR threads (16, or a wavefront; more: the workgroup, through `part`, which the call leaves free for the next one).
template <bool MAX, int TPR, int N> __device__ __forceinline__ void row_reduce(float (&v)[N], float (*part)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_reduce<MAX, TPR < 64 ? TPR : 64>(v[i]);
    if constexpr (TPR > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) part[threadIdx.x >> 6][i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = part[0][i];
#pragma unroll
            for (int w = 1; w < TPR / 64; ++w) v[i] = join<MAX>(v[i], part[w][i]);
        }
    }
}

}  // namespace asteria
