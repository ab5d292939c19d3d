// asteria_attention and asteria_attention_backward: causal attention over packed sequences with grouped heads.
//
// One pass over the keys with the running maximum and sum of the softmax; no matrix of scores reaches memory.  The products
// are arranged so that what comes out of one matrix instruction is an operand of the next without leaving its lane: a
// 32 x 32 result holds, in lane l, column l % 32 and the rows 8 (i / 4) + 4 (l / 32) + i % 4, i = 0 .. 15; as the second
// operand of the next product lane l holds column l % 32 and eight of 16 places of the contraction, whose order is free as long
// as the first operand follows it.  So
//   forward        S^T = K Q^T,  O^T += V^T P^T             a lane holds one query; V^T read from LDS with transposing loads
//   gradient of Q  S^T = K Q^T,  dP^T = V dO^T,  dQ^T += K^T dS^T
//   of K and V     S = Q K^T,  dP = dO V^T,  dV^T += dO^T P,  dK^T += Q^T dS     a lane holds one key
// In bf16 a product takes v_mfma_f32_32x32x16_bf16; in fp32 the same eight values a lane go through eight
// v_mfma_f32_32x32x2_f32, each of which takes the pair of places that the two halves of the wavefront hold.
#include <math.h>
#include <type_traits>

#include "common.h"
#include "rows.h"

using namespace asteria;

namespace {

typedef float acc16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;
constexpr int NT = 256;            // threads of a workgroup: four wavefronts
constexpr int QT = 128;            // rows of a workgroup's tile, 32 a wavefront

template <typename T> struct Op;
template <> struct Op<bf16_elem> {
    typedef __bf16 frag __attribute__((ext_vector_type(8)));
    static constexpr int BK = 64;             // rows of a staged tile
    static constexpr int PAD = 8;             // elements behind a staged row: 16-byte reads of 8 rows side by side meet in no bank
    __device__ static __forceinline__ acc16 mma(frag a, frag b, acc16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    __device__ static __forceinline__ frag rows(const bf16_elem *p) { return *reinterpret_cast<const frag *>(p); }
    // eight rows (4 h + j % 4 + 8 (j / 4)) of column l % 32 of the 16 x 32 piece at p
    __device__ static __forceinline__ frag cols(const bf16_elem *p, int pitch)
    {
        const int l = (int)threadIdx.x & 63, h = l >> 5, i = l & 15;
        const bf16_elem *q = p + (4 * h + (i >> 2)) * pitch + 16 * ((l >> 4) & 1) + 4 * (i & 3);
        union { struct { s16x4 lo, hi; } s; frag f; } u;
        u.s.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)q);
        u.s.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(q + 8 * pitch));
        return u.f;
    }
    __device__ static __forceinline__ frag pack(const acc16 &v, int from)
    {
        frag f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (__bf16)v[from + j];
        return f;
    }
    __device__ static __forceinline__ float get(const frag &f, int j) { return (float)f[j]; }
};
template <> struct Op<float> {
    typedef float frag __attribute__((ext_vector_type(8)));
    static constexpr int BK = 32;
    static constexpr int PAD = 4;
    __device__ static __forceinline__ acc16 mma(frag a, frag b, acc16 c)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
    __device__ static __forceinline__ frag rows(const float *p)
    {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
        return frag{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
    __device__ static __forceinline__ frag cols(const float *p, int pitch)
    {
        const int l = (int)threadIdx.x & 63, h = l >> 5;
        frag f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = p[(4 * h + (j & 3) + 8 * (j >> 2)) * pitch + (l & 31)];
        return f;
    }
    __device__ static __forceinline__ frag pack(const acc16 &v, int from)
    {
        frag f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = v[from + j];
        return f;
    }
    __device__ static __forceinline__ float get(const frag &f, int j) { return f[j]; }
};

__device__ __forceinline__ int acc_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// values of a lane and of the one 32 places away, joined
template <bool MAX> __device__ __forceinline__ float join_halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return join<MAX>(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// An array of rows x heads x dim.
struct Array {
    char *p;
    int64_t ld, hs;
};
struct Args {
    Array Q, K, V, O, dO, dQ, dK, dV;
    float *lse, *delta;
    const int *cu;
    int total, nseq, heads, group, dim;
    float scale;
};

template <typename T> __device__ __forceinline__ T *at(const Array &a, int row, int head)
{
    return reinterpret_cast<T *>(a.p) + (int64_t)row * a.ld + (int64_t)head * a.hs;
}

// ---- which tile a workgroup takes ----------------------------------------------------------------
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_add(int v)
{
    return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
// sums over lanes 0 .. l of the wavefront
__device__ __forceinline__ int scan_lanes(int v)
{
    v = dpp_add<0x111, 0xf>(v);     // from 1, 2, 4, 8 lanes before in a row of 16
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);     // last lane of the row before
    v = dpp_add<0x143, 0xc>(v);     // last lane of the lower half
    return v;
}

struct Tile {
    int start, len, index;          // first row and length of the sequence, which tile of it
};

// Tile `item` of all sequences' tiles of QT rows, those with the most tiles before them in their sequence first (their
// work is longest in a forward pass).  The workgroups beyond the last tile get false.  All lanes of a wavefront take part.
__device__ __forceinline__ bool find_tile(const Args &a, int item, Tile &t)
{
    if (!a.cu) {
        t.start = 0; t.len = a.total;
        t.index = (a.total + QT - 1) / QT - 1 - item;
        return t.index >= 0;
    }
    const int l = (int)threadIdx.x & 63;
    auto load = [&](int s, int &start, int &len) {
        start = len = 0;
        if (s < a.nseq) {
            const int b = a.cu[s], e = a.cu[s + 1];
            start = b < 0 ? 0 : b > a.total ? a.total : b;
            len = (e > a.total ? a.total : e) - start;
            len = len < 0 ? 0 : len;
        }
    };
    int start, len;
    if (a.nseq <= 64) {
        load(l, start, len);
        const int tiles = (len + QT - 1) / QT;
        // the largest index of which more than `item` tiles have it or a larger one
        auto from = [&](int index) {
            const int over = tiles - index;
            return __builtin_amdgcn_readlane(scan_lanes(over > 0 ? over : 0), 63);
        };
        if (from(0) <= item) return false;
        int lo = 0, hi = (a.total + QT - 1) / QT;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (from(mid) > item) lo = mid; else hi = mid;
        }
        const int rank = item - from(lo + 1);
        const uint64_t have = __ballot(tiles > lo);
        const bool mine = tiles > lo && __builtin_popcountll(have & ((1ull << l) - 1)) == rank;
        const int s = __builtin_ctzll(__ballot(mine));
        t.start = __builtin_amdgcn_readlane(start, s);
        t.len = __builtin_amdgcn_readlane(len, s);
        t.index = lo;
        return true;
    }
    // many sequences: one after the other (finding the longest first would read cu several times in every workgroup)
    int before = 0;
    for (int s0 = 0; s0 < a.nseq; s0 += 64) {
        load(s0 + l, start, len);
        const int tiles = (len + QT - 1) / QT, upto = before + scan_lanes(tiles);
        const uint64_t past = __ballot(upto > item);
        if (past) {
            const int s = __builtin_ctzll(past);
            t.start = __builtin_amdgcn_readlane(start, s);
            t.len = __builtin_amdgcn_readlane(len, s);
            t.index = __builtin_amdgcn_readlane(upto, s) - 1 - item;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// ---- staging ------------------------------------------------------------------------------------
// BK rows of dim elements, padded with zeros to DP, from memory through registers to LDS.
template <typename T, int DP> struct Stage {
    static constexpr int BK = Op<T>::BK, PITCH = DP + Op<T>::PAD, CH = BK * DP / 8 / NT;
    Chunk<T> c[CH];
    __device__ __forceinline__ void load(const Array &a, int row0, int head, int rows, int dim)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = (int)threadIdx.x + NT * i, r = k / (DP / 8), d = k % (DP / 8) * 8;
            c[i].zero();
            if (r < rows && d < dim) c[i].load(at<const T>(a, row0 + r, head) + d, dim - d);
        }
    }
    __device__ __forceinline__ void store(T *lds) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = (int)threadIdx.x + NT * i, r = k / (DP / 8), d = k % (DP / 8) * 8;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<u16x8_any *>(__builtin_assume_aligned(lds + r * PITCH + d, 16)) = c[i].a;
            } else {
                *reinterpret_cast<f32x4_any *>(__builtin_assume_aligned(lds + r * PITCH + d, 16)) = c[i].a;
                *reinterpret_cast<f32x4_any *>(__builtin_assume_aligned(lds + r * PITCH + d + 4, 16)) = c[i].b;
            }
        }
    }
};

// The second operand of a product over dim: lane l holds row `row` of the array, elements 16 c + 8 h + j.
template <typename T, int DP>
__device__ __forceinline__ void load_frags(const Array &a, int row, int head, bool valid, int dim, typename Op<T>::frag (&f)[DP / 16])
{
    const int h = ((int)threadIdx.x >> 5) & 1;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        const int d = 16 * c + 8 * h;
        Chunk<T> k;
        k.zero();
        if (valid && d < dim) k.load(at<const T>(a, row, head) + d, dim - d);
        if constexpr (sizeof(T) == 2) {
            f[c] = __builtin_bit_cast(typename Op<T>::frag, k.a);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[c][j] = k.get(j);
        }
    }
}

// Rows `row`, elements 32 t + 8 g + 4 h + 0 .. 3 of a transposed result, times f.
template <typename T, int DP>
__device__ __forceinline__ void store_result(const Array &a, int row, int head, int dim, const acc16 (&o)[DP / 32], float f)
{
    const int h = ((int)threadIdx.x >> 5) & 1;
    T *p = at<T>(a, row, head);
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * t + 8 * g + 4 * h;
            if constexpr (sizeof(T) == 2) {
                typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
                u16x4_any v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = f32_bf16(o[t][4 * g + e] * f);
                if (d + 4 <= dim) *reinterpret_cast<u16x4_any *>(p + d) = v;
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) if (d + e < dim) p[d + e].bits = v[e];
                }
            } else {
                if (d + 4 <= dim) *reinterpret_cast<f32x4_any *>(p + d) = f32x4_any{o[t][4 * g] * f, o[t][4 * g + 1] * f, o[t][4 * g + 2] * f, o[t][4 * g + 3] * f};
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) if (d + e < dim) p[d + e] = o[t][4 * g + e] * f;
                }
            }
        }
}

// ---- forward ------------------------------------------------------------------------------------
template <typename T, int DP>
__global__ __launch_bounds__(NT) void attention_kernel(Args a)
{
    typedef Op<T> M;
    typedef Stage<T, DP> S;
    constexpr int BK = M::BK, PITCH = S::PITCH;
    __shared__ __attribute__((aligned(16))) T lk[BK * PITCH];
    __shared__ __attribute__((aligned(16))) T lv[BK * PITCH];
    Tile tile;
    const int head = (int)blockIdx.x % a.heads, kvh = head / a.group;
    if (!find_tile(a, (int)blockIdx.x / a.heads, tile)) return;
    const int l = (int)threadIdx.x & 63, h = l >> 5, qw = tile.index * QT + ((int)threadIdx.x >> 6) * 32, qi = qw + (l & 31);
    const bool valid = qi < tile.len;
    typename M::frag q[DP / 16];
    load_frags<T, DP>(a.Q, tile.start + qi, head, valid, a.dim, q);
    acc16 o[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) o[t] = 0.0f;
    // the maximum m follows only where the scores have grown by more than 2^8 of it: sums and O are scaled rarely, and
    // exp2 stays below 2^8
    const float c = a.scale * LOG2E, slack = 8.0f / c;
    float m = -INFINITY, sum = 0.0f;
    const int last = min(tile.len, (tile.index + 1) * QT), nk = (last + BK - 1) / BK;
    S sk, sv;
    sk.load(a.K, tile.start, kvh, last, a.dim);
    sv.load(a.V, tile.start, kvh, last, a.dim);
    for (int kt = 0; kt < nk; ++kt) {
        const int k0 = kt * BK;
        __syncthreads();
        sk.store(lk);
        sv.store(lv);
        __syncthreads();
        if (kt + 1 < nk) {
            sk.load(a.K, tile.start + k0 + BK, kvh, last - k0 - BK, a.dim);
            sv.load(a.V, tile.start + k0 + BK, kvh, last - k0 - BK, a.dim);
        }
        if (k0 > qw + 31) continue;              // behind this wavefront's rows
        acc16 s[BK / 32];
#pragma unroll
        for (int b = 0; b < BK / 32; ++b) {
            s[b] = 0.0f;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) s[b] = M::mma(M::rows(lk + (32 * b + (l & 31)) * PITCH + 16 * d + 8 * h), q[d], s[b]);
        }
        if (k0 + BK - 1 > qw) {
#pragma unroll
            for (int b = 0; b < BK / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) if (k0 + 32 * b + acc_row(i, h) > qi) s[b][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < BK / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = join_halves<true>(top);
        if (__any(top > m + slack)) {
            const float to = fmaxf(m, top), f = to == m ? 1.0f : __builtin_amdgcn_exp2f((m - to) * c);
            m = to;
            sum *= f;
#pragma unroll
            for (int t = 0; t < DP / 32; ++t) o[t] *= f;
        }
        const float mc = m == -INFINITY ? 0.0f : m * c;
#pragma unroll
        for (int b = 0; b < BK / 32; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, -mc));
                sum += s[b][i];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const typename M::frag p = M::pack(s[b], 8 * k);
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) o[t] = M::mma(M::cols(lv + (32 * b + 16 * k) * PITCH + 32 * t, PITCH), p, o[t]);
            }
        }
    }
    sum = join_halves<false>(sum);
    if (!valid) return;
    store_result<T, DP>(a.O, tile.start + qi, head, a.dim, o, 1.0f / sum);
    if (a.lse && h == 0) a.lse[(size_t)head * a.total + tile.start + qi] = (m * c + __builtin_amdgcn_logf(sum)) * LN2;
}

// ---- gradient of Q (and D = rowsum(dO o O), which the other kernel reads) ----------------------------
template <typename T, int DP>
__global__ __launch_bounds__(NT) void attention_dq_kernel(Args a)
{
    typedef Op<T> M;
    typedef Stage<T, DP> S;
    constexpr int BK = M::BK, PITCH = S::PITCH;
    __shared__ __attribute__((aligned(16))) T lk[BK * PITCH];
    __shared__ __attribute__((aligned(16))) T lv[BK * PITCH];
    Tile tile;
    const int head = (int)blockIdx.x % a.heads, kvh = head / a.group;
    if (!find_tile(a, (int)blockIdx.x / a.heads, tile)) return;
    const int l = (int)threadIdx.x & 63, h = l >> 5, qw = tile.index * QT + ((int)threadIdx.x >> 6) * 32, qi = qw + (l & 31);
    const bool valid = qi < tile.len;
    typename M::frag q[DP / 16], g[DP / 16];
    float delta = 0.0f;
    {
        load_frags<T, DP>(a.O, tile.start + qi, head, valid, a.dim, q);
        load_frags<T, DP>(a.dO, tile.start + qi, head, valid, a.dim, g);
#pragma unroll
        for (int d = 0; d < DP / 16; ++d)
#pragma unroll
            for (int j = 0; j < 8; ++j) delta += M::get(q[d], j) * M::get(g[d], j);
        delta = join_halves<false>(delta);
    }
    const size_t at_row = (size_t)head * a.total + tile.start + qi;
    if (valid && h == 0) a.delta[at_row] = delta;
    const float lse = valid ? a.lse[at_row] * LOG2E : 0.0f;
    load_frags<T, DP>(a.Q, tile.start + qi, head, valid, a.dim, q);
    acc16 o[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) o[t] = 0.0f;
    const float c = a.scale * LOG2E;
    const int last = min(tile.len, (tile.index + 1) * QT), nk = (last + BK - 1) / BK;
    S sk, sv;
    sk.load(a.K, tile.start, kvh, last, a.dim);
    sv.load(a.V, tile.start, kvh, last, a.dim);
    for (int kt = 0; kt < nk; ++kt) {
        const int k0 = kt * BK;
        __syncthreads();
        sk.store(lk);
        sv.store(lv);
        __syncthreads();
        if (kt + 1 < nk) {
            sk.load(a.K, tile.start + k0 + BK, kvh, last - k0 - BK, a.dim);
            sv.load(a.V, tile.start + k0 + BK, kvh, last - k0 - BK, a.dim);
        }
#pragma unroll
        for (int b = 0; b < BK / 32; ++b) {
            if (k0 + 32 * b > qw + 31) continue;
            acc16 s = 0.0f, dp = 0.0f;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                s = M::mma(M::rows(lk + (32 * b + (l & 31)) * PITCH + 16 * d + 8 * h), q[d], s);
                dp = M::mma(M::rows(lv + (32 * b + (l & 31)) * PITCH + 16 * d + 8 * h), g[d], dp);
            }
            const bool edge = k0 + 32 * b + 31 > qw;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -lse)) * (dp[i] - delta);
                // a row that sees one key has no gradient through the softmax: zero, not the round-off of dP - D
                if (edge && (k0 + 32 * b + acc_row(i, h) > qi || qi == 0)) s[i] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const typename M::frag p = M::pack(s, 8 * k);
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) o[t] = M::mma(M::cols(lk + (32 * b + 16 * k) * PITCH + 32 * t, PITCH), p, o[t]);
            }
        }
    }
    if (valid) store_result<T, DP>(a.dQ, tile.start + qi, head, a.dim, o, a.scale);
}

// ---- gradients of K and V: a wavefront holds 32 keys and passes over the rows that see them ------------
template <typename T, int DP>
__global__ __launch_bounds__(NT) void attention_dkv_kernel(Args a)
{
    typedef Op<T> M;
    typedef Stage<T, DP> S;
    constexpr int BK = M::BK, PITCH = S::PITCH;
    __shared__ __attribute__((aligned(16))) T lq[BK * PITCH];
    __shared__ __attribute__((aligned(16))) T lg[BK * PITCH];
    __shared__ __attribute__((aligned(16))) float rows[2][BK];
    Tile tile;
    const int kv_heads = a.heads / a.group, kvh = (int)blockIdx.x % kv_heads;
    if (!find_tile(a, (int)blockIdx.x / kv_heads, tile)) return;
    tile.index = (tile.len + QT - 1) / QT - 1 - tile.index;      // the first keys are seen by the most rows
    const int l = (int)threadIdx.x & 63, h = l >> 5, kw = tile.index * QT + ((int)threadIdx.x >> 6) * 32, ki = kw + (l & 31);
    const bool valid = ki < tile.len;
    typename M::frag kf[DP / 16], vf[DP / 16];
    load_frags<T, DP>(a.K, tile.start + ki, kvh, valid, a.dim, kf);
    load_frags<T, DP>(a.V, tile.start + ki, kvh, valid, a.dim, vf);
    acc16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) { dk[t] = 0.0f; dv[t] = 0.0f; }
    const float c = a.scale * LOG2E;
    const int first = tile.index * QT / BK, nq = (tile.len + BK - 1) / BK;
    S sq, sg;
    float lse = 0.0f, delta = 0.0f;
    auto load = [&](int head, int q0) {
        sq.load(a.Q, tile.start + q0, head, tile.len - q0, a.dim);
        sg.load(a.dO, tile.start + q0, head, tile.len - q0, a.dim);
        if (threadIdx.x < BK) {
            const bool in = q0 + (int)threadIdx.x < tile.len;
            const size_t at_row = (size_t)head * a.total + tile.start + q0 + threadIdx.x;
            lse = in ? a.lse[at_row] * LOG2E : 0.0f;
            delta = in ? a.delta[at_row] : 0.0f;
        }
    };
    const int steps = (nq - first) * a.group;
    load(kvh * a.group, first * BK);
    int qt = first, head = kvh * a.group;
    for (int step = 0; step < steps; ++step) {
        const int q0 = qt * BK;
        __syncthreads();
        sq.store(lq);
        sg.store(lg);
        if (threadIdx.x < BK) { rows[0][threadIdx.x] = lse; rows[1][threadIdx.x] = delta; }
        __syncthreads();
        if (++qt == nq) { qt = first; ++head; }
        if (step + 1 < steps) load(head, qt * BK);
#pragma unroll
        for (int b = 0; b < BK / 32; ++b) {
            if (q0 + 32 * b + 31 < kw) continue;                 // rows before this wavefront's keys
            acc16 s = 0.0f, dp = 0.0f;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                s = M::mma(M::rows(lq + (32 * b + (l & 31)) * PITCH + 16 * d + 8 * h), kf[d], s);
                dp = M::mma(M::rows(lg + (32 * b + (l & 31)) * PITCH + 16 * d + 8 * h), vf[d], dp);
            }
            const bool edge = q0 + 32 * b < kw + 31;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = 32 * b + acc_row(i, h);
                s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -rows[0][r]));
                dp[i] = s[i] * (dp[i] - rows[1][r]);
                if (edge && q0 + r < ki) { s[i] = 0.0f; dp[i] = 0.0f; }
                if (edge && q0 + r == 0) dp[i] = 0.0f;           // as in the gradient of Q
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const typename M::frag p = M::pack(s, 8 * k), ds = M::pack(dp, 8 * k);
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) {
                    dv[t] = M::mma(M::cols(lg + (32 * b + 16 * k) * PITCH + 32 * t, PITCH), p, dv[t]);
                    dk[t] = M::mma(M::cols(lq + (32 * b + 16 * k) * PITCH + 32 * t, PITCH), ds, dk[t]);
                }
            }
        }
    }
    if (!valid) return;
    store_result<T, DP>(a.dK, tile.start + ki, kvh, a.dim, dk, a.scale);
    store_result<T, DP>(a.dV, tile.start + ki, kvh, a.dim, dv, 1.0f);
}

// ---- host ---------------------------------------------------------------------------------------
// rows x heads x dim elements that share no place
bool apart(int64_t ld, int64_t hs, int64_t total, int64_t heads, int64_t dim)
{
    if (total == 1) return heads == 1 || hs >= dim;
    if (heads == 1) return ld >= dim;
    if (ld <= 0 || hs <= 0) return false;
    return (hs >= dim && ld / hs >= heads - 1 && ld - (heads - 1) * hs >= dim) || (ld >= dim && hs / ld >= total - 1 && hs - (total - 1) * ld >= dim);
}

asteria_status validate(const asteria_attn *a, bool writes_o)
{
    if (!a || !a->Q || !a->K || !a->V || !a->O) return ASTERIA_INVALID_ARG;
    if (a->total <= 0 || a->nseq <= 0 || a->heads <= 0 || a->kv_heads <= 0 || a->dim <= 0) return ASTERIA_INVALID_ARG;
    if (a->heads % a->kv_heads || (!a->cu && a->nseq != 1) || !valid_dtype(a->dtype)) return ASTERIA_INVALID_ARG;
    if (!(a->scale > 0.0f) || !isfinite(a->scale)) return ASTERIA_INVALID_ARG;
    if (a->ldq < 0 || a->ldk < 0 || a->ldv < 0 || a->ldo < 0 || a->hq < 0 || a->hk < 0 || a->hv < 0 || a->ho < 0) return ASTERIA_INVALID_ARG;
    if (writes_o && !apart(a->ldo, a->ho, a->total, a->heads, a->dim)) return ASTERIA_INVALID_ARG;
    if (a->dim > 128) return ASTERIA_UNSUPPORTED;
    if (((int64_t)a->total / QT + 1 + a->nseq) * a->heads > MOST_BLOCKS) return ASTERIA_UNSUPPORTED;
    return ASTERIA_OK;
}

Args args_of(const asteria_attn *a)
{
    Args k = {};
    auto array = [](const void *p, int64_t ld, int64_t hs) { return Array{reinterpret_cast<char *>(const_cast<void *>(p)), ld, hs}; };
    k.Q = array(a->Q, a->ldq, a->hq);
    k.K = array(a->K, a->ldk, a->hk);
    k.V = array(a->V, a->ldv, a->hv);
    k.O = array(a->O, a->ldo, a->ho);
    k.lse = a->lse; k.cu = a->cu;
    k.total = a->total; k.nseq = a->nseq; k.heads = a->heads; k.group = a->heads / a->kv_heads; k.dim = a->dim;
    k.scale = a->scale;
    return k;
}

// Most tiles that sequences of `total` rows together can have (rows / QT whole ones and one more each).
unsigned most_tiles(const asteria_attn *a)
{
    if (!a->cu) return (unsigned)((a->total + QT - 1) / QT);
    return (unsigned)(a->total / QT + (a->nseq < a->total ? a->nseq : a->total));
}

// Kernels for dims padded to 64 or 128.
template <typename F> asteria_status for_type(int dtype, int dim, F f)
{
    if (dtype == ASTERIA_BF16) return dim <= 64 ? f(bf16_elem(), std::integral_constant<int, 64>()) : f(bf16_elem(), std::integral_constant<int, 128>());
    return dim <= 64 ? f(float(), std::integral_constant<int, 64>()) : f(float(), std::integral_constant<int, 128>());
}

}  // namespace

extern "C" asteria_status asteria_attention(const asteria_attn *a, void *stream_)
{
    ASTERIA_TRY(validate(a, true));
    const Args k = args_of(a);
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    return for_type(a->dtype, a->dim, [&](auto t, auto dp) {
        typedef decltype(t) T;
        constexpr int DP = dp();
        hipLaunchKernelGGL((attention_kernel<T, DP>), dim3(most_tiles(a) * a->heads), dim3(NT), 0, stream, k);
        ASTERIA_HIP_TRY(hipGetLastError());
        return ASTERIA_OK;
    });
}

extern "C" size_t asteria_attention_backward_workspace_bytes(const asteria_attn *a)
{
    if (validate(a, false) != ASTERIA_OK) return 0;
    return Carver::need((size_t)a->total * a->heads, sizeof(float));
}

extern "C" asteria_status asteria_attention_backward(const asteria_attn *a, const asteria_attn_grad *g,
                                                     void *ws, size_t ws_bytes, void *stream_)
{
    ASTERIA_TRY(validate(a, false));
    if (!a->lse || !g || !g->dO || !g->dQ || !g->dK || !g->dV || g->lddo < 0 || g->hdo < 0) return ASTERIA_INVALID_ARG;
    if (!apart(g->lddq, g->hdq, a->total, a->heads, a->dim) || !apart(g->lddk, g->hdk, a->total, a->kv_heads, a->dim) ||
        !apart(g->lddv, g->hdv, a->total, a->kv_heads, a->dim)) return ASTERIA_INVALID_ARG;
    if (!ws || ws_bytes < asteria_attention_backward_workspace_bytes(a)) return ASTERIA_WORKSPACE_TOO_SMALL;
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return ASTERIA_INVALID_ARG;   // workspace must be 256-byte aligned
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    Args k = args_of(a);
    auto array = [](const void *p, int64_t ld, int64_t hs) { return Array{reinterpret_cast<char *>(const_cast<void *>(p)), ld, hs}; };
    k.dO = array(g->dO, g->lddo, g->hdo);
    k.dQ = array(g->dQ, g->lddq, g->hdq);
    k.dK = array(g->dK, g->lddk, g->hdk);
    k.dV = array(g->dV, g->lddv, g->hdv);
    Carver cv(ws);
    k.delta = cv.take<float>((size_t)a->total * a->heads);
    return for_type(a->dtype, a->dim, [&](auto t, auto dp) {
        typedef decltype(t) T;
        constexpr int DP = dp();
        hipLaunchKernelGGL((attention_dq_kernel<T, DP>), dim3(most_tiles(a) * a->heads), dim3(NT), 0, stream, k);
        ASTERIA_HIP_TRY(hipGetLastError());
        hipLaunchKernelGGL((attention_dkv_kernel<T, DP>), dim3(most_tiles(a) * a->kv_heads), dim3(NT), 0, stream, k);
        ASTERIA_HIP_TRY(hipGetLastError());
        return ASTERIA_OK;
    });
}
