// Causal attention over packed sequences with grouped heads: what the forward kernel and the two kernels of the backward
// pass share.
//
// One pass over the keys with the running maximum and sum of the softmax; no matrix of scores reaches memory.  The products
// are arranged so that what comes out of one matrix instruction is an operand of the next without leaving its lane: a
// 32 x 32 result holds, in lane l, column l % 32 and the rows 8 (i / 4) + 4 (l / 32) + i % 4, i = 0 .. 15; as the second
// operand of the next product lane l holds column l % 32 and eight of 16 places of the contraction, whose order is free as long
// as the first operand follows it.  So
//   forward        S^T = K Q^T,  O^T += V^T P^T             a lane holds one query; V^T read from LDS with transposing loads
//   gradient of Q  S^T = K Q^T,  dP^T = V dO^T,  dQ^T += K^T dS^T  (bf16: K^T P^T, too)
//   of K and V     S = Q K^T,  dP = dO V^T,  dV^T += dO^T P,  dK^T += Q^T dS     a lane holds one key
// All products run on v_mfma_f32_32x32x16_bf16: bf16 operands as they are, fp32 operands in three terms.
#pragma once
#include <math.h>
#include <type_traits>

#include "common.h"
#include "planes.h"
#include "rows.h"

namespace asteria {

typedef float acc16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f, BF16_MAX = 0x1.fep127f;
constexpr int ATT_THREADS = 256;      // four wavefronts, NA along the tile that the workgroup owns, NB along the rows it passes over

// The place in LDS of a pointer to it: the low half of its address.
__device__ __forceinline__ uint32_t lds_place(const void *p) { return (uint32_t)reinterpret_cast<uintptr_t>(p); }

// ---- operands -----------------------------------------------------------------------------------
// Operands from tiles of rows in LDS.  rows(): eight elements of one row, 8 h .. of the 16 from d on; cols(): of column d + l % 32 the eight rows
// 4 h + j % 4 + 8 (j / 4) from r on - the order in which a 32 x 32 result holds its rows.
template <typename T, int DP> struct Op;

// Tiles of bf16 rows of P (64 or 128) elements, S elements apart (P, or three times that), without padding: piece c (16 bytes) of row r lies
// at place c ^ swz(r).  LDS serves 256 bytes a cycle: reads of one piece from 16 rows side by side, and transposing reads of four
// pieces side by side from four rows, both meet every bank once.
template <int P, int S> struct Swizzled {
    typedef __bf16 piece __attribute__((ext_vector_type(8)));
    __device__ static __forceinline__ int swz(int r) { return (P == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1)) + ((r >> 2) & 3); }
    __device__ static __forceinline__ int place(int r, int c) { return r * S + ((c ^ swz(r)) << 3); }
    // What a lane reads of a tile (at a multiple of 256 bytes): the exclusive or with d goes last, on the address, so that it takes
    // one instruction a read and no register over the loop.
    struct Tile {
        uint32_t r, c;
        __device__ __forceinline__ explicit Tile(const void *tile)
        {
            const int l = (int)threadIdx.x & 63, i = l & 15;
            const uint32_t at = lds_place(tile);
            r = at + 2 * place(l & 31, l >> 5);
            c = at + 2 * (place(4 * (l >> 5) + (i >> 2), 2 * ((l >> 4) & 1) + ((i & 3) >> 1)) + 4 * (i & 1));
        }
    };
    // r a multiple of 32, d of 16; `more`: elements from the tile's beginning
    __device__ static __forceinline__ piece rows(const Tile &t, int r, int d, int more = 0)
    {
        return *reinterpret_cast<__attribute__((address_space(3))) const piece *>((t.r ^ (2 * d)) + (r * S + more) * 2);
    }
    // r a multiple of 16, d of 32: a 16-lane group reads four rows of 16 elements and gets, lane by lane, the columns
    __device__ static __forceinline__ piece cols(const Tile &t, int r, int d, int more = 0)
    {
        union { struct { s16x4 lo, hi; } s; piece f; } u;
        u.s.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>((t.c ^ (2 * d)) + (r * S + more) * 2));
        u.s.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>((t.c ^ (2 * d + 32)) + ((r + 8) * S + more) * 2));   // swz(r + 8) = swz(r) ^ 2
        return u.f;
    }
};

template <int DP> struct Op<bf16_elem, DP> {
    typedef bf16_elem T;
    static constexpr int BLOCKS = 2;          // blocks of 32 staged rows a wavefront takes at a time
    static constexpr int PITCH = DP > 64 ? 128 : 64;
    typedef Swizzled<PITCH, PITCH> Places;
    typedef typename Places::piece frag;
    typedef frag held;                        // the operand that stays in registers
    typedef typename Places::Tile Tile;
    __device__ static __forceinline__ acc16 mma(const frag &a, const held &b, acc16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    __device__ static __forceinline__ frag rows(const Tile &t, int r, int d) { return Places::rows(t, r, d); }
    __device__ static __forceinline__ frag cols(const Tile &t, int r, int d) { return Places::cols(t, r, d); }
    __device__ static __forceinline__ void put(T *tile, int r, int d, const Chunk<T> &c) { *reinterpret_cast<u16x8 *>(tile + Places::place(r, d >> 3)) = c.a; }
    __device__ static __forceinline__ held pack(const acc16 &v, int from)
    {
        held f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (__bf16)v[from + j];
        return f;
    }
    __device__ static __forceinline__ held of(const Chunk<T> &c) { return __builtin_bit_cast(held, c.a); }
};

// fp32: every operand as three bf16 terms, x = hi + mid + lo with the rest below 2^-27 of x, and of the nine products the six above
// 2^-26: six instructions of 32 cycles where the fp32 matrix cores take eight of 64 for the same 16 places, and the sums are fp32.  A
// tile is cut once, on its way to LDS, where the terms of a row lie one behind the other (cut by every wavefront that reads it, the
// vector units were the bound: 580 us instead of 475 us a forward pass of 4 x 2048 rows, 16 heads of 128).  An infinite element has no such terms:
// it counts as no number.
template <int DP> struct Op<float, DP> {
    typedef float T;
    static constexpr int BLOCKS = DP > 64 ? 1 : 2;
    static constexpr int P = DP > 64 ? 128 : 64, PITCH = 3 * P / 2;      // PITCH in floats
    typedef Swizzled<P, 3 * P> Places;
    typedef typename Places::piece term;
    struct held { term hi, mid, lo; };
    typedef held frag;
    typedef typename Places::Tile Tile;
    // FAR: elements that would round to an infinite hi (fp32's lowest and largest) leave the rest to mid and lo.  Of what lies in memory; forward
    // pass of 4 x 2048 rows, 16 heads of 64: 204 -> 209 us, of 128: 481 -> 500.
    template <bool FAR> __device__ static __forceinline__ held cut(float (&r)[8])
    {
        held t;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t.hi[j] = (__bf16)(FAR ? __builtin_amdgcn_fmed3f(r[j], -BF16_MAX, BF16_MAX) : r[j]);
            r[j] -= (float)t.hi[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) { t.mid[j] = (__bf16)r[j]; r[j] -= (float)t.mid[j]; }
#pragma unroll
        for (int j = 0; j < 8; ++j) t.lo[j] = (__bf16)r[j];
        return t;
    }
    __device__ static __forceinline__ acc16 mma(const frag &a, const held &b, acc16 c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.lo, b.hi, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.hi, b.lo, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.mid, b.mid, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.mid, b.hi, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.hi, b.mid, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.hi, b.hi, c, 0, 0, 0);
    }
    __device__ static __forceinline__ frag rows(const Tile &t, int r, int d)
    {
        return frag{Places::rows(t, r, d), Places::rows(t, r, d, P), Places::rows(t, r, d, 2 * P)};
    }
    __device__ static __forceinline__ frag cols(const Tile &t, int r, int d)
    {
        return frag{Places::cols(t, r, d), Places::cols(t, r, d, P), Places::cols(t, r, d, 2 * P)};
    }
    __device__ static __forceinline__ void put(T *tile, int r, int d, const Chunk<T> &c)
    {
        const held t = of(c);
        term *p = reinterpret_cast<term *>(reinterpret_cast<__bf16 *>(tile) + Places::place(r, d >> 3));
        p[0] = t.hi;
        p[P / 8] = t.mid;
        p[2 * P / 8] = t.lo;
    }
    __device__ static __forceinline__ held pack(const acc16 &v, int from)
    {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = v[from + j];
        return cut<false>(f);
    }
    __device__ static __forceinline__ held of(const Chunk<T> &c)
    {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = c.get(j);
        return cut<true>(f);
    }
};

__device__ __forceinline__ int acc_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// values of a lane and of the one 32 places away, joined
template <bool MAX> __device__ __forceinline__ float join_halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return join<MAX>(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// An array of rows x heads x dim.
struct AttArray {
    char *p;
    int64_t ld, hs;
};
struct AttArgs {
    AttArray Q, K, V, O, dO, dQ, dK, dV;
    float *lse;
    float *from;         // gradients: -lse / scale, then -D, heads x total each
    float *part;         // sums over a part of the heads that share keys: 2 x splits x total x kv_heads x dim (dK, then dV), or null
    const int *cu;
    int total, nseq, heads, group, dim, splits;
    float scale;
};

template <typename T> __device__ __forceinline__ T *att_at(const AttArray &a, int row, int head)
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

// Workgroups go round the eight XCDs one by one: so that the heads of an XCD share keys (and its L2 holds them), it takes
// neighbours.  8192 rows, 32 heads on 4: the keys and values of one head of 2 MB each in an L2 of 4 MB, not of four.
__device__ __forceinline__ int att_head(int block, int heads)
{
    const int b = block % heads;
    return heads % 8 ? b : b % 8 * (heads / 8) + b / 8;
}

struct AttTile {
    int start, len, index;          // first row and length of the sequence, which tile of it
};

// Tile `item` of all sequences' tiles of QT rows, those with the most tiles before them in their sequence first (their
// work is longest in a forward pass).  The workgroups beyond the last tile get false.  All lanes of a wavefront take part.
template <int QT> __device__ __forceinline__ bool find_tile(const AttArgs &a, int item, AttTile &t)
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
        // how many tiles have this index or a larger one
        auto from = [&](int index) {
            const int over = tiles - index;
            return __builtin_amdgcn_readlane(scan_lanes(over > 0 ? over : 0), 63);
        };
        if (from(0) <= item) return false;
        int lo = 0, hi = (a.total + QT - 1) / QT;
        while (hi - lo > 1) {                       // the largest index of which there are more than `item`
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
// BK rows of dim elements, padded with zeros to DP, from memory to LDS.  Rows at any place go through registers.  Whole
// 16-byte pieces (DIRECT: att_direct) are loaded to LDS without registers, which is what lets the backward kernels keep two
// wavefronts a SIMD, into one of two stages while the other is read; rows and columns beyond the ends come as zeros from
// the bounds of the descriptor.
template <typename T, int DP, int BK, bool DIRECT> struct AttStage;

template <typename T, int DP, int BK> struct AttStage<T, DP, BK, false> {
    static constexpr int ALL = BK * DP / 8, CH = (ALL + ATT_THREADS - 1) / ATT_THREADS;
    Chunk<T> c[CH];
    // rows row0 .. row0 + rows - 1 of one head
    __device__ __forceinline__ void load(const AttArray &a, int row0, int head, int rows, int dim)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = (int)threadIdx.x + ATT_THREADS * i, r = k / (DP / 8), d = k % (DP / 8) * 8;
            c[i].zero();
            if (r < rows && d < dim && (ALL % ATT_THREADS == 0 || k < ALL)) c[i].load(att_at<const T>(a, row0 + r, head) + d, dim - d);
        }
    }
    __device__ __forceinline__ void store(T *lds) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = (int)threadIdx.x + ATT_THREADS * i, r = k / (DP / 8), d = k % (DP / 8) * 8;
            if (ALL % ATT_THREADS == 0 || k < ALL) Op<T, DP>::put(lds, r, d, c[i]);
        }
    }
};

template <int DP, int BK> struct AttStage<bf16_elem, DP, BK, true> {
    typedef Op<bf16_elem, DP> M;
    static constexpr int CPR = M::PITCH / 8, NI = BK * CPR / ATT_THREADS;      // pieces of a row in LDS, load instructions of a wavefront
    static_assert(NI * ATT_THREADS == BK * CPR, "whole instructions");
    static constexpr int RPI = ATT_THREADS / CPR;                              // rows of an instruction of the workgroup: swz(r + RPI) = swz(r)
    static_assert(RPI % 16 == 0, "one place a lane");
    uint64_t base;
    int left, ld, dim;     // bytes from there to the end, of a row; columns
    // rows row0 + first .. row0 + rows - 1 of one head
    __device__ __forceinline__ void init(const AttArray &a, int row0, int head, int first, int rows, int dim_)
    {
        ld = (int)a.ld * 2;
        const uint64_t at = reinterpret_cast<uint64_t>(att_at<const bf16_elem>(a, row0 + first, head));
        base = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
        dim = dim_;
        left = __builtin_amdgcn_readfirstlane((rows - first - 1) * ld + dim * 2);
    }
    // the next BK rows to `stage`; the rows after them are next.  SPARE: a lane's place is made anew for every tile - kept, it is a
    // register that the gradients of K and V do not have.
    template <bool SPARE> __device__ __forceinline__ void issue(const bf16_elem *stage)
    {
        int t = (int)threadIdx.x;
        if constexpr (SPARE) asm("" : "+v"(t));
        const int r = t / CPR, c = (t % CPR) ^ M::Places::swz(r);
        const uint32_t at = c * 8 < dim ? (uint32_t)(r * ld + c * 16) : 0x80000000u;
        const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_place(stage) + (threadIdx.x & ~63u) * 16u);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            load_to_lds(buffer_rsrc(reinterpret_cast<const void *>(base), (uint32_t)max(left, 0)), lds + ATT_THREADS * 16u * i, at, 0);
            base += (uint32_t)(RPI * ld);
            left -= RPI * ld;
        }
    }
};

// 64 floats from p on, those from `count` on as zeros, to LDS at `to` (counted by wait_lds_loads).
__device__ __forceinline__ void load_floats_to_lds(const float *p, int count, const float *to)
{
    const i32x4 rsrc = buffer_rsrc(p, (uint32_t)max(count, 0) * 4u);
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_place(to));
    uint32_t t = threadIdx.x;
    asm("" : "+v"(t));
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :: "s"(lds), "v"((t & 63u) * 4u), "s"(rsrc) : "memory", "m0");
#pragma clang diagnostic pop
}

// Whether an array's rows can be loaded to LDS directly: whole aligned 16-byte pieces, offsets within 31 bits even of the
// tile beyond the last row.
inline bool att_direct(const AttArray &a, int dtype, int total, int dim)
{
    return dtype == ASTERIA_BF16 && dim % 8 == 0 && a.ld >= dim && a.ld % 8 == 0 && a.hs % 8 == 0 &&
           (reinterpret_cast<uintptr_t>(a.p) & 15) == 0 && ((int64_t)total + 1024) * a.ld < (1 << 30);
}

// The second operand of a product over dim: lane l holds row `row` of the array, elements 16 c + 8 h + j.
template <typename T, int DP>
__device__ __forceinline__ void load_frags(const AttArray &a, int row, int head, bool valid, int dim, typename Op<T, DP>::held (&f)[DP / 16])
{
    const int h = ((int)threadIdx.x >> 5) & 1;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        const int d = 16 * c + 8 * h;
        Chunk<T> k;
        k.zero();
        if (valid && d < dim) k.load(att_at<const T>(a, row, head) + d, dim - d);
        f[c] = Op<T, DP>::of(k);
    }
}

// The loads of f have arrived behind this: left to their first use, which lies in the loop over the tiles, the wait for them would
// hold up every step until the next tile's loads have arrived, too.
template <typename F> __device__ __forceinline__ void arrived(F &f)
{
    if constexpr (sizeof(F) == 16) {
        i32x4 v = __builtin_bit_cast(i32x4, f);
        asm volatile("" : "+v"(v));
        f = __builtin_bit_cast(F, v);
    } else {
        arrived(f.hi); arrived(f.mid); arrived(f.lo);
    }
}
template <typename F, int N> __device__ __forceinline__ void arrived(F (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) arrived(f[i]);
}

// Elements 32 t + 8 g + 4 h + 0 .. 3 of the row at p (of dim elements), times f.
__device__ __forceinline__ void store4(bf16_elem *p_, int n, const float (&v)[4])
{
    typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
    uint16_t *p = reinterpret_cast<uint16_t *>(p_);
    u16x4_any b;
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = f32_bf16(v[e]);
    if (n >= 4) *reinterpret_cast<u16x4_any *>(p) = b;
    else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (e < n) p[e] = b[e];
    }
}
__device__ __forceinline__ void store4(float *p, int n, const float (&v)[4])
{
    if (n >= 4) *reinterpret_cast<f32x4_any *>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
    else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (e < n) p[e] = v[e];
    }
}
template <typename TO, int DP>
__device__ __forceinline__ void store_row(TO *p, int dim, const acc16 (&o)[DP / 32], float f)
{
    const int h = ((int)threadIdx.x >> 5) & 1;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * t + 8 * g + 4 * h;
            const float v[4] = {o[t][4 * g] * f, o[t][4 * g + 1] * f, o[t][4 * g + 2] * f, o[t][4 * g + 3] * f};
            if (d < dim) store4(p + d, dim - d, v);
        }
}

// Adds the results of the NB wavefronts that hold the same 32 rows (wavefronts w, w + NA, ..) into the first one's, through
// NB / 2 x NA x DP x 32 floats of LDS in halves: 4 -> 2 -> 1.
template <int DP, int NA, int NB>
__device__ __forceinline__ void add_wavefronts(float *lds, acc16 (&o)[DP / 32])
{
    const int l = (int)threadIdx.x & 63, w = (int)threadIdx.x >> 6, wa = w % NA, wb = w / NA;
#pragma unroll
    for (int half = NB / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (wb >= half && wb < 2 * half) {
            f32x4 *q = reinterpret_cast<f32x4 *>(lds) + ((wb - half) * NA + wa) * DP * 8;
#pragma unroll
            for (int t = 0; t < DP / 32; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) q[(4 * t + g) * 64 + l] = f32x4{o[t][4 * g], o[t][4 * g + 1], o[t][4 * g + 2], o[t][4 * g + 3]};
        }
        __syncthreads();
        if (wb < half) {
            const f32x4 *q = reinterpret_cast<const f32x4 *>(lds) + (wb * NA + wa) * DP * 8;
#pragma unroll
            for (int t = 0; t < DP / 32; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 v = q[(4 * t + g) * 64 + l];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[t][4 * g + e] += v[e];
                }
        }
    }
}

// Most tiles of qt rows that sequences of `total` rows together can have (total / qt whole ones and one more each).
inline int64_t att_tiles(const AttArgs &a, int qt)
{
    if (!a.cu) return ((int64_t)a.total + qt - 1) / qt;
    return (int64_t)a.total / qt + (a.nseq < a.total ? a.nseq : a.total);
}
// A wavefront for every 32 rows, four of which share a tile of the rows they pass over - or where that gives less than one and a
// half workgroups a CU, four wavefronts (or two) for the same 32 rows, each with a quarter (half) of what is passed over.  Forward and backward, heads of
// 64: at 324 workgroups 103 us so, 107 us otherwise, at 444 160 and 150 us (bf16); 304 and 362, 570 and 524 us (fp32).
inline bool att_few(const AttArgs &a, int heads) { return att_tiles(a, 128) * heads < 384; }

// How many wavefronts the same rows take then.  Tiles of 32 rows for each of them lie in LDS: fp32 ones fill it with two (and a tile that
// one wavefront reads is cut for it alone: 3200 rows, 12 heads of 64, 397 + 128 us with four, 236 + 69 us with two).
template <typename T> constexpr int att_shared = sizeof(T) == 4 ? 2 : 4;
// The last 16 columns of fp32 heads of 65 to 80, which are padding only, are left out of the products over dim (a head of 80: 3 %).
template <typename T, int DP> __device__ __forceinline__ bool att_empty(int d, int dim) { return sizeof(T) == 4 && DP == 96 && d == 5 && dim <= 80; }

// LDS to ask for, in kernels of which PER_CU workgroups fit a CU.  Workgroups that would all run at once are given so much that fewer
// share a CU: the longest then do not share one while others stand idle.  fp32 with two a CU, below 544: one (heads of 64, forward: 390 workgroups
// 225 -> 218 us, 520 484 -> 476; at 756 200 -> 238).  bf16 with three a CU, below 768: two (backward, heads of 64: 740 workgroups 142 -> 133 us;
// at 888 159 -> 160).
template <typename T, int NB, int PER_CU> constexpr size_t att_lds(size_t need, int64_t blocks)
{
    const size_t more = sizeof(T) == 4 ? 84 * 1024 : 56 * 1024;
    return NB == 1 && (sizeof(T) == 4 || PER_CU == 3) && blocks < (sizeof(T) == 4 ? 544 : 768) && need < more ? more : need;
}

// Kernels for dims padded to 64, 96 or 128.
template <typename F> asteria_status att_for_type(int dtype, int dim, bool direct, F f)
{
    auto width = [&](auto t, auto direct_) {
        if (dim <= 64) return f(t, std::integral_constant<int, 64>(), direct_);
        if (dim <= 96) return f(t, std::integral_constant<int, 96>(), direct_);
        return f(t, std::integral_constant<int, 128>(), direct_);
    };
    if (dtype != ASTERIA_BF16) return width(float(), std::false_type());
    return direct ? width(bf16_elem(), std::true_type()) : width(bf16_elem(), std::false_type());
}

asteria_status attention_dq(const AttArgs &a, int dtype, hipStream_t stream);
asteria_status attention_dkv(const AttArgs &a, int dtype, hipStream_t stream);
int attention_splits(const AttArgs &a);       // of the heads that share keys, in attention_dkv

}  // namespace asteria
