// Gradient of Q (attention.h); and for the gradients of K and V, at which their sums begin: -lse / scale and -D, D = rowsum(dO o O).
//
// The tiles and stages of the forward pass, with three products a tile instead of two (four in bf16).  A kernel of its own, beside that
// of K and V, which computes scores and dP once more: one kernel for all would add dQ up over workgroups, by atomics whose order
// changes the result or through partial sums in memory (570 MB for 4 x 2048 rows, 32 heads of 64).  Measured: those rows 147 us, 940
// TFLOP/s of causal products, matrix cores busy 41 % and vector units 47 %, 2.2 wavefronts a SIMD; 8123 packed rows, 16 heads of 128: 146 us.
#include "attention.h"
#include "gemm.h"

using namespace asteria;

namespace {

template <typename T, int DP, int NA, int NB, bool DIRECT> struct DqShape {
    static constexpr bool B16 = sizeof(T) == 2, LONE = B16 && NB > 1 && !DIRECT && DP > 64;
    // 32 keys a stage where registers are short: two blocks side by side take 16 more of them.  8123 packed rows, 16 heads of 128, backward:
    // 316 us so, 399 with 64 keys; 4 x 2048 rows, 16 heads of 65 in rows of no whole pieces: 497 and 528 us.
    static constexpr int BK = 32 * (NB > 1 ? NB : B16 && (DP == 128 || (DP == 96 && !DIRECT)) ? 1 : Op<T, DP>::BLOCKS);
    static constexpr int TILE = BK * Op<T, DP>::PITCH;
    // Pieces of dO that stay in LDS, so that two accumulators of dim x 32 fit the registers of PER_CU workgroups.
    static constexpr int HELD = !B16 || LONE ? 0 : DP == 64 ? (DIRECT && NB == 1 ? 2 : 0) : DP == 96 ? 3 : DIRECT ? 5 : 7;
    static constexpr size_t STAGED = (DIRECT ? 4 : 2) * (size_t)TILE * sizeof(T), LDS = STAGED + HELD * NA * NB * 64 * 16;
    // Workgroups a CU: three with heads of up to 64 in bf16 (backward pass of 4 x 2048 rows, 32 heads: 306 us so, 319 with two), one where
    // the rows that four wavefronts share come through registers (2000 rows, 8 heads of 127, backward: 166 us so, 225 with two, which spill).
    static constexpr int PER_CU = !B16 ? (DP == 64 ? 2 : 1) : LONE ? 1 : DP == 64 && DIRECT && NB == 1 ? 3 : 2;
    static_assert(LDS >= (NB / 2) * NA * DP * 32 * sizeof(float), "room for the sums");
};

template <typename T, int DP, int NA, int NB, bool DIRECT>
__global__ __launch_bounds__(ATT_THREADS, (DqShape<T, DP, NA, NB, DIRECT>::PER_CU)) void attention_dq_kernel(AttArgs a)
{
    typedef Op<T, DP> M;
    typedef DqShape<T, DP, NA, NB, DIRECT> Shape;
    constexpr int BK = Shape::BK;
    extern __shared__ __attribute__((aligned(256))) char lds[];
    constexpr int TILE = Shape::TILE;
    T *lk = reinterpret_cast<T *>(lds), *lv = lk + TILE;
    AttTile tile;
    const int head = att_head((int)blockIdx.x, a.heads), kvh = head / a.group;
    if (!find_tile<32 * NA>(a, (int)blockIdx.x / a.heads, tile)) return;
    const int l = (int)threadIdx.x & 63, h = l >> 5, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wa = NB == 1 ? w : w % NA, wb = NB == 1 ? 0 : w / NA;
    const int q0 = tile.index * 32 * NA, qw = q0 + wa * 32, qi = qw + (l & 31);
    const bool valid = qi < tile.len;
    typename M::held q[DP / 16], g[DP / 16 - Shape::HELD];
    constexpr int HELD = Shape::HELD, REGS = DP / 16 - HELD;
    typename M::held *held = reinterpret_cast<typename M::held *>(lds + Shape::STAGED) + w * HELD * 64 + l;
    float delta = 0.0f;
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
        const int at = 16 * d + 8 * h;
        Chunk<T> o, go;
        o.zero();
        go.zero();
        if (valid && at < a.dim) {
            o.load(att_at<T>(a.O, tile.start + qi, head) + at, a.dim - at);
            go.load(att_at<T>(a.dO, tile.start + qi, head) + at, a.dim - at);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) delta += o.get(j) * go.get(j);
        if (d < REGS) g[d] = M::of(go);
        else held[64 * (d - REGS)] = M::of(go);
    }
    delta = join_halves<false>(delta);
    const size_t at_row = (size_t)head * a.total + tile.start + qi;
    const float lse_ = valid ? a.lse[at_row] : 0.0f, lse = lse_ * LOG2E;
    load_frags<T, DP>(a.Q, tile.start + qi, head, valid, a.dim, q);
    // D of the stored O carries O's rounding, which in bf16 is large beside dP - D where the values have a mean (of 64: dQ off by 14 %).
    // The sum of a row of dS says by how much: P sums to one, so that D + sum(dS) is D without it, at which the gradients of K and V
    // begin.  Here it is known behind the last key, and dQ = scale (dS K - sum(dS) P K): P K is one product more, with K^T as it is
    // read for dS K (4 x 2048 rows, 32 heads of 64: 129 -> 147 us).
    constexpr bool CORRECT = sizeof(T) == 2;
    float more = 0.0f;
    const acc16 from = -delta;                // dP - D: its sums begin at -D
    acc16 o[DP / 32], pk[CORRECT ? DP / 32 : 1];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) {
        o[t] = 0.0f;
        if constexpr (CORRECT) pk[t] = 0.0f;
    }
    const float c = a.scale * LOG2E;
    const int last = min(tile.len, q0 + 32 * NA), nk = (last + BK - 1) / BK;
    AttStage<T, DP, BK, DIRECT> sk, sv;
    if constexpr (DIRECT) {
        sk.init(a.K, tile.start, kvh, 0, last, a.dim);
        sv.init(a.V, tile.start, kvh, 0, last, a.dim);
        sk.template issue<false>(lk);
        sv.template issue<false>(lv);
    } else {
        sk.load(a.K, tile.start, kvh, last, a.dim);
        sv.load(a.V, tile.start, kvh, last, a.dim);
    }
    arrived(q);
    // over the lanes and wavefronts that hold parts of the same row
    __shared__ float parts[4][32];
    auto sum_of_row = [&](float v) {
        v = join_halves<false>(v);
        if constexpr (NB > 1) {
            __syncthreads();
            if (h == 0) parts[w][l] = v;
            __syncthreads();
            v = 0.0f;
#pragma unroll
            for (int k = 0; k < NB; ++k) v += parts[k * NA + wa][l & 31];
        }
        return v;
    };
    for (int kt = 0; kt < nk; ++kt) {
        const int k0 = kt * BK, next = k0 + BK;
        if constexpr (DIRECT) {
            lk = reinterpret_cast<T *>(lds) + (kt & 1) * 2 * TILE;
            lv = lk + TILE;
            wait_lds_loads<0>();
            __syncthreads();
            if (kt + 1 < nk) {
                T *to = reinterpret_cast<T *>(lds) + (~kt & 1) * 2 * TILE;
                sk.template issue<false>(to);
                sv.template issue<false>(to + TILE);
            }
        } else {
            __syncthreads();
            sk.store(lk);
            sv.store(lv);
            __syncthreads();
            if (kt + 1 < nk) {
                sk.load(a.K, tile.start + next, kvh, last - next, a.dim);
                sv.load(a.V, tile.start + next, kvh, last - next, a.dim);
            }
        }
        const typename M::Tile tk(lk + 32 * wb * M::PITCH), tv(lv + 32 * wb * M::PITCH);
#pragma unroll
        for (int b = 0; b < BK / 32; b += NB) {
            const int kb = k0 + 32 * (b + wb);
            if (kb > qw + 31) continue;
            acc16 s = 0.0f, dp = from;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                if (att_empty<T, DP>(d, a.dim)) break;
                s = M::mma(M::rows(tk, 32 * b, 16 * d), q[d], s);
                dp = M::mma(M::rows(tv, 32 * b, 16 * d), d < REGS ? g[d] : held[64 * (d - REGS)], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -lse));
                dp[i] *= s[i];
            }
            if (kb + 31 > qw) {
                // a row that sees one key has no gradient through the softmax: zero, not the round-off of dP - D
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (kb + acc_row(i, h) > qi) s[i] = 0.0f;
                    if (kb + acc_row(i, h) > qi || qi == 0) dp[i] = 0.0f;
                }
            }
            if constexpr (CORRECT) {
#pragma unroll
                for (int i = 0; i < 16; ++i) more += dp[i];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const typename M::held ds = M::pack(dp, 8 * k);
                typename M::held p;
                if constexpr (CORRECT) p = M::pack(s, 8 * k);
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) {
                    const typename M::frag kc = M::cols(tk, 32 * b + 16 * k, 32 * t);
                    o[t] = M::mma(kc, ds, o[t]);
                    if constexpr (CORRECT) pk[t] = M::mma(kc, p, pk[t]);
                }
            }
        }
    }
    if constexpr (CORRECT) {
        const float sum = sum_of_row(more);
        delta += sum;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) o[t] -= pk[t] * sum;
    }
    if (valid && h == 0 && wb == 0) {
        a.from[at_row] = -lse_ / a.scale;
        a.from[(size_t)a.heads * a.total + at_row] = -delta;
    }
    if constexpr (NB > 1) add_wavefronts<DP, NA, NB>(reinterpret_cast<float *>(lds), o);
    if (valid && wb == 0) store_row<T, DP>(att_at<T>(a.dQ, tile.start + qi, head), a.dim, o, a.scale);
}

template <typename T, int DP, int NA, int NB, bool DIRECT> hipError_t launch(const AttArgs &a, hipStream_t stream)
{
    static bool configured[MAX_DEVICES] = {};
    const int64_t blocks = att_tiles(a, 32 * NA) * a.heads;
    typedef DqShape<T, DP, NA, NB, DIRECT> Shape;
    constexpr size_t MOST = att_lds<T, NB, Shape::PER_CU>(Shape::LDS, 0);
    const size_t bytes = att_lds<T, NB, Shape::PER_CU>(Shape::LDS, blocks);
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(attention_dq_kernel<T, DP, NA, NB, DIRECT>), MOST, configured); e != hipSuccess) return e;
    hipLaunchKernelGGL((attention_dq_kernel<T, DP, NA, NB, DIRECT>), dim3((unsigned)blocks), dim3(ATT_THREADS), bytes, stream, a);
    return hipGetLastError();
}

}  // namespace

asteria_status asteria::attention_dq(const AttArgs &a, int dtype, hipStream_t stream)
{
    const bool direct = att_direct(a.K, dtype, a.total, a.dim) && att_direct(a.V, dtype, a.total, a.dim);
    return att_for_type(dtype, a.dim, direct, [&](auto t, auto dp, auto direct_) {
        typedef decltype(t) T;
        constexpr int DP = dp();
        constexpr bool DIRECT = decltype(direct_)::value;
        ASTERIA_HIP_TRY((att_few(a, a.heads) ? launch<T, DP, 4 / att_shared<T>, att_shared<T>, DIRECT>(a, stream) : launch<T, DP, 4, 1, DIRECT>(a, stream)));
        return ASTERIA_OK;
    });
}
