// asteria_attention and asteria_attention_backward (attention.h): the forward kernel and the entry points.
#include "attention.h"
#include "gemm.h"

using namespace asteria;

namespace {

template <typename T, int DP, int NA, int NB, bool DIRECT> struct FwdShape {
    static constexpr int BK = 32 * (NB > 1 ? NB : Op<T, DP>::BLOCKS);
    static constexpr int TILE = BK * Op<T, DP>::PITCH;
    static constexpr size_t LDS = (DIRECT ? 4 : 2) * (size_t)TILE * sizeof(T);
    static constexpr int PER_CU = sizeof(T) == 2 || DP == 64 ? 2 : 1;       // workgroups a CU, or more
    static_assert(LDS >= (NB / 2) * NA * DP * 32 * sizeof(float) && LDS >= NB * NA * 64 * sizeof(float), "room for the sums");
};

// A workgroup takes 128 rows of a head (NA = 4 wavefronts of 32), or fewer rows with NB wavefronts each, and passes over their keys and values, tile
// by tile through two stages of LDS: the next tile is on its way while this one is multiplied, with one barrier a tile.
// Bound by the vector units more than by the matrix cores: 32 x 32 scores and their products with a head of 64 are 256 cycles of the
// latter, their exponentials, sums and roundings 1.5 times as many of the former, and up to four wavefronts a SIMD overlap them.
// Measured, calls back to back: 8192 rows, 32 heads of 64 on 4 (275 GFLOP of causal products): 287 - 292 us, 940 - 960 TFLOP/s, matrix cores
// busy 49 % and vector units 70 % of the time at 1.8 - 1.95 GHz (the power limit), no LDS conflicts; 4 x 2048 rows 85 - 91 us, 8123 packed
// rows, 16 heads of 128: 81 us.  fp32: 4 x 2048 rows, 16 heads of 64: 209 - 215 us.
template <typename T, int DP, int NA, int NB, bool DIRECT>
__global__ __launch_bounds__(ATT_THREADS, (FwdShape<T, DP, NA, NB, DIRECT>::PER_CU)) void attention_kernel(AttArgs a)
{
    typedef Op<T, DP> M;
    constexpr int BK = FwdShape<T, DP, NA, NB, DIRECT>::BK, NBLK = BK / 32 / NB;
    extern __shared__ __attribute__((aligned(256))) char lds[];
    constexpr int TILE = FwdShape<T, DP, NA, NB, DIRECT>::TILE;
    T *lk = reinterpret_cast<T *>(lds), *lv = lk + TILE;
    AttTile tile;
    const int head = att_head((int)blockIdx.x, a.heads), kvh = head / a.group;
    if (!find_tile<32 * NA>(a, (int)blockIdx.x / a.heads, tile)) return;
    const int l = (int)threadIdx.x & 63, h = l >> 5, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wa = NB == 1 ? w : w % NA, wb = NB == 1 ? 0 : w / NA;
    const int q0 = tile.index * 32 * NA, qw = q0 + wa * 32, qi = qw + (l & 31);
    const bool valid = qi < tile.len;
    typename M::held q[DP / 16];
    load_frags<T, DP>(a.Q, tile.start + qi, head, valid, a.dim, q);
    acc16 o[DP / 32];
    // Exponents count from m.  bf16: m is the maximum of the first tile's scores and rises only where the sum has passed 2^20, by that
    // sum's logarithm; no maximum is taken of the other tiles.  Should the scores of one tile lift the sum beyond 2^40, the
    // workgroup begins again, in a pass (SAFE) that takes every tile's maximum before its exponentials and follows it by steps of 2^8
    // or more, and costs the time of both: 303 us for 8192 rows where the first kind takes 289.  fp32, whose six products a tile leave the vector units time, has
    // only the second kind (2013 rows, 8 heads of 80: 67 us, 69 with the first).
    const float c = a.scale * LOG2E;
    float m, sum;
    const int last = min(tile.len, q0 + 32 * NA), nk = (last + BK - 1) / BK;
    AttStage<T, DP, BK, DIRECT> sk, sv;
    auto pass = [&](auto safe_) -> bool {
        constexpr bool SAFE = decltype(safe_)::value;
        bool fails = false;
        m = -INFINITY;
        sum = 0.0f;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) o[t] = 0.0f;
        lk = reinterpret_cast<T *>(lds);
        lv = lk + TILE;
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
        for (int kt = 0; kt < nk; ++kt) {
            const int k0 = kt * BK + wb * 32 * NBLK, next = (kt + 1) * BK;   // k0: of this wavefront's keys
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
            const typename M::Tile tk(lk + 32 * wb * NBLK * M::PITCH), tv(lv + 32 * wb * NBLK * M::PITCH);
            if (k0 > qw + 31) continue;                              // behind its rows
            acc16 s[NBLK];
#pragma unroll
            for (int b = 0; b < NBLK; ++b) s[b] = 0.0f;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                if (att_empty<T, DP>(d, a.dim)) break;
#pragma unroll
                for (int b = 0; b < NBLK; ++b) s[b] = M::mma(M::rows(tk, 32 * b, 16 * d), q[d], s[b]);
            }
            if (k0 + 32 * NBLK - 1 > qw) {
#pragma unroll
                for (int b = 0; b < NBLK; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) if (k0 + 32 * b + acc_row(i, h) > qi) s[b][i] = -INFINITY;
            }
            if (SAFE || kt == 0) {
                float top = s[0][0];
#pragma unroll
                for (int b = 0; b < NBLK; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
                top = join_halves<true>(top) * c;
                if (!SAFE) {
                    m = top;
                    fails = top == -INFINITY && k0 <= qi;            // no score to count from
                } else if (__any(top > m + 8.0f)) {
                    const float to = fmaxf(m, top), f = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);
                    m = to;
                    sum *= f;
#pragma unroll
                    for (int t = 0; t < DP / 32; ++t) o[t] *= f;
                }
            }
            const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int b = 0; b < NBLK; ++b) {
                if (b && k0 + 32 * b > qw + 31) continue;    // behind its rows: P is 0, but 0 V is no number where V is infinite
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, -from));
                    sum += s[b][i];                                  // before the rounding to an operand: lse is fp32
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const typename M::held p = M::pack(s[b], 8 * k);
#pragma unroll
                    for (int t = 0; t < DP / 32; ++t) o[t] = M::mma(M::cols(tv, 32 * b + 16 * k, 32 * t), p, o[t]);
                }
            }
            if (!SAFE && __any(sum > 0x1p20f)) {
                const float all = join_halves<true>(sum), to = all > 0x1p20f ? m + __builtin_amdgcn_logf(all) : m;
                fails |= !(all <= 0x1p40f);
                const float f = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);
                m = to;
                sum *= f;
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) o[t] *= f;
            }
        }
        return fails || !(sum <= 0x1p40f);
    };
    if constexpr (sizeof(T) == 4) {
        pass(std::true_type());
    } else {
        __shared__ int failed;
        if (threadIdx.x == 0) failed = 0;            // the pass has barriers before its end
        if (pass(std::false_type())) failed = 1;
        __syncthreads();
        if (__builtin_amdgcn_readfirstlane(failed)) pass(std::true_type());
    }
    sum = join_halves<false>(sum);
    if constexpr (NB > 1) {
        // to the largest maximum of the wavefronts that passed over the same rows' keys
        float *ms = reinterpret_cast<float *>(lds);
        __syncthreads();
        if (h == 0) { ms[w * 32 + l] = m; ms[(NA * NB + w) * 32 + l] = sum; }
        __syncthreads();
        float top = m, all = 0.0f;
#pragma unroll
        for (int k = 0; k < NB; ++k) top = fmaxf(top, ms[(k * NA + wa) * 32 + (l & 31)]);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            const float mk = ms[(k * NA + wa) * 32 + (l & 31)];
            all += ms[(NA * NB + k * NA + wa) * 32 + (l & 31)] * (mk == top ? 1.0f : __builtin_amdgcn_exp2f(mk - top));
        }
        const float f = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) o[t] *= f;
        m = top;
        sum = all;
        add_wavefronts<DP, NA, NB>(reinterpret_cast<float *>(lds), o);
        if (wb) return;
    }
    if (!valid) return;
    store_row<T, DP>(att_at<T>(a.O, tile.start + qi, head), a.dim, o, 1.0f / sum);
    if (a.lse && h == 0) a.lse[(size_t)head * a.total + tile.start + qi] = (m + __builtin_amdgcn_logf(sum)) * LN2;
}

template <typename T, int DP, int NA, int NB, bool DIRECT> hipError_t launch(const AttArgs &a, hipStream_t stream)
{
    static bool configured[MAX_DEVICES] = {};
    const int64_t blocks = att_tiles(a, 32 * NA) * a.heads;
    typedef FwdShape<T, DP, NA, NB, DIRECT> Shape;
    constexpr size_t MOST = att_lds<T, NB, Shape::PER_CU>(Shape::LDS, 0);
    const size_t bytes = att_lds<T, NB, Shape::PER_CU>(Shape::LDS, blocks);
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(attention_kernel<T, DP, NA, NB, DIRECT>), MOST, configured); e != hipSuccess) return e;
    hipLaunchKernelGGL((attention_kernel<T, DP, NA, NB, DIRECT>), dim3((unsigned)blocks), dim3(ATT_THREADS), bytes, stream, a);
    return hipGetLastError();
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
    if (!(a->scale >= 0x1p-100f && a->scale <= 0x1p100f)) return ASTERIA_INVALID_ARG;      // lse / scale and 8 / scale are numbers
    if (a->ldq < 0 || a->ldk < 0 || a->ldv < 0 || a->ldo < 0 || a->hq < 0 || a->hk < 0 || a->hv < 0 || a->ho < 0) return ASTERIA_INVALID_ARG;
    if (writes_o && (!apart(a->ldo, a->ho, a->total, a->heads, a->dim) || a->O == a->Q || a->O == a->K || a->O == a->V)) return ASTERIA_INVALID_ARG;
    if (a->dim > 128) return ASTERIA_UNSUPPORTED;
    if (((int64_t)a->total / 128 + 1 + a->nseq) * a->heads > MOST_BLOCKS) return ASTERIA_UNSUPPORTED;
    return ASTERIA_OK;
}

AttArgs args_of(const asteria_attn *a)
{
    AttArgs k = {};
    auto array = [](const void *p, int64_t ld, int64_t hs) { return AttArray{reinterpret_cast<char *>(const_cast<void *>(p)), ld, hs}; };
    k.Q = array(a->Q, a->ldq, a->hq);
    k.K = array(a->K, a->ldk, a->hk);
    k.V = array(a->V, a->ldv, a->hv);
    k.O = array(a->O, a->ldo, a->ho);
    k.lse = a->lse; k.cu = a->cu;
    k.total = a->total; k.nseq = a->nseq; k.heads = a->heads; k.group = a->heads / a->kv_heads; k.dim = a->dim;
    k.scale = a->scale;
    return k;
}

size_t part_elems(const AttArgs &a, int splits)
{
    return splits > 1 ? 2 * (size_t)splits * a.total * (a.heads / a.group) * a.dim : 0;
}

}  // namespace

extern "C" asteria_status asteria_attention(const asteria_attn *a, void *stream_)
{
    ASTERIA_TRY(validate(a, true));
    const AttArgs k = args_of(a);
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    const bool direct = att_direct(k.K, a->dtype, k.total, k.dim) && att_direct(k.V, a->dtype, k.total, k.dim);
    return att_for_type(a->dtype, a->dim, direct, [&](auto t, auto dp, auto direct_) {
        typedef decltype(t) T;
        constexpr int DP = dp();
        constexpr bool DIRECT = decltype(direct_)::value;
        ASTERIA_HIP_TRY((att_few(k, k.heads) ? launch<T, DP, 4 / att_shared<T>, att_shared<T>, DIRECT>(k, stream) : launch<T, DP, 4, 1, DIRECT>(k, stream)));
        return ASTERIA_OK;
    });
}

extern "C" size_t asteria_attention_backward_workspace_bytes(const asteria_attn *a)
{
    if (validate(a, false) != ASTERIA_OK) return 0;
    const AttArgs k = args_of(a);
    return Carver::need(2 * (size_t)a->total * a->heads, sizeof(float)) + Carver::need(part_elems(k, attention_splits(k)), sizeof(float));
}

extern "C" asteria_status asteria_attention_backward(const asteria_attn *a, const asteria_attn_grad *g,
                                                     void *ws, size_t ws_bytes, void *stream_)
{
    ASTERIA_TRY(validate(a, false));
    if (!a->lse || !g || !g->dO || !g->dQ || !g->dK || !g->dV || g->lddo < 0 || g->hdo < 0) return ASTERIA_INVALID_ARG;
    if (!apart(g->lddq, g->hdq, a->total, a->heads, a->dim) || !apart(g->lddk, g->hdk, a->total, a->kv_heads, a->dim) ||
        !apart(g->lddv, g->hdv, a->total, a->kv_heads, a->dim)) return ASTERIA_INVALID_ARG;
    for (const void *out : {g->dQ, g->dK, g->dV})
        if (out == a->Q || out == a->K || out == a->V || out == a->O || out == g->dO) return ASTERIA_INVALID_ARG;
    if (g->dQ == g->dK || g->dQ == g->dV || g->dK == g->dV) return ASTERIA_INVALID_ARG;
    if (!ws || ws_bytes < asteria_attention_backward_workspace_bytes(a)) return ASTERIA_WORKSPACE_TOO_SMALL;
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return ASTERIA_INVALID_ARG;   // workspace must be 256-byte aligned
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    AttArgs k = args_of(a);
    auto array = [](const void *p, int64_t ld, int64_t hs) { return AttArray{reinterpret_cast<char *>(const_cast<void *>(p)), ld, hs}; };
    k.dO = array(g->dO, g->lddo, g->hdo);
    k.dQ = array(g->dQ, g->lddq, g->hdq);
    k.dK = array(g->dK, g->lddk, g->hdk);
    k.dV = array(g->dV, g->lddv, g->hdv);
    Carver cv(ws);
    k.from = cv.take<float>(2 * (size_t)a->total * a->heads);
    k.splits = attention_splits(k);
    k.part = k.splits > 1 ? cv.take<float>(part_elems(k, k.splits)) : nullptr;
    ASTERIA_TRY(attention_dq(k, a->dtype, stream));
    return attention_dkv(k, a->dtype, stream);
}
