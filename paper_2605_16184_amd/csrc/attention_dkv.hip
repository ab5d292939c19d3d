// Gradients of K and V (attention.h): a wavefront holds the keys and values of 32 rows in registers and passes over the
// rows that see them, in all the heads that share them.
//
// Four products a tile; accumulators and the held keys and values leave room for three wavefronts a SIMD (heads of up to 64; two
// with longer ones), of which 2.3 (1.6) are resident on average, and that bounds it: matrix cores are busy 43 % (37 %) and vector units 43 % (28 %)
// of the time.  Three registers of a lane (one) lie in scratch memory over the loop.
// Measured: 4 x 2048 rows, 32 heads of 64 on 4: 149 us, 920 TFLOP/s of causal products; 8123 packed rows, 16 heads of 128 on 4: 158 us.
// With 64 keys a wavefront the backward pass of the former took 12 % more.
//
// Where the heads that share keys are many and the tiles are few, several workgroups take a part of these heads each, leave
// their sums in fp32 in the workspace, and a second kernel adds them up: without atomics, in one order.
#include "attention.h"
#include "gemm.h"

using namespace asteria;

namespace {

template <typename T, int DP, int NA, int NB, bool DIRECT> struct DkvShape {
    static constexpr bool WIDE = sizeof(T) == 2 && DP == 128 && DIRECT && NB == 1;
    static constexpr int BQ = 32 * (NB > 1 ? NB : WIDE ? 1 : Op<T, DP>::BLOCKS), ROWS = BQ < 64 ? 64 : BQ;
    static constexpr size_t TILE = (size_t)BQ * Op<T, DP>::PITCH;
    // Pieces of V that stay in LDS: with heads of 128 a wavefront's registers do not hold all, and what the compiler spilled
    // would wait behind the loads of the next tile.
    static constexpr int HELD = WIDE ? 3 : 0;
    static constexpr size_t SUMS = (NB / 2) * NA * DP * 32 * sizeof(float), STAGED = (DIRECT ? 2 : 1) * (2 * TILE * sizeof(T) + 2 * ROWS * sizeof(float)) + HELD * NA * 64 * 16;
    static constexpr size_t LDS = STAGED > SUMS ? STAGED : SUMS;
    // Workgroups a CU.  Three with heads of up to 64 in bf16: the backward pass of 4 x 2048 rows, 32 heads, 326 us with two, 306 us so.
    static constexpr int PER_CU = sizeof(T) == 4 ? 1 : DP == 64 && DIRECT ? 3 : DP == 64 || DIRECT ? 2 : 1;
};

template <typename T, int DP, int NA, int NB, bool DIRECT>
__global__ __launch_bounds__(ATT_THREADS, (DkvShape<T, DP, NA, NB, DIRECT>::PER_CU)) void attention_dkv_kernel(AttArgs a)
{
    typedef Op<T, DP> M;
    typedef DkvShape<T, DP, NA, NB, DIRECT> Shape;
    constexpr int BQ = Shape::BQ, KT = 32 * NA;
    extern __shared__ __attribute__((aligned(256))) char lds[];
    constexpr int STAGES = DIRECT ? 2 : 1;
    constexpr bool FROM = sizeof(T) == 2;
    T *lq = reinterpret_cast<T *>(lds), *lg = lq + Shape::TILE;
    auto rows_of = [&](int stage) { return reinterpret_cast<float *>(reinterpret_cast<T *>(lds) + STAGES * 2 * Shape::TILE) + stage * 2 * Shape::ROWS; };
    AttTile tile;
    const int kv_heads = a.heads / a.group, units = kv_heads * a.splits;
    const int unit = (int)blockIdx.x % units, kvh = unit / a.splits, split = unit % a.splits;
    if (!find_tile<KT>(a, (int)blockIdx.x / units, tile)) return;
    const int per = a.group / a.splits, head0 = kvh * a.group + split * per;
    tile.index = (tile.len + KT - 1) / KT - 1 - tile.index;      // the first keys are seen by the most rows
    const int l = (int)threadIdx.x & 63, h = l >> 5, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wa = NB == 1 ? w : w % NA, wb = NB == 1 ? 0 : w / NA;
    const int kw = tile.index * KT + wa * 32, ki = kw + (l & 31);
    typename M::held kf[DP / 16], vf[DP / 16];
    acc16 dk[DP / 32], dv[DP / 32];
    load_frags<T, DP>(a.K, tile.start + ki, kvh, ki < tile.len, a.dim, kf);
    load_frags<T, DP>(a.V, tile.start + ki, kvh, ki < tile.len, a.dim, vf);
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) { dk[t] = 0.0f; dv[t] = 0.0f; }
    typedef typename M::held piece;
    constexpr int HELD = Shape::HELD, REGS = DP / 16 - HELD;
    piece *held = reinterpret_cast<piece *>(rows_of(STAGES)) + w * HELD * 64 + l;
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[64 * i] = vf[REGS + i];
    const float c = a.scale * LOG2E;
    const int first = tile.index * KT / BQ, nq = (tile.len + BQ - 1) / BQ;
    AttStage<T, DP, BQ, DIRECT> sq, sg;
    float lse = 0.0f, delta = 0.0f;
    auto load = [&](int head, int q0, int stage) {
        if constexpr (DIRECT) {
            if (q0 == first * BQ) {
                sq.init(a.Q, tile.start, head, q0, tile.len, a.dim);
                sg.init(a.dO, tile.start, head, q0, tile.len, a.dim);
            }
            T *to = reinterpret_cast<T *>(lds) + stage * 2 * Shape::TILE;
            sq.template issue<true>(to);
            sg.template issue<true>(to + Shape::TILE);
            // wavefronts 0 and 2 the rows' -lse / scale, 1 and 3 their -D
            const int r = (w >> 1) * 64;
            if (r < BQ) load_floats_to_lds(a.from + ((size_t)(w & 1) * a.heads + head) * a.total + tile.start + q0 + r, tile.len - q0 - r,
                                           rows_of(stage) + (w & 1) * Shape::ROWS + r);
        } else {
            sq.load(a.Q, tile.start + q0, head, tile.len - q0, a.dim);
            sg.load(a.dO, tile.start + q0, head, tile.len - q0, a.dim);
            if (threadIdx.x < BQ) {
                const bool in = q0 + (int)threadIdx.x < tile.len;
                const float *p = a.from + (size_t)head * a.total + tile.start + q0 + threadIdx.x;
                lse = in ? p[0] : 0.0f;
                delta = in ? p[(size_t)a.heads * a.total] : 0.0f;
            }
        }
    };
    const int steps = (nq - first) * per;
    int qt = first, head = head0;
    load(head, qt * BQ, 0);
    arrived(kf);
    arrived(vf);
    for (int step = 0; step < steps; ++step) {
        const int q0 = qt * BQ, stage = DIRECT ? step & 1 : 0;
        lq = reinterpret_cast<T *>(lds) + stage * 2 * Shape::TILE;
        lg = lq + Shape::TILE;
        const float *row_lse = rows_of(stage), *row_delta = row_lse + Shape::ROWS;
        if constexpr (!DIRECT) {
            __syncthreads();
            sq.store(lq);
            sg.store(lg);
            if (threadIdx.x < BQ) { rows_of(0)[threadIdx.x] = lse; rows_of(0)[Shape::ROWS + threadIdx.x] = delta; }
        } else {
            wait_lds_loads<0>();
        }
        __syncthreads();
        if (++qt == nq) { qt = first; ++head; }
        if (step + 1 < steps) load(head, qt * BQ, ~step & 1);
        const typename M::Tile tq(lq + 32 * wb * M::PITCH), tg(lg + 32 * wb * M::PITCH);
        row_lse += 32 * wb;
        row_delta += 32 * wb;
#pragma unroll
        for (int b_ = 0; b_ < BQ / 32 / NB; ++b_) {
            const int b = b_ * NB, qb = q0 + 32 * (b + wb);
            if (qb + 31 < kw) continue;                 // rows before this wavefront's keys
            // the sums begin at -lse / scale and at -D of their rows: one instruction an element less each.  In bf16, where P is rounded to
            // 2^-8 anyway: dim additions on top of a large lse cost fp32 results up to three bits (measured at scores around 100)
            acc16 s, dp;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 rl = *reinterpret_cast<const f32x4 *>(row_lse + 32 * b + 8 * g + 4 * h);
                const f32x4 rd = *reinterpret_cast<const f32x4 *>(row_delta + 32 * b + 8 * g + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) { s[4 * g + e] = FROM ? rl[e] : 0.0f; dp[4 * g + e] = FROM ? rd[e] : 0.0f; }
            }
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                if (att_empty<T, DP>(d, a.dim)) break;
                const typename M::frag q = M::rows(tq, 32 * b, 16 * d), g = M::rows(tg, 32 * b, 16 * d);
                s = M::mma(q, kf[d], s);
                dp = M::mma(g, d < REGS ? vf[d] : held[64 * (d - REGS)], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = 32 * b + acc_row(i, h);
                s[i] = __builtin_amdgcn_exp2f(FROM ? s[i] * c : __builtin_fmaf(s[i], c, row_lse[r] * c));
                dp[i] = s[i] * (FROM ? dp[i] : dp[i] + row_delta[r]);
            }
            if (qb < kw + 31) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = qb + acc_row(i, h);
                    if (r < ki) s[i] = 0.0f;
                    if (r < ki || r == 0) dp[i] = 0.0f;    // row 0: as in the gradient of Q
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const typename M::held p = M::pack(s, 8 * k), ds = M::pack(dp, 8 * k);
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) {
                    const typename M::frag g = M::cols(tg, 32 * b + 16 * k, 32 * t), q = M::cols(tq, 32 * b + 16 * k, 32 * t);
                    dv[t] = M::mma(g, p, dv[t]);
                    dk[t] = M::mma(q, ds, dk[t]);
                }
            }
        }
    }
    if constexpr (NB > 1) {
        add_wavefronts<DP, NA, NB>(reinterpret_cast<float *>(lds), dk);
        add_wavefronts<DP, NA, NB>(reinterpret_cast<float *>(lds), dv);
        if (wb) return;
    }
    if (ki < tile.len) {
        const int row = tile.start + ki;
        if (a.part) {
            float *p = a.part + (((size_t)split * a.total + row) * kv_heads + kvh) * a.dim;
            store_row<float, DP>(p, a.dim, dk, 1.0f);
            store_row<float, DP>(p + (size_t)a.splits * a.total * kv_heads * a.dim, a.dim, dv, 1.0f);
        } else {
            store_row<T, DP>(att_at<T>(a.dK, row, kvh), a.dim, dk, a.scale);
            store_row<T, DP>(att_at<T>(a.dV, row, kvh), a.dim, dv, 1.0f);
        }
    }
}

// Bound by memory: 4 x 2048 rows, 4 heads of 64 from four parts each (75 MB) 12.8 us, 5.9 TB/s; heads of 128 22.6 us.
// Adds up the splits: a chunk of eight elements of a row and head per thread, dK in the first half of the grid's y, dV in the second.
template <typename T>
__global__ __launch_bounds__(256) void attention_sum_kernel(AttArgs a)
{
    const int kv_heads = a.heads / a.group, chunks = (a.dim + 7) / 8, per_row = kv_heads * chunks;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(t / per_row), kvh = (int)(t % per_row) / chunks, d = (int)(t % chunks) * 8;
    const int begin = a.cu ? max(a.cu[0], 0) : 0, end = a.cu ? min(a.cu[a.nseq], a.total) : a.total;
    if (row < begin || row >= end) return;
    const size_t stride = (size_t)a.total * kv_heads * a.dim;
    const float *p = a.part + blockIdx.y * a.splits * stride + ((size_t)row * kv_heads + kvh) * a.dim + d;
    float sum[8] = {};
    for (int s = 0; s < a.splits; ++s) {
        Chunk<float> c;
        c.load(p + s * stride, a.dim - d);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += c.get(e);
    }
    const float f = blockIdx.y == 0 ? a.scale : 1.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] *= f;
    store8(att_at<T>(blockIdx.y == 0 ? a.dK : a.dV, row, kvh) + d, sum, a.dim - d);
}

template <typename T, int DP, int NA, int NB, bool DIRECT> hipError_t launch(const AttArgs &a, hipStream_t stream)
{
    static bool configured[MAX_DEVICES] = {};
    const int64_t blocks = att_tiles(a, 32 * NA) * (a.heads / a.group) * a.splits;
    typedef DkvShape<T, DP, NA, NB, DIRECT> Shape;
    constexpr size_t MOST = att_lds<T, NB, Shape::PER_CU>(Shape::LDS, 0);
    const size_t bytes = att_lds<T, NB, Shape::PER_CU>(Shape::LDS, blocks);
    auto kernel = attention_dkv_kernel<T, DP, NA, NB, DIRECT>;
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), MOST, configured); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(ATT_THREADS), bytes, stream, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
    const int64_t threads = (int64_t)a.total * (a.heads / a.group) * ((a.dim + 7) / 8);
    hipLaunchKernelGGL(attention_sum_kernel<T>, dim3((unsigned)((threads + 255) / 256), 2), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

// The sums of a part of the heads are written and read once more in fp32, so as few parts as give the card four workgroups a CU:
// the backward pass of 4 x 2048 rows, 32 heads on 4, 306 us, 323 with 1536 and 372 with 512 workgroups as the mark.
int asteria::attention_splits(const AttArgs &a)
{
    const int64_t tiles = att_tiles(a, 128) * (a.heads / a.group);
    int splits = 1;
    for (int s = 2; s <= a.group && tiles * splits < 1024; ++s)
        if (a.group % s == 0) splits = s;
    return splits;
}

asteria_status asteria::attention_dkv(const AttArgs &a, int dtype, hipStream_t stream)
{
    const bool direct = att_direct(a.Q, dtype, a.total, a.dim) && att_direct(a.dO, dtype, a.total, a.dim);
    return att_for_type(dtype, a.dim, direct, [&](auto t, auto dp, auto direct_) {
        typedef decltype(t) T;
        constexpr int DP = dp();
        constexpr bool DIRECT = decltype(direct_)::value;
        ASTERIA_HIP_TRY((att_few(a, a.heads / a.group * a.splits) ? launch<T, DP, 4 / att_shared<T>, att_shared<T>, DIRECT>(a, stream)
                                                                   : launch<T, DP, 4, 1, DIRECT>(a, stream)));
        return ASTERIA_OK;
    });
}
