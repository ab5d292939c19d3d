// asteria_rms_norm and asteria_rms_norm_backward.
//
// A row lies in the registers of TPR threads, VPT chunks of eight elements each, chunk v * TPR + thread: every array is read
// and written once, in 16-byte (bf16) or 32-byte (fp32) pieces per thread, and what bounds both passes is memory.  Sums over
// a row (fp32) go over 16 lanes (rows of up to 128 elements), over the lanes of one wavefront (up to 2048) or through LDS.
// Measured: 16384 x 2048, bf16 with residual, sum, dropout and 8-bit output (236 MB) 50.8 us, 4.6 TB/s, a large copy's rate being 4.9;
// 1001 x 777 in fp32 5.1 us; 4 rows of 2048 4.1 us, launch and the latency of one row.  Backward, 16384 x 2048 with fp32 residual
// stream (537 MB): 114 us, 4.7 TB/s, both kernels.
#include <math.h>
#include <type_traits>

#include "common.h"
#include "rows.h"

using namespace asteria;

namespace {

constexpr int MAX_COLS = 16384, MAX_ROWS = 1 << 22;   // so many workgroups of 512 threads a launch takes
constexpr float E4M3_MAX = 448.0f, SCALE_FLOOR = 0x1p-100f;

struct NormArgs {
    const void *X, *R, *W;
    void *H, *Y;
    float *Scale;
    int rows, cols, ldx, ldr, ldh, ldy;
    int y_dtype, w_dtype, group;
    float eps;
    Dropper drop;
};

template <int TPR> constexpr int norm_threads() { return TPR > 256 ? TPR : 256; }

template <int TPR, int VPT, typename TX, typename TH>
__global__ __launch_bounds__(norm_threads<TPR>()) void norm_kernel(NormArgs a)
{
    __shared__ float part[norm_threads<TPR>() / 64][1];
    read_state(a.drop);
    const int t = (int)threadIdx.x % TPR;
    // a wavefront (TPR = 64) or workgroup without a row of its own works on the last one and writes nothing
    const int row_ = (int)blockIdx.x * (norm_threads<TPR>() / TPR) + (int)threadIdx.x / TPR;
    const bool live = row_ < a.rows;
    const int row = live ? row_ : a.rows - 1;
    Chunk<TX> x[VPT];
    Chunk<TH> r[VPT];
    const TX *X = reinterpret_cast<const TX *>(a.X) + (size_t)row * a.ldx;
    const TH *R = reinterpret_cast<const TH *>(a.R) + (size_t)row * a.ldr;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * TPR + t) * 8;
        x[v].zero();
        if (c < a.cols) x[v].load(X + c, a.cols - c);
    }
    if (a.R) {
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * TPR + t) * 8;
            r[v].zero();
            if (c < a.cols) r[v].load(R + c, a.cols - c);
        }
    } else {
#pragma unroll
        for (int v = 0; v < VPT; ++v) r[v].zero();
    }
    float h[VPT][8], sum[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[v][e] = x[v].get(e);
        if (a.drop.threshold) drop_chunk(a.drop, (uint32_t)row, (uint32_t)(v * TPR + t), h[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[v][e] += r[v].get(e);
            sum[0] += h[v][e] * h[v][e];
        }
        const int c = (v * TPR + t) * 8;
        if (live && a.H && c < a.cols) store8(reinterpret_cast<TH *>(a.H) + (size_t)row * a.ldh + c, h[v], a.cols - c);
    }
    row_reduce<false, TPR>(sum, part);
    const float rs = 1.0f / sqrtf(sum[0] / (float)a.cols + a.eps);
    float top[VPT];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * TPR + t) * 8;
        float w[8];
        if (a.W && c < a.cols) load8(a.W, a.w_dtype, (size_t)c, w, a.cols - c);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = 1.0f;
        }
        top[v] = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[v][e] = c + e < a.cols ? h[v][e] * rs * w[e] : 0.0f;
            top[v] = fmaxf(top[v], fabsf(h[v][e]));
        }
        if (a.y_dtype != ASTERIA_E4M3 && live && c < a.cols) store8(a.Y, a.y_dtype, (size_t)row * a.ldy + c, h[v], a.cols - c);
    }
    if (a.y_dtype != ASTERIA_E4M3) return;
    if (a.group) {
        // 128 columns are the chunks of 16 lanes side by side
#pragma unroll
        for (int v = 0; v < VPT; ++v) top[v] = lanes_reduce<true, 16>(top[v]);
    } else {
        float m[1] = {top[0]};
#pragma unroll
        for (int v = 1; v < VPT; ++v) m[0] = fmaxf(m[0], top[v]);
        row_reduce<true, TPR>(m, part);
#pragma unroll
        for (int v = 0; v < VPT; ++v) top[v] = m[0];
    }
    if (!live) return;
    const int groups = a.group ? (a.cols + 127) / 128 : 1;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int ch = v * TPR + t, c = ch * 8;
        if (c >= a.cols) continue;
        const float scale = fmaxf(top[v], SCALE_FLOOR) / E4M3_MAX, inv = 1.0f / scale;
        if (a.group ? (ch & 15) == 0 : ch == 0) a.Scale[(size_t)row * groups + (a.group ? ch >> 4 : 0)] = scale;
        // Quotients: a product with the rounded reciprocal is on the other side of a tie for some elements.  The product's remainder, exact in one
        // multiply-add, times the reciprocal once more rounds it to the quotient (16384 x 2048: 53.7 us, 57 with divisions, where a product took 53) - but not
        // where the remainder can pass below fp32's range or the scale is infinite.  |y / scale| is at most 448 (1 + 2^-22), which rounds to
        // 448; what is no number stays none
        float z[8];
        if (scale >= 0x1p-80f && scale < INFINITY) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float near = h[v][e] * inv;
                z[e] = __builtin_fmaf(-__builtin_fmaf(near, scale, -h[v][e]), inv, near);     // in this order -0 stays -0
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = h[v][e] / scale;
        }
        uint32_t q[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            int p = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * k], z[4 * k + 1], 0, false);
            q[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[4 * k + 2], z[4 * k + 3], p, true);
        }
        uint8_t *Y = reinterpret_cast<uint8_t *>(a.Y) + (size_t)row * a.ldy + c;
        u8x8_any b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = (uint8_t)(q[e >> 2] >> (8 * (e & 3)));
        if (a.cols - c >= 8) *reinterpret_cast<u8x8_any *>(Y) = b;
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (c + e < a.cols) Y[e] = b[e];
        }
    }
}

struct NormGradArgs {
    const void *H, *dY, *W, *dH;
    void *dX, *dR;
    float *part;       // partial sums of dW, one row of cols per workgroup, or null
    int rows, cols, ldh, lddy, lddh, lddx, lddr;
    int x_dtype, w_dtype;
    float eps;
    Dropper drop;
};

// Every workgroup takes rows gridDim.x apart and keeps its columns' share of dW in registers over all of them, so that H and dY are
// read once and dW costs a row of partial sums a workgroup (600 x 5632: 13.4 us, 2.6 TB/s: two rows a workgroup, of which the second's
// loads begin behind the first's two barriers).
template <int TPR, int VPT, typename TH, typename TY>
__global__ __launch_bounds__(norm_threads<TPR>()) void norm_grad_kernel(NormGradArgs a)
{
    constexpr int NT = norm_threads<TPR>(), RPB = NT / TPR;
    __shared__ float part[NT / 64][2];
    read_state(a.drop);
    const int t = (int)threadIdx.x % TPR;
    float dw[VPT][8];
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[v][e] = 0.0f;
    for (int first = (int)blockIdx.x * RPB; first < a.rows; first += (int)gridDim.x * RPB) {
        const int row_ = first + (int)threadIdx.x / TPR;
        const bool live = row_ < a.rows;
        const int row = live ? row_ : a.rows - 1;
        Chunk<TH> h[VPT], g[VPT];
        Chunk<TY> y[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * TPR + t) * 8;
            h[v].zero(); y[v].zero(); g[v].zero();
            if (c < a.cols) {
                h[v].load(reinterpret_cast<const TH *>(a.H) + (size_t)row * a.ldh + c, a.cols - c);
                y[v].load(reinterpret_cast<const TY *>(a.dY) + (size_t)row * a.lddy + c, a.cols - c);
                if (a.dH) g[v].load(reinterpret_cast<const TH *>(a.dH) + (size_t)row * a.lddh + c, a.cols - c);
            }
        }
        float n[VPT][8], sums[2] = {0.0f, 0.0f};            // of h^2, of n h
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * TPR + t) * 8;
            float w[8];
            if (a.W && c < a.cols) load8(a.W, a.w_dtype, (size_t)c, w, a.cols - c);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = 1.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float he = h[v].get(e);
                n[v][e] = y[v].get(e) * w[e];
                sums[0] += he * he;
                sums[1] += n[v][e] * he;
            }
        }
        row_reduce<false, TPR>(sums, part);
        const float rs = 1.0f / sqrtf(sums[0] / (float)a.cols + a.eps);
        const float f = rs * rs * (sums[1] / (float)a.cols);
        if (!live) continue;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int ch = v * TPR + t, c = ch * 8;
            float d[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float he = h[v].get(e);
                dw[v][e] += y[v].get(e) * he * rs;
                d[e] = g[v].get(e) + rs * (n[v][e] - he * f);
            }
            if (c >= a.cols) continue;
            if (a.dR) store8(reinterpret_cast<TH *>(a.dR) + (size_t)row * a.lddr + c, d, a.cols - c);
            if (a.dX) {
                if (a.drop.threshold) drop_chunk(a.drop, (uint32_t)row, (uint32_t)ch, d);
                store8(a.dX, a.x_dtype, (size_t)row * a.lddx + c, d, a.cols - c);
            }
        }
    }
    if (!a.part) return;
    if constexpr (RPB > 1) {
        // the wavefronts of the workgroup hold the same columns
        __shared__ float share[RPB][TPR * 8];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) share[threadIdx.x / TPR][e * TPR + t] = dw[v][e];
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[v][e] = share[0][e * TPR + t];
#pragma unroll
                for (int k = 1; k < RPB; ++k) dw[v][e] += share[k][e * TPR + t];
            }
        }
        if (threadIdx.x >= TPR) return;
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * TPR + t) * 8;
        if (c < a.cols) store8(a.part + (size_t)blockIdx.x * a.cols + c, dw[v], a.cols - c);
    }
}

// dW = sum of the workgroups' partial sums: 32 columns a workgroup, 32 threads a column, eight loads of a thread in flight, so that
// 512 partial sums are two trips to memory (4 us for 5632 columns).
__global__ __launch_bounds__(1024) void norm_weight_grad_kernel(const float *part, int nparts, int cols, void *dW, int w_dtype)
{
    __shared__ float s[32][33];
    const int c = (int)blockIdx.x * 32 + (int)threadIdx.x % 32, k = (int)threadIdx.x / 32;
    float v = 0.0f;
    if (c < cols) {
        for (int p = k; p < nparts; p += 256) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p + 32 * i < nparts ? part[(size_t)(p + 32 * i) * cols + c] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += x[i];
        }
    }
    s[k][threadIdx.x % 32] = v;
    __syncthreads();
    if (k == 0 && c < cols) {
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) v += s[i][threadIdx.x % 32];
        if (w_dtype == ASTERIA_BF16) reinterpret_cast<uint16_t *>(dW)[c] = f32_bf16(v);
        else reinterpret_cast<float *>(dW)[c] = v;
    }
}

// Rows of up to 128 elements take 16 lanes (the norm of queries and keys, a row per head; backward of 16000 x 100: 12.6 us, 25.9
// with a wavefront each), of up to 2048 one wavefront, of up to 8192 four, longer ones eight: at most 32 elements a thread, what the
// backward pass holds of three arrays in registers.
template <typename F> asteria_status for_width(int cols, F f)
{
    if (cols <= 128) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    if (cols <= 512) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    if (cols <= 1024) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    if (cols <= 2048) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
    if (cols <= 4096) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    if (cols <= 8192) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
    return f(std::integral_constant<int, 512>(), std::integral_constant<int, 4>());
}

// As many workgroups as run at a time (two a CU), each with the same number of rows or one less: every one more is a row of
// partial sums to write and to read (16384 x 2048: 115 us so, 124 with 1024 workgroups; 600 x 5632: 16.4 and 24.8).
int grad_blocks(int rows, int cols)
{
    const int rpb = cols <= 128 ? 16 : cols <= 2048 ? 4 : 1, units = (rows + rpb - 1) / rpb, per = (units + 511) / 512;
    return (units + per - 1) / per;
}

bool valid_eps(float eps) { return eps >= 0.0f && isfinite(eps); }

}  // namespace

extern "C" asteria_status asteria_rms_norm(const asteria_norm *n, float eps, const asteria_rng *rng, void *stream_)
{
    if (!n || !n->X || !n->Y || n->rows <= 0 || n->cols <= 0 || !valid_eps(eps)) return ASTERIA_INVALID_ARG;
    if (n->ldx < n->cols || n->ldy < n->cols || (n->R && n->ldr < n->cols) || (n->H && n->ldh < n->cols)) return ASTERIA_INVALID_ARG;
    if (!valid_dtype(n->x_dtype) || !valid_dtype(n->h_dtype) || !valid_dtype(n->w_dtype)) return ASTERIA_INVALID_ARG;
    const bool e4m3 = n->y_dtype == ASTERIA_E4M3;
    if (!e4m3 && !valid_dtype(n->y_dtype)) return ASTERIA_INVALID_ARG;
    if (e4m3 ? !n->Scale || (n->group != 0 && n->group != 128) : n->group != 0) return ASTERIA_INVALID_ARG;
    if (n->H && ((n->H == n->R && n->ldh != n->ldr) || (n->H == n->X && (n->ldh != n->ldx || n->h_dtype != n->x_dtype)))) return ASTERIA_INVALID_ARG;
    if (n->Y == n->H || n->Y == n->R || (n->Y == n->X && (n->ldy != n->ldx || n->y_dtype != n->x_dtype))) return ASTERIA_INVALID_ARG;
    if (n->cols > MAX_COLS || n->rows >= MAX_ROWS) return ASTERIA_UNSUPPORTED;
    NormArgs a;
    if (!make_dropper(rng, a.drop)) return ASTERIA_INVALID_ARG;
    a.X = n->X; a.R = n->R; a.W = n->W; a.H = n->H; a.Y = n->Y; a.Scale = n->Scale;
    a.rows = n->rows; a.cols = n->cols; a.ldx = n->ldx; a.ldr = n->R ? n->ldr : 0; a.ldh = n->ldh; a.ldy = n->ldy;
    a.y_dtype = n->y_dtype; a.w_dtype = n->w_dtype; a.group = n->group; a.eps = eps;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    return for_width(n->cols, [&](auto tpr, auto vpt) {
        constexpr int TPR = tpr(), VPT = vpt(), NT = norm_threads<TPR>(), RPB = NT / TPR;
        const dim3 grid((unsigned)((n->rows + RPB - 1) / RPB));
        const bool xb = n->x_dtype == ASTERIA_BF16, hb = n->h_dtype == ASTERIA_BF16;
        if (xb && hb) hipLaunchKernelGGL((norm_kernel<TPR, VPT, bf16_elem, bf16_elem>), grid, dim3(NT), 0, stream, a);
        else if (xb) hipLaunchKernelGGL((norm_kernel<TPR, VPT, bf16_elem, float>), grid, dim3(NT), 0, stream, a);
        else if (hb) hipLaunchKernelGGL((norm_kernel<TPR, VPT, float, bf16_elem>), grid, dim3(NT), 0, stream, a);
        else hipLaunchKernelGGL((norm_kernel<TPR, VPT, float, float>), grid, dim3(NT), 0, stream, a);
        ASTERIA_HIP_TRY(hipGetLastError());
        return ASTERIA_OK;
    });
}

extern "C" size_t asteria_rms_norm_backward_workspace_bytes(const asteria_norm_grad *n)
{
    if (!n || !n->dW || n->rows <= 0 || n->cols <= 0 || n->cols > MAX_COLS || n->rows >= MAX_ROWS) return 0;
    return Carver::need((size_t)grad_blocks(n->rows, n->cols) * n->cols, sizeof(float));
}

extern "C" asteria_status asteria_rms_norm_backward(const asteria_norm_grad *n, float eps, const asteria_rng *rng,
                                                    void *ws, size_t ws_bytes, void *stream_)
{
    if (!n || !n->H || !n->dY || n->rows <= 0 || n->cols <= 0 || !valid_eps(eps)) return ASTERIA_INVALID_ARG;
    if (n->ldh < n->cols || n->lddy < n->cols || (n->dH && n->lddh < n->cols) || (n->dX && n->lddx < n->cols) ||
        (n->dR && n->lddr < n->cols)) return ASTERIA_INVALID_ARG;
    if (!valid_dtype(n->x_dtype) || !valid_dtype(n->h_dtype) || !valid_dtype(n->y_dtype) || !valid_dtype(n->w_dtype)) return ASTERIA_INVALID_ARG;
    if (n->dR && (n->dR == n->H || n->dR == n->dY || (n->dR == n->dH && n->lddr != n->lddh))) return ASTERIA_INVALID_ARG;
    if (n->dX && (n->dX == n->H || n->dX == n->dH || n->dX == n->dR ||
                  (n->dX == n->dY && (n->lddx != n->lddy || n->x_dtype != n->y_dtype)))) return ASTERIA_INVALID_ARG;
    if (n->cols > MAX_COLS || n->rows >= MAX_ROWS) return ASTERIA_UNSUPPORTED;
    NormGradArgs a;
    if (!make_dropper(rng, a.drop)) return ASTERIA_INVALID_ARG;
    if (n->dW) {
        if (!ws || ws_bytes < asteria_rms_norm_backward_workspace_bytes(n)) return ASTERIA_WORKSPACE_TOO_SMALL;
        if (reinterpret_cast<uintptr_t>(ws) & 255u) return ASTERIA_INVALID_ARG;   // workspace must be 256-byte aligned
    }
    a.H = n->H; a.dY = n->dY; a.W = n->W; a.dH = n->dH; a.dX = n->dX; a.dR = n->dR;
    a.part = n->dW ? reinterpret_cast<float *>(ws) : nullptr;
    a.rows = n->rows; a.cols = n->cols; a.ldh = n->ldh; a.lddy = n->lddy; a.lddh = n->lddh; a.lddx = n->lddx; a.lddr = n->lddr;
    a.x_dtype = n->x_dtype; a.w_dtype = n->w_dtype; a.eps = eps;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    const int blocks = grad_blocks(n->rows, n->cols);
    ASTERIA_TRY(for_width(n->cols, [&](auto tpr, auto vpt) {
        constexpr int TPR = tpr(), VPT = vpt(), NT = norm_threads<TPR>();
        const bool hb = n->h_dtype == ASTERIA_BF16, yb = n->y_dtype == ASTERIA_BF16;
        const dim3 grid((unsigned)blocks);
        if (hb && yb) hipLaunchKernelGGL((norm_grad_kernel<TPR, VPT, bf16_elem, bf16_elem>), grid, dim3(NT), 0, stream, a);
        else if (hb) hipLaunchKernelGGL((norm_grad_kernel<TPR, VPT, bf16_elem, float>), grid, dim3(NT), 0, stream, a);
        else if (yb) hipLaunchKernelGGL((norm_grad_kernel<TPR, VPT, float, bf16_elem>), grid, dim3(NT), 0, stream, a);
        else hipLaunchKernelGGL((norm_grad_kernel<TPR, VPT, float, float>), grid, dim3(NT), 0, stream, a);
        ASTERIA_HIP_TRY(hipGetLastError());
        return ASTERIA_OK;
    }));
    if (n->dW) {
        hipLaunchKernelGGL(norm_weight_grad_kernel, dim3((unsigned)((n->cols + 31) / 32)), dim3(1024), 0, stream, a.part, blocks, n->cols,
                           n->dW, n->w_dtype);
        ASTERIA_HIP_TRY(hipGetLastError());
    }
    return ASTERIA_OK;
}
