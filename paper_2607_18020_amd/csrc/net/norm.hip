// norm.hip -- root-mean-square norm with the residual stream's addition, its
// 8-bit output and its gradients.
//
// Forward: s = x + r, y = w s (mean(s^2) + eps)^-1/2.  A row is held in the
// registers of LPR neighbouring lanes between the sum of its squares and its
// output, so x and r are read once and y and s written once; what bounds it is
// memory.  LPR grows with the width (16 lanes to a workgroup of 256) such that a
// lane holds one or a few 16-byte loads: narrow rows share a wavefront.
//
// Backward: with rho = (mean(s^2) + eps)^-1/2 and g = w dy, differentiating
// y_i = w_i s_i rho gives ds = dsum + rho g - rho^3 mean(g s) s.  Both row means
// come from the registers that hold the row, so again everything is read once; rho
// is recomputed, since s is read anyway.  dw sums dy s rho over the rows: a lane
// keeps the sums of its columns in float32 registers while its workgroup walks
// over rows, the workgroup adds its row groups through LDS and writes one
// partial row, and colsum_kernel adds those in a fixed order.
#include "net_common.hpp"

using namespace fpde_net;

namespace {

constexpr float kF8Max = 448.f, kF8Tiny = 0x1p-126f;

// four float32 values, already in +-448 or NaN, as four e4m3 bytes
__device__ __forceinline__ uint32_t pack_f8(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}

// y / sigma, held in +-448; a NaN stays one
__device__ __forceinline__ float to_f8_range(float y, float sigma) {
    const float q = y / sigma;
    return q > kF8Max ? kF8Max : (q < -kF8Max ? -kF8Max : q);
}

template <int V>
__device__ __forceinline__ void store_f8(uint8_t* p, const float (&y)[V], float sigma, int n) {
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
        w[i] = pack_f8(to_f8_range(y[4 * i], sigma), to_f8_range(y[4 * i + 1], sigma),
                       to_f8_range(y[4 * i + 2], sigma), to_f8_range(y[4 * i + 3], sigma));
    if (n >= V) {
        typedef uint32_t u32a1 __attribute__((aligned(1)));
#pragma unroll
        for (int i = 0; i < V / 4; ++i) ((u32a1*)p)[i] = w[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
    }
}

__device__ __forceinline__ float f8_scale(float amax) { return fmaxf(amax / kF8Max, kF8Tiny); }

__device__ __forceinline__ float rms_scale(float sumsq, float inv_width, float eps) {
    return __builtin_amdgcn_rsqf(fmaf(sumsq, inv_width, eps));
}

struct NormP {
    const void *x, *r, *w;
    void *y, *s;
    float* scales;
    int64_t rows, xs, rs;
    int width, wf32, group, ngroups;
    float eps, inv_width;
};

// A row in LPR lanes x CH chunks of V columns; 256 threads.
template <class T, bool F8, int LPR, int CH>
__global__ __launch_bounds__(256) void norm_fwd_kernel(NormP P) {
    constexpr int V = kVec<T>, RPB = 256 / LPR;
    __shared__ float red[4];
    const int lane = threadIdx.x % LPR;
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR;; row += (int64_t)gridDim.x * RPB) {
        // (a workgroup's threads leave together where they meet at barriers: LPR = 256 is one row)
        if (LPR == 256 ? row >= P.rows : row - threadIdx.x / LPR >= P.rows) break;
        const bool live = row < P.rows;
        float s[CH][V];
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * LPR + lane) * V, n = live ? P.width - c : 0;
            if (n > 0) {
                load_f32<T, V>(s[k], (const T*)P.x + row * P.xs + c, n);
                if (P.r) {
                    float q[V];
                    load_f32<T, V>(q, (const T*)P.r + row * P.rs + c, n);
#pragma unroll
                    for (int i = 0; i < V; ++i) s[k][i] += q[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) s[k][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) ss = fmaf(s[k][i], s[k][i], ss);
        }
        ss = group_reduce<LPR, AddOp>(ss, red);
        const float rho = rms_scale(ss, P.inv_width, P.eps);
        float rowmax = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * LPR + lane) * V, n = live ? P.width - c : 0;
            if (n > 0 && P.s) store_f32<T, V>((T*)P.s + row * P.width + c, s[k], n);
#pragma unroll
            for (int i = 0; i < V; ++i) s[k][i] *= rho;
            if (n > 0 && P.w) {
                float w[V];
                load_param<T, V>(w, P.w, P.wf32, c, n);
#pragma unroll
                for (int i = 0; i < V; ++i) s[k][i] *= w[i];
            }
            if constexpr (F8) {
                // a group of 128 columns is 128 / V neighbouring lanes of one chunk
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) m = fmaxf(m, n > i ? fabsf(s[k][i]) : 0.f);
                if (P.group) {
                    m = lanes_reduce<128 / V, MaxOp>(m);
                    const float sigma = f8_scale(m);
                    if (n > 0) {
                        store_f8<V>((uint8_t*)P.y + row * P.width + c, s[k], sigma, n);
                        if (c % 128 == 0) P.scales[row * P.ngroups + c / 128] = sigma;
                    }
                } else {
                    rowmax = fmaxf(rowmax, m);
                }
            } else if (n > 0) {
                store_f32<T, V>((T*)P.y + row * P.width + c, s[k], n);
            }
        }
        if constexpr (F8) {
            if (!P.group) {
                const float sigma = f8_scale(group_reduce<LPR, MaxOp>(rowmax, red));
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    const int c = (k * LPR + lane) * V, n = live ? P.width - c : 0;
                    if (n > 0) store_f8<V>((uint8_t*)P.y + row * P.width + c, s[k], sigma, n);
                }
                if (live && lane == 0) P.scales[row] = sigma;
            }
        }
    }
}

// Rows wider than the registers hold: a workgroup of 1024 per row reads it once
// for the sum of squares and again (from the caches) for each output pass.
template <class T, bool F8>
__global__ __launch_bounds__(1024) void norm_fwd_wide_kernel(NormP P) {
    constexpr int V = kVec<T>;
    __shared__ float red[16];
    for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x) {
        auto load = [&](int c, int n, float (&s)[V]) {
            load_f32<T, V>(s, (const T*)P.x + row * P.xs + c, n);
            if (P.r) {
                float q[V];
                load_f32<T, V>(q, (const T*)P.r + row * P.rs + c, n);
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] += q[i];
            }
        };
        float ss = 0.f;
        for (int c = threadIdx.x * V; c < P.width; c += 1024 * V) {
            float s[V];
            load(c, P.width - c, s);
#pragma unroll
            for (int i = 0; i < V; ++i) ss = fmaf(s[i], s[i], ss);
        }
        const float rho = rms_scale(group_reduce<1024, AddOp>(ss, red), P.inv_width, P.eps);
        auto scaled = [&](int c, int n, float (&s)[V]) {
            load(c, n, s);
            float w[V];
            if (P.w) load_param<T, V>(w, P.w, P.wf32, c, n);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = P.w ? s[i] * rho * w[i] : s[i] * rho;
        };
        float rowmax = 0.f;
        if (F8 && !P.group) {
            for (int c = threadIdx.x * V; c < P.width; c += 1024 * V) {
                float s[V];
                scaled(c, P.width - c, s);
#pragma unroll
                for (int i = 0; i < V; ++i) rowmax = fmaxf(rowmax, P.width - c > i ? fabsf(s[i]) : 0.f);
            }
            rowmax = group_reduce<1024, MaxOp>(rowmax, red);
            if (threadIdx.x == 0) P.scales[row] = f8_scale(rowmax);
        }
        // (every lane of a wavefront takes part in the groups' maxima; s may be the x or r that
        // this pass reads, so it is written element for element where it was read)
        const int end = (P.width + 1024 * V - 1) / (1024 * V) * (1024 * V);
        for (int c = threadIdx.x * V; c < end; c += 1024 * V) {
            const int n = P.width - c;
            float s[V];
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = 0.f;
            if (n > 0) {
                if (P.s) {
                    float q[V];
                    load(c, n, q);
                    scaled(c, n, s);
                    store_f32<T, V>((T*)P.s + row * P.width + c, q, n);
                } else {
                    scaled(c, n, s);
                }
            }
            if constexpr (F8) {
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) m = fmaxf(m, n > i ? fabsf(s[i]) : 0.f);
                if (P.group) m = lanes_reduce<128 / V, MaxOp>(m);
                const float sigma = f8_scale(P.group ? m : rowmax);
                if (n > 0) {
                    store_f8<V>((uint8_t*)P.y + row * P.width + c, s, sigma, n);
                    if (P.group && c % 128 == 0) P.scales[row * P.ngroups + c / 128] = sigma;
                }
            } else if (n > 0) {
                store_f32<T, V>((T*)P.y + row * P.width + c, s, n);
            }
        }
    }
}

struct NormBwdP {
    const void *dy, *s, *dsum, *w;
    void* ds;
    float* part;      // [gridDim.x][width], or nullptr
    float* rho;       // wide rows: [rows], or nullptr
    int64_t rows, dys, ss, dss;
    int width, wf32;
    float eps, inv_width;
};

template <class T, int LPR, int CH>
__global__ __launch_bounds__(256) void norm_bwd_kernel(NormBwdP P) {
    constexpr int V = kVec<T>, RPB = 256 / LPR;
    __shared__ float red[4], red2[4];
    __shared__ float acc[LPR == 256 ? 1 : RPB][LPR == 256 ? 1 : LPR * CH * V];
    const int lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
    float w[CH][V], dw[CH][V];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * LPR + lane) * V, n = P.width - c;
#pragma unroll
        for (int i = 0; i < V; ++i) w[k][i] = 1.f, dw[k][i] = 0.f;
        if (P.w && n > 0) load_param<T, V>(w[k], P.w, P.wf32, c, n);
    }
    for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < P.rows; row0 += (int64_t)gridDim.x * RPB) {
        const int64_t row = row0 + sub;
        const bool live = row < P.rows;
        float s[CH][V], g[CH][V];
        float ss = 0.f, gs = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * LPR + lane) * V, n = live ? P.width - c : 0;
#pragma unroll
            for (int i = 0; i < V; ++i) s[k][i] = 0.f, g[k][i] = 0.f;
            if (n > 0) {
                load_f32<T, V>(s[k], (const T*)P.s + row * P.ss + c, n);
                load_f32<T, V>(g[k], (const T*)P.dy + row * P.dys + c, n);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                ss = fmaf(s[k][i], s[k][i], ss);
                gs = fmaf(g[k][i] * w[k][i], s[k][i], gs);
            }
        }
        ss = group_reduce<LPR, AddOp>(ss, red);
        gs = group_reduce<LPR, AddOp>(gs, red2);
        const float rho = rms_scale(ss, P.inv_width, P.eps);
        const float c3 = rho * rho * rho * gs * P.inv_width;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * LPR + lane) * V, n = live ? P.width - c : 0;
            if (n > 0) {
                float d[V];
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] = 0.f;
                if (P.dsum) load_f32<T, V>(d, (const T*)P.dsum + row * P.dss + c, n);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float t = rho * g[k][i];
                    dw[k][i] = fmaf(t, s[k][i], dw[k][i]);
                    d[i] += fmaf(t, w[k][i], -c3 * s[k][i]);
                }
                store_f32<T, V>((T*)P.ds + row * P.width + c, d, n);
            }
        }
    }
    if (!P.part) return;
    float* out = P.part + (int64_t)blockIdx.x * P.width;
    if constexpr (LPR == 256) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * LPR + lane) * V, n = P.width - c;
            if (n > 0) store_f32<float, V>(out + c, dw[k], n);
        }
    } else {
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[sub][(k * LPR + lane) * V + i] = dw[k][i];
        __syncthreads();
        for (int c = threadIdx.x; c < P.width; c += 256) {
            float t = acc[0][c];
#pragma unroll
            for (int r = 1; r < RPB; ++r) t += acc[r][c];
            out[c] = t;
        }
    }
}

// Wide rows: ds a row at a time, re-read from the caches, and rho kept for the
// column sums, which walk down the rows (without ds: rho alone).
template <class T>
__global__ __launch_bounds__(1024) void norm_bwd_wide_kernel(NormBwdP P) {
    constexpr int V = kVec<T>;
    __shared__ float red[16], red2[16];
    for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x) {
        float ss = 0.f, gs = 0.f;
        auto load = [&](int c, int n, float (&s)[V], float (&g)[V], float (&w)[V]) {
            load_f32<T, V>(s, (const T*)P.s + row * P.ss + c, n);
            load_f32<T, V>(g, (const T*)P.dy + row * P.dys + c, n);
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = 1.f;
            if (P.w) load_param<T, V>(w, P.w, P.wf32, c, n);
        };
        for (int c = threadIdx.x * V; c < P.width; c += 1024 * V) {
            float s[V], g[V], w[V];
            load(c, P.width - c, s, g, w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                ss = fmaf(s[i], s[i], ss);
                gs = fmaf(g[i] * w[i], s[i], gs);
            }
        }
        ss = group_reduce<1024, AddOp>(ss, red);
        gs = group_reduce<1024, AddOp>(gs, red2);
        const float rho = rms_scale(ss, P.inv_width, P.eps);
        const float c3 = rho * rho * rho * gs * P.inv_width;
        if (P.rho && threadIdx.x == 0) P.rho[row] = rho;
        if (!P.ds) continue;
        for (int c = threadIdx.x * V; c < P.width; c += 1024 * V) {
            const int n = P.width - c;
            float s[V], g[V], w[V], d[V];
            load(c, n, s, g, w);
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] = 0.f;
            if (P.dsum) load_f32<T, V>(d, (const T*)P.dsum + row * P.dss + c, n);
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] += fmaf(rho * g[i], w[i], -c3 * s[i]);
            store_f32<T, V>((T*)P.ds + row * P.width + c, d, n);
        }
    }
}

// Wide rows: dw partials.  Workgroup (x, y) sums rows y, y + gridDim.y, ... of 256 chunks of
// V columns.
template <class T>
__global__ __launch_bounds__(256) void norm_dw_wide_kernel(NormBwdP P) {
    constexpr int V = kVec<T>;
    const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * V, n = P.width - c;
    if (n <= 0) return;
    float dw[V];
#pragma unroll
    for (int i = 0; i < V; ++i) dw[i] = 0.f;
    for (int64_t row = blockIdx.y; row < P.rows; row += gridDim.y) {
        float s[V], g[V];
        load_f32<T, V>(s, (const T*)P.s + row * P.ss + c, n);
        load_f32<T, V>(g, (const T*)P.dy + row * P.dys + c, n);
        const float rho = P.rho[row];
#pragma unroll
        for (int i = 0; i < V; ++i) dw[i] = fmaf(rho * g[i], s[i], dw[i]);
    }
    store_f32<float, V>(P.part + (int64_t)blockIdx.y * P.width + c, dw, n);
}

// ---------------------------------------------------------------------------
// Host side.

constexpr int64_t kMaxRows = (int64_t)1 << 40, kMaxWidth = 1 << 20;

// lanes a row and 16-byte chunks a lane: f(LPR, CH) for the narrowest that holds the row;
// f(0, 0) if none does
template <class F>
int with_layout(int64_t chunks, F f) {
#define FPDE_L(L, C) f(std::integral_constant<int, L>{}, std::integral_constant<int, C>{})
    if (chunks <= 16) return FPDE_L(16, 1);
    if (chunks <= 32) return FPDE_L(32, 1);
    if (chunks <= 64) return FPDE_L(64, 1);
    if (chunks <= 128) return FPDE_L(64, 2);
    if (chunks <= 256) return FPDE_L(64, 4);
    if (chunks <= 512) return FPDE_L(256, 2);
    if (chunks <= 1024) return FPDE_L(256, 4);
    if (chunks <= 2048) return FPDE_L(256, 8);
    return FPDE_L(0, 0);
#undef FPDE_L
}

// Workgroups of the backward, which each write one partial row of dw: 4 for every
// compute unit keep the loads in flight, and few partial rows keep their sum short.
constexpr int64_t kBwdBlocks = 1024;
// Row groups of the wide rows' column sums.
constexpr int64_t kWideGroups = 128;
// Most workgroups of a launch: past it they loop over rows.
constexpr int64_t kMaxBlocks = 1 << 21;

bool known(int dtype) { return size_of(dtype) != 0; }

int check_norm(int dtype, int wdtype, int64_t rows, int64_t width, double eps) {
    if (!known(dtype) || !(wdtype == FPDE_F32 || wdtype == dtype)) return FPDE_ERR_UNSUPPORTED;
    if (rows < 0 || rows > kMaxRows || width < 1 || width > kMaxWidth) return FPDE_ERR_SHAPE;
    if (!(eps >= 0.0) || !(eps <= 3.0e38)) return FPDE_ERR_COEFF;
    return FPDE_OK;
}

bool stride_ok(int64_t stride, int64_t width) { return stride >= width && stride <= (int64_t)1 << 40; }

int64_t bwd_blocks(int64_t rows, int rows_per_block) {
    const int64_t n = cdiv(rows, rows_per_block);
    return n < 1 ? 1 : (n > kBwdBlocks ? kBwdBlocks : n);
}

template <class T>
int queue_dw_wide(const NormBwdP& P, int64_t parts, hipStream_t s) {
    return launch(norm_dw_wide_kernel<T>,
                  dim3((unsigned)cdiv(P.width, 256 * kVec<T>), (unsigned)parts), dim3(256), s, P);
}

}  // namespace

extern "C" int fpde_rms_norm(const fpde_norm_args* a, void* stream) {
    if (!a) return FPDE_ERR_ARG;
    int st = check_norm(a->dtype, a->weight_dtype, a->rows, a->width, a->eps);
    if (st != FPDE_OK) return st;
    const bool f8 = a->out_dtype == FPDE_F8E4M3;
    if (!f8 && a->out_dtype != a->dtype) return FPDE_ERR_UNSUPPORTED;
    if (f8 && a->group != 128 && a->group != 0) return FPDE_ERR_UNSUPPORTED;
    if (!stride_ok(a->x_stride, a->width) || (a->residual && !stride_ok(a->residual_stride, a->width)))
        return FPDE_ERR_SHAPE;
    if (a->rows == 0) return FPDE_OK;
    if (!a->x || !a->y || (f8 && !a->scales)) return FPDE_ERR_ARG;
    const int e = size_of(a->dtype);
    const int64_t ng = f8 && a->group ? cdiv(a->width, a->group) : 1;
    const int64_t dense = a->rows * a->width;
    Spans sp;
    sp.add(a->x, span3(1, a->rows, a->width, 0, a->x_stride, e), e, false);
    sp.add(a->residual, span3(1, a->rows, a->width, 0, a->residual_stride, e), e, false);
    sp.add(a->weight, a->width * size_of(a->weight_dtype), size_of(a->weight_dtype), false);
    sp.add(a->y, dense * (f8 ? 1 : e), f8 ? 1 : e, true);
    sp.add(a->sum, dense * e, e, true);
    if (f8) sp.add(a->scales, a->rows * ng * 4, 4, true);
    // (in place: the whole dense x or residual)
    const void* twin = a->sum == a->x ? a->x : a->residual;
    st = sp.check(a->sum, twin);
    if (st != FPDE_OK) return st;
    NormP P{a->x, a->residual, a->weight, a->y, a->sum, a->scales, a->rows, a->x_stride,
            a->residual_stride, (int)a->width, a->weight_dtype == FPDE_F32, a->group, (int)ng,
            (float)a->eps, (float)(1.0 / (double)a->width)};
    return with_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        return with_layout(cdiv(a->width, kVec<T>), [&](auto lpr, auto ch) {
            constexpr int L = decltype(lpr)::value, C = decltype(ch)::value;
            hipStream_t s = (hipStream_t)stream;
            if constexpr (L == 0) {
                const dim3 g((unsigned)(a->rows < kMaxBlocks ? a->rows : kMaxBlocks));
                return f8 ? launch(norm_fwd_wide_kernel<T, true>, g, dim3(1024), s, P)
                          : launch(norm_fwd_wide_kernel<T, false>, g, dim3(1024), s, P);
            } else {
                // (8 bits in 16-lane rows of float32: a group of 128 columns needs 32 lanes)
                constexpr int L8 = L < 128 / kVec<T> ? 128 / kVec<T> : L;
                const int64_t n = cdiv(a->rows, f8 ? 256 / L8 : 256 / L);
                const dim3 g((unsigned)(n < kMaxBlocks ? n : kMaxBlocks));
                return f8 ? launch(norm_fwd_kernel<T, true, L8, C>, g, dim3(256), s, P)
                          : launch(norm_fwd_kernel<T, false, L, C>, g, dim3(256), s, P);
            }
        });
    });
}

extern "C" int64_t fpde_rms_norm_bwd_workspace(const fpde_norm_bwd_args* a) {
    if (!a) return FPDE_ERR_ARG;
    const int st = check_norm(a->dtype, a->weight_dtype, a->rows, a->width, a->eps);
    if (st != FPDE_OK) return st;
    if (!a->dweight) return 0;
    const int64_t chunks = cdiv(a->width, 16 / size_of(a->dtype));
    return with_layout(chunks, [&](auto lpr, auto) { return (int)decltype(lpr)::value; }) == 0
               ? (kWideGroups * a->width + a->rows) * 4
               : kBwdBlocks * a->width * 4;
}

extern "C" int fpde_rms_norm_bwd(const fpde_norm_bwd_args* a, void* stream) {
    if (!a) return FPDE_ERR_ARG;
    int st = check_norm(a->dtype, a->weight_dtype, a->rows, a->width, a->eps);
    if (st != FPDE_OK) return st;
    if (!stride_ok(a->dy_stride, a->width) || !stride_ok(a->sum_stride, a->width) ||
        (a->dsum && !stride_ok(a->dsum_stride, a->width)))
        return FPDE_ERR_SHAPE;
    if (a->rows > 0 && (!a->dy || !a->sum || !a->ds)) return FPDE_ERR_ARG;
    const int64_t need = fpde_rms_norm_bwd_workspace(a);
    if (need > 0 && (!a->workspace || a->workspace_bytes < need)) return FPDE_ERR_ARG;
    const int e = size_of(a->dtype), we = size_of(a->weight_dtype);
    Spans sp;
    sp.add(a->dy, span3(1, a->rows, a->width, 0, a->dy_stride, e), e, false);
    sp.add(a->sum, span3(1, a->rows, a->width, 0, a->sum_stride, e), e, false);
    sp.add(a->dsum, span3(1, a->rows, a->width, 0, a->dsum_stride, e), e, false);
    sp.add(a->weight, a->width * we, we, false);
    sp.add(a->ds, a->rows * a->width * e, e, true);
    sp.add(a->dweight, a->width * we, we, true);
    if (need > 0) sp.add(a->workspace, need, 16, true);
    st = sp.check(a->ds, a->ds == a->dy ? a->dy : a->dsum);
    if (st != FPDE_OK) return st;
    hipStream_t s = (hipStream_t)stream;
    NormBwdP P{a->dy, a->sum, a->dsum, a->weight, a->ds, a->dweight ? (float*)a->workspace : nullptr,
               nullptr, a->rows, a->dy_stride, a->sum_stride, a->dsum_stride, (int)a->width,
               a->weight_dtype == FPDE_F32, (float)a->eps, (float)(1.0 / (double)a->width)};
    if (a->rows == 0)
        return a->dweight ? queue_colsum(P.part, 0, a->width, a->width, a->dweight, a->weight_dtype, s)
                          : FPDE_OK;
    return with_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        return with_layout(cdiv(a->width, kVec<T>), [&](auto lpr, auto ch) {
            constexpr int L = decltype(lpr)::value, C = decltype(ch)::value;
            int64_t parts;
            int r;
            if constexpr (L == 0) {
                parts = a->rows < kWideGroups ? a->rows : kWideGroups;
                if (P.part) P.rho = P.part + kWideGroups * a->width;
                const dim3 g((unsigned)(a->rows < kMaxBlocks ? a->rows : kMaxBlocks));
                // where ds takes dy's place the column sums have to read dy before it goes
                const bool first = P.part && a->ds == a->dy;
                r = FPDE_OK;
                if (first) {
                    NormBwdP Q = P;
                    Q.ds = nullptr;
                    r = launch(norm_bwd_wide_kernel<T>, g, dim3(1024), s, Q);
                    P.rho = nullptr;
                    if (r == FPDE_OK) r = queue_dw_wide<T>(Q, parts, s);
                }
                if (r == FPDE_OK) r = launch(norm_bwd_wide_kernel<T>, g, dim3(1024), s, P);
                if (r == FPDE_OK && P.part && !first) r = queue_dw_wide<T>(P, parts, s);
            } else {
                parts = bwd_blocks(a->rows, 256 / L);
                r = launch(norm_bwd_kernel<T, L, C>, dim3((unsigned)parts), dim3(256), s, P);
            }
            if (r != FPDE_OK || !P.part) return r;
            return queue_colsum(P.part, parts, a->width, a->width, a->dweight, a->weight_dtype, s);
        });
    });
}
