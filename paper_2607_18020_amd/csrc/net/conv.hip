// conv.hip -- short causal convolution along time, per channel, and its gradients.
//
//   p_t = b + sum_k w_k x_{t - W + 1 + k},  y = p or silu(p) = p sigmoid(p)
//   dp = dy (silu'(p) = q (1 + p (1 - q)), q = sigmoid(p));  dx_t = sum_k w_k dp_{t + W - 1 - k}
//   dw_k = sum_t dp_t x_{t - W + 1 + k},  db = sum_t dp_t
//
// A lane owns 2 neighbouring channels and marches a chunk of levels, the last W - 1 of
// them in registers, so x is read once but for the W - 1 levels before a chunk; the
// next kBlock levels are on their way while those before them are worked on.  What
// bounds both directions is memory, and how many loads are in flight: 2 channels (a
// wavefront's load of 16-bit data is 256 bytes), since the filters, windows and sums of
// 4 leave the backward two wavefronts a SIMD, of 8 one.  Where the channels are no
// multiple of 2 the last lane's two begin earlier, and what two lanes own they write with
// the same values.  The backward recomputes p from x instead of reading it, and runs
// W - 1 levels past its chunk for the dp that dx needs there.
//
// Measured, 256 x 128 x 512 bf16, 4 taps, with 2, 4 and 8 channels a lane: forward 15.6 us
// (4.3 TB/s), 17.6, -, backward with 5 for the partial sums 30.8, 35.2, 130; 8 x 2048 x
// 1024: 14.6 and 17.2, 28.1 and 33.8.
#include "net_common.hpp"

using namespace fpde_net;

namespace {

constexpr int kBlock = 8;  // levels whose loads are in flight together
constexpr int kLane = 2;   // channels of a lane

struct ConvP {
    const void *x, *dy, *w, *b, *state;
    const int32_t* lengths;
    void *y, *state_out;  // y: dx in the backward
    float* part;          // [slots][channels * taps + channels]
    int64_t batch, chunks, xb, xt, dyb, dyt;
    int length, channels, chunk, wf32, silu;
};

__device__ __forceinline__ int levels(const ConvP& P, int64_t b) {
    if (!P.lengths) return P.length;
    const int n = P.lengths[b];
    return n < 0 ? 0 : (n < P.length ? n : P.length);
}

// x at level t of sequence b, which holds len: its own levels, the carried state before
// them, or zero
template <class T, int W, int V>
__device__ __forceinline__ void x_at(const ConvP& P, int64_t b, int t, int len, int c, float (&v)[V]) {
    if (t >= 0 && t < len)
        load_f32<T, V>(v, (const T*)P.x + b * P.xb + (int64_t)t * P.xt + c, V);
    else if (t < 0 && P.state)
        load_f32<T, V>(v, (const T*)P.state + (b * (W - 1) + (W - 1 + t)) * P.channels + c, V);
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.f;
    }
}

// the filters of V channels: w[k][i], and the bias
template <class T, int W, int V>
__device__ __forceinline__ void load_filters(const ConvP& P, int c, float (&w)[W][V], float (&b)[V]) {
    float q[W * V];
    load_param<T, W * V>(q, P.w, P.wf32, (int64_t)c * W, W * V);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int k = 0; k < W; ++k) w[k][i] = q[i * W + k];
        b[i] = 0.f;
    }
    if (P.b) load_param<T, V>(b, P.b, P.wf32, c, V);
}

// The first of a lane's V channels, or -1 past the last.
template <int V>
__device__ __forceinline__ int lane_channel(const ConvP& P) {
    const int c = ((int)blockIdx.x * 64 + (int)threadIdx.x) * V;
    return c >= P.channels ? -1 : (c < P.channels - V ? c : P.channels - V);
}

// kBlock levels from t on (clamped to the sequence's last, which exists)
template <class T, int V>
__device__ __forceinline__ void load_block(Raw<T, V> (&q)[kBlock], const void* x, int64_t b, int64_t bs, int64_t ts,
                                           int t, int len, int c) {
#pragma unroll
    for (int j = 0; j < kBlock; ++j) {
        const int s = t + j < len ? t + j : len - 1;
        q[j] = load_raw<T, V>((const T*)x + b * bs + (int64_t)s * ts + c);
    }
}

template <class T, int W, int V>
__global__ __launch_bounds__(64) void conv_fwd_kernel(ConvP P) {
    const int c = lane_channel<V>(P);
    if (c < 0) return;
    float w[W][V], bias[V];
    load_filters<T, W, V>(P, c, w, bias);
    for (int64_t job = blockIdx.y; job < P.batch * P.chunks; job += gridDim.y) {
        const int64_t b = job / P.chunks;
        const int t0 = (int)(job - b * P.chunks) * P.chunk, len = levels(P, b);
        const int t1 = t0 + P.chunk < P.length ? t0 + P.chunk : P.length, te = t1 < len ? t1 : len;
        Raw<T, V> x[kBlock], nx[kBlock];
        if (t0 < te) load_block<T, V>(x, P.x, b, P.xb, P.xt, t0, len, c);
        float win[W][V];  // win[k]: x at t - W + 1 + k
#pragma unroll
        for (int k = 0; k < W - 1; ++k) x_at<T, W, V>(P, b, t0 - (W - 1) + k, len, c, win[k + 1]);
        if (t0 == 0 && P.state_out) {
            // The lane that reads the state is the one that replaces it, after its reads.
            float last[W - 1][V];
#pragma unroll
            for (int i = 0; i < W - 1; ++i) x_at<T, W, V>(P, b, len - (W - 1) + i, len, c, last[i]);
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                store_f32<T, V>((T*)P.state_out + (b * (W - 1) + i) * P.channels + c, last[i], V);
        }
        T* y = (T*)P.y + (b * P.length) * P.channels + c;
        for (int t = t0; t < te; t += kBlock) {
            if (t + kBlock < te) load_block<T, V>(nx, P.x, b, P.xb, P.xt, t + kBlock, len, c);
#pragma unroll
            for (int j = 0; j < kBlock; ++j) {
                if (t + j >= te) break;
                float p[V], v[V];
                unpack<T, V>(v, x[j]);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    p[i] = bias[i];
#pragma unroll
                    for (int k = 0; k < W - 1; ++k) {
                        win[k][i] = win[k + 1][i];
                        p[i] = fmaf(w[k][i], win[k][i], p[i]);
                    }
                    win[W - 1][i] = v[i];
                    p[i] = fmaf(w[W - 1][i], v[i], p[i]);
                    if (P.silu) p[i] = silu(p[i]);
                }
                store_f32<T, V>(y + (int64_t)(t + j) * P.channels, p, V);
            }
#pragma unroll
            for (int j = 0; j < kBlock; ++j) x[j] = nx[j];
        }
        const float zero[V] = {};
        for (int t = te > t0 ? te : t0; t < t1; ++t) store_f32<T, V>(y + (int64_t)t * P.channels, zero, V);
    }
}

template <class T, int W, int V>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(3))) void conv_bwd_kernel(ConvP P) {
    const int c = lane_channel<V>(P);
    if (c < 0) return;
    float w[W][V], bias[V], dw[W][V], db[V];
    load_filters<T, W, V>(P, c, w, bias);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        db[i] = 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) dw[k][i] = 0.f;
    }
    for (int64_t job = blockIdx.y; job < P.batch * P.chunks; job += gridDim.y) {
        const int64_t b = job / P.chunks;
        const int t0 = (int)(job - b * P.chunks) * P.chunk, len = levels(P, b);
        const int t1 = t0 + P.chunk < P.length ? t0 + P.chunk : P.length;
        // dx at level t - W + 1 is complete with dp at t: W - 1 levels more than the chunk has
        const int tn = t1 + W - 1;
        Raw<T, V> x[kBlock], g[kBlock], nx[kBlock], ng[kBlock];
        if (t0 < len) {
            load_block<T, V>(x, P.x, b, P.xb, P.xt, t0, len, c);
            load_block<T, V>(g, P.dy, b, P.dyb, P.dyt, t0, len, c);
        }
        float win[W][V];  // win[k]: x at t - W + 1 + k
        float dps[W][V];  // dps[k]: dp at t - W + 1 + k
#pragma unroll
        for (int k = 0; k < W - 1; ++k) {
            x_at<T, W, V>(P, b, t0 - (W - 1) + k, len, c, win[k + 1]);
#pragma unroll
            for (int i = 0; i < V; ++i) dps[k + 1][i] = 0.f;
        }
        T* dx = (T*)P.y + (b * P.length) * P.channels + c;
        for (int t = t0; t < tn; t += kBlock) {
            if (t + kBlock < tn && t + kBlock < len) {
                load_block<T, V>(nx, P.x, b, P.xb, P.xt, t + kBlock, len, c);
                load_block<T, V>(ng, P.dy, b, P.dyb, P.dyt, t + kBlock, len, c);
            }
            // WHOLE: a level of the chunk that exists.  A block of them runs without a branch but that of the
            // chunk's first stores, so the windows' shifts are names of registers and no moves.
            auto level = [&](auto whole, int j) {
                constexpr bool WHOLE = decltype(whole)::value;
                float d[V], o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] = 0.f;
                if (WHOLE || t + j < len) {
                    float v[V];
                    unpack<T, V>(v, x[j]);
                    unpack<T, V>(d, g[j]);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float p = bias[i];
#pragma unroll
                        for (int k = 0; k < W - 1; ++k) {
                            win[k][i] = win[k + 1][i];
                            p = fmaf(w[k][i], win[k][i], p);
                        }
                        win[W - 1][i] = v[i];
                        p = fmaf(w[W - 1][i], v[i], p);
                        if (P.silu) {
                            const float q = sigmoid(p);
                            d[i] *= q * fmaf(p, 1.f - q, 1.f);
                        }
                        // (the levels past the chunk count in the next one's dw)
                        if (WHOLE || t + j < t1) {
                            db[i] += d[i];
#pragma unroll
                            for (int k = 0; k < W; ++k) dw[k][i] = fmaf(d[i], win[k][i], dw[k][i]);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    o[i] = 0.f;
#pragma unroll
                    for (int k = 0; k < W - 1; ++k) dps[k][i] = dps[k + 1][i];
                    dps[W - 1][i] = d[i];
                    // dx_s = sum_k w_k dp_{s + W - 1 - k}, s = t - W + 1
#pragma unroll
                    for (int k = 0; k < W; ++k) o[i] = fmaf(w[k][i], dps[W - 1 - k][i], o[i]);
                }
                const int s = t + j - (W - 1);
                if ((WHOLE && j >= W - 1) || s >= t0) {
                    if (!WHOLE && s >= len) {
#pragma unroll
                        for (int i = 0; i < V; ++i) o[i] = 0.f;
                    }
                    store_f32<T, V>(dx + (int64_t)s * P.channels, o, V);
                }
            };
            if (t + kBlock <= t1 && t + kBlock <= len) {
#pragma unroll
                for (int j = 0; j < kBlock; ++j) level(std::true_type{}, j);
            } else {
#pragma unroll
                for (int j = 0; j < kBlock; ++j) {
                    if (t + j >= tn) break;
                    level(std::false_type{}, j);
                }
            }
#pragma unroll
            for (int j = 0; j < kBlock; ++j) x[j] = nx[j], g[j] = ng[j];
        }
    }
    // a partial row: every channel's taps, then the biases
    float* pw = P.part + (int64_t)blockIdx.y * P.channels * (W + 1);
    float q[W * V];
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) q[i * W + k] = dw[k][i];
    store_f32<float, W * V>(pw + (int64_t)c * W, q, W * V);
    store_f32<float, V>(pw + (int64_t)P.channels * W + c, db, V);
}

// ---------------------------------------------------------------------------
// Host side.

constexpr int64_t kMaxChannels = 1 << 20, kMaxLevels = (int64_t)1 << 34;
// Wavefronts of a launch before they loop over chunks.  The backward's partial
// sums grow with them (half and twice as many within 2% of these at 256 x 128 x 512).
constexpr int64_t kFwdWaves = 1 << 21, kBwdWaves = 8192;

// Levels of a chunk: 32, where the W - 1 levels read twice cost little, or 16 or 8 where
// there would be fewer than one wavefront a SIMD.  Backward: 1 x 1024 x 512 19 us with 8 and 23 with 32;
// 8 x 2048 x 1024 28 with 32, 34 with 16, 30 with 64.
int chunk_of(int64_t batch, int64_t length, int64_t channels) {
    int c = 32;
    while (c > 8 && batch * cdiv(length, c) * cdiv(channels, 64 * kLane) < 1024) c /= 2;
    return c;
}

int check_conv(int dtype, int wdtype, int taps, int act, int64_t batch, int64_t length, int64_t channels) {
    if (size_of(dtype) == 0 || !(wdtype == FPDE_F32 || wdtype == dtype)) return FPDE_ERR_UNSUPPORTED;
    if (act != 0 && act != 1) return FPDE_ERR_ARG;
    if (taps < 2 || taps > 4) return FPDE_ERR_UNSUPPORTED;
    if (batch < 0 || length < 0 || length >= ((int64_t)1 << 31) - 256 || channels < 1 ||
        channels > kMaxChannels)
        return FPDE_ERR_SHAPE;
    if (length > 0 && batch > kMaxLevels / length) return FPDE_ERR_SHAPE;
    if (batch > kMaxLevels) return FPDE_ERR_SHAPE;
    return FPDE_OK;
}

bool strides_ok(int64_t bs, int64_t ts, int64_t batch, int64_t length, int64_t channels) {
    const int64_t most = (int64_t)1 << 50;
    if (length > 1 && (ts < channels || ts > most / length)) return false;
    return batch <= 1 || (bs >= 0 && bs <= most / batch);
}

int64_t slots(int64_t jobs, int64_t channels, int64_t waves) {
    const int64_t n = waves / cdiv(channels, 64 * kLane);
    const int64_t m = n < 1 ? 1 : (n > 65535 ? 65535 : n);
    return jobs < m ? (jobs < 1 ? 1 : jobs) : m;
}

// f(T{}, integral_constant<int, taps>, integral_constant<int, channels a lane>): 2, or 1 where there
// is one, or where lanes that share channels would read a state that the other replaces
template <class F>
int with_taps(int dtype, int taps, bool one, F f) {
    return with_type(dtype, [&](auto t) {
        auto v = [&](auto w) {
            return one ? f(t, w, std::integral_constant<int, 1>{}) : f(t, w, std::integral_constant<int, kLane>{});
        };
        switch (taps) {
        case 2: return v(std::integral_constant<int, 2>{});
        case 3: return v(std::integral_constant<int, 3>{});
        default: return v(std::integral_constant<int, 4>{});
        }
    });
}

}  // namespace

extern "C" int fpde_causal_conv(const fpde_conv_args* a, void* stream) {
    if (!a) return FPDE_ERR_ARG;
    int st = check_conv(a->dtype, a->weight_dtype, a->taps, a->silu, a->batch, a->length, a->channels);
    if (st != FPDE_OK) return st;
    if (!strides_ok(a->x_batch_stride, a->x_time_stride, a->batch, a->length, a->channels))
        return FPDE_ERR_SHAPE;
    if (a->batch == 0 || (a->length == 0 && !a->state_out)) return FPDE_OK;
    if (!a->weight || (a->length > 0 && (!a->x || !a->y))) return FPDE_ERR_ARG;
    const int e = size_of(a->dtype), we = size_of(a->weight_dtype);
    const int64_t hist = a->batch * (a->taps - 1) * a->channels * e;
    Spans sp;
    sp.add(a->x, span3(a->batch, a->length, a->channels, a->x_batch_stride, a->x_time_stride, e), e, false);
    sp.add(a->weight, a->channels * a->taps * we, we, false);
    sp.add(a->bias, a->channels * we, we, false);
    sp.add(a->lengths, a->batch * 4, 4, false);
    sp.add(a->state, hist, e, false);
    sp.add(a->y, a->batch * a->length * a->channels * e, e, true);
    sp.add(a->state_out, hist, e, true);
    st = sp.check(a->state_out, a->state);
    if (st != FPDE_OK) return st;
    ConvP P{};
    P.x = a->x, P.w = a->weight, P.b = a->bias, P.state = a->state, P.lengths = a->lengths;
    P.y = a->y, P.state_out = a->state_out;
    P.batch = a->batch, P.xb = a->x_batch_stride, P.xt = a->x_time_stride;
    P.length = (int)a->length, P.channels = (int)a->channels;
    P.wf32 = a->weight_dtype == FPDE_F32, P.silu = a->silu;
    P.chunk = chunk_of(a->batch, a->length, a->channels);
    P.chunks = a->length > 0 ? cdiv(a->length, P.chunk) : 1;
    const bool one = a->channels < kLane || (a->channels % kLane && a->state && a->state == a->state_out);
    return with_taps(a->dtype, a->taps, one, [&](auto t, auto w, auto v) {
        constexpr int V = decltype(v)::value;
        const dim3 g((unsigned)cdiv(a->channels, 64 * V),
                     (unsigned)slots(a->batch * P.chunks, a->channels, kFwdWaves));
        return launch(conv_fwd_kernel<decltype(t), decltype(w)::value, V>, g, dim3(64), (hipStream_t)stream, P);
    });
}

extern "C" int64_t fpde_causal_conv_bwd_workspace(const fpde_conv_bwd_args* a) {
    if (!a) return FPDE_ERR_ARG;
    const int st = check_conv(a->dtype, a->weight_dtype, a->taps, a->silu, a->batch, a->length, a->channels);
    if (st != FPDE_OK) return st;
    const int64_t jobs = a->batch * cdiv(a->length, chunk_of(a->batch, a->length, a->channels));
    return slots(jobs, a->channels, kBwdWaves) * a->channels * (a->taps + 1) * 4;
}

extern "C" int fpde_causal_conv_bwd(const fpde_conv_bwd_args* a, void* stream) {
    if (!a) return FPDE_ERR_ARG;
    int st = check_conv(a->dtype, a->weight_dtype, a->taps, a->silu, a->batch, a->length, a->channels);
    if (st != FPDE_OK) return st;
    if (!strides_ok(a->x_batch_stride, a->x_time_stride, a->batch, a->length, a->channels) ||
        !strides_ok(a->dy_batch_stride, a->dy_time_stride, a->batch, a->length, a->channels))
        return FPDE_ERR_SHAPE;
    const int64_t total = a->batch * a->length;
    if (!a->weight || !a->dweight || (total > 0 && (!a->x || !a->dy || !a->dx))) return FPDE_ERR_ARG;
    const int64_t need = fpde_causal_conv_bwd_workspace(a);
    if (!a->workspace || a->workspace_bytes < need) return FPDE_ERR_ARG;
    const int e = size_of(a->dtype), we = size_of(a->weight_dtype);
    Spans sp;
    sp.add(a->x, span3(a->batch, a->length, a->channels, a->x_batch_stride, a->x_time_stride, e), e, false);
    sp.add(a->dy, span3(a->batch, a->length, a->channels, a->dy_batch_stride, a->dy_time_stride, e), e, false);
    sp.add(a->weight, a->channels * a->taps * we, we, false);
    sp.add(a->bias, a->channels * we, we, false);
    sp.add(a->lengths, a->batch * 4, 4, false);
    sp.add(a->state, a->batch * (a->taps - 1) * a->channels * e, e, false);
    sp.add(a->dx, total * a->channels * e, e, true);
    sp.add(a->dweight, a->channels * a->taps * we, we, true);
    sp.add(a->dbias, a->channels * we, we, true);
    sp.add(a->workspace, need, 16, true);
    st = sp.check();
    if (st != FPDE_OK) return st;
    ConvP P{};
    P.x = a->x, P.dy = a->dy, P.w = a->weight, P.b = a->bias, P.state = a->state, P.lengths = a->lengths;
    P.y = a->dx;
    P.batch = a->batch, P.xb = a->x_batch_stride, P.xt = a->x_time_stride;
    P.dyb = a->dy_batch_stride, P.dyt = a->dy_time_stride;
    P.length = (int)a->length, P.channels = (int)a->channels;
    P.wf32 = a->weight_dtype == FPDE_F32, P.silu = a->silu;
    P.chunk = chunk_of(a->batch, a->length, a->channels);
    P.chunks = cdiv(a->length, P.chunk);
    const int64_t jobs = a->batch * P.chunks, n = slots(jobs, a->channels, kBwdWaves);
    P.part = (float*)a->workspace;
    hipStream_t s = (hipStream_t)stream;
    if (jobs > 0) {
        st = with_taps(a->dtype, a->taps, a->channels < kLane, [&](auto t, auto w, auto v) {
            constexpr int V = decltype(v)::value;
            return launch(conv_bwd_kernel<decltype(t), decltype(w)::value, V>,
                          dim3((unsigned)cdiv(a->channels, 64 * V), (unsigned)n), dim3(64), s, P);
        });
        if (st != FPDE_OK) return st;
    }
    return queue_colsum(P.part, jobs > 0 ? n : 0, a->channels * (a->taps + 1), a->dweight, a->channels * a->taps,
                        a->dbias, a->dbias ? a->channels : 0, a->weight_dtype, s);
}
