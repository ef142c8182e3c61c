// scan.hip -- selective state space scan along time, its single-level step and
// its gradients.
//
//   dt_t = softplus(delta_t + bias),  a_t = exp(dt_t A),  h_t = a_t h_{t-1} + dt_t u_t B_t
//   y_t = sum_n C_t h_t + D u_t,  out_t = y_t silu(z_t)
//
// A lane owns one channel and keeps its NS states in registers; neighbouring lanes
// own neighbouring channels, so every access to u, delta, z and out is dense, and B
// and C, the same for all channels of a group, are staged through LDS in float32
// and read by broadcast.  Per level, channel and state: one product and one exp2
// for a, then one product and two multiply-adds; the exponential counts as four of
// those, so 16 states cost about 130 VALU slots and the operator is bound by the
// VALU, not by its 4 reads and writes an element.
//
// Few sequences and channels leave the card empty, since time is serial: the window
// is then split in chunks.  A first pass finds what each chunk adds to the state
// from zero and the sum of its dt; as the product of a chunk's a_t is exp(A sum dt),
// a short scan over the chunks (chunk_kernel) gives the state each starts from, and
// the main pass runs all chunks at once.  This costs the exponentials twice, so it is
// done only where whole windows are fewer wavefronts than the card has SIMDs.
//
// Backward: with dy_t = dout_t silu(z_t) and g_t = dL/dh_t,
//   g_t = C_t dy_t + a_{t+1} g_{t+1};  dC_t = sum_c h_t dy_t;  dB_t = sum_c g_t dt_t u_t
//   du_t = D dy_t + dt_t sum_n g_t B_t
//   ddt_t = sum_n g_t (A a_t h_{t-1} + B_t u_t);  dA = sum_t dt_t g_t a_t h_{t-1}
// One pass forward leaves the state at the start of every block of KB levels; the
// main pass walks the blocks backward, runs each block forward again from its state
// with all a_t h_{t-1} of the block in registers, and then backward.  The window is
// split in chunks as above, with the same scan over chunks for g.  The sums over
// channels (dB, dC) halve the values and the lanes together (reduce_lanes): one
// swap or DPP and one addition for each value that goes; the wavefronts' sums meet
// in LDS and the workgroups' in partial rows that a last launch adds in order.
#include "net_common.hpp"

using namespace fpde_net;

namespace {

constexpr int kTile = 16;        // levels of B and C staged together
constexpr int kSub = 8;          // levels whose loads are in flight together
constexpr float kLn2 = 0.69314718055994530942f;

struct Seq {  // a [batch][length][...] array
    const void* p;
    int64_t bs, ts;
};

struct ScanP {
    Seq u, delta, z, B, C, dy;
    const float *A, *D, *bias, *state;
    const int32_t* lengths;
    void *y, *ddelta, *dz;                // y: du in the backward
    float* state_out;
    float *hend, *gend, *sdt;             // [batch][chunks][states][channels], [batch][chunks][channels]
    float* ck;                            // [batch][blocks][states][channels]
    float *pbc, *pA, *pD, *pbias;         // partial sums
    int64_t batch;
    int length, channels, states, groups, softplus;
    int chunk, chunks, per, nblk, slots;  // per: channels a group; nblk: workgroups a group
};

__device__ __forceinline__ int lane_levels(const int32_t* lengths, int64_t b, int length) {
    if (!lengths) return length;
    const int n = lengths[b];
    return n < 0 ? 0 : (n < length ? n : length);
}
// (for a b that is the wavefront's)
__device__ __forceinline__ int levels(const int32_t* lengths, int64_t b, int length) {
    return __builtin_amdgcn_readfirstlane(lane_levels(lengths, b, length));
}

// log(1 + exp(x)) = max(x, 0) + log1p(e), e = exp(-|x|) in (0, 1].  The product with
// log2(e) is carried to twice the precision, so that small results keep their digits;
// log1p(e) = 2 artanh(e / (2 + e)), whose series in s^2 <= 1/9 is cut below 2^-26.
__device__ __forceinline__ float softplus(float x) {
    const float ax = -fabsf(x), hi = ax * kLog2e;
    const float lo = fmaf(ax, kLog2e, -hi) + ax * 1.92596299e-8f;  // log2(e) - float(log2(e))
    float e = __builtin_amdgcn_exp2f(hi);
    e = fmaf(e, lo * kLn2, e);
    const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
    float r = 1.f / 15;
    r = fmaf(r, q, 1.f / 13);
    r = fmaf(r, q, 1.f / 11);
    r = fmaf(r, q, 1.f / 9);
    r = fmaf(r, q, 1.f / 7);
    r = fmaf(r, q, 1.f / 5);
    r = fmaf(r, q, 1.f / 3);
    r = fmaf(r, q, 1.f);
    const float v = fmaf(2.f * s, r, fmaxf(x, 0.f));
    return x != x ? x : (ax < -3.0e38f ? fmaxf(x, 0.f) : v);  // (infinite x: no 0 * inf above)
}

// ---------------------------------------------------------------------------
// A workgroup's place: its channels within one group, and one lane's channel.

struct Place {
    int g, c;
    bool live;
};
template <int TPB>
__device__ __forceinline__ Place place(const ScanP& P, int blk) {
    Place q;
    q.g = blk / P.nblk;
    const int l = (blk - q.g * P.nblk) * TPB + (int)threadIdx.x;
    q.live = l < P.per;
    q.c = q.g * P.per + (q.live ? l : P.per - 1);  // (idle lanes repeat the last channel and store nothing)
    return q;
}

// B and C of levels t .. t + TL - 1 (those before t1; zeros after) into bc[TL][2 NS]
template <class T, int NS, int TPB, int TL, bool WITH_C>
__device__ __forceinline__ void stage_bc(const ScanP& P, int64_t b, int g, int t, int t1, float* bc) {
    constexpr int E = TL * NS;
#pragma unroll
    for (int h = 0; h < (WITH_C ? 2 : 1); ++h) {
        const Seq& s = h ? P.C : P.B;
        const T* p = (const T*)s.p + b * s.bs + (int64_t)g * P.states;
#pragma unroll
        for (int e0 = 0; e0 < E; e0 += TPB) {
            const int e = e0 + (int)threadIdx.x, j = e / NS, n = e % NS;
            if (E % TPB == 0 || e < E) {
                const bool in = n < P.states && t + j < t1;
                bc[j * 2 * NS + h * NS + n] = in ? to_f32<T>(p[(int64_t)(t + j) * s.ts + n]) : 0.f;
            }
        }
    }
}

// (the row's address is the workgroup's, so only the channel takes a lane's register)
template <class T>
__device__ __forceinline__ T at(const Seq& s, int64_t b, int t, int c) {
    return ((const T*)s.p + b * s.bs + (int64_t)t * s.ts)[(unsigned)c];
}
template <class T>
__device__ __forceinline__ void put(void* p, int64_t row, int channels, int c, float v) {
    ((T*)p + row * channels)[(unsigned)c] = from_f32<T>(v);
}

// A * log2(e) of one channel (0 past the states that exist)
template <int NS>
__device__ __forceinline__ void load_a2(const ScanP& P, int c, float (&a2)[NS]) {
#pragma unroll
    for (int n = 0; n < NS; ++n) a2[n] = n < P.states ? P.A[(int64_t)c * P.states + n] * kLog2e : 0.f;
}

// ---------------------------------------------------------------------------
// Forward.  OUT: the outputs.  ENDS: a chunk's own contribution to the state, from zero,
// and its sum of dt.  CHECKS: the state at the start of every block of KB levels.
enum { OUT, ENDS, CHECKS };

template <class T, int NS, int TPB, int MODE, int KB>
__global__ __launch_bounds__(TPB) void scan_fwd_kernel(ScanP P) {
    __shared__ __attribute__((aligned(16))) float bc[kTile * 2 * NS];
    const int64_t job = (int64_t)(blockIdx.x / (P.nblk * P.groups));
    const Place q = place<TPB>(P, (int)(blockIdx.x % (P.nblk * P.groups)));
    const int64_t b = job / P.chunks;
    const int ch = (int)(job - b * P.chunks), c = q.c;
    const int len = levels(P.lengths, b, P.length);
    const int t0 = ch * P.chunk, tn = t0 + P.chunk < P.length ? t0 + P.chunk : P.length;
    const int t1 = tn < len ? tn : len;
    float a2[NS], h[NS];
    load_a2<NS>(P, c, a2);
    const float bias = P.bias ? P.bias[c] : 0.f, dd = MODE == OUT && P.D ? P.D[c] : 0.f;
    if (MODE != ENDS && P.chunks > 1) {
        const float* s = P.hend + job * P.states * P.channels + c;
#pragma unroll
        for (int n = 0; n < NS; ++n) h[n] = n < P.states ? s[(int64_t)n * P.channels] : 0.f;
    } else {
        const float* s = MODE != ENDS && P.state ? P.state + (b * P.channels + c) * P.states : nullptr;
#pragma unroll
        for (int n = 0; n < NS; ++n) h[n] = s && n < P.states ? s[n] : 0.f;
    }
    float sum = 0.f;
    const int64_t row = b * P.length;
    for (int tt = t0; tt < t1; tt += kTile) {
        __syncthreads();
        stage_bc<T, NS, TPB, kTile, MODE == OUT>(P, b, q.g, tt, t1, bc);
        __syncthreads();
#pragma unroll 1
        for (int t = tt; t < tt + kTile && t < t1; t += kSub) {
            T ru[kSub], rd[kSub], rz[kSub];
#pragma unroll
            for (int j = 0; j < kSub; ++j) {
                const int s = t + j < t1 ? t + j : t1 - 1;
                ru[j] = at<T>(P.u, b, s, c);
                rd[j] = at<T>(P.delta, b, s, c);
                if (MODE == OUT && P.z.p) rz[j] = at<T>(P.z, b, s, c);
            }
#pragma unroll
            for (int j = 0; j < kSub; ++j) {
                if (t + j >= t1) break;
                if (MODE == CHECKS && (t + j - t0) % KB == 0 && q.live) {
                    const int64_t blocks = (P.length + KB - 1) / KB;
                    float* s = P.ck + (b * blocks + (t + j) / KB) * P.states * P.channels;
#pragma unroll
                    for (int n = 0; n < NS; ++n)
                        if (n < P.states) (s + (int64_t)n * P.channels)[(unsigned)c] = h[n];
                }
                const float* w = bc + (t - tt + j) * 2 * NS;
                const float u = to_f32<T>(ru[j]), raw = to_f32<T>(rd[j]) + bias;
                const float dt = P.softplus ? softplus(raw) : raw, du = dt * u;
                float acc = 0.f;
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    const float a = __builtin_amdgcn_exp2f(dt * a2[n]);
                    h[n] = fmaf(a, h[n], du * w[n]);
                    if (MODE == OUT) acc = fmaf(h[n], w[NS + n], acc);
                }
                if (MODE == ENDS) sum += dt;
                if (MODE == OUT) {
                    acc = fmaf(dd, u, acc);
                    if (P.z.p) acc *= silu(to_f32<T>(rz[j]));
                    if (q.live) put<T>(P.y, row + t + j, P.channels, c, acc);
                }
            }
        }
    }
    if (!q.live) return;
    if (MODE == OUT) {
        for (int t = t1 > t0 ? t1 : t0; t < tn; ++t) put<T>(P.y, row + t, P.channels, c, 0.f);
        if (P.state_out && ch == P.chunks - 1) {
            float* s = P.state_out + (b * P.channels + c) * P.states;
#pragma unroll
            for (int n = 0; n < NS; ++n)
                if (n < P.states) s[n] = h[n];
        }
    }
    if (MODE == ENDS) {
        float* s = P.hend + job * P.states * P.channels + c;
#pragma unroll
        for (int n = 0; n < NS; ++n)
            if (n < P.states) s[(int64_t)n * P.channels] = h[n];
        P.sdt[job * P.channels + c] = sum;
    }
}

// The state that every chunk starts from (e: what the chunks add, replaced by what they
// start from), forward in time, or backward for the adjoint.  One lane a state.
__global__ __launch_bounds__(256) void chunk_kernel(ScanP P, float* e, int backward) {
    const int c = (int)(blockIdx.x * 256 + threadIdx.x), n = (int)blockIdx.y;
    if (c >= P.channels) return;
    const float a2 = P.A[(int64_t)c * P.states + n] * kLog2e;
    for (int64_t b = blockIdx.z; b < P.batch; b += gridDim.z) {
        float h = !backward && P.state ? P.state[(b * P.channels + c) * P.states + n] : 0.f;
#pragma unroll 4
        for (int i = 0; i < P.chunks; ++i) {
            const int64_t job = b * P.chunks + (backward ? P.chunks - 1 - i : i);
            float* s = e + (job * P.states + n) * P.channels + c;
            const float add = *s, sum = P.sdt[job * P.channels + c];
            *s = h;
            h = fmaf(sum == 0.f ? 1.f : __builtin_amdgcn_exp2f(sum * a2), h, add);
        }
    }
}

// ---------------------------------------------------------------------------
// One level from a carried state: NS / 4 neighbouring lanes own a channel, four
// states each, so that the states' reads and writes, all but the whole of the
// traffic, are dense.
template <class T, int NS>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanP P) {
    constexpr int LPC = NS / 4;
    const int i = (int)(blockIdx.x * 256 + threadIdx.x), c = i / LPC, n0 = i % LPC * 4;
    const bool live = c < P.channels;
    const int cc = live ? c : P.channels - 1, k = P.states - n0;  // (a channel's lanes stay together)
    float a[4] = {0.f, 0.f, 0.f, 0.f};
    if (k > 0) load_f32<float, 4>(a, P.A + (int64_t)cc * P.states + n0, k);
    const float bias = P.bias ? P.bias[cc] : 0.f, dd = P.D ? P.D[cc] : 0.f;
    const int g = cc / P.per;
    for (int64_t b = blockIdx.y; b < P.batch; b += gridDim.y) {
        const bool on = levels(P.lengths, b, 1) > 0;
        float h[4] = {0.f, 0.f, 0.f, 0.f}, B[4] = {0.f, 0.f, 0.f, 0.f}, C[4] = {0.f, 0.f, 0.f, 0.f};
        const int64_t at_h = (b * P.channels + cc) * P.states + n0;
        float y = 0.f;
        if (k > 0 && P.state) load_f32<float, 4>(h, P.state + at_h, k);
        if (on) {
            if (k > 0) {
                load_f32<T, 4>(B, (const T*)P.B.p + b * P.B.bs + (int64_t)g * P.states + n0, k);
                load_f32<T, 4>(C, (const T*)P.C.p + b * P.C.bs + (int64_t)g * P.states + n0, k);
            }
            const float u = to_f32<T>(at<T>(P.u, b, 0, cc)), raw = to_f32<T>(at<T>(P.delta, b, 0, cc)) + bias;
            const float dt = P.softplus ? softplus(raw) : raw, du = dt * u;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                h[n] = fmaf(__builtin_amdgcn_exp2f(dt * (a[n] * kLog2e)), h[n], du * B[n]);
                y = fmaf(h[n], C[n], y);
            }
            y = fmaf(dd, u, lanes_reduce<LPC, AddOp>(y));
            if (P.z.p) y *= silu(to_f32<T>(at<T>(P.z, b, 0, cc)));
        }
        if (live && n0 == 0) ((T*)P.y)[b * P.channels + c] = from_f32<T>(y);
        if (live && k > 0 && P.state_out) store_f32<float, 4>(P.state_out + at_h, h, k);
    }
}

// ---------------------------------------------------------------------------
// Backward.

// What a chunk adds to the adjoint state that leaves it at its start: g through it
// from zero at its end.
template <class T, int NS, int TPB>
__global__ __launch_bounds__(TPB) void scan_adj_kernel(ScanP P) {
    __shared__ __attribute__((aligned(16))) float bc[kTile * 2 * NS];
    const int64_t job = (int64_t)(blockIdx.x / (P.nblk * P.groups));
    const Place q = place<TPB>(P, (int)(blockIdx.x % (P.nblk * P.groups)));
    const int64_t b = job / P.chunks;
    const int ch = (int)(job - b * P.chunks), c = q.c;
    const int len = levels(P.lengths, b, P.length);
    const int t0 = ch * P.chunk, tn = t0 + P.chunk < P.length ? t0 + P.chunk : P.length;
    const int t1 = tn < len ? tn : len;
    float a2[NS], g[NS];
    load_a2<NS>(P, c, a2);
    const float bias = P.bias ? P.bias[c] : 0.f;
#pragma unroll
    for (int n = 0; n < NS; ++n) g[n] = 0.f;
    for (int tt = t0 + (t1 - t0 - 1) / kTile * kTile; t1 > t0 && tt >= t0; tt -= kTile) {
        __syncthreads();
        stage_bc<T, NS, TPB, kTile, true>(P, b, q.g, tt, t1, bc);
        __syncthreads();
#pragma unroll 1
        for (int t = tt + kTile - kSub; t >= tt; t -= kSub) {
            if (t >= t1) continue;
            T ry[kSub], rd[kSub], rz[kSub];
#pragma unroll
            for (int j = 0; j < kSub; ++j) {
                const int s = t + j < t1 ? t + j : t1 - 1;
                ry[j] = at<T>(P.dy, b, s, c);
                rd[j] = at<T>(P.delta, b, s, c);
                if (P.z.p) rz[j] = at<T>(P.z, b, s, c);
            }
#pragma unroll
            for (int j = kSub - 1; j >= 0; --j) {
                if (t + j >= t1) continue;
                const float* w = bc + (t - tt + j) * 2 * NS + NS;
                const float raw = to_f32<T>(rd[j]) + bias, dt = P.softplus ? softplus(raw) : raw;
                float dy = to_f32<T>(ry[j]);
                if (P.z.p) dy *= silu(to_f32<T>(rz[j]));
#pragma unroll
                for (int n = 0; n < NS; ++n)
                    g[n] = __builtin_amdgcn_exp2f(dt * a2[n]) * fmaf(w[n], dy, g[n]);
            }
        }
    }
    if (!q.live) return;
    float* s = P.gend + job * P.states * P.channels + c;
#pragma unroll
    for (int n = 0; n < NS; ++n)
        if (n < P.states) s[(int64_t)n * P.channels] = g[n];
}

// Sums of NV values over the 64 lanes, NV a power of two up to 64: lane l ends with the
// sum of value l / (64 / NV).  A step takes the values in pairs and keeps one of each on
// the lanes with a bit clear and the other on those with it set, with the partner's
// share added, so values and lanes halve together.
__device__ __forceinline__ float pair_sum32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a),
                                                    __builtin_bit_cast(unsigned, b), false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float pair_sum16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a),
                                                    __builtin_bit_cast(unsigned, b), false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
template <int CTRL>
__device__ __forceinline__ float pair_sum(float a, float b, bool upper) {
    return (upper ? b : a) + dpp<CTRL>(upper ? a : b);
}
template <int CTRL>  // (row_half_mirror: the partner lane holds the other of its own pair)
__device__ __forceinline__ float pair_sum_mirror(float a, float b, bool upper) {
    const float x = a + dpp<CTRL>(a), y = b + dpp<CTRL>(b);
    return upper ? y : x;
}

template <int NV>
__device__ __forceinline__ float reduce_lanes(float (&v)[NV]) {
    const int lane = (int)(threadIdx.x & 63);
    constexpr int N1 = NV > 1 ? NV / 2 : 1;
#pragma unroll
    for (int i = 0; i < N1; ++i) v[i] = pair_sum32(v[i], v[NV > 1 ? i + N1 : i]);
    constexpr int N2 = N1 > 1 ? N1 / 2 : 1;
#pragma unroll
    for (int i = 0; i < N2; ++i) v[i] = pair_sum16(v[i], v[N1 > 1 ? i + N2 : i]);
    constexpr int N3 = N2 > 1 ? N2 / 2 : 1;
#pragma unroll
    for (int i = 0; i < N3; ++i)
        v[i] = N2 > 1 ? pair_sum<0x128>(v[i], v[N2 > 1 ? i + N3 : i], lane & 8) : v[i] + dpp<0x128>(v[i]);
    constexpr int N4 = N3 > 1 ? N3 / 2 : 1;
#pragma unroll
    for (int i = 0; i < N4; ++i)
        v[i] = N3 > 1 ? pair_sum_mirror<0x141>(v[i], v[N3 > 1 ? i + N4 : i], lane & 4)
                      : v[i] + dpp<0x141>(v[i]);
    constexpr int N5 = N4 > 1 ? N4 / 2 : 1;
#pragma unroll
    for (int i = 0; i < N5; ++i)
        v[i] = N4 > 1 ? pair_sum<0x4E>(v[i], v[N4 > 1 ? i + N5 : i], lane & 2) : v[i] + dpp<0x4E>(v[i]);
    return N5 > 1 ? pair_sum<0xB1>(v[0], v[N5 > 1 ? 1 : 0], lane & 1) : v[0] + dpp<0xB1>(v[0]);
}

template <class T, int NS, int TPB, int KB>
__global__ __launch_bounds__(TPB) void scan_bwd_kernel(ScanP P) {
    constexpr int WAVES = TPB / 64, NV = 2 * NS;
    __shared__ __attribute__((aligned(16))) float bc[KB * NV];
    __shared__ float red[WAVES][KB][NV];
    const int slot = (int)(blockIdx.x / (P.nblk * P.groups));
    const int blk = (int)(blockIdx.x % (P.nblk * P.groups));
    const Place q = place<TPB>(P, blk);
    const int c = q.c, lane = (int)(threadIdx.x & 63), wave = (int)(threadIdx.x >> 6);
    const int64_t blocks = (P.length + KB - 1) / KB;
    float a2[NS], dA[NS];
    load_a2<NS>(P, c, a2);
#pragma unroll
    for (int n = 0; n < NS; ++n) dA[n] = 0.f;
    const float bias = P.bias ? P.bias[c] : 0.f, dd = P.D ? P.D[c] : 0.f;
    float dD = 0.f, dbias = 0.f;
    for (int64_t job = slot; job < P.batch * P.chunks; job += P.slots) {
        const int64_t b = job / P.chunks;
        const int ch = (int)(job - b * P.chunks);
        const int len = levels(P.lengths, b, P.length);
        const int t0 = ch * P.chunk, tn = t0 + P.chunk < P.length ? t0 + P.chunk : P.length;
        const int t1 = tn < len ? tn : len;
        float G[NS];  // a_{t+1} g_{t+1} (0 with dy in idle lanes: they add nothing to dB and dC)
        const float* ge = P.gend + job * P.states * P.channels + c;
#pragma unroll
        for (int n = 0; n < NS; ++n)
            G[n] = P.chunks > 1 && q.live && n < P.states ? ge[(int64_t)n * P.channels] : 0.f;
        const int64_t row = b * P.length;
        for (int t = t0 + (t1 - t0 - 1) / KB * KB; t1 > t0 && t >= t0; t -= KB) {
            float h[NS], p[KB][NS];
            float u[KB], raw[KB], dts[KB], dy[KB];
            T rz[KB], ry[KB];
#pragma unroll
            for (int j = 0; j < KB; ++j) {
                const int s = t + j < t1 ? t + j : t1 - 1;
                u[j] = to_f32<T>(at<T>(P.u, b, s, c));
                raw[j] = to_f32<T>(at<T>(P.delta, b, s, c)) + bias;
                ry[j] = at<T>(P.dy, b, s, c);
                if (P.z.p) rz[j] = at<T>(P.z, b, s, c);
            }
            const float* ck = P.ck + (b * blocks + t / KB) * P.states * P.channels;
#pragma unroll
            for (int n = 0; n < NS; ++n) h[n] = n < P.states ? (ck + (int64_t)n * P.channels)[(unsigned)c] : 0.f;
            __syncthreads();
            stage_bc<T, NS, TPB, KB, true>(P, b, q.g, t, t1, bc);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < KB; ++j) {
                if (t + j >= t1) break;
                const float* w = bc + j * NV;
                dts[j] = P.softplus ? softplus(raw[j]) : raw[j];
                const float du = dts[j] * u[j];
                float y = 0.f;
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    p[j][n] = __builtin_amdgcn_exp2f(dts[j] * a2[n]) * h[n];
                    h[n] = fmaf(du, w[n], p[j][n]);
                    y = fmaf(h[n], w[NS + n], y);
                }
                dy[j] = q.live ? to_f32<T>(ry[j]) : 0.f;
                if (P.z.p) {
                    const float z = to_f32<T>(rz[j]), s = sigmoid(z), dz = dy[j] * fmaf(dd, u[j], y);
                    if (q.live) put<T>(P.dz, row + t + j, P.channels, c, dz * (s * fmaf(z, 1.f - s, 1.f)));
                    dy[j] *= z * s;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int j = KB - 1; j >= 0; --j) {
                if (t + j >= t1) continue;
                const float* w = bc + j * NV;
                // a_t and h_t are formed again, not kept: with them the block would not fit the registers
                float dt = dts[j];
                asm volatile("" : "+v"(dt));
                const float du = dt * u[j];
                float v[NS], gB = 0.f, gA = 0.f;
#pragma unroll
                for (int n = 0; n < NS; ++n) v[n] = fmaf(du, w[n], p[j][n]) * dy[j];
                const float sc = reduce_lanes<NS>(v);
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    const float g = fmaf(w[NS + n], dy[j], G[n]);
                    const float gp = g * p[j][n];
                    v[n] = g * du;
                    gB = fmaf(g, w[n], gB);
                    gA = fmaf(gp, a2[n], gA);
                    dA[n] = fmaf(dt, gp, dA[n]);
                    G[n] = __builtin_amdgcn_exp2f(dt * a2[n]) * g;
                }
                const float sb = reduce_lanes<NS>(v);
                float dl = fmaf(gA, kLn2, gB * u[j]);
                if (P.softplus) dl *= sigmoid(raw[j]);
                dD = fmaf(dy[j], u[j], dD);
                dbias += dl;
                if (q.live) {
                    put<T>(P.y, row + t + j, P.channels, c, fmaf(dt, gB, dd * dy[j]));
                    put<T>(P.ddelta, row + t + j, P.channels, c, dl);
                }
                if (lane % (64 / NS) == 0) {
                    red[wave][j][lane / (64 / NS)] = sb;
                    red[wave][j][NS + lane / (64 / NS)] = sc;
                }
                __builtin_amdgcn_sched_barrier(0);  // (one level's values at a time)
            }
            __syncthreads();
            // the workgroup's sums of this block
            const int m = (t1 - t < KB ? t1 - t : KB) * NV;
            float* out = P.pbc + (((int64_t)blk * P.batch + b) * P.length + t) * NV;
            for (int e = (int)threadIdx.x; e < m; e += TPB) {
                float s = red[0][e / NV][e % NV];
#pragma unroll
                for (int k = 1; k < WAVES; ++k) s += red[k][e / NV][e % NV];
                out[e] = s;
            }
        }
        if (q.live)
            for (int t = t1 > t0 ? t1 : t0; t < tn; ++t) {
                put<T>(P.y, row + t, P.channels, c, 0.f);
                put<T>(P.ddelta, row + t, P.channels, c, 0.f);
                if (P.z.p) put<T>(P.dz, row + t, P.channels, c, 0.f);
            }
    }
    if (!q.live) return;
    float* s = P.pA + ((int64_t)slot * P.channels + c) * P.states;
#pragma unroll
    for (int n = 0; n < NS; ++n)
        if (n < P.states) s[n] = dA[n];
    if (P.pD) P.pD[(int64_t)slot * P.channels + c] = dD;
    if (P.pbias) P.pbias[(int64_t)slot * P.channels + c] = dbias;
}

// dB and dC from the workgroups' partial sums: one lane a (level, group, n, which).
template <class T>
__global__ __launch_bounds__(256) void scan_bc_kernel(ScanP P, int ns, T* dB, T* dC) {
    const int per = P.groups * 2 * ns;
    const int64_t total = P.batch * P.length * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t lv = i / per;
        const int r = (int)(i - lv * per), g = r / (2 * ns), v = r - g * 2 * ns, n = v % ns;
        if (n >= P.states) continue;
        const int64_t b = lv / P.length;
        float s = 0.f;
        if ((int)(lv - b * P.length) < lane_levels(P.lengths, b, P.length)) {
            const int64_t step = P.batch * P.length * 2 * ns;
            const float* p = P.pbc + (int64_t)g * P.nblk * step + lv * 2 * ns + v;
            for (int k = 0; k < P.nblk; ++k) s += p[k * step];
        }
        (v < ns ? dB : dC)[(lv * P.groups + g) * P.states + n] = from_f32<T>(s);
    }
}

// ---------------------------------------------------------------------------
// Host side.

constexpr int64_t kMaxChannels = 1 << 20, kMaxLevels = (int64_t)1 << 40;

int lanes_of(int64_t per) { return per <= 64 ? 64 : per <= 128 ? 128 : 256; }
int states_of(int states) { return states <= 4 ? 4 : states <= 8 ? 8 : states <= 16 ? 16 : 32; }
int block_of(int ns) { return ns == 32 ? 4 : 8; }

struct Plan {
    int tpb, nblk, per, ns, chunk, chunks, slots;
};

// Wavefronts that fill the card: one for each SIMD.  Whole windows with fewer are
// split in chunks, as long as a chunk keeps kMinChunk levels.
constexpr int64_t kFill = 1024;
constexpr int kMinChunk = 64;
// Workgroup rows of partial dA sums.
constexpr int64_t kSlots = 2048;

Plan plan(int64_t batch, int64_t length, int64_t channels, int states, int groups) {
    Plan p;
    p.per = (int)(channels / groups);
    p.tpb = lanes_of(p.per);
    p.nblk = (int)cdiv(p.per, p.tpb);
    p.ns = states_of(states);
    const int64_t waves = (batch < 1 ? 1 : batch) * groups * p.nblk * (p.tpb / 64);
    int64_t n = waves >= kFill ? 1 : cdiv(2 * kFill, waves);
    const int64_t most = length / kMinChunk;
    if (n > most) n = most < 1 ? 1 : most;
    p.chunk = (int)(cdiv(cdiv(length < 1 ? 1 : length, n), kTile) * kTile);
    p.chunks = (int)cdiv(length < 1 ? 1 : length, p.chunk);
    const int64_t jobs = batch * p.chunks, wg = (int64_t)groups * p.nblk;
    int64_t s = kSlots / wg;
    if (s < 64) s = 64;
    p.slots = (int)(jobs < s ? (jobs < 1 ? 1 : jobs) : s);
    return p;
}

int check_scan(int dtype, int states, int groups, int sp, int64_t batch, int64_t length, int64_t channels) {
    if (size_of(dtype) == 0) return FPDE_ERR_UNSUPPORTED;
    if (sp != 0 && sp != 1) return FPDE_ERR_ARG;
    if (states < 1 || batch < 0 || length < 0 || length >= ((int64_t)1 << 31) - 256 || channels < 1 ||
        channels > kMaxChannels || groups < 1 || channels % groups)
        return FPDE_ERR_SHAPE;
    if (states > 32) return FPDE_ERR_UNSUPPORTED;
    if (batch > kMaxLevels || (length > 0 && batch > kMaxLevels / length)) return FPDE_ERR_SHAPE;
    const Plan p = plan(batch, length, channels, states, groups);
    if (batch * p.chunks > (((int64_t)1 << 31) - 1) / ((int64_t)p.nblk * groups * p.tpb)) return FPDE_ERR_SHAPE;
    return FPDE_OK;
}

bool seq_ok(const Seq& s, int64_t batch, int64_t length, int64_t width) {
    const int64_t most = (int64_t)1 << 50;
    if (length > 1 && (s.ts < width || s.ts > most / length)) return false;
    return batch <= 1 || (s.bs >= 0 && s.bs <= most / batch);
}

// f(T{}, NS, TPB)
template <class F>
int with_scan(int dtype, const Plan& p, F f) {
    return with_type(dtype, [&](auto t) {
        auto wg = [&](auto ns) {
            switch (p.tpb) {
            case 64: return f(t, ns, std::integral_constant<int, 64>{});
            case 128: return f(t, ns, std::integral_constant<int, 128>{});
            default: return f(t, ns, std::integral_constant<int, 256>{});
            }
        };
        switch (p.ns) {
        case 4: return wg(std::integral_constant<int, 4>{});
        case 8: return wg(std::integral_constant<int, 8>{});
        case 16: return wg(std::integral_constant<int, 16>{});
        default: return wg(std::integral_constant<int, 32>{});
        }
    });
}

template <class A>
ScanP params(const A* a, const Plan& p) {
    ScanP P{};
    P.u = Seq{a->u, a->u_batch_stride, a->u_time_stride};
    P.delta = Seq{a->delta, a->delta_batch_stride, a->delta_time_stride};
    P.z = Seq{a->z, a->z_batch_stride, a->z_time_stride};
    P.B = Seq{a->B, a->b_batch_stride, a->b_time_stride};
    P.C = Seq{a->C, a->c_batch_stride, a->c_time_stride};
    P.A = a->A, P.D = a->D, P.bias = a->delta_bias, P.state = a->state, P.lengths = a->lengths;
    P.batch = a->batch, P.length = (int)a->length, P.channels = (int)a->channels;
    P.states = a->states, P.groups = a->groups, P.softplus = a->softplus;
    P.chunk = p.chunk, P.chunks = p.chunks, P.per = p.per, P.nblk = p.nblk, P.slots = p.slots;
    return P;
}

template <class A>
int check_inputs(const A* a, const ScanP& P, Spans* sp) {
    const int e = size_of(a->dtype);
    const int64_t bc = (int64_t)a->groups * a->states;
    if (!seq_ok(P.u, a->batch, a->length, a->channels) || !seq_ok(P.delta, a->batch, a->length, a->channels) ||
        (a->z && !seq_ok(P.z, a->batch, a->length, a->channels)) || !seq_ok(P.B, a->batch, a->length, bc) ||
        !seq_ok(P.C, a->batch, a->length, bc))
        return FPDE_ERR_SHAPE;
    if (!a->A || (a->batch * a->length > 0 && (!a->u || !a->delta || !a->B || !a->C))) return FPDE_ERR_ARG;
    auto seq = [&](const Seq& s, int64_t w) { sp->add(s.p, span3(a->batch, a->length, w, s.bs, s.ts, e), e, false); };
    seq(P.u, a->channels), seq(P.delta, a->channels), seq(P.z, a->channels), seq(P.B, bc), seq(P.C, bc);
    sp->add(a->A, a->channels * a->states * 4, 4, false);
    sp->add(a->D, a->channels * 4, 4, false);
    sp->add(a->delta_bias, a->channels * 4, 4, false);
    sp->add(a->lengths, a->batch * 4, 4, false);
    sp->add(a->state, a->batch * a->channels * a->states * 4, 4, false);
    return FPDE_OK;
}

unsigned grid_of(const ScanP& P, int64_t rows) { return (unsigned)(rows * P.nblk * P.groups); }

int queue_chunks(const ScanP& P, float* e, int backward, hipStream_t s) {
    const dim3 g((unsigned)cdiv(P.channels, 256), (unsigned)P.states,
                 (unsigned)(P.batch < 65535 ? P.batch : 65535));
    return launch(chunk_kernel, g, dim3(256), s, P, e, backward);
}

// floats of one [batch][chunks][states][channels] array and of the sums of dt
int64_t ends_of(int64_t batch, int64_t channels, int states, const Plan& p) {
    return p.chunks > 1 ? batch * p.chunks * states * channels : 0;
}
int64_t sums_of(int64_t batch, int64_t channels, const Plan& p) {
    return p.chunks > 1 ? batch * p.chunks * channels : 0;
}

struct BwdSpace {
    int64_t hend, gend, sdt, ck, pbc, pA, pD, total;
};
BwdSpace bwd_space(int64_t batch, int64_t length, int64_t channels, int states, int groups, const Plan& p) {
    BwdSpace w;
    int64_t n = 0;
    auto take = [&](int64_t k) {
        const int64_t at = n;
        n += (k + 3) / 4 * 4;
        return at;
    };
    w.hend = take(ends_of(batch, channels, states, p));
    w.gend = take(ends_of(batch, channels, states, p));
    w.sdt = take(sums_of(batch, channels, p));
    w.ck = take(batch * cdiv(length, block_of(p.ns)) * states * channels);
    w.pbc = take((int64_t)groups * p.nblk * batch * length * 2 * p.ns);
    w.pA = take((int64_t)p.slots * channels * states);
    w.pD = take((int64_t)p.slots * channels * 2);
    w.total = n * 4;
    return w;
}

}  // namespace

extern "C" int64_t fpde_selective_scan_workspace(const fpde_scan_args* a) {
    if (!a) return FPDE_ERR_ARG;
    const int st = check_scan(a->dtype, a->states, a->groups, a->softplus, a->batch, a->length, a->channels);
    if (st != FPDE_OK) return st;
    const Plan p = plan(a->batch, a->length, a->channels, a->states, a->groups);
    return (ends_of(a->batch, a->channels, a->states, p) + sums_of(a->batch, a->channels, p)) * 4;
}

extern "C" int fpde_selective_scan(const fpde_scan_args* a, void* stream) {
    const int64_t need = fpde_selective_scan_workspace(a);
    if (need < 0) return (int)need;
    const Plan p = plan(a->batch, a->length, a->channels, a->states, a->groups);
    ScanP P = params(a, p);
    Spans sp;
    int st = check_inputs(a, P, &sp);
    if (st != FPDE_OK) return st;
    if (a->batch * a->length > 0 && !a->y) return FPDE_ERR_ARG;
    if (need > 0 && (!a->workspace || a->workspace_bytes < need)) return FPDE_ERR_ARG;
    sp.add(a->y, a->batch * a->length * a->channels * size_of(a->dtype), size_of(a->dtype), true);
    sp.add(a->state_out, a->batch * a->channels * a->states * 4, 4, true);
    if (need > 0) sp.add(a->workspace, need, 16, true);
    st = sp.check(a->state_out, a->state);
    if (st != FPDE_OK) return st;
    if (a->batch == 0 || (a->length == 0 && !a->state_out)) return FPDE_OK;
    P.y = a->y, P.state_out = a->state_out;
    P.hend = (float*)a->workspace;
    if (need > 0) P.sdt = P.hend + ends_of(a->batch, a->channels, a->states, p);
    hipStream_t s = (hipStream_t)stream;
    return with_scan(a->dtype, p, [&](auto t, auto nsc, auto tpbc) {
        using T = decltype(t);
        constexpr int NS = decltype(nsc)::value, TPB = decltype(tpbc)::value;
        if (a->length == 1) {
            const dim3 g((unsigned)cdiv(a->channels * (NS / 4), 256),
                         (unsigned)(a->batch < 65535 ? a->batch : 65535));
            return launch(scan_step_kernel<T, NS>, g, dim3(256), s, P);
        }
        const dim3 g(grid_of(P, a->batch * P.chunks));
        if (P.chunks > 1) {
            int r = launch(scan_fwd_kernel<T, NS, TPB, ENDS, 8>, g, dim3(TPB), s, P);
            if (r == FPDE_OK) r = queue_chunks(P, P.hend, 0, s);
            if (r != FPDE_OK) return r;
        }
        return launch(scan_fwd_kernel<T, NS, TPB, OUT, 8>, g, dim3(TPB), s, P);
    });
}

extern "C" int64_t fpde_selective_scan_bwd_workspace(const fpde_scan_bwd_args* a) {
    if (!a) return FPDE_ERR_ARG;
    const int st = check_scan(a->dtype, a->states, a->groups, a->softplus, a->batch, a->length, a->channels);
    if (st != FPDE_OK) return st;
    const Plan p = plan(a->batch, a->length, a->channels, a->states, a->groups);
    return bwd_space(a->batch, a->length, a->channels, a->states, a->groups, p).total;
}

extern "C" int fpde_selective_scan_bwd(const fpde_scan_bwd_args* a, void* stream) {
    const int64_t need = fpde_selective_scan_bwd_workspace(a);
    if (need < 0) return (int)need;
    const Plan p = plan(a->batch, a->length, a->channels, a->states, a->groups);
    ScanP P = params(a, p);
    P.dy = Seq{a->dy, a->dy_batch_stride, a->dy_time_stride};
    Spans sp;
    int st = check_inputs(a, P, &sp);
    if (st != FPDE_OK) return st;
    if (!seq_ok(P.dy, a->batch, a->length, a->channels)) return FPDE_ERR_SHAPE;
    const int64_t n = a->batch * a->length;
    if (!a->dA || (n > 0 && (!a->dy || !a->du || !a->ddelta || !a->dB || !a->dC)) ||
        (a->D == nullptr) != (a->dD == nullptr) || (n > 0 && (a->z == nullptr) != (a->dz == nullptr)) ||
        (a->delta_bias == nullptr) != (a->ddelta_bias == nullptr))
        return FPDE_ERR_ARG;
    if (!a->workspace || a->workspace_bytes < need) return FPDE_ERR_ARG;
    const int e = size_of(a->dtype);
    const int64_t data = n * a->channels * e, bc = n * a->groups * a->states * e;
    sp.add(a->dy, span3(a->batch, a->length, a->channels, P.dy.bs, P.dy.ts, e), e, false);
    sp.add(a->du, data, e, true);
    sp.add(a->ddelta, data, e, true);
    sp.add(a->dz, data, e, true);
    sp.add(a->dB, bc, e, true);
    sp.add(a->dC, bc, e, true);
    sp.add(a->dA, a->channels * a->states * 4, 4, true);
    sp.add(a->dD, a->channels * 4, 4, true);
    sp.add(a->ddelta_bias, a->channels * 4, 4, true);
    sp.add(a->workspace, need, 16, true);
    st = sp.check();
    if (st != FPDE_OK) return st;
    const BwdSpace w = bwd_space(a->batch, a->length, a->channels, a->states, a->groups, p);
    float* ws = (float*)a->workspace;
    P.hend = ws + w.hend, P.gend = ws + w.gend, P.sdt = ws + w.sdt, P.ck = ws + w.ck, P.pbc = ws + w.pbc;
    P.pA = ws + w.pA;
    P.pD = a->D ? ws + w.pD : nullptr;
    P.pbias = a->delta_bias ? ws + w.pD + (int64_t)p.slots * a->channels : nullptr;
    P.y = a->du, P.ddelta = a->ddelta, P.dz = a->dz;
    hipStream_t s = (hipStream_t)stream;
    if (n > 0) {
        st = with_scan(a->dtype, p, [&](auto t, auto nsc, auto tpbc) {
            using T = decltype(t);
            constexpr int NS = decltype(nsc)::value, TPB = decltype(tpbc)::value, KB = NS == 32 ? 4 : 8;
            const dim3 g(grid_of(P, a->batch * P.chunks));
            int r = FPDE_OK;
            if (P.chunks > 1) {
                r = launch(scan_fwd_kernel<T, NS, TPB, ENDS, KB>, g, dim3(TPB), s, P);
                if (r == FPDE_OK) r = launch(scan_adj_kernel<T, NS, TPB>, g, dim3(TPB), s, P);
                if (r == FPDE_OK) r = queue_chunks(P, P.hend, 0, s);
                if (r == FPDE_OK) r = queue_chunks(P, P.gend, 1, s);
            }
            if (r == FPDE_OK) r = launch(scan_fwd_kernel<T, NS, TPB, CHECKS, KB>, g, dim3(TPB), s, P);
            if (r == FPDE_OK)
                r = launch(scan_bwd_kernel<T, NS, TPB, KB>, dim3(grid_of(P, P.slots)), dim3(TPB), s, P);
            if (r != FPDE_OK) return r;
            const int64_t bcs = cdiv(n * a->groups * 2 * NS, 256);
            return launch(scan_bc_kernel<T>, dim3((unsigned)(bcs < 65536 ? bcs : 65536)), dim3(256), s, P, NS,
                          (T*)a->dB, (T*)a->dC);
        });
        if (st != FPDE_OK) return st;
    }
    const int64_t rows = n > 0 ? p.slots : 0, cols = a->channels * a->states;
    st = queue_colsum(P.pA, rows, cols, a->dA, cols, nullptr, 0, FPDE_F32, s);
    if (st == FPDE_OK && P.pD)
        st = queue_colsum(P.pD, rows, a->channels, a->dD, a->channels, nullptr, 0, FPDE_F32, s);
    if (st == FPDE_OK && P.pbias)
        st = queue_colsum(P.pbias, rows, a->channels, a->ddelta_bias, a->channels, nullptr, 0, FPDE_F32, s);
    return st;
}
