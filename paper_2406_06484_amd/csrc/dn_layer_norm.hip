// The norms behind a mixer and between two blocks, and their gradients.
//
// Output norm, a row o of one head, its gate g, a the gate's factor g sigmoid(g) or sigmoid(g), r = 1 / sqrt(mean(o^2) + eps), n = r o:
//
//     y = n w a ;   dn = dy a w ,  do = r (dn - n mean(dn n)) ,  dw = sum dy a n ,  dg = dy n w a'(g)
//
// Block norm, x the branch that a block adds to the stream, m = x or its RMS norm, u the branch's gate per channel (or ones):
//
//     h = keep residual + scale u m ,  y = r h w ,  r = 1 / sqrt(mean(h^2) + eps) ;  with  q = r h ,  dz = dy w :
//     H = dh + r (dz - q mean(dz q)) ,  dresidual = keep H ,  B = scale u H ,  dx = B, or r_x (B - m mean(B m)) ,  dw = sum dy q ,  du = scale sum H m
//
// Bound by HBM: about ten operations an element forward and thirty backward.  In bf16, 16384 tokens of 16 heads of 128: output norm 37 us forward (201 MB), 59 backward (336 MB, 5.7 TB/s) and 5 for the weight's sums; 16384 rows of 2048: block norm
// 45 (268 MB, 6.0 TB/s), 56 (273 MB) and 5; 4101 rows of 4104 with an fp32 stream and a normed, gated branch 43 (202 MB), 64 (303 MB) and 5.  Each element is fetched once and written once; sums over a row stay in registers and lane swaps (a row wider than
// two words a lane: and the LDS).  y comes from the sum before it is rounded to the stream's type, and the backward pass, which forms r and q again, from the stream as it was stored.
#include "dn_layer_device.hpp"

namespace dn {

// Outputs that the caches would not hold until they are read are stored past them: gradients, and the stream, which the next block's end reads, of over kPastCaches bytes.  (Both passes in a row 10 % faster at 16384 rows of
// 2048; a pass and the product that reads its result: 175 us instead of 178 to 184 at 16384 rows, output norm backward, and at 2048 rows 39 instead of 36, block norm backward.  y, which the next product reads, stays: 141 us
// instead of 143.)
constexpr long kPastCaches = 32l << 20;

// --- output norm: a wave has 64 16 / (D sizeof(T)) rows (token and head) at a time

template <typename T, int D> struct HeadRow {
    static constexpr int V = 16 / (int)sizeof(T), LPR = D / V, RPW = 64 / LPR;
};

// a(g), and a'(g)
__device__ inline float gate_of(int act, float g, float *d) {
    const float s = sigmoid_fast_f32(g);
    if (act == 2) { if (d) *d = s * (1.f - s); return s; }
    if (d) *d = s * fmaf(g, 1.f - s, 1.f);
    return g * s;
}

// Elements from a tensor's start to row r's.
__device__ inline long head_row(const OutNormArgs &a, int D, int r, long stride) {
    if (stride == (long)a.H * D) return (long)r * D;
    const int t = a.H == 1 ? r : (int)(__umulhi((unsigned)r, a.magic) >> a.shift);
    return t * stride + (r - t * a.H) * D;
}

constexpr int kOutBatch = 4, kOutBwdBatch = 2;

template <typename T, int D>
__global__ __launch_bounds__(256) void k_out_norm_fwd(OutNormArgs a) {
    using L = HeadRow<T, D>;
    constexpr int V = L::V;
    const int lane = threadIdx.x & 63, e0 = (lane % L::LPR) * V, sub = lane / L::LPR;
    const int rows = a.T * a.H;
    const T *o = static_cast<const T *>(a.o) + e0, *gate = static_cast<const T *>(a.gate) + e0;
    T *y = static_cast<T *>(a.y) + e0;
    Word<T, V> ww;
    float w[V];
    if (a.w) { ww.load(static_cast<const T *>(a.w) + e0); ww.unpack(w); }
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = 1.f;
    }
    constexpr int STEP = kOutBatch * L::RPW;
    for (long r0 = ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) * STEP + sub; r0 - sub < rows; r0 += (long)gridDim.x * 4 * STEP) {
        Word<T, V> xo[kOutBatch], xg[kOutBatch];
#pragma unroll
        for (int b = 0; b < kOutBatch; ++b) {
            const int r = (int)min(r0 + b * L::RPW, (long)rows - 1);
            xo[b].load(o + head_row(a, D, r, a.o_stride));
            if (a.gate) xg[b].load(gate + head_row(a, D, r, a.gate_stride));
        }
#pragma unroll
        for (int b = 0; b < kOutBatch; ++b) {
            float f[V], ss = 0.f;
            xo[b].unpack(f);
#pragma unroll
            for (int i = 0; i < V; ++i) ss = fmaf(f[i], f[i], ss);
            const float r = rsqrtf(lanes_sum<L::LPR>(ss) * (1.f / D) + a.eps);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = f[i] * r * w[i];
            if (a.gate)
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] *= gate_of(a.act, xg[b].get(i), nullptr);
            Word<T, V> out;
            out.pack(f);
            if (r0 + b * L::RPW < rows) out.store(y + (r0 + b * L::RPW) * D);
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void k_out_norm_bwd(OutNormArgs a) {
    using L = HeadRow<T, D>;
    constexpr int V = L::V;
    __shared__ float part[4][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e0 = (lane % L::LPR) * V, sub = lane / L::LPR;
    const int rows = a.T * a.H;
    const T *o = static_cast<const T *>(a.o) + e0, *gate = static_cast<const T *>(a.gate) + e0, *dy = static_cast<const T *>(a.dy) + e0;
    T *d_o = static_cast<T *>(a.d_o) + e0, *dgate = static_cast<T *>(a.dgate) + e0;
    Word<T, V> ww;
    float w[V], dw[V];
    if (a.w) { ww.load(static_cast<const T *>(a.w) + e0); ww.unpack(w); }
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = 1.f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) dw[i] = 0.f;
    constexpr int STEP = kOutBwdBatch * L::RPW;
    for (long r0 = ((long)blockIdx.x * 4 + wave) * STEP + sub; r0 - sub < rows; r0 += (long)gridDim.x * 4 * STEP) {
        Word<T, V> xo[kOutBwdBatch], xg[kOutBwdBatch], xy[kOutBwdBatch];
#pragma unroll
        for (int b = 0; b < kOutBwdBatch; ++b) {
            const int r = (int)min(r0 + b * L::RPW, (long)rows - 1);
            xo[b].load(o + head_row(a, D, r, a.o_stride));
            if (a.gate) xg[b].load(gate + head_row(a, D, r, a.gate_stride));
            xy[b].load(dy + (long)r * D);
        }
#pragma unroll
        for (int b = 0; b < kOutBwdBatch; ++b) {
            const bool live = r0 + b * L::RPW < rows;
            const int row = (int)min(r0 + b * L::RPW, (long)rows - 1);
            float f[V], g[V], dg[V], ss = 0.f, dot = 0.f;
            xo[b].unpack(f);
            xy[b].unpack(g);
            if (a.gate) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float d;
                    const float act = gate_of(a.act, xg[b].get(i), &d);
                    dg[i] = g[i] * w[i] * f[i] * d;
                    g[i] *= act;
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                ss = fmaf(f[i], f[i], ss);
                dot = fmaf(g[i] * w[i], f[i], dot);
            }
            const float r = rsqrtf(lanes_sum<L::LPR>(ss) * (1.f / D) + a.eps), m = lanes_sum<L::LPR>(dot) * r * (1.f / D);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float n = f[i] * r;
                if (live) dw[i] = fmaf(g[i], n, dw[i]);
                if (a.gate) dg[i] *= r;
                f[i] = r * fmaf(-n, m, g[i] * w[i]);
            }
            Word<T, V> out;
            out.pack(f);
            if (live) out.store(d_o + (long)row * D, a.once);
            if (a.gate) {
                out.pack(dg);
                if (live) out.store(dgate + head_row(a, D, row, a.dgate_stride), a.once);
            }
        }
    }
    if (!a.dw) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int m = L::LPR; m < 64; m <<= 1) dw[i] += __shfl_xor(dw[i], m);
        if (sub == 0) part[wave][e0 + i] = dw[i];
    }
    __syncthreads();
    float *to = gridDim.x == 1 ? a.dw : a.partial + (long)blockIdx.x * D;
    for (int e = threadIdx.x; e < D; e += 256) to[e] = (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
}

// --- block norm: LANES lanes to a row (a part of a wave, one, or some waves), NW words of 16 bytes (of T) a lane

// Sums over a row's lanes; `part` has a place for each of its waves, and is free for the next sum when a later barrier has passed.
template <int LANES> __device__ inline float row_sum(float x, float *part) {
    x = lanes_sum<LANES < 64 ? LANES : 64>(x);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
        lds_barrier();
        x = part[0];
#pragma unroll
        for (int i = 1; i < LANES / 64; ++i) x += part[i];
    }
    return x;
}
template <int LANES> __device__ inline float2 row_sums(float x, float y, float *part) {
    constexpr int WAVES = LANES / 64;
    x = lanes_sum<LANES < 64 ? LANES : 64>(x);
    y = lanes_sum<LANES < 64 ? LANES : 64>(y);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) { part[threadIdx.x >> 6] = x; part[WAVES + (threadIdx.x >> 6)] = y; }
        lds_barrier();
        x = part[0];
        y = part[WAVES];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) { x += part[i]; y += part[WAVES + i]; }
    }
    return make_float2(x, y);
}

template <int LANES> constexpr int kBlockRows = LANES > 64 ? 1 : 256 / LANES; // rows of a workgroup
template <int LANES> constexpr int kBlockThreads = LANES > 64 ? LANES : 256;

template <typename T, typename RT, int LANES, int NW, bool POST>
__global__ __launch_bounds__(kBlockThreads<LANES>) void k_block_norm_fwd(BlockNormArgs a) {
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float part[2][LANES > 64 ? LANES / 64 : 1];
    const int lane = threadIdx.x % LANES, sub = LANES < 64 ? (threadIdx.x & 63) / LANES : 0; // (sub: the row among those of the wave, which goes on to the last of them)
    const int words = a.D / V;
    const float inv = 1.f / (float)a.D;
    const int step = gridDim.x * kBlockRows<LANES>;
    for (int first = blockIdx.x * kBlockRows<LANES> + (LANES > 64 ? 0 : (threadIdx.x >> 6) * (LANES < 64 ? 64 / LANES : 1)); first < a.T; first += step) {
        const int row = min(first + sub, a.T - 1);
        const bool live = LANES >= 64 || first + sub < a.T;
        Word<T, V> x[NW];
        Word<RT, V> r[NW];
        float h[NW][V];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int e = (lane + i * LANES) * V;
            if (lane + i * LANES < words) {
                x[i].load(static_cast<const T *>(a.x) + row * a.x_stride + e);
                if (a.res) r[i].load(static_cast<const RT *>(a.res) + row * a.res_stride + e);
                else r[i].zero();
            } else { x[i].zero(); r[i].zero(); }
        }
        float rx = 1.f;
        if constexpr (POST) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < NW; ++i)
#pragma unroll
                for (int v = 0; v < V; ++v) ss = fmaf(x[i].get(v), x[i].get(v), ss);
            rx = rsqrtf(row_sum<LANES>(ss, part[0]) * inv + a.eps);
        }
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int e = (lane + i * LANES) * V;
            Word<T, V> u;
            u.zero();
            if (a.gate && lane + i * LANES < words) u.load(static_cast<const T *>(a.gate) + e);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float f = a.gate ? a.scale * u.get(v) : a.scale, m = POST ? x[i].get(v) * rx : x[i].get(v);
                h[i][v] = a.res ? fmaf(f, m, a.res_scale * r[i].get(v)) : f * m;
            }
            if (lane + i * LANES < words) {
#pragma unroll
                for (int v = 0; v < V; ++v) ss = fmaf(h[i][v], h[i][v], ss);
                if (a.h_out && live) {
                    Word<RT, V> out;
                    out.pack(h[i]);
                    out.store(static_cast<RT *>(a.h_out) + (long)row * a.D + e, a.once);
                }
            }
        }
        const float rh = rsqrtf(row_sum<LANES>(ss, part[1]) * inv + a.eps);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int e = (lane + i * LANES) * V;
            if (lane + i * LANES < words && live) {
                Word<T, V> w;
                if (a.w) w.load(static_cast<const T *>(a.w) + e);
#pragma unroll
                for (int v = 0; v < V; ++v) h[i][v] *= a.w ? rh * w.get(v) : rh;
                w.pack(h[i]);
                w.store(static_cast<T *>(a.y) + (long)row * a.D + e);
            }
        }
        if constexpr (LANES > 64 && !POST) lds_barrier(); // (the next row's sum takes the same place)
    }
}

template <typename T, typename RT, int LANES, int NW, bool POST>
__global__ __launch_bounds__(kBlockThreads<LANES>) void k_block_norm_bwd(BlockNormArgs a) {
    constexpr int V = 16 / (int)sizeof(T), ROWS = kBlockRows<LANES>;
    constexpr bool AHEAD = NW <= 2; // (a next row's words as well would not fit beside four and their sums)
    __shared__ float part[2][LANES > 64 ? LANES / 32 : 1];
    const int lane = threadIdx.x % LANES, mine = LANES > 64 ? 0 : threadIdx.x >> 6, sub = LANES < 64 ? (threadIdx.x & 63) / LANES : 0; // (the wave; the row among its rows)
    const int words = a.D / V;
    const float inv = 1.f / (float)a.D;
    const bool branch = POST || a.gate;
    float dw[NW][V], du[NW][V];
    Word<T, V> w[NW], u[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const int e = (lane + i * LANES) * V;
        w[i].zero();
        u[i].zero();
        if (lane + i * LANES < words) {
            if (a.w) w[i].load(static_cast<const T *>(a.w) + e);
            if (a.gate) u[i].load(static_cast<const T *>(a.gate) + e);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) dw[i][v] = du[i][v] = 0.f;
    }
    const int step = gridDim.x * ROWS;
    int first = blockIdx.x * ROWS + mine * (LANES < 64 ? 64 / LANES : 1);
    struct Row {
        Word<T, V> dy[NW], x[NW];
        Word<RT, V> h[NW], dh[NW];
    } buffer[AHEAD ? 2 : 1];
    auto load = [&](Row &r, int of) __attribute__((always_inline)) {
        const int at_row = min(of + sub, a.T - 1);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int e = (lane + i * LANES) * V;
            const long at = (long)at_row * a.D + e;
            r.dy[i].zero(); r.x[i].zero(); r.h[i].zero(); r.dh[i].zero();
            if (lane + i * LANES < words) {
                r.dy[i].load(static_cast<const T *>(a.dy) + at);
                r.h[i].load(static_cast<const RT *>(a.h) + at);
                if (a.dh) r.dh[i].load(static_cast<const RT *>(a.dh) + at);
                if (branch) r.x[i].load(static_cast<const T *>(a.x) + at_row * a.x_stride + e);
            }
        }
    };
    auto work = [&](Row &now, Row &next) __attribute__((always_inline)) {
        auto &dy = now.dy; auto &x = now.x; auto &h = now.h; auto &dh = now.dh;
        const int row = first + sub;
        const bool live = LANES >= 64 || row < a.T;
        if constexpr (AHEAD) load(next, min(first + step, a.T - 1));
        else load(now, first);
        // mean(h^2), mean(dz h), and of the branch mean(x^2)
        float ss = 0.f, dot = 0.f, xx = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float f = h[i].get(v), g = a.w ? dy[i].get(v) * w[i].get(v) : dy[i].get(v);
                ss = fmaf(f, f, ss);
                dot = fmaf(g, f, dot);
                if constexpr (POST) xx = fmaf(x[i].get(v), x[i].get(v), xx);
            }
        const float2 s = row_sums<LANES>(ss, dot, part[0]);
        const float r = rsqrtf(s.x * inv + a.eps), m = s.y * r * inv;
        float H[NW][V];
#pragma unroll
        for (int i = 0; i < NW; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float q = h[i].get(v) * r, g = dy[i].get(v);
                H[i][v] = fmaf(r, fmaf(-q, m, a.w ? g * w[i].get(v) : g), dh[i].get(v));
                if (live) dw[i][v] = fmaf(g, q, dw[i][v]);
            }
        float rx = 1.f, mx = 0.f;
        if constexpr (POST) {
            float bx = 0.f;
#pragma unroll
            for (int i = 0; i < NW; ++i)
#pragma unroll
                for (int v = 0; v < V; ++v) bx = fmaf(a.gate ? H[i][v] * u[i].get(v) : H[i][v], x[i].get(v), bx);
            const float2 sx = row_sums<LANES>(xx, bx * a.scale, part[1]);
            rx = rsqrtf(sx.x * inv + a.eps);
            mx = sx.y * rx * inv;
        }
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int e = (lane + i * LANES) * V;
            const long at = (long)row * a.D + e;
            float d[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float n = x[i].get(v) * rx, b = a.scale * (a.gate ? u[i].get(v) * H[i][v] : H[i][v]);
                if (live) du[i][v] = fmaf(H[i][v], n, du[i][v]);
                d[v] = POST ? rx * fmaf(-n, mx, b) : b;
                H[i][v] *= a.res_scale;
            }
            if (lane + i * LANES < words && live) {
                if (a.dx) {
                    Word<T, V> out;
                    out.pack(d);
                    out.store(static_cast<T *>(a.dx) + at, a.once);
                }
                if (a.dres) {
                    Word<RT, V> out;
                    out.pack(H[i]);
                    out.store(static_cast<RT *>(a.dres) + at, a.once);
                }
            }
        }
        if constexpr (LANES > 64 && !POST) lds_barrier(); // (the next row's sums take the same place)
        first += step;
    };
    if constexpr (AHEAD) {
        if (first < a.T) load(buffer[0], first);
        while (first < a.T) {
            work(buffer[0], buffer[1]);
            if (first >= a.T) break;
            work(buffer[1], buffer[0]);
        }
    } else
        while (first < a.T) work(buffer[0], buffer[0]);
    if (!a.dw && !a.dgate) return;
    const bool alone = gridDim.x == 1;
    float *at = a.partial + (long)blockIdx.x * 2 * a.D, *tw = alone || !a.dw ? a.dw : at, *tu = alone || !a.dgate ? a.dgate : at + a.D;
    if constexpr (LANES > 64) {
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int e = (lane + i * LANES) * V;
            if (lane + i * LANES < words) {
#pragma unroll
                for (int v = 0; v < V; v += 4) {
                    if (tw) *reinterpret_cast<float4 *>(tw + e + v) = make_float4(dw[i][v], dw[i][v + 1], dw[i][v + 2], dw[i][v + 3]);
                    if (tu) *reinterpret_cast<float4 *>(tu + e + v) = make_float4(du[i][v] * a.scale, du[i][v + 1] * a.scale, du[i][v + 2] * a.scale, du[i][v + 3] * a.scale);
                }
            }
        }
    } else {
        // the rows of a wave, then the four waves, in their order
        __shared__ float sums[3][2 * NW * V][LANES];
#pragma unroll
        for (int i = 0; i < NW; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int m = LANES; m < 64; m <<= 1) { dw[i][v] += __shfl_xor(dw[i][v], m); du[i][v] += __shfl_xor(du[i][v], m); }
        if (mine && sub == 0)
#pragma unroll
            for (int i = 0; i < NW; ++i)
#pragma unroll
                for (int v = 0; v < V; ++v) { sums[mine - 1][i * V + v][lane] = dw[i][v]; sums[mine - 1][NW * V + i * V + v][lane] = du[i][v]; }
        __syncthreads();
        if (mine || sub) return;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int e = (lane + i * LANES) * V;
            if (lane + i * LANES >= words) continue;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int k = i * V + v;
                if (tw) tw[e + v] = ((dw[i][v] + sums[0][k][lane]) + sums[1][k][lane]) + sums[2][k][lane];
                if (tu) tu[e + v] = (((du[i][v] + sums[0][NW * V + k][lane]) + sums[1][NW * V + k][lane]) + sums[2][NW * V + k][lane]) * a.scale;
            }
        }
    }
}

namespace {

int launch(const char *name, const void *fn, int blocks, int threads, void **args, hipStream_t stream) {
    prof_begin(name, stream);
    const hipError_t e = hipLaunchKernel(fn, dim3(blocks), dim3(threads), args, 0, stream);
    prof_end(stream);
    return (int)e;
}

int fewer(long a, long b) { return (int)(a < b ? a : b); }

template <typename F> int by_head(int dtype, int d, F f) {
    if (dtype == 0) {
        if (d == 32) return f.template operator()<float, 32>();
        if (d == 64) return f.template operator()<float, 64>();
        if (d == 128) return f.template operator()<float, 128>();
        if (d == 256) return f.template operator()<float, 256>();
    } else {
        if (d == 32) return f.template operator()<bf16, 32>();
        if (d == 64) return f.template operator()<bf16, 64>();
        if (d == 128) return f.template operator()<bf16, 128>();
        if (d == 256) return f.template operator()<bf16, 256>();
    }
    return (int)hipErrorInvalidValue;
}
// Rows that a workgroup of the output norm's passes has at a time.
int out_rows(int dtype, int d, int batch) { return 4 * batch * (64 * (dtype == 0 ? 4 : 8) / d); }

struct OutFwd {
    OutNormArgs a;
    hipStream_t stream;
    template <typename T, int D> int operator()() {
        const long rows = (long)a.T * a.H, per = 4 * kOutBatch * HeadRow<T, D>::RPW;
        void *args[] = {&a};
        return launch("k_out_norm_fwd", reinterpret_cast<const void *>(k_out_norm_fwd<T, D>), fewer((rows + per - 1) / per, 4096), 256, args, stream);
    }
};
struct OutBwd {
    OutNormArgs a;
    hipStream_t stream;
    template <typename T, int D> int operator()() {
        const int blocks = out_norm_bwd_blocks(sizeof(T) == 4 ? 0 : 1, D, a.T, a.H);
        void *args[] = {&a};
        const int e = launch("k_out_norm_bwd", reinterpret_cast<const void *>(k_out_norm_bwd<T, D>), blocks, 256, args, stream);
        return e || blocks == 1 || !a.dw ? e : run_sum_partials(a.partial, blocks, D, D, a.dw, nullptr, stream);
    }
};

// f<T, LANES, NW>() for rows of D elements
template <typename T, typename F> int by_width(int D, F f) {
    const int words = D / (16 / (int)sizeof(T));
    if (words <= 8) return f.template operator()<T, 8, 1>();
    if (words <= 16) return f.template operator()<T, 16, 1>();
    if (words <= 32) return f.template operator()<T, 32, 1>();
    if (words <= 64) return f.template operator()<T, 64, 1>();
    if (words <= 128) return f.template operator()<T, 64, 2>();
    if (words <= 256) return f.template operator()<T, 256, 1>();
    if (words <= 512) return f.template operator()<T, 256, 2>();
    if (words <= 1024) return f.template operator()<T, 512, 2>();
    if constexpr (sizeof(T) == 4) // (bf16 rows of that many words would not fit a wave's registers)
        if (words <= 2048) return f.template operator()<T, 512, 4>();
    return (int)hipErrorInvalidValue;
}
int rows_of_workgroup(int words) { return words <= 8 ? 32 : words <= 16 ? 16 : words <= 32 ? 8 : words <= 128 ? 4 : 1; }

template <typename RT, bool POST> struct BlockFwd {
    BlockNormArgs a;
    hipStream_t stream;
    template <typename T, int LANES, int NW> int operator()() {
        void *args[] = {&a};
        return launch("k_block_norm_fwd", reinterpret_cast<const void *>(k_block_norm_fwd<T, RT, LANES, NW, POST>), fewer(((long)a.T + kBlockRows<LANES> - 1) / kBlockRows<LANES>, 1 << 16),
                      kBlockThreads<LANES>, args, stream);
    }
};
template <typename RT, bool POST> struct BlockBwd {
    BlockNormArgs a;
    hipStream_t stream;
    template <typename T, int LANES, int NW> int operator()() {
        const int blocks = block_norm_bwd_blocks(sizeof(T) == 4 ? 0 : 1, a.T, a.D);
        void *args[] = {&a};
        const int e = launch("k_block_norm_bwd", reinterpret_cast<const void *>(k_block_norm_bwd<T, RT, LANES, NW, POST>), blocks, kBlockThreads<LANES>, args, stream);
        return e || blocks == 1 || (!a.dw && !a.dgate) ? e : run_sum_partials(a.partial, blocks, 2 * (long)a.D, a.D, a.dw, a.dgate, stream);
    }
};
template <template <typename, bool> class L> int block_norm(int dtype, bool wide_stream, bool post, const BlockNormArgs &a, hipStream_t stream) {
    if (dtype == 0) return post ? by_width<float>(a.D, L<float, true>{a, stream}) : by_width<float>(a.D, L<float, false>{a, stream});
    if (wide_stream) return post ? by_width<bf16>(a.D, L<float, true>{a, stream}) : by_width<bf16>(a.D, L<float, false>{a, stream});
    return post ? by_width<bf16>(a.D, L<bf16, true>{a, stream}) : by_width<bf16>(a.D, L<bf16, false>{a, stream});
}

} // namespace

// Rounds of a workgroup's rows up to which one workgroup has all of a backward pass and so its vectors' sums: it saves a launch and the partial sums' memory
// (block norm, 16 rows of 256: 4.3 us by one workgroup, 8.6 by two launches; output norm, 16 tokens of 4 heads: 5.6 and 10.0).
constexpr int kAloneRounds = 4;

int out_norm_bwd_blocks(int dtype, int d, int T, int H) {
    const long rows = (long)T * H, per = out_rows(dtype, d, kOutBwdBatch);
    return rows > kAloneRounds * per ? fewer((rows + per - 1) / per, 1024) : 1;
}
int block_norm_bwd_blocks(int dtype, int T, int D) {
    // Eight waves to a CU, so that their sums are few: with twice as many workgroups 4101 rows of 4104 (fp32 stream, normed and gated branch) take 110 us instead of 105, with half as many 16384 rows of 2048 in
    // bf16 118 instead of 101 (both passes).
    const int words = D / (dtype == 0 ? 4 : 8), rows = rows_of_workgroup(words);
    return T > kAloneRounds * rows ? fewer(((long)T + rows - 1) / rows, words > 512 ? 256 : 512) : 1;
}

namespace {
bool past_caches(long elements, bool wide) { return elements * (wide ? 4 : 2) > kPastCaches; }
} // namespace

int run_out_norm_fwd(int dtype, int d, const OutNormArgs &a, hipStream_t stream) { return a.T == 0 ? 0 : by_head(dtype, d, OutFwd{a, stream}); }
int run_out_norm_bwd(int dtype, int d, const OutNormArgs &a, hipStream_t stream) {
    OutNormArgs b = a;
    b.once = past_caches((long)a.T * a.H * d, dtype == 0);
    return a.T == 0 && !a.dw ? 0 : by_head(dtype, d, OutBwd{b, stream});
}
int run_block_norm_fwd(int dtype, bool wide_stream, bool post, const BlockNormArgs &a, hipStream_t stream) {
    BlockNormArgs b = a;
    b.once = past_caches((long)a.T * a.D, dtype == 0 || wide_stream);
    return a.T == 0 ? 0 : block_norm<BlockFwd>(dtype, wide_stream, post, b, stream);
}
int run_block_norm_bwd(int dtype, bool wide_stream, bool post, const BlockNormArgs &a, hipStream_t stream) {
    BlockNormArgs b = a;
    b.once = past_caches((long)a.T * a.D, dtype == 0 || wide_stream);
    return a.T == 0 && !a.dw && !a.dgate ? 0 : block_norm<BlockBwd>(dtype, wide_stream, post, b, stream);
}

} // namespace dn
