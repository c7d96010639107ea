// The short causal convolution in front of a mixer, per channel c with W taps, and its gradient:
//
//     z_t = b + sum_j w_j X_{t-W+1+j} ,  y = z or z sigmoid(z) ;   X: the sequence's rows, in front of them those of initial_state (or zeros)
//     dz = dy act'(z) ,  dX_e = sum_j w_{W-1-j} dz_{e+j} ,  dw_j = sum_t dz_t X_{t-W+1+j} ,  db = sum_t dz_t
//
// A sequence's W - 1 last rows are its final_state; rows in front of it take their gradient to dinitial_state, and a gradient with respect to final_state is
// added to those rows' own.  z is formed again in the backward pass (W products an element, where keeping it would be another tensor of traffic).
//
// Bound by HBM: 16384 rows of 6144 channels in bf16 take 72 us forward (403 MB, 5.6 TB/s), 124 backward (604 MB, 4.9 TB/s) and 5 for the weights' sums under a trace, 193 together without (5.2 TB/s).  Workgroups that follow each other have neighbouring columns of the same
// rows, so that what is under way at a time is whole rows (the other way round, with a kilobyte of a row each, 237 us for both passes instead of 218), and outputs are stored past the caches (193).
// A wave has V channels per lane and walks down a strip of a sequence's rows with the W - 1 rows behind it in registers, so that a row is fetched once, and W - 1
// more at the ends of a strip.  Strips are cut from each sequence's start: strip i of sequence n is at slot cu[n] / S + n + i, slots that are left over have
// nothing to do, and the place of a slot is found by a search of the offsets alone.  Only a sequence's first strip touches its states, which may so be updated in place.
#include "dn_layer_device.hpp"

namespace dn {

struct Strip {
    int n, row0, len;      // the sequence, its first row in the tensors and its length
    int first, rows;       // this strip's rows, counted from row0
    bool none;             // rows that lie in no sequence
};

__device__ inline int strips_of(int len, int S) { return len > S ? (len + S - 1) / S : 1; }

// The strip at a slot (the wave's); false where there is none.  Whatever the offsets hold, its rows lie in the tensors.
__device__ inline bool strip_at(const ConvArgs &a, int S, int slot, Strip *s) {
    int i;
    if (!a.cu) {
        const int per = strips_of(a.L, S);
        s->n = slot / per;
        i = slot - s->n * per;
        if (s->n >= a.N) return false;
        s->row0 = s->n * a.L;
        s->len = a.L;
        s->none = false;
    } else {
        // rows in front of the first sequence and behind the last one count as sequences, too: offsets 0, cu[0], .. cu[N], T
        auto offset = [&](int k) { return k == 0 ? 0 : k == a.N + 2 ? a.T : min(max(a.cu[k - 1], 0), a.T); };
        const int lane = threadIdx.x & 63;
        int k; // the answer, the last one with offset(k) / S + k <= slot
        if (a.N + 3 <= 64) { // (one fetch)
            const int own = offset(min(lane, a.N + 2));
            k = __builtin_popcountll(__ballot(lane <= a.N + 1 && own / S + lane <= slot)) - 1;
            k = max(k, 0);
            s->row0 = __builtin_amdgcn_readlane(own, k);
            s->len = max(__builtin_amdgcn_readlane(own, k + 1) - s->row0, 0);
        } else {
            int lo = 0, hi = a.N + 1; // it lies in [lo, hi]
            while (lo < hi) {
                const int step = (hi - lo + 63) >> 6, at = lo + (lane + 1) * step;
                const bool over = at <= hi && offset(min(at, hi)) / S + at <= slot;
                lo += __builtin_popcountll(__ballot(over)) * step;
                hi = min(hi, lo + step - 1);
            }
            k = __builtin_amdgcn_readfirstlane(lo);
            s->row0 = offset(k);
            s->len = max(offset(k + 1) - s->row0, 0);
        }
        s->n = k - 1;
        s->none = k == 0 || k == a.N + 1;
        i = slot - (s->row0 / S + k);
        if (i < 0 || (s->none && s->len == 0)) return false;
    }
    if (i >= strips_of(s->len, S)) return false;
    s->first = i * S;
    s->rows = min(S, s->len - s->first);
    return true;
}

// The lane's channels: their part, the place in it, and whether it is activated.
struct Lane {
    int c, part, width, off;
    bool live, silu;
    template <int V> __device__ inline void find(const ConvArgs &a) {
        c = (blockIdx.x * 64 + (threadIdx.x & 63)) * V;
        live = c < a.C;
        c = live ? c : a.C - V; // (loads what another lane has, stores nothing)
        part = (c >= a.at[1]) + (c >= a.at[2]);
        off = c - (part == 0 ? 0 : part == 1 ? a.at[1] : a.at[2]);
        width = part == 0 ? a.at[1] : part == 1 ? a.at[2] - a.at[1] : a.at[3] - a.at[2];
        silu = a.silu >> part & 1;
    }
    template <typename P> __device__ inline P *of(P *const (&p)[kMostParts]) const { return part == 0 ? p[0] : part == 1 ? p[1] : p[2]; }
};

template <typename T, int W, int V> struct Taps {
    Word<T, V> w[W]; // V W weights as they lie in memory: channel v's are elements v W ..
    Word<T, V> b;
    __device__ inline void load(const ConvArgs &a, int c) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i].load(static_cast<const T *>(a.w) + (long)c * W + i * V);
        if (a.b) b.load(static_cast<const T *>(a.b) + c);
        else b.zero();
    }
    __device__ inline float get(int v, int j) const { return w[(v * W + j) / V].get((v * W + j) % V); }
};

// Rows of a strip of the forward pass (R), and where sequences have few rows.
constexpr int kFwdRows = 8, kFewRows = 4;
template <typename T, int W, int V, int R>
__global__ __launch_bounds__(256) void k_short_conv_fwd(ConvArgs a, int slots) {
    Lane ln;
    ln.find<V>(a);
    Taps<T, W, V> taps;
    taps.load(a, ln.c);
    const bool act = __any(ln.silu);
    const T *x = static_cast<const T *>(a.x) + ln.c;
    T *y = static_cast<T *>(ln.of(a.y)) + ln.off;
    for (int slot = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); slot < slots; slot += gridDim.y * 4) {
        Strip s;
        if (!strip_at(a, R, slot, &s)) continue;
        T *to = y + (long)(s.row0 + s.first) * ln.width;
        if (s.none) {
            Word<T, V> zero;
            zero.zero();
            for (int r = 0; r < s.rows; ++r)
                if (ln.live) zero.store(to + (long)r * ln.width);
            continue;
        }
        Word<T, V> in[W - 1 + R];
        const T *from = x + s.row0 * a.x_stride;
        const long state = (long)s.n * (W - 1) * a.C + ln.c;
#pragma unroll
        for (int r = 0; r < R; ++r) in[W - 1 + r].zero();
        if (s.rows > 0)
#pragma unroll
            for (int r = 0; r < R; ++r) in[W - 1 + r].load(from + (s.first + min(r, s.rows - 1)) * a.x_stride);
        if (s.first > 0) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) in[j].load(from + (s.first - (W - 1) + j) * a.x_stride);
        } else {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                if (a.s0) in[j].load(static_cast<const T *>(a.s0) + state + (long)j * a.C);
                else in[j].zero();
            }
            if (a.sT) {
                Word<T, V> last[W - 1];
#pragma unroll
                for (int j = 0; j < W - 1; ++j) {
                    const int e = s.len - (W - 1) + j;
                    if (e >= 0) last[j].load(from + e * a.x_stride);
                    else {
                        last[j] = in[0];
#pragma unroll
                        for (int i = 1; i < W - 1; ++i)
                            if (W - 1 + e == i) last[j] = in[i];
                    }
                }
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
                    if (ln.live) last[j].store(static_cast<T *>(a.sT) + state + (long)j * a.C);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (R > kFewRows || r < s.rows) { // (in a long strip the branch costs more than the last strip's missing rows)
                float z[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    z[v] = taps.b.get(v);
#pragma unroll
                    for (int j = 0; j < W; ++j) z[v] = fmaf(taps.get(v, j), in[r + j].get(v), z[v]);
                }
                if (act)
#pragma unroll
                    for (int v = 0; v < V; ++v) z[v] = ln.silu ? z[v] * sigmoid_fast_f32(z[v]) : z[v];
                Word<T, V> out;
                out.pack(z);
                if (ln.live && r < s.rows) {
                    if constexpr (R > kFewRows) out.store_once(to + (long)r * ln.width);
                    else out.store(to + (long)r * ln.width);
                }
            }
    }
}

// Rows that are requested together in the backward pass; strips are S rows, a multiple of it.
constexpr int kBwdBatch = 8;


template <typename T, int W, int V>
__global__ __launch_bounds__(256) void k_short_conv_bwd(ConvArgs a, int slots, int S) {
    constexpr int K = (W + 1) * V;
    __shared__ float part[3][K][64];
    Lane ln;
    ln.find<V>(a);
    Taps<T, W, V> taps;
    taps.load(a, ln.c);
    const bool act = __any(ln.silu);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const T *x = static_cast<const T *>(a.x) + ln.c, *dy = static_cast<const T *>(ln.of(a.dy)) + ln.off;
    T *dx = static_cast<T *>(a.dx) + ln.c;
    float dw[W][V], db[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        db[v] = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][v] = 0.f;
    }
    for (int slot = blockIdx.y * 4 + wave; slot < slots; slot += gridDim.y * 4) {
        Strip s;
        if (!strip_at(a, S, slot, &s)) continue;
        T *to = dx + s.row0 * a.dx_stride;
        if (s.none) {
            Word<T, V> zero;
            zero.zero();
            for (int r = 0; r < s.rows; ++r)
                if (ln.live) zero.store(to + (s.first + r) * a.dx_stride);
            continue;
        }
        const T *from = x + s.row0 * a.x_stride, *grad = dy + (long)s.row0 * ln.width;
        const long state = (long)s.n * (W - 1) * a.C + ln.c;
        const int own = s.first + s.rows, tail = s.len - (W - 1); // rows below `own` are this strip's; final_state's are those from `tail` on
        float xw[W][V], zw[W][V]; // the last W rows of X and of dz, the present one last
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            Word<T, V> w;
            if (s.first > 0) w.load(from + (s.first - (W - 1) + j) * a.x_stride);
            else if (a.s0) w.load(static_cast<const T *>(a.s0) + state + (long)j * a.C);
            else w.zero();
            w.unpack(xw[j + 1]);
#pragma unroll
            for (int v = 0; v < V; ++v) zw[j + 1][v] = 0.f;
        }
        for (int t0 = s.first; t0 < own + W - 1; t0 += kBwdBatch) {
            Word<T, V> xr[kBwdBatch], gr[kBwdBatch];
#pragma unroll
            for (int u = 0; u < kBwdBatch; ++u) { xr[u].zero(); gr[u].zero(); }
            if (s.len > 0)
#pragma unroll
                for (int u = 0; u < kBwdBatch; ++u) {
                    const int t = min(t0 + u, min(own + W - 2, s.len - 1));
                    xr[u].load(from + t * a.x_stride);
                    gr[u].load(grad + (long)t * ln.width);
                }
#pragma unroll
            for (int u = 0; u < kBwdBatch; ++u) {
                const int t = t0 + u, e = t - (W - 1);
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) { xw[j][v] = xw[j + 1][v]; zw[j][v] = zw[j + 1][v]; }
                xr[u].unpack(xw[W - 1]);
                gr[u].unpack(zw[W - 1]);
                if (act)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float z = taps.b.get(v);
#pragma unroll
                        for (int j = 0; j < W; ++j) z = fmaf(taps.get(v, j), xw[j][v], z);
                        const float g = sigmoid_fast_f32(z), d = g * fmaf(z, 1.f - g, 1.f);
                        zw[W - 1][v] *= ln.silu ? d : 1.f;
                    }
#pragma unroll
                for (int v = 0; v < V; ++v) zw[W - 1][v] = t < s.len ? zw[W - 1][v] : 0.f;
                if (t < own)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        db[v] += zw[W - 1][v];
#pragma unroll
                        for (int j = 0; j < W; ++j) dw[j][v] = fmaf(zw[W - 1][v], xw[j][v], dw[j][v]);
                    }
                if (e < own && (e >= s.first || (e < 0 && a.ds0))) { // (the strip before has the rows in front)
                    float d[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        d[v] = 0.f;
#pragma unroll
                        for (int j = 0; j < W; ++j) d[v] = fmaf(taps.get(v, W - 1 - j), zw[j][v], d[v]);
                    }
                    if (a.dsT && e >= tail) {
                        Word<T, V> w;
                        w.load(static_cast<const T *>(a.dsT) + state + (long)(e - tail) * a.C);
#pragma unroll
                        for (int v = 0; v < V; ++v) d[v] += w.get(v);
                    }
                    Word<T, V> out;
                    out.pack(d);
                    if (ln.live) {
                        if (e >= 0) out.store_once(to + e * a.dx_stride);
                        else out.store(static_cast<T *>(a.ds0) + state + (long)(W - 1 + e) * a.C);
                    }
                }
            }
        }
    }
    if (!a.partial && !a.dw && !a.db) return;
    // the four waves' sums, in their order
    if (wave)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            part[wave - 1][W * V + v][lane] = db[v];
#pragma unroll
            for (int j = 0; j < W; ++j) part[wave - 1][v * W + j][lane] = dw[j][v];
        }
    __syncthreads();
    if (wave || !ln.live) return;
    const bool alone = gridDim.y == 1; // (then these are the gradients)
    float *tw = alone ? a.dw : a.partial + (long)blockIdx.y * ((long)a.C * (W + 1)), *tb = alone ? a.db : tw + (long)a.C * W;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (tw)
#pragma unroll
            for (int j = 0; j < W; ++j) tw[(long)(ln.c + v) * W + j] = ((dw[j][v] + part[0][v * W + j][lane]) + part[1][v * W + j][lane]) + part[2][v * W + j][lane];
        if (tb) tb[ln.c + v] = ((db[v] + part[0][W * V + v][lane]) + part[1][W * V + v][lane]) + part[2][W * V + v][lane];
    }
}

// Sums of partial vectors: E elements a workgroup, P = 1024 / E threads for each, the p-th of which has vectors p, p + P, ..
template <int E>
__global__ __launch_bounds__(1024) void k_sum_partials(const float *partial, int count, long n, long n1, float *out1, float *out2) {
    constexpr int P = 1024 / E;
    __shared__ float part[P][E + 1];
    const int i = threadIdx.x % E, p = threadIdx.x / E;
    const long e = (long)blockIdx.x * E + i;
    float *to = e < n1 ? out1 + e : out2 ? out2 + (e - n1) : nullptr;
    const bool live = e < n && (e < n1 ? out1 != nullptr : out2 != nullptr);
    float s = 0.f;
    if (live)
#pragma unroll 4
        for (int k = p; k < count; k += P) s += partial[k * n + e];
    part[p][i] = s;
    __syncthreads();
    if (p || !live) return;
    for (int k = 1; k < P; ++k) s += part[k][i];
    *to = s;
}

namespace {

int launch(const char *name, const void *fn, dim3 grid, int threads, void **args, hipStream_t stream) {
    prof_begin(name, stream);
    const hipError_t e = hipLaunchKernel(fn, grid, dim3(threads), args, 0, stream);
    prof_end(stream);
    return (int)e;
}

// Slots of strips of S rows (see strip_at).
long slots_of(const ConvArgs &a, int S) {
    if (!a.cu) return (long)a.N * (a.L > S ? (a.L + S - 1) / S : 1);
    return (long)a.T / S + a.N + 2;
}
int column_blocks(const ConvArgs &a, int V) { return (a.C / V + 63) / 64; }

constexpr int kMostBlocks = 1 << 15; // along the rows; waves go on to further slots

// Bytes of a row that a lane has: 16 forward and 8 backward (more registers), half of that where there are no two waves for each SIMD, which a strip's instructions then keep busy longer than the memory does
// (32 sequences of one row of 6144 channels, backward: 6.1 us instead of 8.6).
constexpr long kFewWaves = 2048;

template <typename T, int W, int R> const void *fwd_of(bool thin) {
    return thin ? reinterpret_cast<const void *>(k_short_conv_fwd<T, W, 8 / (int)sizeof(T), R>) : reinterpret_cast<const void *>(k_short_conv_fwd<T, W, 16 / (int)sizeof(T), R>);
}
template <typename T, int W> int launch_fwd(ConvArgs a, hipStream_t stream) {
    const bool few = (long)a.T <= (long)kFewRows * a.N;
    int slots = (int)slots_of(a, few ? kFewRows : kFwdRows);
    if (!slots) return 0;
    const bool thin = (long)slots * column_blocks(a, 16 / (int)sizeof(T)) < kFewWaves;
    const int blocks = (slots + 3) / 4, columns = column_blocks(a, (thin ? 8 : 16) / (int)sizeof(T));
    void *args[] = {&a, &slots};
    return launch("k_short_conv_fwd", few ? fwd_of<T, W, kFewRows>(thin) : fwd_of<T, W, kFwdRows>(thin), dim3(columns, blocks < kMostBlocks ? blocks : kMostBlocks), 256, args, stream);
}

// The backward pass's split.  Strips are as long as there are 4096 of them and columns.  Workgroups along the rows: up to 1024 in all, or 64 where there are many columns (their sums are traffic, too):
// 16000 rows of 64 channels, both passes, by 64 workgroups 42 us, by 500 16.
struct BwdPlan { int strip, slots, blocks, columns; bool thin; };
BwdPlan bwd_plan(int dtype, const ConvArgs &a) {
    const int V = dtype == 0 ? 2 : 4, wide = column_blocks(a, V);
    BwdPlan p;
    p.strip = 64;
    while (p.strip > kBwdBatch && (long)a.T / p.strip * wide < 4096) p.strip /= 2;
    p.slots = (int)slots_of(a, p.strip);
    p.thin = (long)p.slots * wide < kFewWaves;
    p.columns = p.thin ? column_blocks(a, V / 2) : wide;
    const int blocks = (p.slots + 3) / 4, most = 1024 / p.columns > 64 ? 1024 / p.columns : 64;
    p.blocks = blocks < 1 ? 1 : blocks < most ? blocks : most; // (with no sequence the gradients of weight and bias are zero)
    return p;
}

template <typename T, int W> int launch_bwd(ConvArgs a, hipStream_t stream) {
    BwdPlan p = bwd_plan(sizeof(T) == 4 ? 0 : 1, a);
    void *args[] = {&a, &p.slots, &p.strip};
    const void *fn = p.thin ? reinterpret_cast<const void *>(k_short_conv_bwd<T, W, 4 / (int)sizeof(T)>) : reinterpret_cast<const void *>(k_short_conv_bwd<T, W, 8 / (int)sizeof(T)>);
    const int e = launch("k_short_conv_bwd", fn, dim3(p.columns, p.blocks), 256, args, stream);
    if (e || p.blocks == 1 || (!a.dw && !a.db)) return e;
    return run_sum_partials(a.partial, p.blocks, (long)a.C * (W + 1), (long)a.C * W, a.dw, a.db, stream);
}

} // namespace

int short_conv_bwd_blocks(int dtype, const ConvArgs &a) { return bwd_plan(dtype, a).blocks; }

int run_short_conv_fwd(int dtype, const ConvArgs &a, hipStream_t stream) {
    if (dtype == 0) return a.W == 2 ? launch_fwd<float, 2>(a, stream) : a.W == 3 ? launch_fwd<float, 3>(a, stream) : launch_fwd<float, 4>(a, stream);
    return a.W == 2 ? launch_fwd<bf16, 2>(a, stream) : a.W == 3 ? launch_fwd<bf16, 3>(a, stream) : launch_fwd<bf16, 4>(a, stream);
}
int run_short_conv_bwd(int dtype, const ConvArgs &a, hipStream_t stream) {
    if (dtype == 0) return a.W == 2 ? launch_bwd<float, 2>(a, stream) : a.W == 3 ? launch_bwd<float, 3>(a, stream) : launch_bwd<float, 4>(a, stream);
    return a.W == 2 ? launch_bwd<bf16, 2>(a, stream) : a.W == 3 ? launch_bwd<bf16, 3>(a, stream) : launch_bwd<bf16, 4>(a, stream);
}

int run_sum_partials(const float *partial, int count, long n, long n1, float *out1, float *out2, hipStream_t stream) {
    void *args[] = {&partial, &count, &n, &n1, &out1, &out2};
    const bool wide = n >= 16384;
    const int E = wide ? 64 : 16;
    return launch("k_sum_partials", wide ? reinterpret_cast<const void *>(k_sum_partials<64>) : reinterpret_cast<const void *>(k_sum_partials<16>),
                  dim3((unsigned)((n + E - 1) / E)), 1024, args, stream);
}

} // namespace dn
