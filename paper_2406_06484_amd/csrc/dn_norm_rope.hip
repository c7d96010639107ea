// The pass between an attention layer's projections and the attention: RMS norm of every head's query and key with the position
// rotation, its gradient, and the serving forms that quantise k and v and write them to the paged cache, or read them back.
//
// With r = 1 / sqrt(mean(x^2) + eps), xhat = r x, z = xhat * w and the rotation R of a position (orthogonal on its pairs),
//
//     y = R z ;    backward:  dz = R^T dy ,  dw = sum dz * xhat ,  g = dz * w ,  dx = r (g - xhat mean(g * xhat)).
//
// Everything is bound by HBM (about ten operations per element of two or four bytes): each row is read once, in 16-byte words,
// and written once.  A row of one head is D * sizeof(T) / 16 lanes wide, so a wave holds 64 * 16 / (D * sizeof(T)) heads of one
// token at a time and its sums are lane swaps inside a row.  A wave stays with one token and one tensor (q, k or v is
// blockIdx.y), so that the token's cosines and sines and the weight are fetched once for all heads.
#include "dn_attn_device.hpp"

namespace dn {

template <typename T, int D> struct RowLayout {
    static constexpr int V = 16 / (int)sizeof(T); // elements per lane
    static constexpr int LPR = D / V;             // lanes per row
    static constexpr int RPW = 64 / LPR;          // rows (heads) per wave and step
};

// What a lane needs to turn its V elements: out_i = own_i c_i + other_i s_i, where `other` is the pair's other element and the
// sign is in s; the transposed turn is own_i c_i - other_i s_i.  Elements past the rotated ones have c = 1, s = 0.
// IL: pairs are neighbours, else halves.
template <int V, bool IL> struct Turn {
    float c[V], s[V];
    int from; // the lane that holds the others (halves); unused for neighbours
    __device__ static inline const float *row_of(const RowArgs &a, int pos) { return a.cs + (long)min(max(pos, 0), a.max_pos - 1) * a.rot; }
    __device__ inline void load(const RowArgs &a, int e0, const float *row) {
        const int lane = threadIdx.x & 63, half = a.rot >> 1;
        from = lane;
#pragma unroll
        for (int i = 0; i < V; ++i) { c[i] = 1.f; s[i] = 0.f; }
        if (e0 >= a.rot) return;
        if constexpr (IL) {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float co = row[e0 / 2 + i], si = row[half + e0 / 2 + i];
                c[2 * i] = c[2 * i + 1] = co;
                s[2 * i] = -si; s[2 * i + 1] = si;
            }
            return;
        }
        const bool second = e0 >= half;
        const int at = second ? e0 - half : e0;
        from = second ? lane - half / V : lane + half / V;
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 co = *reinterpret_cast<const float4 *>(row + at + i), si = *reinterpret_cast<const float4 *>(row + half + at + i);
            c[i] = co.x; c[i + 1] = co.y; c[i + 2] = co.z; c[i + 3] = co.w;
            s[i] = second ? si.x : -si.x; s[i + 1] = second ? si.y : -si.y; s[i + 2] = second ? si.z : -si.z; s[i + 3] = second ? si.w : -si.w;
        }
    }
    // the others of the elements in word w (the whole wave takes part)
    template <typename T> __device__ inline void others(const uint4 &w, const float (&own)[V], float (&o)[V]) const {
        if constexpr (IL) {
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = own[i ^ 1];
            return;
        }
        auto get = [this](unsigned v) { return (unsigned)__builtin_amdgcn_ds_bpermute(4 * from, (int)v); };
        unpack16<T>(make_uint4(get(w.x), get(w.y), get(w.z), get(w.w)), o);
    }
};

template <typename T, int V> __device__ inline void load_weight(const void *w, int e0, float (&f)[V]) {
    if (w) unpack16<T>(*reinterpret_cast<const uint4 *>(static_cast<const T *>(w) + e0), f);
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = 1.f;
    }
}

// Waves of the workgroup that has all of a tensor's gradient to itself, its steps (of a wave's rows) under way together, and the elements per lane, in rounds of those, up to
// which it has: it saves a launch, but has one CU.  Backward alone, by one workgroup per tensor and by two launches, in us: fp32, 2 + 2 heads of 64, three rounds (192 tokens) 8.2 and 10.6,
// four 9.4 and 10.8, five 11.0 and 10.7, six 12.7 and 10.8; bf16, 16 + 16 heads of 128 (eight elements a lane), one round (8 tokens) 7.8 and 10.5, two 8.2 and 10.5, three 10.6 and 10.4, four 12.9
// and 10.5; other numbers and sizes of heads within 0.3 of these.
constexpr int kAloneWaves = 16, kAloneBatch = 2, kAloneElements = 16;

// Loads of up to this many steps (64 / lanes of a row heads each) are requested before the first is worked on.
constexpr int kRowBatch = 4;

// The weight at the lane's elements and at their pairs' other ones.
template <typename T, int D, bool IL> struct Weights {
    using L = RowLayout<T, D>;
    float w[L::V], wo[L::V];
    __device__ inline void load(const RowArgs &a, const void *weight, int e0) {
        load_weight<T>(weight, e0, w);
        if (!IL && e0 < a.rot) load_weight<T>(weight, e0 < (a.rot >> 1) ? e0 + (a.rot >> 1) : e0 - (a.rot >> 1), wo);
        else {
#pragma unroll
            for (int i = 0; i < L::V; ++i) wo[i] = w[i ^ 1];
        }
    }
};

// y of a row: r (x c w + other s wo), with the factors of a token's heads formed once (they are the same for all of a tensor's heads, and the
// vector ALU, not only the memory, would bound a pass that forms them for each).
template <typename T, int D, bool IL> struct NormTurn {
    using L = RowLayout<T, D>;
    Turn<L::V, IL> turn; // c w, s wo
    __device__ inline void load(const RowArgs &a, const Weights<T, D, IL> &w, int e0, const float *row) {
        turn.load(a, e0, row);
#pragma unroll
        for (int i = 0; i < L::V; ++i) { turn.c[i] *= w.w[i]; turn.s[i] *= w.wo[i]; }
    }
    __device__ inline void apply(const RowArgs &a, const uint4 &x, float (&y)[L::V]) const {
        float own[L::V], oth[L::V], ss = 0.f;
        unpack16<T>(x, own);
#pragma unroll
        for (int i = 0; i < L::V; ++i) ss = fmaf(own[i], own[i], ss);
        const float r = rsqrtf(lanes_sum<L::LPR>(ss) * (1.f / D) + a.eps);
        turn.template others<T>(x, own, oth);
#pragma unroll
        for (int i = 0; i < L::V; ++i) y[i] = r * fmaf(own[i], turn.c[i], oth[i] * turn.s[i]);
    }
};

// y of every row.  16384 tokens of 16 + 16 heads of 128 in bf16 (268 MB): 47 us, 5.7 TB/s, the rate of a copy; 256 tokens of 2 + 2 of 64 in fp32: 3.2 us.
template <typename T, int D, bool IL>
__global__ __launch_bounds__(256) void k_norm_rope_fwd(RowArgs a) {
    using L = RowLayout<T, D>;
    const int lane = threadIdx.x & 63, e0 = (lane % L::LPR) * L::V, sub = lane / L::LPR;
    const bool is_q = blockIdx.y == 0;
    const int H = is_q ? a.Hq : a.Hkv;
    const long stride = is_q ? a.q_stride : a.k_stride;
    const T *in = static_cast<const T *>(is_q ? a.q : a.k);
    T *out = static_cast<T *>(is_q ? a.q_out : a.k_out);
    NormTurn<T, D, IL> nt;
    Weights<T, D, IL> w;
    w.load(a, is_q ? a.qw : a.kw, e0);
    for (int t = blockIdx.x * 4 + (threadIdx.x >> 6); t < a.T; t += gridDim.x * 4) {
        const T *row = in + t * stride;
        T *to = out + (long)t * H * D;
        nt.load(a, w, e0, nt.turn.row_of(a, a.positions ? a.positions[t] : t % a.seq_len));
        for (int h0 = 0; h0 < H; h0 += kRowBatch * L::RPW) {
            uint4 x[kRowBatch];
#pragma unroll
            for (int b = 0; b < kRowBatch; ++b) {
                const int h = h0 + b * L::RPW + sub;
                x[b] = h < H ? *reinterpret_cast<const uint4 *>(row + h * D + e0) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int b = 0; b < kRowBatch; ++b) {
                if (h0 + b * L::RPW >= H) break;
                const int h = h0 + b * L::RPW + sub;
                float y[L::V];
                nt.apply(a, x[b], y);
                if (h < H) *reinterpret_cast<uint4 *>(to + h * D + e0) = pack16<T>(y);
            }
        }
    }
}

// dx of a row, and its dz * xhat added to dw if it is one.
template <typename T, int D, bool IL>
__device__ __forceinline__ void row_gradient(const RowArgs &a, const Turn<RowLayout<T, D>::V, IL> &turn, const float (&w)[RowLayout<T, D>::V], const uint4 &x, const uint4 &g, bool is_row,
                                             float (&dw)[RowLayout<T, D>::V], float (&dx)[RowLayout<T, D>::V]) {
    using L = RowLayout<T, D>;
    float xf[L::V], own[L::V], oth[L::V], ss = 0.f, gx = 0.f;
    unpack16<T>(x, xf);
    unpack16<T>(g, own);
    turn.template others<T>(g, own, oth);
#pragma unroll
    for (int i = 0; i < L::V; ++i) {
        ss = fmaf(xf[i], xf[i], ss);
        own[i] = fmaf(own[i], turn.c[i], -oth[i] * turn.s[i]); // dz
        gx = fmaf(own[i] * w[i], xf[i], gx);
    }
    const float r = rsqrtf(lanes_sum<L::LPR>(ss) * (1.f / D) + a.eps);
    const float m = lanes_sum<L::LPR>(gx) * r * (1.f / D);
#pragma unroll
    for (int i = 0; i < L::V; ++i) {
        const float xh = xf[i] * r;
        if (is_row) dw[i] = fmaf(own[i], xh, dw[i]);
        dx[i] = r * fmaf(-xh, m, own[i] * w[i]);
    }
}

// Rows' gradients: 403 MB for the same tokens in 78 us, 5.2 TB/s.  The norm is formed again from x, which has to be read anyway.  Every workgroup also leaves its sum of dz * xhat,
// which k_weight_grad adds up in the workgroups' order (atomics would change the result from run to run); 512 workgroups, so that their sums are few.
template <typename T, int D, bool IL>
__global__ __launch_bounds__(256) void k_norm_rope_bwd(RowArgs a) {
    using L = RowLayout<T, D>;
    __shared__ float part[4][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e0 = (lane % L::LPR) * L::V, sub = lane / L::LPR;
    const bool is_q = blockIdx.y == 0;
    const int H = is_q ? a.Hq : a.Hkv;
    const long stride = is_q ? a.q_stride : a.k_stride;
    const T *in = static_cast<const T *>(is_q ? a.q : a.k), *grad = static_cast<const T *>(is_q ? a.dq_out : a.dk_out);
    T *out = static_cast<T *>(is_q ? a.q_out : a.k_out);
    float w[L::V], dw[L::V];
    load_weight<T>(is_q ? a.qw : a.kw, e0, w);
#pragma unroll
    for (int i = 0; i < L::V; ++i) dw[i] = 0.f;
    Turn<L::V, IL> turn;
    for (int t = blockIdx.x * 4 + wave; t < a.T; t += gridDim.x * 4) {
        const T *row = in + t * stride, *dy = grad + (long)t * H * D;
        T *to = out + (long)t * H * D;
        turn.load(a, e0, turn.row_of(a, a.positions ? a.positions[t] : t % a.seq_len));
        for (int h0 = 0; h0 < H; h0 += kRowBatch * L::RPW) {
            uint4 x[kRowBatch], g[kRowBatch];
#pragma unroll
            for (int b = 0; b < kRowBatch; ++b) {
                const int h = h0 + b * L::RPW + sub;
                x[b] = h < H ? *reinterpret_cast<const uint4 *>(row + h * D + e0) : make_uint4(0, 0, 0, 0);
                g[b] = h < H ? *reinterpret_cast<const uint4 *>(dy + h * D + e0) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int b = 0; b < kRowBatch; ++b) {
                if (h0 + b * L::RPW >= H) break;
                const int h = h0 + b * L::RPW + sub;
                float dx[L::V];
                row_gradient<T, D, IL>(a, turn, w, x[b], g[b], h < H, dw, dx);
                if (h < H) *reinterpret_cast<uint4 *>(to + h * D + e0) = pack16<T>(dx);
            }
        }
    }
    if (!a.partial) return;
    // the wave's rows side by side, then the four waves
#pragma unroll
    for (int i = 0; i < L::V; ++i) {
#pragma unroll
        for (int m = L::LPR; m < 64; m <<= 1) dw[i] += __shfl_xor(dw[i], m);
        if (sub == 0) part[wave][e0 + i] = dw[i];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < D; e += 256)
        a.partial[((long)blockIdx.x * 2 + blockIdx.y) * D + e] = (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
}

// The same for few tokens, a workgroup per tensor (blockIdx.x), which so has the weight's gradient, too.  Rows (token and head) stand side by side in a wave, whatever
// the number of heads.
template <typename T, int D, bool IL>
__global__ __launch_bounds__(64 * kAloneWaves) void k_norm_rope_bwd_alone(RowArgs a) {
    using L = RowLayout<T, D>;
    __shared__ float part[kAloneWaves][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e0 = (lane % L::LPR) * L::V, sub = lane / L::LPR;
    const bool is_q = blockIdx.x == 0;
    const int H = is_q ? a.Hq : a.Hkv, rows = a.T * H;
    const long stride = is_q ? a.q_stride : a.k_stride;
    const T *in = static_cast<const T *>(is_q ? a.q : a.k), *grad = static_cast<const T *>(is_q ? a.dq_out : a.dk_out);
    T *out = static_cast<T *>(is_q ? a.q_out : a.k_out);
    float w[L::V], dw[L::V];
    load_weight<T>(is_q ? a.qw : a.kw, e0, w);
#pragma unroll
    for (int i = 0; i < L::V; ++i) dw[i] = 0.f;
    for (int r0 = wave * kAloneBatch * L::RPW; r0 < rows; r0 += kAloneWaves * kAloneBatch * L::RPW) {
        uint4 x[kAloneBatch], g[kAloneBatch];
        Turn<L::V, IL> turn[kAloneBatch];
#pragma unroll
        for (int b = 0; b < kAloneBatch; ++b) {
            const int r = min(r0 + b * L::RPW + sub, rows - 1), t = r / H;
            x[b] = *reinterpret_cast<const uint4 *>(in + t * stride + (r - t * H) * D + e0);
            g[b] = *reinterpret_cast<const uint4 *>(grad + (long)r * D + e0);
            turn[b].load(a, e0, turn[b].row_of(a, a.positions ? a.positions[t] : t % a.seq_len));
        }
#pragma unroll
        for (int b = 0; b < kAloneBatch; ++b) {
            const int r = r0 + b * L::RPW + sub;
            float dx[L::V];
            row_gradient<T, D, IL>(a, turn[b], w, x[b], g[b], r < rows, dw, dx);
            if (r < rows) *reinterpret_cast<uint4 *>(out + (long)r * D + e0) = pack16<T>(dx);
        }
    }
    float *to = is_q ? a.dqw : a.dkw;
    if (!to) return;
#pragma unroll
    for (int i = 0; i < L::V; ++i) {
#pragma unroll
        for (int m = L::LPR; m < 64; m <<= 1) dw[i] += __shfl_xor(dw[i], m);
        if (sub == 0) part[wave][e0 + i] = dw[i];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < D; e += 64 * kAloneWaves) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kAloneWaves; ++i) s += part[i][e];
        to[e] = s;
    }
}

// Sums the workgroups' partial weight gradients: 64 threads per element, each every 64th partial.  A launch's time, 3 to 5 us.
__global__ __launch_bounds__(1024) void k_weight_grad(RowArgs a, int D, int blocks) {
    __shared__ float part[64][17];
    const int e = blockIdx.x * 16 + (threadIdx.x & 15), of = threadIdx.x >> 4; // D is a multiple of 16
    float *to = blockIdx.y == 0 ? a.dqw : a.dkw;
    if (!to) return;
    float s = 0.f;
#pragma unroll 8
    for (int b = of; b < blocks; b += 64) s += a.partial[((long)b * 2 + blockIdx.y) * D + e];
    part[of][threadIdx.x & 15] = s;
    __syncthreads();
    if (of == 0) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 64; ++i) s += part[i][threadIdx.x];
        to[e] = s;
    }
}

// The position of the wave's packed row t of sequence n, counted back from the context's end whether or not the table has room for all of it.
__device__ inline int position_of(const PagedArgs &c, int n, int t) {
    const long pos = (long)c.kv_len[n] - c.cu[n + 1] + t;
    return (int)(pos < -1 ? -1 : pos > 0x7fffffff ? 0x7fffffff : pos);
}
// Where it stands in the cache; false for a row that has no place there.
struct Slot { long base; int stride; }; // of head 0, in rows of d elements; rows between heads
__device__ inline bool slot_of(const PagedArgs &c, int n, int pos, int Hkv, bool clamp, Slot *s) {
    if (pos < 0 || pos >= c.max_kv) return false; // (max_kv tokens need max_pages pages at most)
    int id = c.table[(long)n * c.max_pages + (pos >> c.page_shift)];
    if (clamp) id = min(max(id, 0), c.num_pages - 1);
    else if (id < 0 || id >= c.num_pages) return false;
    s->base = (((long)id * Hkv) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
    s->stride = 1 << c.page_shift;
    return true;
}

// Where the wave's rows of one tensor go: a descriptor from the token's first head on that ends behind its last one (stores past it, of heads that
// are not there, and all stores of a token without a place are dropped; offsets stand in the vector operand alone, where the range is checked), this
// lane's offset, and the step between `RPW` heads.
struct Rows { __amdgpu_buffer_rsrc_t rs; int off, step; };

__device__ inline void store16(const Rows &to, int step, const uint4 &w) {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{w.x, w.y, w.z, w.w}, to.rs, to.off + step * to.step, 0, 0);
}

// Quantises the row that `y` is part of (LPR lanes) and writes it to the cache.
template <typename T, typename CT, int D>
__device__ inline void cache_row(const Rows &to, const Rows &scale, int step, int e0, const float (&y)[RowLayout<T, D>::V]) {
    using L = RowLayout<T, D>;
    if constexpr (__is_same(CT, fp8)) {
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < L::V; ++i) amax = fmaxf(amax, fabsf(y[i]));
        amax = lanes_max<L::LPR>(amax);
        // Quotients to the last bit (the product with the reciprocal, corrected once: rows of bf16 values meet ties often): amax / 448, then y / s.  A row
        // under 2^-100, whose factor would leave the range of normal numbers, is held as zeros.
        constexpr float c = 1.f / 448.f;
        float s = amax * c;
        s = amax < INFINITY ? fmaf(fmaf(-s, 448.f, amax), c, s) : amax;
        float inv = __builtin_amdgcn_rcpf(s);
        inv = fmaf(fmaf(-s, inv, 1.f), inv, inv);
        const bool none = amax < 0x1p-100f;
        s = none ? 0.f : s;
        inv = none || s == INFINITY ? 0.f : inv;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = y[i] * inv;
            v[i] = fmaf(fmaf(-x, s, y[i]), inv, x);
        }
        const uint2 w = to_fp8x8(v);
        typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{w.x, w.y}, to.rs, to.off + step * to.step, 0, 0);
        if (e0 == 0) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(s), scale.rs, scale.off + step * scale.step, 0, 0);
    } else if constexpr (__is_same(CT, fp4)) {
        // A group's factor is a power of two: quotients are exact but for the one rounding to e2m1, which the conversion does.
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < L::V; ++i) amax = fmaxf(amax, fabsf(y[i]));
        bool whole = amax < INFINITY;
#pragma unroll
        for (int i = 0; i < L::V; ++i) whole = whole && y[i] == y[i];
        amax = lanes_max<kGroup / L::V>(whole ? amax : INFINITY); // (a maximum passes over NaN)
        const unsigned byte = fp4_factor_byte(amax);
        const unsigned w = amax < 0x1p-100f ? 0u : to_fp4x8(y, fp4_factor(byte));
        __builtin_amdgcn_raw_buffer_store_b32(w, to.rs, to.off + step * to.step, 0, 0);
        if (e0 % kGroup == 0) __builtin_amdgcn_raw_buffer_store_b8((unsigned char)byte, scale.rs, scale.off + step * scale.step, 0, 0);
    } else store16(to, step, pack16<T>(y));
}

// The workgroup's four tokens; its part of their steps is blockIdx.y.  (A launch of 2^32 threads or more along one dimension of its grid is cut to the low 32 bits
// without an error, so workgroups past kGridRow stand in further rows.)
constexpr int kGridRowShift = 22, kGridRow = 1 << kGridRowShift;
__device__ inline int token_block() { return (blockIdx.z << kGridRowShift) + blockIdx.x; }

// New tokens: a wave takes up to kAppendSteps steps (a step: as many heads as a wave holds) of one token's q, k and v (q only with NORM, which also
// normalises and rotates k).  Finding the token's place takes three loads in a row (its sequence, the context's length, the page),
// and that latency, not the bytes, would be the time: all rows are requested before the search, and what the norm needs waits in the LDS, because a load
// issued behind the first stores would wait for those.  8192 tokens of 16 + 4 + 4 heads of 128 into e4m3 pages (94 MB): 21 to 22 us, 4.3 TB/s, the vector ALU (norm,
// rotation, maximum, quotients) busy for 0.37 of it, of 4 + 4 heads as they are into 4-bit pages (21 MB) 7.5; 32 single tokens of 16 + 16 + 16: 4.5 us.
constexpr int kAppendSteps = 2;
template <typename T, typename CT, int D, bool NORM, bool IL>
__global__ __launch_bounds__(256) void k_paged_append(RowArgs a, PagedArgs c, int per) {
    using L = RowLayout<T, D>;
    constexpr int ES = (int)sizeof(T), CB = Held<CT, D>::BYTES, FB = Held<CT, D>::FACTORS; // bytes of an element; of a row and of its factors in the cache
    __shared__ __align__(16) float turns[NORM ? 4 : 1][NORM ? D : 4];
    __shared__ __align__(16) T weight[NORM ? 2 : 1][NORM ? D : 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), e0 = (lane % L::LPR) * L::V, sub = lane / L::LPR;
    const int t = token_block() * 4 + wave;
    // steps: those of q, then k, then v
    const int sq = NORM ? (a.Hq + L::RPW - 1) / L::RPW : 0, skv = (a.Hkv + L::RPW - 1) / L::RPW;
    const int first = blockIdx.y * per, last = min(first + per, sq + 2 * skv);
    uint4 x[kAppendSteps];
    if (t < a.T) {
#pragma unroll
        for (int i = 0; i < kAppendSteps; ++i) {
            const int at = min(first + i, last - 1), what = at < sq ? 0 : at < sq + skv ? 1 : 2, step = at - (what == 0 ? 0 : what == 1 ? sq : sq + skv);
            const T *row = static_cast<const T *>(what == 0 ? a.q : what == 1 ? a.k : a.v) + t * (what == 0 ? a.q_stride : what == 1 ? a.k_stride : a.v_stride);
            const auto w = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(row, (what == 0 ? a.Hq : a.Hkv) * D * ES), ((sub + step * L::RPW) * D + e0) * ES, 0, 0);
            x[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    int n = c.N, pos = -1;
    Slot s{0, 0};
    bool live = false;
    if (t < a.T) n = seq_of_row(c.cu, c.N, t);
    if (n < c.N) {
        pos = position_of(c, n, t);
        live = slot_of(c, n, pos, a.Hkv, false, &s);
    }
    if constexpr (NORM) {
        if (first < sq + skv) {
            for (int i = threadIdx.x; i < 2 * D / L::V; i += 256) {
                const void *w = i < D / L::V ? a.qw : a.kw;
                float f[L::V];
                load_weight<T>(w, i % (D / L::V) * L::V, f);
                *reinterpret_cast<uint4 *>(&weight[i / (D / L::V)][i % (D / L::V) * L::V]) = pack16<T>(f);
            }
            if (a.rot && 4 * lane < a.rot)
                *reinterpret_cast<float4 *>(&turns[wave][4 * lane]) = *reinterpret_cast<const float4 *>(Turn<L::V, IL>::row_of(a, pos) + 4 * lane);
            __syncthreads();
        }
    }
    if (t >= a.T) return;
    NormTurn<T, D, IL> nt;
    int with = -1;
#pragma unroll
    for (int i = 0; i < kAppendSteps; ++i) {
        const int at = first + i;
        if (at < last) {
            const int what = at < sq ? 0 : at < sq + skv ? 1 : 2, step = at - (what == 0 ? 0 : what == 1 ? sq : sq + skv);
            float y[L::V];
            if (NORM && what != 2) {
                if (what != with) {
                    Weights<T, D, IL> w;
                    w.load(a, weight[what], e0);
                    nt.load(a, w, e0, turns[wave]);
                    with = what;
                }
                nt.apply(a, x[i], y);
            } else unpack16<T>(x[i], y);
            if (what == 0) {
                const Rows to{make_rsrc(static_cast<T *>(a.q_out) + (long)t * a.Hq * D, a.Hq * D * ES), (sub * D + e0) * ES, L::RPW * D * ES};
                store16(to, step, pack16<T>(y));
            } else { // head h of the token is row s.base + h s.stride
                const int rows = live ? (a.Hkv - 1) * s.stride + 1 : 0;
                const Rows to{make_rsrc(static_cast<char *>(what == 1 ? c.kp : c.vp) + s.base * CB, rows * CB), sub * s.stride * CB + e0 * CB / D, L::RPW * s.stride * CB};
                const Rows scale{make_rsrc(reinterpret_cast<char *>(what == 1 ? c.ks : c.vs) + s.base * FB, rows * FB), sub * s.stride * FB + (__is_same(CT, fp4) ? e0 / kGroup : 0), L::RPW * s.stride * FB};
                cache_row<T, CT, D>(to, scale, step, e0, y);
            }
        }
    }
}

// Tokens read back: a.T rows of output, c.cu their offsets.  A wave takes up to `per` steps (kReadSteps at most) of one token's k and v: finding the token's place, three loads in a row, is
// most of its time.  8192 tokens of 4 heads of 128 from e4m3 pages (27 MB, just written): 7 us.
constexpr int kReadSteps = 4;
template <typename T, typename CT, int D>
__global__ __launch_bounds__(256) void k_paged_read(RowArgs a, PagedArgs c, int per) {
    using L = RowLayout<T, D>;
    const int lane = threadIdx.x & 63, e0 = (lane % L::LPR) * L::V, sub = lane / L::LPR;
    const int t = token_block() * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    const int skv = (a.Hkv + L::RPW - 1) / L::RPW; // steps: those of k, then v
    const int first = blockIdx.y * per, last = min(first + per, 2 * skv);
    const int n = seq_of_row(c.cu, c.N, t);
    Slot s{0, 0};
    const bool live = n < c.N && slot_of(c, n, position_of(c, n, t), a.Hkv, true, &s);
    uint4 x[kReadSteps];
    float f[kReadSteps];
#pragma unroll
    for (int b = 0; b < kReadSteps; ++b) {
        const int at = first + b;
        const bool is_k = at < skv;
        const int h = (is_k ? at : at - skv) * L::RPW + sub;
        const long row = s.base + (long)h * s.stride;
        const void *pages = is_k ? c.kp : c.vp;
        x[b] = make_uint4(0, 0, 0, 0);
        f[b] = 0.f;
        if (live && at < last && h < a.Hkv) {
            if constexpr (__is_same(CT, fp8)) {
                const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const unsigned char *>(pages) + row * D + e0);
                x[b].x = w.x; x[b].y = w.y;
                f[b] = (is_k ? c.ks : c.vs)[row];
            } else if constexpr (__is_same(CT, fp4)) {
                x[b].x = *reinterpret_cast<const unsigned *>(static_cast<const unsigned char *>(pages) + row * (D / 2) + e0 / 2);
                f[b] = fp4_factor(reinterpret_cast<const unsigned char *>(is_k ? c.ks : c.vs)[row * (D / kGroup) + e0 / kGroup]);
            } else x[b] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(pages) + row * D + e0);
        }
    }
#pragma unroll
    for (int b = 0; b < kReadSteps; ++b) {
        const int at = first + b;
        if (at >= last) break;
        const bool is_k = at < skv;
        const int h = (is_k ? at : at - skv) * L::RPW + sub;
        if constexpr (__is_same(CT, fp8)) {
            float y[8];
            from_fp8x8(make_uint2(x[b].x, x[b].y), y);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= f[b];
            x[b] = pack16<T>(y);
        }
        if constexpr (__is_same(CT, fp4)) x[b] = __builtin_bit_cast(uint4, from_fp4x8(x[b].x, live ? f[b] : 1.f)); // (rows without a place: zeros)
        if (h < a.Hkv) *reinterpret_cast<uint4 *>(static_cast<T *>(is_k ? a.k_out : a.v_out) + ((long)t * a.Hkv + h) * D + e0) = x[b];
    }
}

namespace {

int launch(const char *name, const void *fn, dim3 grid, void **args, hipStream_t stream, int threads = 256) {
    prof_begin(name, stream);
    const hipError_t e = hipLaunchKernel(fn, grid, dim3(threads), args, 0, stream);
    prof_end(stream);
    return (int)e;
}

// One workgroup per four tokens up to the number that fills the chip, from where on they loop (and keep the weight).
int token_blocks(int T) { const int b = (T + 3) / 4; return b < 4096 ? b : 4096; }

// f<T, D>() for the given (dtype, d); with a cache fp32 ends at 128 and bf16 starts at 64, as the attention does
template <bool PAGED, typename F> int by_type(int dtype, int d, F f) {
    if (dtype == 0) {
        if (d == 32) return f.template operator()<float, 32>();
        if (d == 64) return f.template operator()<float, 64>();
        if (d == 128) return f.template operator()<float, 128>();
        if constexpr (!PAGED) if (d == 256) return f.template operator()<float, 256>();
    } else {
        if constexpr (!PAGED) if (d == 32) return f.template operator()<bf16, 32>();
        if (d == 64) return f.template operator()<bf16, 64>();
        if (d == 128) return f.template operator()<bf16, 128>();
        if (d == 256) return f.template operator()<bf16, 256>();
    }
    return (int)hipErrorInvalidValue;
}

struct FwdLaunch {
    RowArgs a;
    hipStream_t stream;
    template <typename T, int D> int operator()() {
        void *args[] = {&a};
        return launch("k_norm_rope_fwd", a.interleaved ? reinterpret_cast<const void *>(k_norm_rope_fwd<T, D, true>) : reinterpret_cast<const void *>(k_norm_rope_fwd<T, D, false>), dim3(token_blocks(a.T), 2), args, stream);
    }
};
struct BwdLaunch {
    RowArgs a;
    hipStream_t stream;
    template <typename T, int D, bool IL> static const void *of(bool alone) {
        return alone ? reinterpret_cast<const void *>(k_norm_rope_bwd_alone<T, D, IL>) : reinterpret_cast<const void *>(k_norm_rope_bwd<T, D, IL>);
    }
    template <typename T, int D> int operator()() {
        using L = RowLayout<T, D>;
        int blocks = norm_rope_bwd_blocks(a.T), d = D;
        const int H = a.Hq > a.Hkv ? a.Hq : a.Hkv;
        const long rows = (long)a.T * H, round = kAloneWaves * kAloneBatch * L::RPW;
        const bool alone = a.T > 0 && rows <= kAloneElements / L::V * round && (a.dqw || a.dkw);
        if (a.T > 0) {
            void *args[] = {&a};
            const void *fn = a.interleaved ? of<T, D, true>(alone) : of<T, D, false>(alone);
            const int e = alone ? launch("k_norm_rope_bwd", fn, dim3(2), args, stream, 64 * kAloneWaves) : launch("k_norm_rope_bwd", fn, dim3(blocks, 2), args, stream);
            if (e || alone) return e;
        }
        if (!a.dqw && !a.dkw) return 0;
        void *args[] = {&a, &d, &blocks};
        return launch("k_weight_grad", reinterpret_cast<const void *>(k_weight_grad), dim3(D / 16, 2), args, stream, 1024);
    }
};
// The grid of token_block.
dim3 token_grid(int T, int parts) {
    const int blocks = (T + 3) / 4;
    return dim3(blocks < kGridRow ? blocks : kGridRow, parts, (blocks + kGridRow - 1) / kGridRow);
}
// Steps of k_paged_append and k_paged_read per wave: all of a token's, in equal parts of at most `most`; one where there are few tokens.
template <typename T, int D> int steps_per_wave(int tokens, int Hq, int Hkv, int most, int *waves) {
    constexpr int RPW = RowLayout<T, D>::RPW;
    const int all = (Hq + RPW - 1) / RPW + 2 * ((Hkv + RPW - 1) / RPW);
    const int parts = tokens < 512 ? all : (all + most - 1) / most, per = (all + parts - 1) / parts;
    *waves = (all + per - 1) / per;
    return per;
}
struct AppendLaunch {
    RowArgs a;
    PagedArgs c;
    bool fp8_pages, norm;
    hipStream_t stream;
    template <typename T, int D, typename CT> const void *of() const {
        if (!norm) return reinterpret_cast<const void *>(k_paged_append<T, CT, D, false, false>);
        return a.interleaved ? reinterpret_cast<const void *>(k_paged_append<T, CT, D, true, true>) : reinterpret_cast<const void *>(k_paged_append<T, CT, D, true, false>);
    }
    template <typename T, int D> int operator()() {
        int waves, per = steps_per_wave<T, D>(a.T, norm ? a.Hq : 0, a.Hkv, kAppendSteps, &waves);
        void *args[] = {&a, &c, &per};
        const void *fn = of<T, D, T>();
        if constexpr (sizeof(T) == 2) {
            if (c.fp4) fn = of<T, D, fp4>();
            else if (fp8_pages) fn = of<T, D, fp8>();
        }
        return launch("k_paged_append", fn, token_grid(a.T, waves), args, stream);
    }
};
struct ReadLaunch {
    RowArgs a;
    PagedArgs c;
    bool fp8_pages;
    hipStream_t stream;
    template <typename T, int D> int operator()() {
        // Two waves per token, or one where k and v are a step each: 16384 tokens of 2 heads of 64 read back (with a small append) in 12.4 us instead of 15.0; of 8 heads
        // of 128 by one wave 29.0 instead of 28.0.
        const int skv = (a.Hkv + RowLayout<T, D>::RPW - 1) / RowLayout<T, D>::RPW;
        int waves, per = steps_per_wave<T, D>(a.T, 0, a.Hkv, skv < 2 ? 2 : skv < kReadSteps ? skv : kReadSteps, &waves);
        void *args[] = {&a, &c, &per};
        const void *fn = reinterpret_cast<const void *>(k_paged_read<T, T, D>);
        if constexpr (sizeof(T) == 2) {
            if (c.fp4) fn = reinterpret_cast<const void *>(k_paged_read<T, fp4, D>);
            else if (fp8_pages) fn = reinterpret_cast<const void *>(k_paged_read<T, fp8, D>);
        }
        return launch("k_paged_read", fn, token_grid(a.T, waves), args, stream);
    }
};

} // namespace

int run_norm_rope_fwd(int dtype, int d, const RowArgs &a, hipStream_t stream) { return a.T == 0 ? 0 : by_type<false>(dtype, d, FwdLaunch{a, stream}); }
int run_norm_rope_bwd(int dtype, int d, const RowArgs &a, hipStream_t stream) { return by_type<false>(dtype, d, BwdLaunch{a, stream}); }
int run_paged_append(int dtype, int d, bool fp8, bool norm, const RowArgs &a, const PagedArgs &c, hipStream_t stream) {
    return a.T == 0 ? 0 : by_type<true>(dtype, d, AppendLaunch{a, c, fp8, norm, stream});
}
int run_paged_read(int dtype, int d, bool fp8, const RowArgs &a, const PagedArgs &c, hipStream_t stream) {
    return a.T == 0 ? 0 : by_type<true>(dtype, d, ReadLaunch{a, c, fp8, stream});
}

} // namespace dn
