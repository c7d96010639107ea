// Attention of new tokens over the paged cache.  The rows of a sequence that read one key/value head, q_len tokens times
// G = Hq / Hkv query heads, are taken together (row = token * G + head), so that each key and value is fetched once for all of them.
// Softmax runs over the keys in one pass with the running maximum m and sum l per row (in powers of two, the scale folded in):
//
//     m' = max(m, max_j s_j) ,  l' = l 2^(m - m') + sum_j 2^(s_j - m') ,  o' = o 2^(m - m') + sum_j 2^(s_j - m') v_j
//
// and splits of the key axis are joined by the same formula.  All products run transposed, S^T = K Q^T and O^T = V^T P^T: the
// matrix cores leave S^T with a lane's values all in one row (the lane's query) and at the keys that P^T's operand wants from
// that lane, so that P never leaves its registers.
#include "dn_attn_device.hpp"

namespace dn {

constexpr float kNoScore = -1e30f; // the running maximum before the first key: finite, so that differences are never NaN

// The rows of sequence n and its context, held inside the tensors whatever the arrays say.
struct SeqRows {
    int r0, r1, kv;
    __device__ inline void load(const AttnArgs &a, int n) {
        r0 = min(max(a.c.cu[n], 0), a.r.T);
        r1 = min(max(a.c.cu[n + 1], r0), a.r.T);
        kv = min(max(a.c.kv_len[n], 0), a.c.max_kv);
    }
};

// The keys that rows [row0, row1) of a sequence see between them: [lo, hi), lo a multiple of `step`.
__device__ inline void key_range(const AttnArgs &a, const SeqRows &s, int G, int row0, int row1, int step, int &lo, int &hi) {
    const int before = s.kv - (s.r1 - s.r0); // position of the first new token
    hi = max(before + (row1 - 1) / G + 1, 0);
    const int first = max(before + row0 / G, 0);
    lo = a.window > 0 ? max(first - a.window + 1, 0) / step * step : 0;
}

// Cache row (of d elements) of key kk, a multiple of 16 (a page holds at least 16): the same for the whole wave.
__device__ inline int page_of(const PagedArgs &c, int n, int kk) {
    const int id = c.table[(long)n * c.max_pages + min(kk >> c.page_shift, c.max_pages - 1)];
    return __builtin_amdgcn_readfirstlane(min(max(id, 0), c.num_pages - 1));
}
__device__ inline long row_of(const PagedArgs &c, int page, int kk, int kvh, int Hkv) {
    return (((long)page * Hkv + kvh) << c.page_shift) + (kk & ((1 << c.page_shift) - 1));
}

// Zeroes the outputs of rows that lie in no sequence.
template <typename T, int D> __device__ inline void zero_rest(const AttnArgs &a, int kvh, int G) {
    const int from = min(max(a.c.N ? a.c.cu[a.c.N] : 0, 0), a.r.T);
    constexpr int W = D * (int)sizeof(T) / 16; // words of a row
    for (long i = threadIdx.x; i < (long)(a.r.T - from) * G * W; i += blockDim.x) {
        const long row = (from + i / (G * W)) * a.r.Hq + kvh * G + i / W % G;
        reinterpret_cast<uint4 *>(a.r.q_out)[row * W + i % W] = make_uint4(0, 0, 0, 0);
    }
}

// --- Few rows: generation, and short chunks.
//
// Bound by the reading of the cache.  A wave takes 32 keys at a time straight from memory to its registers, in the order in which
// the products want them: for S^T lane l holds a quarter (l / 16) of the elements of key l % 16 of each half; for O^T it holds a
// sixteenth (l % 16) of the elements of the eight keys whose probabilities it has, which a 16-bit transposition among its own
// registers turns into the operands of D / 16 products.  No LDS traffic and no barrier until the waves of a workgroup, which share out the
// keys of one split, join their sums.
constexpr int kFewTile = 16, kFewKeys = 32, kFewWaves = 4;

template <typename T, typename CT> struct PageElem { typedef CT type; static constexpr int bytes = (int)sizeof(CT); };
template <typename T> struct PageElem<T, fp8> { typedef unsigned char type; static constexpr int bytes = 1; };

template <int W> __device__ inline void load_words(unsigned (&w)[W], const void *p) {
    if constexpr (W == 1) w[0] = *static_cast<const unsigned *>(p);
    else if constexpr (W == 2) { const uint2 x = *static_cast<const uint2 *>(p); w[0] = x.x; w[1] = x.y; }
    else {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const uint4 x = static_cast<const uint4 *>(p)[i];
            w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
        }
    }
}
// two neighbouring e4m3 numbers as two bf16 (exact)
__device__ inline unsigned bf16_pair(unsigned w, bool hi) {
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
    return __builtin_bit_cast(unsigned, v);
}
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

template <typename T, typename CT, int D>
__global__ __launch_bounds__(64 * kFewWaves) void k_attn_few(AttnArgs a, int tiles, int splits, int split_keys, int max_rows) {
    constexpr int EB = PageElem<T, CT>::bytes;
    constexpr int KE = D / 4, VE = D / 16;              // elements of a key, of a value, that a lane holds
    constexpr int KW = KE * EB / 4, VW = VE * EB / 4;   // in words
    constexpr bool FP8 = __is_same(CT, fp8);
    extern __shared__ __align__(16) float smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int Hkv = a.r.Hkv, G = a.r.Hq / Hkv;
    int b = blockIdx.x;
    const int kvh = b % Hkv; b /= Hkv;
    const int split = b % splits; b /= splits;
    const int tile = b % tiles, n = b / tiles;
    if (n == a.c.N) {
        if (split == 0 && tile == 0) zero_rest<T, D>(a, kvh, G);
        return;
    }
    SeqRows s;
    s.load(a, n);
    const int R = (s.r1 - s.r0) * G, row0 = tile * kFewTile;
    if (R > max_rows || row0 >= R) return;
    const int row1 = min(row0 + kFewTile, R);
    int lo, hi;
    key_range(a, s, G, row0, row1, kFewKeys, lo, hi);
    const int k_begin = lo + split * split_keys, k_end = min(hi, k_begin + split_keys);
    if (splits > 1 && k_begin >= k_end) return; // (the rows' other splits know)
    const bool valid = row0 + col < row1;
    const int tok = (valid ? row0 + col : row0) / G, head = kvh * G + (valid ? row0 + col : row0) % G;
    const int before = s.kv - (s.r1 - s.r0), p = before + tok;              // the lane's query's position
    const int p_lo = a.window > 0 ? p - a.window + 1 : 0;                   // first key it sees
    const int all_from = a.window > 0 ? before + (row1 - 1) / G - a.window + 1 : 0, all_to = before + row0 / G; // keys in [all_from, all_to] are seen by every row

    // the query: elements g KE .. g KE + KE - 1
    unsigned qw[KE * sizeof(T) / 4];
    load_words(qw, static_cast<const T *>(a.r.q) + (long)(s.r0 + tok) * a.r.q_stride + head * D + g * KE);
    const float c = a.scale * 1.4426950408889634f;

    const char *kp = static_cast<const char *>(a.c.kp), *vp = static_cast<const char *>(a.c.vp);
    unsigned kw[2][KW], vw[8][VW];
    float4 ks[2], vs[2];
    auto load_k = [&](int k0, const int (&page)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long row = row_of(a.c, page[h], k0 + 16 * h, kvh, Hkv);
            load_words(kw[h], kp + (row * D * EB + (col * D + g * KE) * EB));
            if constexpr (FP8) ks[h] = *reinterpret_cast<const float4 *>(a.c.ks + row + 4 * g);
        }
    };
    auto load_v = [&](int k0, const int (&page)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long row = row_of(a.c, page[h], k0 + 16 * h, kvh, Hkv);
#pragma unroll
            for (int i = 0; i < 4; ++i) load_words(vw[4 * h + i], vp + (row * D * EB + ((4 * g + i) * D + col * VE) * EB));
            if constexpr (FP8) vs[h] = *reinterpret_cast<const float4 *>(a.c.vs + row + 4 * g);
        }
    };

    f32x4 o[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNoScore, l = 0.f;

    constexpr int STEP = kFewWaves * kFewKeys;
    int k0 = k_begin + wave * kFewKeys;
    int page[2], next[2];
    if (k0 < k_end) {
#pragma unroll
        for (int h = 0; h < 2; ++h) { page[h] = page_of(a.c, n, k0 + 16 * h); next[h] = page_of(a.c, n, k0 + STEP + 16 * h); }
        load_k(k0, page);
        load_v(k0, page);
    }
    for (; k0 < k_end; k0 += STEP) {
        const bool more = k0 + STEP < k_end;
        f32x4 st[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < KE; ++e)
                    st[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[h][e]), __uint_as_float(qw[e]), st[h], 0, 0, 0);
            } else {
#pragma unroll
                for (int e = 0; e < KE / 8; ++e) {
                    u32x4 kk;
                    if constexpr (FP8) kk = u32x4{bf16_pair(kw[h][2 * e], false), bf16_pair(kw[h][2 * e], true), bf16_pair(kw[h][2 * e + 1], false), bf16_pair(kw[h][2 * e + 1], true)};
                    else kk = u32x4{kw[h][4 * e], kw[h][4 * e + 1], kw[h][4 * e + 2], kw[h][4 * e + 3]};
                    const u32x4 qq = u32x4{qw[4 * e], qw[4 * e + 1], qw[4 * e + 2], qw[4 * e + 3]};
                    st[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk), __builtin_bit_cast(bf16x8, qq), st[h], 0, 0, 0);
                }
            }
            if constexpr (FP8) { st[h][0] *= ks[h].x; st[h][1] *= ks[h].y; st[h][2] *= ks[h].z; st[h][3] *= ks[h].w; }
        }
        if (more) load_k(k0 + STEP, next);
        if (k0 < all_from || k0 + kFewKeys - 1 > all_to) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = k0 + 16 * h + 4 * g + i;
                    if (key > p || key < p_lo) st[h][i] = -INFINITY;
                }
        }
        float mt = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])), fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3])));
        {
            const unsigned u = __float_as_uint(mt);
            const auto x = __builtin_amdgcn_permlane16_swap(u, u, false, false);
            const unsigned v = __float_as_uint(fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])));
            const auto y = __builtin_amdgcn_permlane32_swap(v, v, false, false);
            mt = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
        }
        const float mn = fmaxf(m, mt * c);
        if (__any(mn > m)) {
            const float f = __builtin_amdgcn_exp2f(m - mn);
            l *= f;
#pragma unroll
            for (int j = 0; j < VE; ++j) o[j] *= f;
            m = mn;
        }
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) { st[h][i] = __builtin_amdgcn_exp2f(fmaf(st[h][i], c, -m)); sum += st[h][i]; }
        l += sum;
        if (k0 + kFewKeys > hi) { // nothing past the last key that a row sees is read into a result, whatever stands there
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool dead = k0 + 16 * h + 4 * g + i >= hi;
#pragma unroll
                    for (int w = 0; w < VW; ++w) vw[4 * h + i][w] = dead ? 0u : vw[4 * h + i][w];
                    if constexpr (FP8) if (dead) reinterpret_cast<float *>(&vs[h])[i] = 0.f;
                }
        }
        if constexpr (FP8)
#pragma unroll
            for (int h = 0; h < 2; ++h) { st[h][0] *= vs[h].x; st[h][1] *= vs[h].y; st[h][2] *= vs[h].z; st[h][3] *= vs[h].w; }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < VE; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vw[i][j]), st[i >> 2][i & 3], o[j], 0, 0, 0);
        } else {
            bf16x8 pt;
#pragma unroll
            for (int i = 0; i < 8; ++i) pt[i] = (bf16)st[i >> 2][i & 3];
#pragma unroll
            for (int w = 0; w < VE / 2; ++w) { // a pair of elements of eight keys -> eight keys of each element
                unsigned x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (FP8) x[i] = bf16_pair(vw[i][w / 2], w & 1);
                    else x[i] = vw[i][w];
                }
                u32x4 even, odd;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    even[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100);
                    odd[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302);
                }
                o[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pt, o[2 * w], 0, 0, 0);
                o[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pt, o[2 * w + 1], 0, 0, 0);
            }
        }
        if (more) {
            load_v(k0 + STEP, next);
#pragma unroll
            for (int h = 0; h < 2; ++h) next[h] = page_of(a.c, n, k0 + 2 * STEP + 16 * h);
        }
    }

    // the waves' sums: o of element (4 g + r) VE + j and query col stands at o[j][r]
    constexpr int LD = D + 4;
    float *so = smem, *sm = smem + kFewWaves * kFewTile * LD, *sl = sm + kFewWaves * kFewTile;
    {
        const unsigned u = __float_as_uint(l);
        const auto x = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        const unsigned v = __float_as_uint(__uint_as_float(x[0]) + __uint_as_float(x[1]));
        const auto y = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        l = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    if (g == 0) { sm[wave * kFewTile + col] = m; sl[wave * kFewTile + col] = l; }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VE; ++j) so[(wave * kFewTile + col) * LD + (4 * g + r) * VE + j] = o[j][r];
    __syncthreads();
    const int q = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * VE; // sixteen threads per query
    if (row0 + q >= row1) return;
    float M = kNoScore, L = 0.f, acc[VE];
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) M = fmaxf(M, sm[w * kFewTile + q]);
#pragma unroll
    for (int j = 0; j < VE; ++j) acc[j] = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm[w * kFewTile + q] - M);
        L = fmaf(sl[w * kFewTile + q], f, L);
#pragma unroll
        for (int j = 0; j < VE; ++j) acc[j] = fmaf(so[(w * kFewTile + q) * LD + e0 + j], f, acc[j]);
    }
    const long row = (long)(s.r0 + (row0 + q) / G) * a.r.Hq + kvh * G + (row0 + q) % G;
    if (splits == 1) {
        const float inv = L > 0.f ? 1.f / L : (L == L ? 0.f : L);
        T *to = static_cast<T *>(a.r.q_out) + row * D + e0;
#pragma unroll
        for (int j = 0; j < VE; ++j) to[j] = (T)(acc[j] * inv);
    } else {
        const long at = (long)split * a.r.T * a.r.Hq + row, all = (long)splits * a.r.T * a.r.Hq;
        float *ml = static_cast<float *>(a.workspace), *po = ml + ((2 * all + 3) & ~3l);
        if (e0 == 0) *reinterpret_cast<float2 *>(ml + 2 * at) = make_float2(M, L);
#pragma unroll
        for (int j = 0; j < VE; j += 2) *reinterpret_cast<float2 *>(po + at * D + e0 + j) = make_float2(acc[j], acc[j + 1]);
    }
}

// Joins the splits of every row (a wave per row and head).
template <typename T, int D>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, int splits, int split_keys) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long row = (long)blockIdx.x * 4 + wave;
    if (row >= (long)a.r.T * a.r.Hq) return;
    const int t = (int)(row / a.r.Hq), h = (int)(row % a.r.Hq), G = a.r.Hq / a.r.Hkv;
    constexpr int E = D >= 64 ? D / 64 : 1;
    const bool on = lane * E < D;
    T *to = static_cast<T *>(a.r.q_out) + row * D + lane * E;
    const int n = seq_of_row(a.c.cu, a.c.N, t);
    int live = 0;
    if (n < a.c.N) {
        SeqRows s;
        s.load(a, n);
        const int R = (s.r1 - s.r0) * G, r = max(t - s.r0, 0) * G + h % G, row0 = r / kFewTile * kFewTile;
        int lo, hi;
        key_range(a, s, G, row0, min(row0 + kFewTile, R), kFewKeys, lo, hi);
        live = hi > lo ? min((hi - lo + split_keys - 1) / split_keys, splits) : 0;
    }
    const long rows = (long)a.r.T * a.r.Hq;
    const float *ml = static_cast<const float *>(a.workspace), *po = ml + ((2 * splits * rows + 3) & ~3l);
    float M = kNoScore, L = 0.f, acc[E];
    for (int i = lane; i < live; i += 64) M = fmaxf(M, ml[2 * (i * rows + row)]);
    M = lanes_max<64>(M);
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] = 0.f;
    for (int i = 0; i < live; ++i) {
        const float2 x = *reinterpret_cast<const float2 *>(ml + 2 * (i * rows + row));
        const float f = __builtin_amdgcn_exp2f(x.x - M);
        L = fmaf(x.y, f, L);
        if (on) {
#pragma unroll
            for (int j = 0; j < E; ++j) acc[j] = fmaf(po[(i * rows + row) * D + lane * E + j], f, acc[j]);
        }
    }
    const float inv = L > 0.f ? 1.f / L : (L == L ? 0.f : L);
    if (on) {
#pragma unroll
        for (int j = 0; j < E; ++j) to[j] = (T)(acc[j] * inv);
    }
}

namespace {

struct Plan { int tiles, splits, split_keys; };

// Tiles and splits by the bounds that the host knows.
Plan plan_few(const AttnArgs &a) {
    const int G = a.r.Hq / a.r.Hkv;
    Plan p;
    p.tiles = (int)(((long)a.max_q * G + kFewTile - 1) / kFewTile);
    if (p.tiles < 1) p.tiles = 1;
    const long range = a.window > 0 ? (a.c.max_kv < (long)a.window + a.max_q + kFewKeys ? a.c.max_kv : (long)a.window + a.max_q + kFewKeys) : a.c.max_kv;
    const long base = (long)(a.c.N > 0 ? a.c.N : 1) * p.tiles * a.r.Hkv;
    long splits = 1024 / base, most = (range + 255) / 256;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    if (splits > 64) splits = 64;
    long keys = (range + splits - 1) / splits;
    keys = (keys + 127) / 128 * 128;
    if (keys < 128) keys = 128;
    p.split_keys = (int)keys;
    p.splits = (int)((range + keys - 1) / keys);
    if (p.splits < 1) p.splits = 1;
    return p;
}

size_t workspace_of(const AttnArgs &a, int d, int splits) {
    if (splits == 1) return 0;
    const size_t rows = (size_t)splits * a.r.T * a.r.Hq;
    return (((2 * rows + 3) & ~size_t(3)) + rows * d) * sizeof(float);
}

template <typename T, typename CT, int D> int launch_attn(AttnArgs a, hipStream_t stream) {
    Plan p = plan_few(a);
    int max_rows = 1 << 30;
    constexpr int lds = kFewWaves * kFewTile * (D + 4 + 2) * 4;
    const void *fn = reinterpret_cast<const void *>(k_attn_few<T, CT, D>);
    if constexpr (lds > 64 * 1024)
        if (const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds)) return (int)e;
    void *args[] = {&a, &p.tiles, &p.splits, &p.split_keys, &max_rows};
    const long blocks = ((long)a.c.N * p.tiles + 1) * p.splits * a.r.Hkv;
    if (blocks >= (1l << 31)) return (int)hipErrorInvalidConfiguration;
    prof_begin("k_attn_few", stream);
    hipError_t e = hipLaunchKernel(fn, dim3((unsigned)blocks), dim3(64 * kFewWaves), args, lds, stream);
    prof_end(stream);
    if (e != hipSuccess || p.splits == 1) return (int)e;
    void *jargs[] = {&a, &p.splits, &p.split_keys};
    const long rows = (long)a.r.T * a.r.Hq;
    prof_begin("k_attn_join", stream);
    e = hipLaunchKernel(reinterpret_cast<const void *>(k_attn_join<T, D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), jargs, 0, stream);
    prof_end(stream);
    return (int)e;
}

} // namespace

size_t paged_attn_workspace(int, int d, const AttnArgs &a) { return a.r.T == 0 ? 0 : workspace_of(a, d, plan_few(a).splits); }

int run_paged_attn(int dtype, int d, bool fp8_pages, const AttnArgs &a, hipStream_t stream) {
    if (a.r.T == 0) return 0;
    if (dtype == 0) {
        if (d == 32) return launch_attn<float, float, 32>(a, stream);
        if (d == 64) return launch_attn<float, float, 64>(a, stream);
        if (d == 128) return launch_attn<float, float, 128>(a, stream);
    } else if (fp8_pages) {
        if (d == 64) return launch_attn<bf16, fp8, 64>(a, stream);
        if (d == 128) return launch_attn<bf16, fp8, 128>(a, stream);
        if (d == 256) return launch_attn<bf16, fp8, 256>(a, stream);
    } else {
        if (d == 64) return launch_attn<bf16, bf16, 64>(a, stream);
        if (d == 128) return launch_attn<bf16, bf16, 128>(a, stream);
        if (d == 256) return launch_attn<bf16, bf16, 256>(a, stream);
    }
    return (int)hipErrorInvalidValue;
}

} // namespace dn
