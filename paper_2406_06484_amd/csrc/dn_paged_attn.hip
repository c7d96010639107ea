// Attention of new tokens over the paged cache.  The rows of a sequence that read one key/value head, q_len tokens times
// G = Hq / Hkv query heads, are taken together (row = token * G + head), so that each key and value is fetched once for all of them.
// Softmax runs over the keys in one pass with the running maximum m and sum l per row (in powers of two, c = scale / log 2):
//
//     m' = max(m, max_j s_j) ,  l' = l 2^(c (m - m')) + sum_j 2^(c (s_j - m')) ,  o' = o 2^(c (m - m')) + sum_j 2^(c (s_j - m')) v_j
//
// (m is a score, not its multiple: s_j - m is right to its last bits however large both are, where c s_j less a rounded c m may be off by more than the
// exponential's range) and splits of the key axis are joined by the same formula.  All products run transposed, S^T = K Q^T and O^T = V^T P^T: the
// matrix cores leave S^T with a lane's values all in one row (the lane's query) and at the keys that P^T's operand wants from
// that lane, so that P never leaves its registers.
#include "dn_attn_device.hpp"

namespace dn {

// How the key axis is cut: `splits` pieces of `keys` keys from the first that a row tile sees.
struct Cut { int splits, keys; };

constexpr float kNoScore = -3.4028235e38f; // the running maximum before the first key: finite, so that differences are never NaN, and under every other score
constexpr float kLog2e = 1.4426950408889634f;

// The rows of sequence n, its context, held inside the tensors whatever the arrays say, and the position of its first row (tokens that the table has no room
// for have theirs behind the context's end, and move nobody's).
struct SeqRows {
    int r0, r1, kv, before;
    __device__ inline void load(const AttnArgs &a, int n) {
        r0 = min(max(a.c.cu[n], 0), a.r.T);
        r1 = min(max(a.c.cu[n + 1], r0), a.r.T);
        const int len = max(a.c.kv_len[n], 0);
        kv = min(len, a.c.max_kv);
        before = len - (r1 - r0);
    }
};

// The keys that rows [row0, row1) of a sequence see between them: [from, hi); lo is `from` rounded down to a multiple of `step`.  Values outside, which a
// window may have left to other sequences, enter no product, whatever stands there.
__device__ inline void key_range(const AttnArgs &a, const SeqRows &s, int G, int row0, int row1, int step, int &lo, int &from, int &hi) {
    hi = min(max(s.before + (row1 - 1) / G + 1, 0), s.kv);
    const int first = max(s.before + row0 / G, 0);
    from = a.window > 0 ? min(max(first - a.window + 1, 0), hi) : 0;
    lo = from / step * step;
}

// The page table's entry for key kk, the page that it stands for, and (the wave's key kk, a multiple of 16: a page holds at least 16) the
// cache row of d elements.
__device__ inline int page_entry(const PagedArgs &c, int n, int kk) { return c.table[(long)n * c.max_pages + min(kk >> c.page_shift, c.max_pages - 1)]; }
__device__ inline int page_id(const PagedArgs &c, int entry) { return min(max(entry, 0), c.num_pages - 1); }
__device__ inline int page_of(const PagedArgs &c, int n, int kk) { return __builtin_amdgcn_readfirstlane(page_id(c, page_entry(c, n, kk))); }
__device__ inline long row_of(const PagedArgs &c, int page, int kk, int kvh, int Hkv) {
    return (((long)page * Hkv + kvh) << c.page_shift) + (kk & ((1 << c.page_shift) - 1));
}

// Zeroes the outputs of rows that lie in no sequence: those in front of the first one and those past the last one.
template <typename T, int D> __device__ inline void zero_rest(const AttnArgs &a, int kvh, int G) {
    int front = a.c.N ? min(max(a.c.cu[0], 0), a.r.T) : 0, from = a.c.N ? min(max(a.c.cu[a.c.N], front), a.r.T) : 0;
    if (!a.zero_front) front = 0;
    if (!a.zero_rest) from = a.r.T;
    constexpr int W = D * (int)sizeof(T) / 16; // words of a row
    for (long i = threadIdx.x; i < (long)(front + a.r.T - from) * G * W; i += blockDim.x) {
        const long t = i / (G * W), row = (t < front ? t : from + t - front) * a.r.Hq + kvh * G + i / W % G;
        reinterpret_cast<uint4 *>(a.r.q_out)[row * W + i % W] = make_uint4(0, 0, 0, 0);
    }
}

// What a sum of weights divides by: nothing where there is nothing, and NaN stays NaN.
__device__ inline float inverse_sum(float l) { return l > 0.f ? 1.f / l : (l == l ? 0.f : l); }

// Where a split's (maximum, sum) and unnormalised output of a row (token and head) stand in the workspace.
__device__ inline void partial_of(const AttnArgs &a, int split, long row, int D, float **ml, float **po) {
    const long rows = (long)a.r.T * a.r.Hq, at = split * rows + row;
    float *base = static_cast<float *>(a.workspace);
    *ml = base + 2 * at;
    *po = base + ((2 * a.splits * rows + 3) & ~3l) + at * D;
}

// --- Few rows: generation, and short chunks.
//
// Bound by the reading of the cache.  A wave takes 32 keys at a time straight from memory to its registers, in the order in which
// the products want them: for S^T lane l holds a quarter of the elements of key l % 16 of each half, every fourth 16-byte piece from l / 16 on; for O^T it
// holds a sixteenth of the elements of the eight keys whose probabilities it has, one 16-byte piece (or less) of each 16, from l % 16 on, which a 16-bit
// transposition among its own registers turns into the operands of D / 16 products.  (So the lanes of one load stand side by side.)  No LDS traffic and no barrier until the waves of a workgroup, which share out the
// keys of one split, join their sums.  32 sequences of 16 heads of 128 over up to 2048 keys in bf16 (374 MB): 72 us, 5.2 TB/s; one over 32768 e4m3 keys of 4 heads (34 MB):
// 11 us and 4 for the join.
constexpr int kFewTile = 16, kFewKeys = 32, kFewWaves = 4;
// Twice as many waves per workgroup where there are few workgroups, if their registers allow it.
template <typename T> constexpr bool few_twice(int d) { return d * sizeof(T) <= 256; }

template <typename T, typename CT> struct PageElem { typedef CT type; static constexpr int bytes = (int)sizeof(CT); };
template <typename T> struct PageElem<T, fp8> { typedef unsigned char type; static constexpr int bytes = 1; };

// W words, from `off` bytes behind a descriptor's base on, in pieces of 16 bytes that are `step` bytes apart.  (Buffer loads: the base, the same for the whole wave, stays in scalar registers, where a global load
// would have a 64-bit address per lane and load.)
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
template <int W> __device__ inline void load_words(unsigned (&w)[W], __amdgpu_buffer_rsrc_t rs, int off, int step = 16) {
    if constexpr (W == 1) w[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0);
    else if constexpr (W == 2) { const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0); w[0] = x[0]; w[1] = x[1]; }
    else {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rs, off + step * i, 0, 0);
            w[4 * i] = x[0]; w[4 * i + 1] = x[1]; w[4 * i + 2] = x[2]; w[4 * i + 3] = x[3];
        }
    }
}
// two neighbouring e4m3 numbers as two bf16 (exact)
__device__ inline unsigned bf16_pair(unsigned w, bool hi) {
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
    return __builtin_bit_cast(unsigned, v);
}
// eight e4m3 numbers as bf16
__device__ inline u32x4 widen(unsigned lo, unsigned hi) { return u32x4{bf16_pair(lo, false), bf16_pair(lo, true), bf16_pair(hi, false), bf16_pair(hi, true)}; }

template <typename T, typename CT, int D, int WAVES>
__device__ __forceinline__ void attend_few(const AttnArgs &a, int tiles, Cut cut, int max_rows, int block, float *smem) {
    const int splits = cut.splits, split_keys = cut.keys;
    constexpr int EB = PageElem<T, CT>::bytes;
    constexpr int KE = D / 4, VE = D / 16;              // elements of a key, of a value, that a lane holds
    constexpr int KW = KE * EB / 4, VW = VE * EB / 4;   // in words
    constexpr int KV = 16 / EB;                         // elements of a piece of a key: (4 piece + g) KV ..
    constexpr int VV = VE * EB > 16 ? 16 / EB : VE;     // ... and of a value: (16 piece + col) VV ..
    constexpr bool FP8 = __is_same(CT, fp8);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int Hkv = a.r.Hkv, G = a.r.Hq / Hkv;
    int b = block;
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
    int lo, from, hi;
    key_range(a, s, G, row0, row1, kFewKeys, lo, from, hi);
    const int k_begin = lo + split * split_keys, k_end = min(hi, k_begin + split_keys);
    if (splits > 1 && k_begin >= k_end) return; // (the rows' other splits know)
    const bool valid = row0 + col < row1;
    const int tok = (valid ? row0 + col : row0) / G, head = kvh * G + (valid ? row0 + col : row0) % G;
    const int pos = s.before + tok, p = min(pos, s.kv - 1);                 // the lane's query's position, and the last key it sees
    const int p_lo = a.window > 0 ? pos - a.window + 1 : 0;                 // the first one
    const int all_from = a.window > 0 ? s.before + (row1 - 1) / G - a.window + 1 : 0, all_to = min(s.before + row0 / G, s.kv - 1); // keys in [all_from, all_to] are seen by every row

    // the query, in the same order as a key
    unsigned qw[KE * sizeof(T) / 4];
    {
        const T *src = static_cast<const T *>(a.r.q) + (long)(s.r0 + tok) * a.r.q_stride + head * D;
        constexpr int PW = KV * (int)sizeof(T) / 16; // 16-byte words of a piece
#pragma unroll
        for (int i = 0; i < KE / KV * PW; ++i) {
            const uint4 x = reinterpret_cast<const uint4 *>(src + (4 * (i / PW) + g) * KV)[i % PW];
            qw[4 * i] = x.x; qw[4 * i + 1] = x.y; qw[4 * i + 2] = x.z; qw[4 * i + 3] = x.w;
        }
    }
    const float c = a.scale * kLog2e;

    const char *kp = static_cast<const char *>(a.c.kp), *vp = static_cast<const char *>(a.c.vp);
    unsigned kw[2][KW], vw[8][VW];
    float4 ks[2], vs[2];
    auto load_k = [&](int k0, const int (&page)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long row = row_of(a.c, page[h], k0 + 16 * h, kvh, Hkv);
            load_words(kw[h], make_rsrc(kp + row * (D * EB)), col * D * EB + 16 * g, 64);
            if constexpr (FP8) ks[h] = *reinterpret_cast<const float4 *>(a.c.ks + row + 4 * g);
        }
    };
    auto load_v = [&](int k0, const int (&page)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long row = row_of(a.c, page[h], k0 + 16 * h, kvh, Hkv);
            const __amdgpu_buffer_rsrc_t va = make_rsrc(vp + row * (D * EB));
#pragma unroll
            for (int i = 0; i < 4; ++i) load_words(vw[4 * h + i], va, ((4 * g + i) * D + col * VV) * EB, 256);
            if constexpr (FP8) vs[h] = *reinterpret_cast<const float4 *>(a.c.vs + row + 4 * g);
        }
    };

    f32x4 o[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNoScore, l = 0.f;

    constexpr int STEP = WAVES * kFewKeys;
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
                    if constexpr (FP8) kk = widen(kw[h][2 * e], kw[h][2 * e + 1]);
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
        const float mn = fmaxf(m, mt);
        if (__any(mn > m)) {
            const float f = __builtin_amdgcn_exp2f((m - mn) * c);
            l *= f;
#pragma unroll
            for (int j = 0; j < VE; ++j) o[j] *= f;
            m = mn;
        }
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) { st[h][i] = __builtin_amdgcn_exp2f((st[h][i] - m) * c); sum += st[h][i]; }
        l += sum;
        if (k0 + kFewKeys > hi || k0 < from) { // what no row sees enters no result
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = k0 + 16 * h + 4 * g + i;
                    const bool dead = key >= hi || key < from;
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
            // Probabilities as two bf16 terms: the products wait for memory anyway, and the output then carries the one rounding of its own (in one
            // term, 1.4 times its error).
            bf16x8 pt, pl;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = st[i >> 2][i & 3];
                pt[i] = (bf16)x;
                pl[i] = (bf16)(x - (float)pt[i]);
            }
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
                o[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pl, o[2 * w], 0, 0, 0);
                o[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pl, o[2 * w + 1], 0, 0, 0);
            }
        }
        if (more) {
            load_v(k0 + STEP, next);
#pragma unroll
            for (int h = 0; h < 2; ++h) next[h] = page_of(a.c, n, k0 + 2 * STEP + 16 * h);
        }
    }

    // the waves' sums: o of element (16 piece + 4 g + r) VV + j and query col stands at o[piece VV + j][r]
    constexpr int LD = D + 4;
    float *so = smem, *sm = smem + WAVES * kFewTile * LD, *sl = sm + WAVES * kFewTile;
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
        for (int j = 0; j < VE; ++j) so[(wave * kFewTile + col) * LD + (16 * (j / VV) + 4 * g + r) * VV + j % VV] = o[j][r];
    __syncthreads();
    const int q = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * VE; // sixteen threads per query
    if (q >= kFewTile || row0 + q >= row1) return;
    float M = kNoScore, L = 0.f, acc[VE];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) M = fmaxf(M, sm[w * kFewTile + q]);
#pragma unroll
    for (int j = 0; j < VE; ++j) acc[j] = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f((sm[w * kFewTile + q] - M) * c);
        L = fmaf(sl[w * kFewTile + q], f, L);
#pragma unroll
        for (int j = 0; j < VE; ++j) acc[j] = fmaf(so[(w * kFewTile + q) * LD + e0 + j], f, acc[j]);
    }
    const long row = (long)(s.r0 + (row0 + q) / G) * a.r.Hq + kvh * G + (row0 + q) % G;
    if (splits == 1) {
        const float inv = inverse_sum(L);
        T *to = static_cast<T *>(a.r.q_out) + row * D + e0;
#pragma unroll
        for (int j = 0; j < VE; ++j) to[j] = (T)(acc[j] * inv);
    } else {
        float *ml, *po;
        partial_of(a, split, row, D, &ml, &po);
        if (e0 == 0) *reinterpret_cast<float2 *>(ml) = make_float2(M, L);
#pragma unroll
        for (int j = 0; j < VE; j += 2) *reinterpret_cast<float2 *>(po + e0 + j) = make_float2(acc[j], acc[j + 1]);
    }
}

// --- Many rows: prompts and long chunks.
//
// Products, softmax, products in turn: prompts of 4 x 2048 tokens, 16 heads of 128, 88 to 91 us (760 TFLOP/s of the 1195 of a large matrix product), the matrix pipes busy for 0.32 of the time, the
// vector ALU for 0.33 or more (exponentials count as one instruction), the LDS for 0.16; the waves wait for 0.27 of theirs and are ready but not issued for 0.31.  512 tokens of 16 heads (4 of keys)
// behind 15872, 86 us with the join (10), 0.37, 0.34, 0.19, 0.22, 0.32.  Without the requests, the exponentials or half of the products it would still take 90 % (80 %).  A workgroup has 128
// rows, 32 per wave, and walks over its keys 64 at a time: K and V travel straight, 8-bit pages through registers (they become bf16 on the way, exactly), into one of two LDS buffers while the other
// is worked on, so that a tile costs one barrier.  Rows of a tile are not padded: their 16-byte pieces are permuted by an XOR with the row, which spreads both the row
// reads (K) and the transposing reads (V, four rows at a time) over the banks.
constexpr int kWideRows = 128, kWideWaves = 4;
constexpr float kFarScore = 0x1p20f; // (a number of this size is rounded by 2^-4 at most)
// keys of a tile (at d = 256 twice as many would need more registers than there are)
constexpr int wide_keys(int d) { return d > 128 ? 32 : 64; }

// 64 lanes' 16 bytes from global memory to a kilobyte of the LDS, without registers in between: lane l's land 16 l behind `lds` (M0 holds it); lanes past
// the descriptor's range leave zeros.  The compiler does not know of the transfer (told of it, it would have every read of the LDS wait for it): wait_moved
// before the barrier that makes the tile readable.  Nor does it keep the hardware's distances inside the text: M0 needs one wait state, a scalar
// register written on the vector unit (readfirstlane) five before a buffer access reads it.  tests/test_attention_dma_host.py reads both from the compiled code.
__device__ __forceinline__ void move16(__amdgpu_buffer_rsrc_t rs, int off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(rs) : "memory");
}
__device__ inline unsigned lds_place(const unsigned char *p) {
    typedef __attribute__((address_space(3))) const unsigned char lds_t;
    return __builtin_amdgcn_readfirstlane((unsigned)(size_t)(lds_t *)p);
}
__device__ __forceinline__ void wait_moved() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <typename CT, int D> struct WideTile {
    static constexpr bool FP8 = __is_same(CT, fp8);
    static constexpr int KEYS = wide_keys(D);
    static constexpr int CH = D / 8, ROWB = 2 * D;                 // 16-byte pieces, bytes of a row in the LDS
    static constexpr int PER = FP8 ? 2 : 1, LPR = CH / PER;        // pieces per load, lanes per row
    static constexpr int NL = KEYS * LPR / (64 * kWideWaves); // loads per thread and tensor
    static constexpr int BYTES = KEYS * ROWB;
    static constexpr int oV = BYTES, oKS = 2 * BYTES, oVS = oKS + (FP8 ? 4 * KEYS : 0), SIZE = oVS + (FP8 ? 4 * KEYS : 0);
    __device__ static inline int swizzle(int row) { return D == 64 ? ((row >> 1) & 1) << 2 | ((row >> 2) & 3) : (row & 3) << 2 | ((row >> 2) & 3); }
};

// The sequence and the row tile that a slot stands for: slots count the tiles of 128 rows of the sequences with more than `few` rows.
// Later tiles see more keys and come first, so that the workgroups that start last are short: of each 64 sequences the last tiles, then the ones
// before those, and so on (in the order of the sequences, prompts of 4 x 2048 tokens took 160 us instead of 126).  False past the last slot.
__device__ inline bool tile_of_slot(const AttnArgs &a, int G, int few, int slot, int *seq, int *tile) {
    const int lane = threadIdx.x & 63;
    int next0 = 0, next1 = 0; // offsets of the 64 sequences to come, on their way while the present ones are gone through
    auto ahead = [&](int n) { if (n < a.c.N) { next0 = a.c.cu[n]; next1 = a.c.cu[n + 1]; } };
    ahead(lane);
    for (int base = 0; base < a.c.N; base += 64) {
        const int n = base + lane, r0 = min(max(next0, 0), a.r.T), r1 = min(max(next1, r0), a.r.T), R = (r1 - r0) * G;
        const int tiles = n < a.c.N && R > few ? (R + kWideRows - 1) / kWideRows : 0;
        ahead(n + 64);
        int rank = 0; // tiles behind this one in its sequence
        for (unsigned long long on = __ballot(tiles > 0); on; on = __ballot(tiles > rank)) {
            const int count = __builtin_popcountll(on);
            if (slot < count) {
                const bool mine = (on >> lane & 1) && __builtin_popcountll(on & ((1ull << lane) - 1)) == slot;
                const int at = __builtin_ctzll(__ballot(mine));
                *seq = base + at;
                *tile = __shfl(tiles, at) - 1 - rank;
                return true;
            }
            // the ranks up to the shortest sequence's first tile hold as many
            int least = tiles > rank ? tiles : 0x7fffffff;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) least = min(least, __shfl_xor(least, o));
            const int steps = min(least - rank, slot / count);
            rank += steps;
            slot -= steps * count;
        }
    }
    return false;
}

template <typename CT, int D>
__device__ __forceinline__ void attend_wide(const AttnArgs &a, Cut cut, int few, bool zero, int block, unsigned char *wsmem) {
    const int splits = cut.splits, split_keys = cut.keys;
    using W = WideTile<CT, D>;
    constexpr bool FP8 = W::FP8;
    constexpr int EB = FP8 ? 1 : 2, NB = D / 32, KEYS = W::KEYS, NX = KEYS / 32;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 31, h = lane >> 5;
    const int Hkv = a.r.Hkv, G = a.r.Hq / Hkv;
    int b = block;
    const int kvh = b % Hkv; b /= Hkv;
    const int split = b % splits, slot = b / splits;
    int n, tile;
    if (zero && block < Hkv) zero_rest<bf16, D>(a, kvh, G);
    if (!tile_of_slot(a, G, few, slot, &n, &tile)) return;
    n = __builtin_amdgcn_readfirstlane(n);
    tile = __builtin_amdgcn_readfirstlane(tile);
    SeqRows s;
    s.load(a, n);
    const int R = (s.r1 - s.r0) * G, row0 = tile * kWideRows, row1 = min(row0 + kWideRows, R);
    int lo, from, hi;
    key_range(a, s, G, row0, row1, KEYS, lo, from, hi);
    const int k_begin = lo + split * split_keys, k_end = min(hi, k_begin + split_keys);
    if (splits > 1 && k_begin >= k_end) return; // (the rows' other splits know)
    const int wrow = row0 + 32 * wave;
    const int row = min(wrow + col, row1 - 1), tok = row / G, head = kvh * G + row % G;
    const int pos = s.before + tok, p = min(pos, s.kv - 1), p_lo = a.window > 0 ? pos - a.window + 1 : 0; // the lane's query's position, the last and the first key it sees
    // keys that some row, that every row of the wave sees
    const int last = s.before + (min(wrow + 32, row1) - 1) / G, first = s.before + min(wrow, row1 - 1) / G;
    const int some_from = a.window > 0 ? first - a.window + 1 : 0, some_to = wrow < row1 ? min(last, s.kv - 1) : -1;
    const int all_from = a.window > 0 ? last - a.window + 1 : 0, all_to = min(first, s.kv - 1);
    const float c = a.scale * kLog2e;

    bf16x8 q[D / 16];
    {
        const bf16 *src = static_cast<const bf16 *>(a.r.q) + (long)(s.r0 + tok) * a.r.q_stride + head * D + 8 * h;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) q[i] = *reinterpret_cast<const bf16x8 *>(src + 16 * i);
    }
    f32x16 o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    // A score's exponent is c s - off, one operation, where c m is rounded by a small part of a power of two (the same for all of a row's scores); with a row
    // whose scores are larger, the wave subtracts m first.  (off is finite also before the first key: masked scores are -infinity.)
    float m = kNoScore, l = 0.f, off;
    bool far;
    auto set_off = [&]() __attribute__((always_inline)) { off = fmaxf(m * c, kNoScore); far = __any(m > kNoScore && fabsf(off) > kFarScore); };
    set_off();

    // this thread's pieces of a tile on their way (8-bit pages; 16-bit ones go straight to the LDS)
    u32x4 rk[W::NL], rv[W::NL];
    float rs = 0.f;
    const char *kp = static_cast<const char *>(a.c.kp), *vp = static_cast<const char *>(a.c.vp);
    const int piece = t % W::LPR;
    int page[W::NL], spage = 0; // of the next tile to fetch, looked up a tile ahead
    const unsigned page_bytes = (unsigned)(Hkv << a.c.page_shift) * (D * EB);
    auto look_up = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < W::NL; ++i) page[i] = page_entry(a.c, n, k0 + ((i * 256 + wave * 64) / W::LPR & ~15));
        if constexpr (FP8) spage = page_entry(a.c, n, k0 + (lane & 48));
    };
    // load i of a tile's NL (of K and of V)
    auto fetch = [&](unsigned char *buf, int k0, int i) __attribute__((always_inline)) {
        const int r0 = (i * 256 + wave * 64) / W::LPR, kk = k0 + (r0 & ~15); // the wave's rows lie in one group of 16 keys
        const unsigned id = __builtin_amdgcn_readfirstlane(page_id(a.c, page[i]));
        const long at = (long)((unsigned long)id * page_bytes) + ((kvh << a.c.page_shift) + (kk & ((1 << a.c.page_shift) - 1))) * (D * EB);
        const int r = r0 + lane / W::LPR;
        if constexpr (FP8) {
            const int off = (r & 15) * (D * EB) + piece * 16;
            rk[i] = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(kp + at), off, 0, 0);
            rv[i] = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(vp + at), off, 0, 0);
            if (i == 0 && wave < 2 && lane < KEYS)
                rs = (wave ? a.c.vs : a.c.ks)[row_of(a.c, page_id(a.c, spage), k0 + (lane & 48), kvh, Hkv) + (lane & 15)];
        } else {
            // values that no row sees arrive as zeros
            const int off = (r & 15) * (D * EB) + ((piece ^ W::swizzle(r)) << 4);
            const unsigned to = lds_place(buf) + (i * 256 + wave * 64) * 16;
            move16(make_rsrc(kp + at), off, to);
            move16(make_rsrc(vp + at), (unsigned)(k0 + r - from) < (unsigned)(hi - from) ? off : kBufRange, to + W::oV);
        }
    };
    auto fetch_all = [&](unsigned char *buf, int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < W::NL; ++i) fetch(buf, k0, i);
        look_up(k0 + KEYS);
    };
    auto park = [&](unsigned char *buf, int k0) __attribute__((always_inline)) {
        const bool ends = k0 + KEYS > hi || k0 < from; // values that no row sees become zeros
        auto dead = [&](int key) { return key >= hi || key < from; };
#pragma unroll
        for (int i = 0; i < W::NL; ++i) {
            const int r = (i * 256 + t) / W::LPR;
            u32x4 v = rv[i];
            if (ends && dead(k0 + r)) v = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                unsigned char *at = buf + r * W::ROWB + (((2 * piece + u) ^ W::swizzle(r)) << 4);
                *reinterpret_cast<u32x4 *>(at) = widen(rk[i][2 * u], rk[i][2 * u + 1]);
                *reinterpret_cast<u32x4 *>(at + W::oV) = widen(v[2 * u], v[2 * u + 1]);
            }
        }
        if (wave < 2 && lane < KEYS) reinterpret_cast<float *>(buf + (wave ? W::oVS : W::oKS))[lane] = ends && dead(k0 + lane) ? 0.f : rs;
    };
    // a tile's work, and between its first products the requests for tile `next` (16 bits: into `to`), if `more`
    auto work = [&](const unsigned char *buf, int k0, unsigned char *to, int next, bool more) __attribute__((always_inline)) {
        f32x16 st[NX];
        {
            // all operands are requested before the first product: one LDS latency instead of one per product (the compiler's own order)
            bf16x8 kf[NX][D / 16];
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int x = 0; x < NX; ++x) kf[x][i] = *reinterpret_cast<const bf16x8 *>(buf + (32 * x + col) * W::ROWB + (((2 * i + h) ^ W::swizzle(col)) << 4));
            __builtin_amdgcn_s_setprio(1); // (over the other workgroup's softmax: a chunk of 512 behind 15872 keys 88.6 -> 85.2 us)
            __builtin_amdgcn_sched_barrier(0);
            constexpr int EVERY = D / 16 / W::NL;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
#pragma unroll
                for (int x = 0; x < NX; ++x) st[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[x][i], q[i], i ? st[x] : f32x16{}, 0, 0, 0);
                if (i % EVERY == EVERY - 1) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (more) fetch(to, next, i / EVERY);
                }
            }
            if (more) look_up(next + KEYS);
            __builtin_amdgcn_s_setprio(0);
        }
        if constexpr (FP8)
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 f = *reinterpret_cast<const float4 *>(buf + W::oKS + (32 * x + 8 * g + 4 * h) * 4);
                    st[x][4 * g] *= f.x; st[x][4 * g + 1] *= f.y; st[x][4 * g + 2] *= f.z; st[x][4 * g + 3] *= f.w;
                }
        if (k0 < all_from || k0 + KEYS - 1 > all_to) {
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = k0 + 32 * x + 8 * (r >> 2) + 4 * h + (r & 3);
                    if (key > p || key < p_lo) st[x][r] = -INFINITY;
                }
        }
        float mt = -INFINITY;
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) mt = fmaxf(mt, st[x][r]);
        {
            const unsigned u = __float_as_uint(mt);
            const auto x = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            mt = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
        }
        // m need not be the maximum, only near it: sums are rescaled when a row's has grown by 2^8 or more
        if (__any((mt - m) * c > 8.f)) {
            const float mn = fmaxf(m, mt), f = __builtin_amdgcn_exp2f((m - mn) * c);
            l *= f;
#pragma unroll
            for (int i = 0; i < NB; ++i) o[i] *= f;
            m = mn;
            set_off();
        }
        float sub = off, sum[4] = {0.f, 0.f, 0.f, 0.f};
        if (far) {
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[x][r] -= m;
            sub = 0.f;
        }
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                st[x][r] = __builtin_amdgcn_exp2f(fmaf(st[x][r], c, -sub));
                sum[r & 3] += st[x][r];
            }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        const int i = lane & 15;
        const int sw[2] = {W::swizzle((i >> 2) + 4 * h), W::swizzle((i >> 2) + 4 * h + 8)};
        const int c0 = ((lane & 16) >> 3) + ((i & 3) >> 1);
        if constexpr (FP8) __builtin_amdgcn_s_setprio(1); // (mixed batch, d = 64: 42.3 -> 39.6 us; with 16-bit pages a chunk behind 15872 keys 85.2 -> 88.7)
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            if constexpr (FP8) {
                __builtin_amdgcn_sched_barrier(0); // (the factors would be fetched for both halves, into registers that are not there)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 f = *reinterpret_cast<const float4 *>(buf + W::oVS + (32 * x + 8 * g + 4 * h) * 4);
                    st[x][4 * g] *= f.x; st[x][4 * g + 1] *= f.y; st[x][4 * g + 2] *= f.z; st[x][4 * g + 3] *= f.w;
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                bf16x8 pt;
#pragma unroll
                for (int u = 0; u < 8; ++u) pt[u] = (bf16)st[x][8 * y + u];
                const unsigned char *vr = buf + W::oV + (32 * x + 16 * y + 4 * h + (i >> 2)) * W::ROWB + 8 * (i & 1);
#pragma unroll
                for (int d = 0; d < NB; ++d) {
                    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                    const s16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vr + (((4 * d + c0) ^ sw[0]) << 4)));
                    const s16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vr + 8 * W::ROWB + (((4 * d + c0) ^ sw[1]) << 4)));
                    const s16x8 v = __builtin_shufflevector(va, vb, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), pt, o[d], 0, 0, 0);
                }
            }
        }
    };

    // One barrier per tile: the other buffer was last read before the barrier in front of this tile.
    auto seen = [&](int k0) { return k0 <= some_to && k0 + KEYS > some_from; };
    if (k_begin < k_end) {
        look_up(k_begin);
        if constexpr (FP8) {
            fetch_all(wsmem, k_begin);
            park(wsmem, k_begin);
            if (k_begin + KEYS < k_end) fetch_all(wsmem, k_begin + KEYS);
            lds_barrier();
            for (int k0 = k_begin, j = 0; k0 < k_end; k0 += KEYS, j ^= 1) {
                if (k0 + KEYS < k_end) park(wsmem + (j ^ 1) * W::SIZE, k0 + KEYS);
                const bool more = k0 + 2 * KEYS < k_end;
                if (seen(k0)) work(wsmem + j * W::SIZE, k0, wsmem, k0 + 2 * KEYS, more);
                else if (more) fetch_all(wsmem, k0 + 2 * KEYS);
                lds_barrier();
            }
        } else {
            fetch_all(wsmem, k_begin);
            for (int k0 = k_begin, j = 0; k0 < k_end; k0 += KEYS, j ^= 1) {
                wait_moved();
                lds_barrier();
                const bool more = k0 + KEYS < k_end;
                if (seen(k0)) work(wsmem + j * W::SIZE, k0, wsmem + (j ^ 1) * W::SIZE, k0 + KEYS, more);
                else if (more) fetch_all(wsmem + (j ^ 1) * W::SIZE, k0 + KEYS);
            }
        }
    }
    {
        const unsigned u = __float_as_uint(l);
        const auto x = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    if (wrow + col >= row1) return;
    // element 32 d + 8 g + 4 h + i of the lane's row stands at o[d][4 g + i]
    const long out = (long)(s.r0 + tok) * a.r.Hq + head;
    if (splits == 1) {
        const float inv = inverse_sum(l);
        bf16 *to = static_cast<bf16 *>(a.r.q_out) + out * D + 4 * h;
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<bf16x4 *>(to + 32 * d + 8 * g) = bf16x4{(bf16)(o[d][4 * g] * inv), (bf16)(o[d][4 * g + 1] * inv), (bf16)(o[d][4 * g + 2] * inv), (bf16)(o[d][4 * g + 3] * inv)};
    } else {
        float *ml, *po;
        partial_of(a, split, out, D, &ml, &po);
        if (h == 0) *reinterpret_cast<float2 *>(ml) = make_float2(m, l);
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4 *>(po + 32 * d + 8 * g + 4 * h) = make_float4(o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]);
    }
}

template <typename T, typename CT, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_attn_few(AttnArgs a, int tiles, Cut cut, int max_rows) {
    extern __shared__ __align__(16) unsigned char lds[];
    attend_few<T, CT, D, WAVES>(a, tiles, cut, max_rows, blockIdx.x, reinterpret_cast<float *>(lds));
}
template <typename CT, int D>
__global__ __launch_bounds__(64 * kWideWaves, D > 128 ? 1 : 2) void k_attn_wide(AttnArgs a, Cut cut, int few_rows) {
    extern __shared__ __align__(16) unsigned char lds[];
    attend_wide<CT, D>(a, cut, few_rows, true, blockIdx.x, lds);
}
// Chunks beside single tokens: both kinds of workgroup in one launch, the long ones first, so that the short ones, which wait for memory, run under them.  12 chunks of up to 256 tokens
// and 12 single ones, 32 heads (8 of keys) of 64, e4m3, window 1024: 39.5 us, the matrix pipes busy for 0.13, the vector ALU for 0.34, the waves waiting for 0.44 of their time: with 8-bit pages at d = 64 and 128 the compiled
// loop waits for the tile that it has just requested before it takes the first maximum, so that no request is under way under the softmax.
template <typename CT, int D>
__global__ __launch_bounds__(64 * kWideWaves, D > 128 ? 1 : 2) void k_attn_both(AttnArgs a, int tiles, Cut few, Cut wide, int few_rows, int wide_blocks) {
    extern __shared__ __align__(16) unsigned char lds[];
    if ((int)blockIdx.x < wide_blocks) attend_wide<CT, D>(a, wide, few_rows, false, blockIdx.x, lds);
    else attend_few<bf16, CT, D, kFewWaves>(a, tiles, few, few_rows, blockIdx.x - wide_blocks, reinterpret_cast<float *>(lds));
}

// Joins the splits of a row (token and head): 8192 rows of 128 in eight pieces (36 MB) 10 us, 16 rows in 64 pieces 4 us.  ALL: a wave for each row, of either kind; else of the sequences that attend_few takes, where there are no others.
// WHOLE: a workgroup per row, for few rows with many splits (16 rows of 128, 64 splits: a wave per row took 17 us, one load after the other).
template <typename T, int D, bool ALL, bool WHOLE>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, Cut few, Cut wide, int few_rows, int per_seq) {
    constexpr int LPR = D / 4, TPR = WHOLE ? 256 : 64, SIDE = TPR / LPR; // lanes of a row, threads of a row, splits side by side
    __shared__ float part[WHOLE ? 4 : 1][D + 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = a.r.Hq / a.r.Hkv;
    int n, kvh, r;
    SeqRows s;
    if (ALL) {
        const long row = (long)blockIdx.x * 4 + wave;
        if (row >= (long)a.r.T * a.r.Hq) return;
        const int t = (int)(row / a.r.Hq), h = (int)(row % a.r.Hq);
        n = seq_of_row(a.c.cu, a.c.N, t);
        if (n >= a.c.N) return; // (zeroed)
        s.load(a, n);
        kvh = h / G; r = max(t - s.r0, 0) * G + h % G;
    } else {
        long b = WHOLE ? (long)blockIdx.x : (long)blockIdx.x * 4 + wave;
        r = (int)(b % per_seq); b /= per_seq;
        kvh = (int)(b % a.r.Hkv); n = (int)(b / a.r.Hkv);
        if (n >= a.c.N) return;
        s.load(a, n);
    }
    const int R = (s.r1 - s.r0) * G;
    if (!ALL && (r >= R || R > few_rows)) return;
    const bool is_few = !ALL || R <= few_rows;
    const Cut cut = is_few ? few : wide;
    if (cut.splits == 1) return; // (stored as they are)
    const int rows = is_few ? kFewTile : kWideRows;
    int lo, from, hi;
    key_range(a, s, G, r / rows * rows, min(r / rows * rows + rows, R), is_few ? kFewKeys : wide_keys(D), lo, from, hi);
    const int live = hi > lo ? min((hi - lo + cut.keys - 1) / cut.keys, cut.splits) : 0;
    const long row = (long)(s.r0 + r / G) * a.r.Hq + kvh * G + r % G;
    const int in = WHOLE ? threadIdx.x : lane, e0 = in % LPR * 4, side = in / LPR;
    // the first pieces are on their way while the maximum is found
    constexpr int AHEAD = 4;
    float *ml, *po;
    float2 wl[AHEAD];
    f32x4 w[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        partial_of(a, min(side + u * SIDE, max(live - 1, 0)), row, D, &ml, &po);
        wl[u] = *reinterpret_cast<const float2 *>(ml);
        w[u] = *reinterpret_cast<const f32x4 *>(po + e0);
    }
    float M = kNoScore;
    for (int i = lane; i < live; i += 64) {
        partial_of(a, i, row, D, &ml, &po);
        M = fmaxf(M, ml[0]);
    }
    M = lanes_max<64>(M);
    const float c = a.scale * kLog2e;
    float L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (side + u * SIDE < live) {
            const float f = __builtin_amdgcn_exp2f((wl[u].x - M) * c);
            L = fmaf(wl[u].y, f, L);
            acc += w[u] * f;
        }
#pragma unroll 4
    for (int i = side + AHEAD * SIDE; i < live; i += SIDE) {
        partial_of(a, i, row, D, &ml, &po);
        const float f = __builtin_amdgcn_exp2f((ml[0] - M) * c);
        L = fmaf(ml[1], f, L);
        acc += *reinterpret_cast<const f32x4 *>(po + e0) * f;
    }
#pragma unroll
    for (int m = LPR; m < 64; m <<= 1) {
        L += __shfl_xor(L, m);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], m);
    }
    if constexpr (WHOLE) {
        if (lane < LPR) {
#pragma unroll
            for (int j = 0; j < 4; ++j) part[wave][e0 + j] = acc[j];
            if (lane == 0) part[wave][D] = L;
        }
        __syncthreads();
        if (threadIdx.x >= LPR) return;
        L = (part[0][D] + part[1][D]) + (part[2][D] + part[3][D]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = (part[0][e0 + j] + part[1][e0 + j]) + (part[2][e0 + j] + part[3][e0 + j]);
    } else if (lane >= LPR) return;
    const float inv = inverse_sum(L);
    typedef T out4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<out4 *>(static_cast<T *>(a.r.q_out) + row * D + e0) = out4{(T)(acc[0] * inv), (T)(acc[1] * inv), (T)(acc[2] * inv), (T)(acc[3] * inv)};
}

namespace {

// Rows of a sequence and key/value head up to which the kernel for few rows takes them (fp32: always).
constexpr int kFewMost = 32;
constexpr int kMostSplits = 128;
constexpr int kUncut = 640 * 128;

// waves: of a workgroup of attend_few; per_seq: most rows of a sequence and key/value head that attend_few has; tiles: its tiles of them (0: there is none); slots: row tiles of attend_wide
struct Plan { int few_rows, per_seq, tiles, slots, waves; Cut few, wide; };

// `range` keys at most, in `blocks` workgroups without a cut: as many splits as make up to `want` workgroups, each of `least` keys or more.
Cut cut_keys(long range, long blocks, long want, long least, int step) {
    long splits = want / blocks, most = (range + least - 1) / least;
    splits = splits < most ? splits : most;
    splits = splits < 1 ? 1 : splits > kMostSplits ? kMostSplits : splits;
    long keys = (range + splits - 1) / splits;
    keys = (keys + step - 1) / step * step;
    Cut c;
    c.keys = (int)(keys < step ? step : keys);
    c.splits = (int)((range + c.keys - 1) / c.keys);
    c.splits = c.splits < 1 ? 1 : c.splits;
    return c;
}

// Tiles and splits by the bounds that the host knows.
Plan plan_attn(int dtype, int d, const AttnArgs &a) {
    const int G = a.r.Hq / a.r.Hkv;
    const long most = (long)a.max_q * G, rows = (long)a.r.T * G, N = a.c.N;
    Plan p;
    // A batch of equal chunks has none of few rows where the bounds are exact; should they not be (padded rows), k_attn_wide is right for those too.
    const bool equal = dtype != 0 && most > kFewMost && N * a.max_q == a.r.T;
    p.few_rows = dtype == 0 ? 0x7fffffff : equal ? 0 : kFewMost;
    p.per_seq = (int)(most < p.few_rows ? most : p.few_rows);
    p.tiles = (p.per_seq + kFewTile - 1) / kFewTile;
    p.slots = 0;
    if (most > p.few_rows) { // sum of ceil(R / 128) over the sequences
        const long by_rows = rows / kWideRows + N, by_most = N * ((most + kWideRows - 1) / kWideRows);
        p.slots = (int)(by_rows < by_most ? by_rows : by_most);
    }
    if (p.tiles < 1 && !p.slots) p.tiles = 1; // (it also zeroes the rows that lie in no sequence)
    auto range = [&](int step) {
        const long seen = a.window > 0 ? (long)a.window + a.max_q + step : a.c.max_kv;
        return seen < a.c.max_kv ? seen : (long)a.c.max_kv;
    };
    const long full = rows / kWideRows;
    p.wide = p.slots ? cut_keys(range(wide_keys(d)), (full > 0 ? full : 1) * a.r.Hkv, d > 128 ? 256 : d > 64 ? 512 : 768, 512, wide_keys(d)) : Cut{1, 64};
    // A second launch for the join and the splits' way through memory cost 4 to 5 us, a walk 1 us for each 128 keys of d = 128: contexts up to kUncut / d are not cut
    // (one token over 300 keys, d = 128: 7.5 us instead of 10.5; over 500, 8.9 instead of 10.6; over 1000 it would take 13.0 instead of 11.0), and never into more
    // than 64 (32768 keys, e4m3, 4 heads: 15.1 us, in 128 pieces 16.4).  Beside chunks, whose walks take longer per key, no finer than twice as long as those, and not at
    // all where those are not: the join would cost more than it brought.  (Most of these sequences are single tokens: one tile.)
    const long seen = range(kFewKeys), blocks = (N > 0 ? N : 1) * (p.slots ? 1 : p.tiles) * a.r.Hkv, uncut = kUncut / (dtype == 0 ? 2 * d : d);
    const long least = !p.slots ? (seen <= uncut ? seen : 256) : p.wide.splits == 1 ? seen : 2l * p.wide.keys;
    // Workgroups of eight waves, one per CU: a CU has more loads under way and rounds end closer together (equal contexts of 1000 keys, d = 128, 256 workgroups: 22.6 us instead of 26.2, e4m3 14.8
    // instead of 18.1), except between one and two workgroups per CU, where two of four waves are all under way at once (320 of 1000 keys: 31.3 us instead of 33.9, e4m3 19.3 instead of 23.4; 496: 40.5
    // instead of 40.8, 23.2 instead of 25.7).  At 512, where one round still holds all, equal contexts are 2 and 8 % faster by four waves, ragged ones (a quarter of the longest up, mean of eight
    // batches) 2 % slower at d = 128 and 5 % faster in e4m3, 3 % faster at d = 64 and 10 % slower in e4m3; at 528 eight waves take 0.98, 1.03, 0.92 of the time of four (16 bits, e4m3, d = 64), at
    // 640 0.98, 0.96, 0.97.  (Between 256 and 512 ragged batches go either way: at 320 0.89, 0.92, 1.07.)
    const bool twice = !p.slots && (dtype == 0 ? few_twice<float>(d) : few_twice<bf16>(d)) && (blocks <= 256 || blocks >= 512) && seen > kFewWaves * kFewKeys;
    p.waves = twice ? 2 * kFewWaves : kFewWaves;
    const long want = twice ? 256 : 512;
    p.few = p.per_seq && N ? cut_keys(seen, blocks, 64 * blocks < want ? 64 * blocks : want, least > 256 ? least : 256, kFewKeys * p.waves) : Cut{1, 128};
    return p;
}

int most_splits(const Plan &p) { return p.few.splits > p.wide.splits ? p.few.splits : p.wide.splits; }
size_t workspace_of(const AttnArgs &a, int d, const Plan &p) {
    const int splits = most_splits(p);
    if (splits == 1 || a.r.T == 0) return 0;
    const size_t rows = (size_t)splits * a.r.T * a.r.Hq;
    return (((2 * rows + 3) & ~size_t(3)) + rows * d) * sizeof(float);
}

// Workgroups of a launch: one of 2^32 threads or more is cut to the low 32 bits without an error.
long most_blocks(int threads) { return ((1l << 32) - 1) / threads; }
int launch(const char *name, const void *fn, long blocks, int threads, int lds, void **args, hipStream_t stream) {
    if (blocks > most_blocks(threads)) return (int)hipErrorInvalidConfiguration;
    if (lds > 64 * 1024)
        if (const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds)) return (int)e;
    prof_begin(name, stream);
    const hipError_t e = hipLaunchKernel(fn, dim3((unsigned)blocks), dim3(threads), args, lds, stream);
    prof_end(stream);
    return (int)e;
}

template <typename T, typename CT, int D> int launch_attn(int dtype, AttnArgs a, hipStream_t stream) {
    Plan p = plan_attn(dtype, D, a);
    a.splits = most_splits(p);
    const int few_lds = p.waves * kFewTile * (D + 4 + 2) * 4;
    const long few_blocks = p.tiles ? ((long)a.c.N * p.tiles + 1) * p.few.splits * a.r.Hkv : 0, wide_blocks = (long)p.slots * p.wide.splits * a.r.Hkv;
    int e = 0;
    if (few_blocks + wide_blocks > most_blocks(64 * p.waves) && a.c.N > 1) {
        // One half of the sequences after the other.  (So many are not cut more finely by halves: the workspace suffices for each.)
        AttnArgs b = a;
        a.c.N /= 2;
        a.zero_rest = 0;
        b.c.cu += a.c.N; b.c.kv_len += a.c.N; b.c.table += (long)a.c.N * a.c.max_pages; b.c.N -= a.c.N;
        b.zero_front = 0;
        e = launch_attn<T, CT, D>(dtype, a, stream);
        return e ? e : launch_attn<T, CT, D>(dtype, b, stream);
    }
    if (p.slots == 0) {
        void *args[] = {&a, &p.tiles, &p.few, &p.few_rows};
        const void *fn = reinterpret_cast<const void *>(k_attn_few<T, CT, D, kFewWaves>);
        if constexpr (few_twice<T>(D))
            if (p.waves != kFewWaves) fn = reinterpret_cast<const void *>(k_attn_few<T, CT, D, 2 * kFewWaves>);
        e = launch("k_attn_few", fn, few_blocks, 64 * p.waves, few_lds, args, stream);
    }
    if constexpr (sizeof(T) == 2)
        if (p.slots) {
            constexpr int wide_lds = 2 * WideTile<CT, D>::SIZE;
            int first = (int)wide_blocks;
            if (p.tiles) {
                void *args[] = {&a, &p.tiles, &p.few, &p.wide, &p.few_rows, &first};
                e = launch("k_attn_both", reinterpret_cast<const void *>(k_attn_both<CT, D>), wide_blocks + few_blocks, 64 * kWideWaves, wide_lds > few_lds ? wide_lds : few_lds, args, stream);
            } else {
                void *args[] = {&a, &p.wide, &p.few_rows};
                e = launch("k_attn_wide", reinterpret_cast<const void *>(k_attn_wide<CT, D>), wide_blocks, 64 * kWideWaves, wide_lds, args, stream);
            }
            if (e || a.splits == 1) return e;
            void *join[] = {&a, &p.few, &p.wide, &p.few_rows, &p.per_seq};
            return launch("k_attn_join", reinterpret_cast<const void *>(k_attn_join<T, D, true, false>), ((long)a.r.T * a.r.Hq + 3) / 4, 256, 0, join, stream);
        }
    if (e || a.splits == 1) return e;
    const long rows = (long)a.c.N * a.r.Hkv * p.per_seq;
    const bool whole = rows <= 2048;
    void *join[] = {&a, &p.few, &p.wide, &p.few_rows, &p.per_seq};
    return launch("k_attn_join", whole ? reinterpret_cast<const void *>(k_attn_join<T, D, false, true>) : reinterpret_cast<const void *>(k_attn_join<T, D, false, false>),
                  whole ? rows : (rows + 3) / 4, 256, 0, join, stream);
}

} // namespace

size_t paged_attn_workspace(int dtype, int d, const AttnArgs &a) { return workspace_of(a, d, plan_attn(dtype, d, a)); }

int run_paged_attn(int dtype, int d, bool fp8_pages, const AttnArgs &a, hipStream_t stream) {
    if (a.r.T == 0) return 0;
    if (dtype == 0) {
        if (d == 32) return launch_attn<float, float, 32>(dtype, a, stream);
        if (d == 64) return launch_attn<float, float, 64>(dtype, a, stream);
        if (d == 128) return launch_attn<float, float, 128>(dtype, a, stream);
    } else if (fp8_pages) {
        if (d == 64) return launch_attn<bf16, fp8, 64>(dtype, a, stream);
        if (d == 128) return launch_attn<bf16, fp8, 128>(dtype, a, stream);
        if (d == 256) return launch_attn<bf16, fp8, 256>(dtype, a, stream);
    } else {
        if (d == 64) return launch_attn<bf16, bf16, 64>(dtype, a, stream);
        if (d == 128) return launch_attn<bf16, bf16, 128>(dtype, a, stream);
        if (d == 256) return launch_attn<bf16, bf16, 256>(dtype, a, stream);
    }
    return (int)hipErrorInvalidValue;
}

} // namespace dn
