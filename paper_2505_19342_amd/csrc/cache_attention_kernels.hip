// Attention of new tokens over the paged cache of 8-bit values (include/astra.h, astra_cache_attention).
#include "cache_common.h"

#include <type_traits>

namespace astra {

// ------------------------------------------------------------------------------------------------
// The query rows of a sequence that share a KV head (H_q / H_kv heads of each new token) are the 16 columns of the products, so
// that a page is read once for all of them.  A wavefront walks tiles of 32 tokens with its own running maximum.
//
// Both contractions of a tile run on 16x16x32 bf16 MFMAs: e4m3 codes convert to bf16 exactly, a block's scale is applied in fp32 to the
// scores (keys) and to the probabilities (values).  S^T = K . Q^T has tokens on the M side and query rows on the N side, so a
// lane's scores all belong to one row and already are the B operand of O^T += V^T . P^T: lane l (column l % 16, l / 16 = g)
// holds tokens 4g .. 4g+3 and 16+4g .. 16+4g+3.  Channels may be dealt to the contraction index in any way that keys and
// queries share: 16 neighbouring ones per lane make 16-byte loads.  Values come as DH / 16 neighbouring channels of each of a
// lane's eight tokens; byte permutes put two tokens side by side before the conversion.
// fp32 operands keep their precision as sums of bf16 parts: queries of three (8 + 8 + 8 mantissa bits), probabilities of three, or of two for bf16 results
// (16 bits, 2^-17 relative, beside the result's own 2^-9).
// ------------------------------------------------------------------------------------------------
#define CA_INLINE __attribute__((always_inline))
constexpr int kCaTile = 32;
constexpr float kCaLazy = 8.f;       // base-2 units a score may exceed the running reference by before the sums are rescaled
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef const __attribute__((address_space(1))) char* gbytes;
typedef const __attribute__((address_space(4))) int32_t* cints;      // read as one by a wavefront: scalar loads
typedef const __attribute__((address_space(4))) float* cfloats;
template <typename V>
__device__ __forceinline__ V ld_global(gbytes at) { return *reinterpret_cast<const __attribute__((address_space(1))) V*>(at); }

__device__ __forceinline__ f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

struct CacheAttnParams {
    CacheStep c;
    const void* q;
    const uint8_t* k_pages;
    const uint8_t* v_pages;
    const float* k_scales;
    const float* v_scales;
    const void* prior_out;
    const float* prior_lse;
    void* out;
    float* lse;
    int32_t q_stride;
    float scale;
};

template <bool HIGH>
__device__ __forceinline__ uint32_t two_codes(uint32_t w) {          // bytes 0 and 1 (2 and 3) as bf16
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HIGH));
}
__device__ __forceinline__ bf16x8 eight_codes(uint32_t lo, uint32_t hi) {
    u32x4 w;
    w.x = two_codes<false>(lo);
    w.y = two_codes<true>(lo);
    w.z = two_codes<false>(hi);
    w.w = two_codes<true>(hi);
    return __builtin_bit_cast(bf16x8, w);
}
// any of four e4m3 bytes a NaN (all seven bits below the sign set)
__device__ __forceinline__ bool any_nan(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; }

// What a wavefront knows of its query rows: a block of 16 rows (new token, head) of one sequence and KV head
struct RowBlock {
    int seq, kv_head;
    int len, n_new, from;        // cached tokens, new tokens, first row of the sequence
    int row0, n_rows;            // first (token, head) row of the block, rows of the sequence in all
    int least, all;              // tokens that the block's first row and its last one attend to
};

template <int DH, typename T>
struct CacheWalk {
    static constexpr int KJ = DH / 64;         // 16-byte pieces of a key row per lane
    static constexpr int KC = DH / 32;         // contraction steps of a score
    static constexpr int VCH = DH / 16;        // value channels per lane
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int QP = F32 ? 3 : 1, PP = F32 ? 3 : 2;
    using Piece = std::conditional_t<DH == 256, u32x4, std::conditional_t<DH == 128, u32x2, uint32_t>>;

    struct Tile {
        u32x4 k[2][KJ];                        // codes of the two 16-token halves
        Piece v[8];
        float ks[2], vs[2];
        bool there[2];
    };

    bf16x8 q[QP][KC];
    f32x4 acc[VCH];
    float m, l;
    int sees;                                  // tokens that this lane's row attends to

    __device__ __forceinline__ void start(const CacheAttnParams& p, const RowBlock& b) {
        const int lane = lane_id(), col = lane & 15, g = lane >> 4;
        const int share = p.c.Hq / p.c.Hkv;
        const int row = min(b.row0 + col, b.n_rows - 1), token = row / share, head = b.kv_head * share + row - token * share;
        sees = min(b.len + token + 1, p.c.capacity());
        const gbytes at = (gbytes)p.q + ((int64_t)(b.from + token) * p.q_stride + head * DH + 16 * g) * (int64_t)sizeof(T);
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
            const gbytes a = at + (64 * (kc >> 1) + 8 * (kc & 1)) * (int)sizeof(T);
            if constexpr (!F32) {
                q[0][kc] = __builtin_bit_cast(bf16x8, ld_global<u32x4>(a));
            } else {
                const f32x4 x0 = ld_global<f32x4>(a), x1 = ld_global<f32x4>(a + 16);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = e < 4 ? x0[e & 3] : x1[e & 3];
#pragma unroll
                    for (int i = 0; i < QP; ++i) {             // every difference is exact
                        const float part = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
                        q[i][kc][e] = (__bf16)part;
                        x -= part;
                    }
                }
            }
        }
#pragma unroll
        for (int c = 0; c < VCH; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = -INFINITY;
        l = 0.f;
    }

    // token of score / value element e inside a tile
    static __device__ __forceinline__ int tok(int e, int g) { return (e < 4 ? 0 : 12) + 4 * g + e; }

    __device__ __forceinline__ void load(const CacheAttnParams& p, const RowBlock& b, int t, Tile& x) const {
        const CacheStep& c = p.c;
        const int lane = lane_id(), col = lane & 15, g = lane >> 4;
        const int last = b.all - 1, in_page = (1 << c.page_shift) - 1;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int first = min(t * kCaTile + 16 * hf, last);                     // tokens beyond the last repeat it
            const int id = __builtin_amdgcn_readfirstlane(((cints)c.table)[(int64_t)b.seq * c.table_stride + (first >> c.page_shift)]);
            x.there[hf] = id >= 0 && id < c.n_pages;
            const int64_t block = (int64_t)(x.there[hf] ? id : 0) * c.Hkv + b.kv_head;
            // a page that is not there: page 0's codes are asked for and count for nothing, whatever they and its scales are
            x.ks[hf] = x.there[hf] ? ((cfloats)p.k_scales)[block] : 0.f;
            x.vs[hf] = x.there[hf] ? ((cfloats)p.v_scales)[block] : 0.f;
            const gbytes kb = (gbytes)p.k_pages + (block << c.page_shift) * DH, vb = (gbytes)p.v_pages + (block << c.page_shift) * DH;
            const uint32_t row = (uint32_t)(min(t * kCaTile + 16 * hf + col, last) & in_page);
#pragma unroll
            for (int j = 0; j < KJ; ++j) x.k[hf][j] = ld_global<u32x4>(kb + (row * DH + 16u * g + 64u * j));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t r = (uint32_t)(min(t * kCaTile + 16 * hf + 4 * g + e, last) & in_page);
                x.v[4 * hf + e] = ld_global<Piece>(vb + (r * DH + (uint32_t)VCH * col));
            }
        }
    }

    __device__ __forceinline__ static uint32_t word(const Piece& v, int d) {
        if constexpr (DH == 64) return v;
        else return v[d];
    }

    // a tile's scores into the running sums
    __device__ __forceinline__ void absorb(const CacheAttnParams& p, const RowBlock& b, int t, Tile& x) {
        const int g = lane_id() >> 4;
        const float sl2 = p.scale * kLog2e;
        float s[8];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kc = 0; kc < KC; ++kc) {
                const u32x4& w = x.k[hf][kc >> 1];
                const bf16x8 kf = kc & 1 ? eight_codes(w.z, w.w) : eight_codes(w.x, w.y);
#pragma unroll
                for (int i = 0; i < QP; ++i) d = mfma_16x16x32(kf, q[i][kc], d);
            }
            const float f = sl2 * x.ks[hf];
#pragma unroll
            for (int v = 0; v < 4; ++v) s[4 * hf + v] = d[v] * f;
        }
        const bool masked = t * kCaTile + kCaTile > b.least || !x.there[0] || !x.there[1];        // of the whole wavefront
        if (masked)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = x.there[e >> 2] && t * kCaTile + tok(e, g) < sees ? s[e] : -INFINITY;
        float mx = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[e]);
        if (__builtin_amdgcn_ballot_w64(mx > m + kCaLazy) != 0) {
            mx = fmaxf(mx, __shfl_xor(mx, 16));              // the four lanes of a column share one reference
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m, mx);
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
            l *= alpha;
#pragma unroll
            for (int c = 0; c < VCH; ++c) acc[c] *= alpha;
            m = m_new;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        u32x4 part[PP];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float a = __builtin_amdgcn_exp2f(s[e] - ref), c = __builtin_amdgcn_exp2f(s[e + 1] - ref);
            l += a;
            l += c;
            a *= x.vs[e >> 2];
            c *= x.vs[e >> 2];
#pragma unroll
            for (int i = 0; i < PP; ++i) {                    // the upper halves of both; what is left of them is exact
                part[i][e >> 1] = __builtin_amdgcn_perm(__float_as_uint(c), __float_as_uint(a), 0x07060302u);
                a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
                c -= __uint_as_float(__float_as_uint(c) & 0xffff0000u);
            }
        }
        bool odd = false;
        if (masked) {
            uint32_t bad = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!x.there[e >> 2]) x.v[e] = Piece{};
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int d = 0; d < VCH / 4; ++d) bad |= any_nan(word(x.v[e], d)) ? 1u : 0u;
            odd = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
        }
        if (__builtin_expect(odd, 0)) {
            careful(b, t, x, part);
            return;
        }
#pragma unroll
        for (int c2 = 0; c2 < VCH / 2; ++c2) {                // two neighbouring channels
            const uint32_t sel = c2 & 1 ? 0x07030602u : 0x05010400u;
            u32x4 lo, hi;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint32_t w = __builtin_amdgcn_perm(word(x.v[e + 1], c2 >> 1), word(x.v[e], c2 >> 1), sel);
                lo[e >> 1] = two_codes<false>(w);
                hi[e >> 1] = two_codes<true>(w);
            }
#pragma unroll
            for (int i = 0; i < PP; ++i) {
                acc[2 * c2] = mfma_16x16x32(__builtin_bit_cast(bf16x8, lo), __builtin_bit_cast(bf16x8, part[i]), acc[2 * c2]);
                acc[2 * c2 + 1] = mfma_16x16x32(__builtin_bit_cast(bf16x8, hi), __builtin_bit_cast(bf16x8, part[i]), acc[2 * c2 + 1]);
            }
        }
    }

    // A tile that hides some token from some row and holds a NaN among its values: zero times NaN would reach rows that do not attend to it.
    // Token by token, a row takes only the products of those it sees.
    __device__ __forceinline__ void careful(const RowBlock& b, int t, const Tile& x, const u32x4 (&part)[PP]) {
        const int g = lane_id() >> 4;
#pragma unroll 1
        for (int e = 0; e < 8; ++e)
#pragma unroll 1
            for (int gg = 0; gg < 4; ++gg) {
                const int token = t * kCaTile + tok(e, gg);
                if (!(e < 4 ? x.there[0] : x.there[1]) || token >= b.all) continue;
#pragma unroll
                for (int c = 0; c < VCH; ++c) {
                    uint32_t code = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) code = k == e ? (word(x.v[k], c >> 2) >> (8 * (c & 3))) & 0xffu : code;
                    const uint32_t one = g == gg ? two_codes<false>(code) & 0xffffu : 0u;
                    u32x4 w;
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = k == e >> 1 ? (e & 1 ? one << 16 : one) : 0u;
                    f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < PP; ++i) d = mfma_16x16x32(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, part[i]), d);
                    if (token < sees) acc[c] += d;
                }
            }
    }

    // of a column, once all tiles are in
    __device__ __forceinline__ void finish_sum() {
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
    }
};

template <typename T>
__device__ __forceinline__ float as_float(T v) {
    if constexpr (sizeof(T) == 2) return bf16_bits_to_f32(v);
    else return v;
}

// A wavefront per block of 16 query rows
template <int DH, typename T>
__global__ __launch_bounds__(64) void cache_attn_kernel(const CacheAttnParams p) {
    using Walk = CacheWalk<DH, T>;
    const CacheStep& c = p.c;
    RowBlock b;
    b.seq = blockIdx.z;
    b.kv_head = blockIdx.y;
    b.len = cache_len(c, b.seq);
    b.from = cache_row(c, b.seq);
    b.n_new = max(cache_row(c, b.seq + 1) - b.from, 0);
    const int share = c.Hq / c.Hkv;
    b.n_rows = b.n_new * share;
    b.row0 = blockIdx.x * 16;
    if (b.row0 >= b.n_rows) return;
    b.least = min(b.len + b.row0 / share + 1, c.capacity());
    b.all = min(b.len + min(b.row0 + 15, b.n_rows - 1) / share + 1, c.capacity());
    Walk w;
    w.start(p, b);
    for (int t = 0; t * kCaTile < b.all; ++t) {
        typename Walk::Tile x;
        w.load(p, b, t, x);
        w.absorb(p, b, t, x);
    }
    w.finish_sum();
    const int lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int row = b.row0 + col;
    if (row >= b.n_rows) return;
    const int token = row / share, head = b.kv_head * share + row - token * share;
    const int64_t at = (int64_t)(b.from + token) * c.Hq + head;
    float m = w.m, wo = w.l > 0.f ? 1.f / w.l : 0.f, wp = 0.f;
    if (w.l != w.l) wo = w.l;
    float lse = w.l == 0.f ? -INFINITY : kLn2 * m + logf(w.l);
    if (p.prior_lse) {
        const float lp = p.prior_lse[at];
        const float top = fmaxf(lse, lp), top0 = top == -INFINITY ? 0.f : top;
        const float a = expf(lse - top0), bb = expf(lp - top0), all = a + bb;
        wo = all == 0.f ? 0.f : wo * a / all;
        wp = all == 0.f ? 0.f : bb / all;
        lse = all == 0.f ? -INFINITY : top0 + logf(all);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int ch = 0; ch < Walk::VCH; ++ch) {
            const int64_t i = at * DH + Walk::VCH * (4 * g + v) + ch;
            float o = w.l == 0.f ? 0.f : w.acc[ch][v] * wo;
            if (p.prior_lse && wp != 0.f) o += wp * as_float<T>(((const T*)p.prior_out)[i]);
            if constexpr (sizeof(T) == 2) ((uint16_t*)p.out)[i] = f32_to_bf16_bits(o);
            else ((float*)p.out)[i] = o;
        }
    if (g == 0 && p.lse) p.lse[at] = lse;
}

// ---- host ---------------------------------------------------------------------------------------
template <typename T>
static int launch_cache_attention(const CacheAttnParams& p, int dh, hipStream_t s) {
    const int64_t blocks = ceil_div((int64_t)p.c.n_tokens * (p.c.Hq / p.c.Hkv), 16);
    if (blocks > 0x7fffffff) return ASTRA_ERR_SHAPE;
    const dim3 grid((unsigned)blocks, p.c.Hkv, p.c.n_seqs);
    if (dh == 64) cache_attn_kernel<64, T><<<grid, 64, 0, s>>>(p);
    else if (dh == 128) cache_attn_kernel<128, T><<<grid, 64, 0, s>>>(p);
    else cache_attn_kernel<256, T><<<grid, 64, 0, s>>>(p);
    return launch_status();
}

}  // namespace astra

using namespace astra;

extern "C" {

size_t astra_cache_attention_workspace_bytes(const astra_cache_desc* desc) {
    if (check_cache_desc(desc) != ASTRA_OK) return 0;
    return 256;
}

int astra_cache_attention(const astra_cache_desc* desc, const int32_t* page_table, const int32_t* lens, const int32_t* first_row,
                          const void* q, const uint8_t* k_pages, const uint8_t* v_pages, const float* k_scales, const float* v_scales,
                          const void* prior_out, const float* prior_lse, void* out, float* lse_out, void* workspace,
                          size_t workspace_bytes, void* stream) {
    const int rc = check_cache_desc(desc);
    if (rc) return rc;
    if (desc->n_tokens == 0 || desc->n_seqs == 0) return ASTRA_OK;
    if (!page_table || !lens || !first_row || !q || !k_pages || !v_pages || !k_scales || !v_scales || !out || !prior_out != !prior_lse) return ASTRA_ERR_NULL;
    if (!workspace || workspace_bytes < astra_cache_attention_workspace_bytes(desc)) return ASTRA_ERR_WORKSPACE;
    for (const void* a : {q, (const void*)k_pages, (const void*)v_pages, prior_out, (const void*)out, (const void*)workspace})
        if ((uintptr_t)a % 16 != 0) return ASTRA_ERR_UNSUPPORTED;
    CacheAttnParams p{};
    p.c = cache_step(*desc, page_table, lens, first_row);
    p.q = q; p.k_pages = k_pages; p.v_pages = v_pages; p.k_scales = k_scales; p.v_scales = v_scales;
    p.prior_out = prior_out; p.prior_lse = prior_lse; p.out = out; p.lse = lse_out;
    p.q_stride = desc->q_stride ? desc->q_stride : desc->n_q_heads * desc->head_dim;
    p.scale = desc->scale != 0.f ? desc->scale : 1.f / sqrtf((float)desc->head_dim);
    if (desc->dtype == ASTRA_BF16) return launch_cache_attention<uint16_t>(p, desc->head_dim, (hipStream_t)stream);
    return launch_cache_attention<float>(p, desc->head_dim, (hipStream_t)stream);
}

}  // extern "C"
