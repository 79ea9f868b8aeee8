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
    // scratch, see CacheAttnScratch
    float* part_o;
    float* part_ml;
    int4* joins;
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
// the value of the lane 32 or 16 away
template <int X>
__device__ __forceinline__ float xor_rows(float v) {
    const uint32_t w = __float_as_uint(v);
    if constexpr (X == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);        // lower halves of both, upper halves of both
        return __uint_as_float(lane_id() & 32 ? r[0] : r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane16_swap(w, w, false, false);
        return __uint_as_float(lane_id() & 16 ? r[0] : r[1]);
    }
}
// 1 in each byte of w that is NaN (all seven bits below the sign set)
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u; }

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

    // a tile's codes and the scales of its two 16-token halves
    struct Keys {
        u32x4 k[2][KJ];
        float scale[2];
    };
    struct Values {
        Piece v[8];
        float scale[2];
    };
    struct Pages {                             // of the two halves
        int id[2];
        __device__ __forceinline__ bool there(const CacheStep& c, int hf) const { return id[hf] >= 0 && id[hf] < c.n_pages; }
        // a page that is not there: page 0's codes are asked for and count for nothing, whatever they and its scales are
        __device__ __forceinline__ int64_t block(const CacheStep& c, int hf, int kv_head) const { return (int64_t)(there(c, hf) ? id[hf] : 0) * c.Hkv + kv_head; }
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

    // a tile beyond the last repeats its last token
    __device__ __forceinline__ static Pages pages(const CacheAttnParams& p, const RowBlock& b, int t) {
        const cints row = (cints)p.c.table + (int64_t)b.seq * p.c.table_stride;
        const int last = b.all - 1;
        return Pages{{row[min(t * kCaTile, last) >> p.c.page_shift], row[min(t * kCaTile + 16, last) >> p.c.page_shift]}};
    }
    // Rows of a half as they lie in its page, whether or not a token is there yet (the page is): what is read beyond the last token is masked like any other.
    // bytes before the half's first row
    __device__ __forceinline__ static int64_t half_at(const CacheAttnParams& p, int64_t block, int t, int hf) {
        return ((block << p.c.page_shift) + ((t * kCaTile + 16 * hf) & ((1 << p.c.page_shift) - 1))) * DH;
    }
    __device__ __forceinline__ static void load(const CacheAttnParams& p, const RowBlock& b, int t, const Pages& pg, Keys& x) {
        const uint32_t lane_at = (uint32_t)(lane_id() & 15) * DH + (uint32_t)(lane_id() >> 4) * 16u;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int64_t block = pg.block(p.c, hf, b.kv_head);
            x.scale[hf] = ld_global<float>((gbytes)(p.k_scales + block));
            const gbytes kb = (gbytes)p.k_pages + half_at(p, block, t, hf);
#pragma unroll
            for (int j = 0; j < KJ; ++j) x.k[hf][j] = ld_global<u32x4>(kb + lane_at + 64 * j);
        }
    }
    __device__ __forceinline__ static void load(const CacheAttnParams& p, const RowBlock& b, int t, const Pages& pg, Values& x) {
        const uint32_t lane_at = (uint32_t)(lane_id() >> 4) * 4u * DH + (uint32_t)(lane_id() & 15) * VCH;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int64_t block = pg.block(p.c, hf, b.kv_head);
            x.scale[hf] = ld_global<float>((gbytes)(p.v_scales + block));
            const gbytes vb = (gbytes)p.v_pages + half_at(p, block, t, hf);
#pragma unroll
            for (int e = 0; e < 4; ++e) x.v[4 * hf + e] = ld_global<Piece>(vb + lane_at + e * DH);
        }
    }

    __device__ __forceinline__ static uint32_t word(const Piece& v, int d) {
        if constexpr (DH == 64) return v;
        else return v[d];
    }

    // scores of a tile in base-2 units, not yet masked
    __device__ __forceinline__ void score(const CacheAttnParams& p, const Keys& x, float (&s)[8]) const {
        const float sl2 = p.scale * kLog2e;
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
            const float f = sl2 * x.scale[hf];
#pragma unroll
            for (int v = 0; v < 4; ++v) s[4 * hf + v] = d[v] * f;
        }
    }

    // scores and values of a tile into the running sums
    __device__ __forceinline__ void absorb(const CacheAttnParams& p, const RowBlock& b, int t, const Pages& pg, float (&s)[8], Values& x) {
        const int g = lane_id() >> 4;
        const bool there[2] = {pg.there(p.c, 0), pg.there(p.c, 1)};
        if (t * kCaTile + kCaTile > b.least || !there[0] || !there[1]) {        // of the whole wavefront
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[e] = there[e >> 2] && t * kCaTile + tok(e, g) < sees ? s[e] : -INFINITY;
                if (!there[e >> 2]) x.v[e] = Piece{};
            }
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                if (!there[hf]) x.scale[hf] = 0.f;
            uint32_t bad = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int d = 0; d < VCH / 4; ++d) bad |= nan_bytes(word(x.v[e], d));
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(bad != 0) != 0, 0)) careful(t, x);
        }
        float mx = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[e]);
        mx = fmaxf(mx, xor_rows<32>(mx));                    // the four lanes of a column share one reference
        mx = fmaxf(mx, xor_rows<16>(mx));
        const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - ref);
        l *= alpha;
#pragma unroll
        for (int c = 0; c < VCH; ++c) acc[c] *= alpha;
        m = m_new;
        u32x4 part[PP];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float a = __builtin_amdgcn_exp2f(s[e] - ref), c = __builtin_amdgcn_exp2f(s[e + 1] - ref);
            l += a;
            l += c;
            a *= x.scale[e >> 2];
            c *= x.scale[e >> 2];
#pragma unroll
            for (int i = 0; i < PP; ++i) {                    // the upper halves of both; what is left of them is exact
                part[i][e >> 1] = __builtin_amdgcn_perm(__float_as_uint(c), __float_as_uint(a), 0x07060302u);
                a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
                c -= __uint_as_float(__float_as_uint(c) & 0xffff0000u);
            }
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
    // Products of ones (NaN here, token seen there) tell which sums become NaN; the NaN values themselves become zeros.
    __device__ __forceinline__ void careful(int t, Values& x) {
        const int g = lane_id() >> 4;
        u32x4 seen;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const int token = t * kCaTile + tok(e, g);
            seen[e >> 1] = (token < sees ? 0x3f80u : 0u) | (token + 1 < sees ? 0x3f800000u : 0u);          // values that are not there are zeros
        }
#pragma unroll
        for (int c2 = 0; c2 < VCH / 2; ++c2) {
            u32x4 lo, hi;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint32_t w = 0x38u * nan_bytes(__builtin_amdgcn_perm(word(x.v[e + 1], c2 >> 1), word(x.v[e], c2 >> 1), c2 & 1 ? 0x07030602u : 0x05010400u));
                lo[e >> 1] = two_codes<false>(w);
                hi[e >> 1] = two_codes<true>(w);
            }
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            const f32x4 a = mfma_16x16x32(__builtin_bit_cast(bf16x8, lo), __builtin_bit_cast(bf16x8, seen), zero);
            const f32x4 b = mfma_16x16x32(__builtin_bit_cast(bf16x8, hi), __builtin_bit_cast(bf16x8, seen), zero);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                acc[2 * c2][v] = a[v] > 0.f ? NAN : acc[2 * c2][v];
                acc[2 * c2 + 1][v] = b[v] > 0.f ? NAN : acc[2 * c2 + 1][v];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (DH == 64) x.v[e] &= ~(0xffu * nan_bytes(x.v[e]));
            else
#pragma unroll
                for (int d = 0; d < VCH / 4; ++d) x.v[e][d] &= ~(0xffu * nan_bytes(x.v[e][d]));
        }
    }

    // of a column, once all tiles are in
    __device__ __forceinline__ void finish_sum() {
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
    }
};

// ---- the work of a launch, dealt out --------------------------------------------------------------
// A unit is a tile of 32 tokens for one row block.  The units of all row blocks (sequence by sequence, head by head, block by block of 16 rows, the tiles of a
// block in order) are cut into equal shares, one per workgroup: ragged batches keep every workgroup busy equally long, and one long context is
// walked by all of them.  Only the device knows the lengths, so every workgroup adds them up itself.  The four wavefronts take the tiles
// of a share in turn and are joined in LDS.  Where a share ends inside a row block, the unnormalised sums go to the scratch array:
// a workgroup has at most two such pieces, one that ends a row block begun by others (slot 2w) and one that begins one (slot 2w + 1).
// The workgroup that begins a block notes how many pieces there are, and a second launch joins them in order.
constexpr int kCaWaves = 4, kCaThreads = kCaWaves * kWave;
constexpr int kCaMinShare = 8;        // tiles, two per wavefront
constexpr int kCaRows = 16;

// what their registers leave room for
template <int DH, typename T>
constexpr int kCaWgsPerCu = (DH == 64 ? 4 : DH == 128 ? 3 : 2) - (sizeof(T) == 4 ? 1 : 0);
constexpr int kCaCus = 256;

__device__ __forceinline__ int n_blocks(int n_rows) { return (n_rows + kCaRows - 1) / kCaRows; }

struct SequencePlan {
    int len, from, n_new, tiles, blocks;
    __device__ __forceinline__ SequencePlan(const CacheStep& c, int s) {
        len = cache_len(c, s);
        from = cache_row(c, s);
        n_new = max(cache_row(c, s + 1) - from, 0);
        tiles = (int)((min((int64_t)len + n_new, (int64_t)c.capacity()) + kCaTile - 1) / kCaTile);
        blocks = n_blocks(n_new * (c.Hq / c.Hkv));
    }
    __device__ __forceinline__ int64_t units(const CacheStep& c) const { return (int64_t)tiles * blocks * c.Hkv; }
};

template <typename T>
__device__ __forceinline__ float as_float(T v) {
    if constexpr (sizeof(T) == 2) return bf16_bits_to_f32(v);
    else return v;
}

// A row's result from its sums (reference m in base-2 units, sum l, values o of N neighbouring channels from `channel` on), joined to the prior
template <typename T>
struct RowResult {
    int64_t at;
    float wo, wp, lse;
    __device__ __forceinline__ RowResult(const CacheAttnParams& p, int64_t row_head, float m, float l) : at(row_head), wp(0.f) {
        wo = l != 0.f ? 1.f / l : 0.f;
        lse = l != 0.f ? kLn2 * m + logf(l) : -INFINITY;
        if (p.prior_lse) {
            const float lp = p.prior_lse[at], top = fmaxf(lse, lp), ref = top == -INFINITY ? 0.f : top;
            const float a = expf(lse - ref), b = expf(lp - ref), all = a + b;
            wo = all != 0.f ? wo * a / all : 0.f;
            wp = all != 0.f ? b / all : 0.f;
            lse = all != 0.f ? ref + logf(all) : -INFINITY;
        }
    }
    template <int N>
    __device__ __forceinline__ void store(const CacheAttnParams& p, int dh, int channel, float (&o)[N]) const {
        const int64_t i = at * dh + channel;
        T* out = (T*)p.out + i;
        const T* prior = (const T*)p.prior_out + i;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            o[e] *= wo;
            if (wp != 0.f) o[e] = fmaf(wp, as_float<T>(prior[e]), o[e]);
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < N; e += 2) *reinterpret_cast<uint32_t*>(out + e) = pack_bf16x2(o[e], o[e + 1]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) out[e] = o[e];
        }
    }
};

template <int DH, typename T>
__global__ __launch_bounds__(kCaThreads, (kCaWgsPerCu<DH, T>)) void cache_attn_kernel(const CacheAttnParams p) {
    using Walk = CacheWalk<DH, T>;
    constexpr int PASS = 4;                                       // channels per thread and pass when the wavefronts are joined
    constexpr int STRIDE = 16 * PASS + 4;
    __shared__ int64_t before[kCacheMaxSeqs + 1];                 // units before a sequence
    __shared__ int64_t wave_sum[kCaWaves];
    __shared__ float ml[kCaWaves][kCaRows][2];
    __shared__ __align__(16) float sums[kCaWaves][kCaRows][STRIDE];
    const CacheStep& c = p.c;
    const int tid = threadIdx.x, lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int share_h = c.Hq / c.Hkv;

    {
        constexpr int PER = kCacheMaxSeqs / kCaThreads;
        int64_t mine[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int s = tid * PER + i;
            mine[i] = sum;
            if (s < c.n_seqs) sum += SequencePlan(c, s).units(c);
        }
        int64_t scan = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t up = __shfl_up(scan, o);
            if (lane >= o) scan += up;
        }
        if (lane == 63) wave_sum[wave] = scan;
        __syncthreads();
        int64_t base = scan - sum;
        for (int w = 0; w < wave; ++w) base += wave_sum[w];
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (tid * PER + i <= c.n_seqs) before[tid * PER + i] = base + mine[i];
        if (tid == kCaThreads - 1 && c.n_seqs == kCacheMaxSeqs) before[kCacheMaxSeqs] = base + sum;
        __syncthreads();
    }
    const int64_t all = before[c.n_seqs];
    const int64_t share = max((all + gridDim.x - 1) / (int64_t)gridDim.x, (int64_t)kCaMinShare);
    int64_t u = (int64_t)blockIdx.x * share;
    const int64_t end = min(u + share, all);
    int4 join = {0, 0, 0, 0};

    while (u < end) {
        int lo = 0, n = c.n_seqs;                // the last sequence that begins at or before u; those without units are behind it
        while (n > 0) {
            const int half = n >> 1;
            if (before[lo + half] <= u) {
                lo += half + 1;
                n -= half + 1;
            } else {
                n = half;
            }
        }
        const int s = __builtin_amdgcn_readfirstlane(lo - 1);
        const SequencePlan sp(c, s);
        const int64_t in = u - before[s], row = in / sp.tiles;
        const int tile0 = __builtin_amdgcn_readfirstlane((int)(in - row * sp.tiles));
        const int count = __builtin_amdgcn_readfirstlane((int)min((int64_t)(sp.tiles - tile0), end - u));
        RowBlock b;
        b.seq = s;
        b.kv_head = __builtin_amdgcn_readfirstlane((int)(row / sp.blocks));
        b.len = __builtin_amdgcn_readfirstlane(sp.len);
        b.n_new = __builtin_amdgcn_readfirstlane(sp.n_new);
        b.from = __builtin_amdgcn_readfirstlane(sp.from);
        b.n_rows = b.n_new * share_h;
        b.row0 = __builtin_amdgcn_readfirstlane((int)(row % sp.blocks)) * kCaRows;
        b.least = (int)min((int64_t)b.len + b.row0 / share_h + 1, (int64_t)c.capacity());
        b.all = (int)min((int64_t)b.len + min(b.row0 + kCaRows - 1, b.n_rows - 1) / share_h + 1, (int64_t)c.capacity());

        Walk w;
        w.start(p, b);
        {
            // The next tile's keys are asked for as soon as this one's have become scores, its values once this one's are in the sums, the numbers of
            // its pages a tile earlier; beyond the last tile it is asked for again, so that there is one body and no wait covers more than it is for.
            const int stop = min(tile0 + count, (b.all + kCaTile - 1) / kCaTile);
            int t = tile0 + wave;
            if (t < stop) {
                typename Walk::Keys k;
                typename Walk::Values v;
                typename Walk::Pages now = Walk::pages(p, b, t);
                Walk::load(p, b, t, now, k);
                Walk::load(p, b, t, now, v);
                typename Walk::Pages next = Walk::pages(p, b, min(t + kCaWaves, stop - 1));
                for (;;) {
                    const int then = min(t + kCaWaves, stop - 1);
                    float s[8];
                    w.score(p, k, s);
                    Walk::load(p, b, then, next, k);
                    w.absorb(p, b, t, now, s, v);
                    Walk::load(p, b, then, next, v);
                    t += kCaWaves;
                    if (t >= stop) break;
                    now = next;
                    next = Walk::pages(p, b, min(t + kCaWaves, stop - 1));
                }
            }
        }
        w.finish_sum();

        // the wavefronts' sums, under the largest of their references
        if (g == 0) {
            ml[wave][col][0] = w.m;
            ml[wave][col][1] = w.l;
        }
        __syncthreads();
        float m = ml[0][col][0];
#pragma unroll
        for (int i = 1; i < kCaWaves; ++i) m = fmaxf(m, ml[i][col][0]);
        const float f = w.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.m - m);
        // from here on a thread has a row and a 16th of its channels
        const int r = tid >> 4, piece = tid & 15;
        float mr = ml[0][r][0], lr = 0.f;
#pragma unroll
        for (int i = 1; i < kCaWaves; ++i) mr = fmaxf(mr, ml[i][r][0]);
#pragma unroll
        for (int i = 0; i < kCaWaves; ++i) lr += ml[i][r][0] == -INFINITY ? 0.f : ml[i][r][1] * __builtin_amdgcn_exp2f(ml[i][r][0] - mr);
        const int my_row = b.row0 + r;
        const bool mine = my_row < b.n_rows, whole = count == sp.tiles;
        const int token = mine ? my_row / share_h : 0, head = b.kv_head * share_h + my_row - token * share_h;
        const int64_t at = (int64_t)(b.from + token) * c.Hq + head;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (tile0 == 0 ? 1 : 0);
        auto channels = [&](int pass, float(&o)[PASS]) __attribute__((always_inline)) {
            __syncthreads();                     // the pass before has been read
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int e = 0; e < PASS; e += 4)
                    *reinterpret_cast<f32x4*>(&sums[wave][col][(4 * g + v) * PASS + e]) =
                        f32x4{w.acc[pass * PASS + e][v] * f, w.acc[pass * PASS + e + 1][v] * f, w.acc[pass * PASS + e + 2][v] * f, w.acc[pass * PASS + e + 3][v] * f};
            __syncthreads();
#pragma unroll
            for (int e = 0; e < PASS; e += 4) {
                f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < kCaWaves; ++i) t += *reinterpret_cast<const f32x4*>(&sums[i][r][piece * PASS + e]);
#pragma unroll
                for (int k = 0; k < 4; ++k) o[e + k] = t[k];
            }
        };
        if (whole) {
            float o[Walk::VCH / PASS][PASS];
#pragma unroll
            for (int pass = 0; pass < Walk::VCH / PASS; ++pass) channels(pass, o[pass]);
            if (mine) {
                const RowResult<T> res(p, at, mr, lr);
#pragma unroll
                for (int pass = 0; pass < Walk::VCH / PASS; ++pass) res.store(p, DH, Walk::VCH * piece + pass * PASS, o[pass]);
                if (p.lse && piece == 0) p.lse[at] = res.lse;
            }
        } else {
#pragma unroll
            for (int pass = 0; pass < Walk::VCH / PASS; ++pass) {
                float o[PASS];
                channels(pass, o);
                if (mine)
#pragma unroll
                    for (int e = 0; e < PASS; e += 4)
                        *reinterpret_cast<f32x4*>(p.part_o + (slot * kCaRows + r) * DH + Walk::VCH * piece + pass * PASS + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
            }
            if (mine && piece == 0) {
                p.part_ml[(slot * kCaRows + r) * 2] = mr;
                p.part_ml[(slot * kCaRows + r) * 2 + 1] = lr;
            }
            if (tile0 == 0) {
                const int64_t last = (u + sp.tiles - 1) / share;         // the workgroup with the block's last tile
                join = int4{(int)(last - blockIdx.x) + 1, b.row0, b.kv_head, s};
            }
        }
        u += count;
        __syncthreads();                         // before the next block's sums
    }
    if (tid == 0) p.joins[blockIdx.x] = join;
}

// The pieces of a row block that was cut, joined in the order of its tokens: a wavefront per row
template <int DH, typename T>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(const CacheAttnParams p) {
    constexpr int N = DH / 64;
    const CacheStep& c = p.c;
    const int4 join = p.joins[blockIdx.x];
    const int pieces = join.x;
    if (pieces == 0) return;
    const int share_h = c.Hq / c.Hkv, lane = lane_id(), r = blockIdx.y * 4 + (threadIdx.x >> 6), s = join.w;
    const int from = cache_row(c, s), n_rows = max(cache_row(c, s + 1) - from, 0) * share_h, row = join.y + r;
    if (row >= n_rows) return;
    const int token = row / share_h, head = join.z * share_h + row - token * share_h;
    const int64_t first = blockIdx.x;
    auto slot = [&](int i) { return (2 * (first + i) + (i == 0 ? 1 : 0)) * kCaRows + r; };
    float m = -INFINITY, l = 0.f, o[N] = {};
    for (int i0 = 0; i0 < pieces; i0 += 64) {
        const int n = min(pieces - i0, 64);
        const int64_t mine = slot(min(i0 + lane, pieces - 1));
        const float mi = p.part_ml[2 * mine], li = p.part_ml[2 * mine + 1];
        float top = mi;
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        top = fmaxf(top, m);
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        const float f = mi == -INFINITY || lane >= n ? 0.f : __builtin_amdgcn_exp2f(mi - top);
        l *= keep;
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] *= keep;
        m = top;
        constexpr int U = 8;
        for (int i = 0; i < n; i += U) {
            float x[U][N];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const float* at = p.part_o + slot(i0 + min(i + k, n - 1)) * DH + N * lane;
#pragma unroll
                for (int e = 0; e < N; ++e) x[k][e] = at[e];
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (i + k >= n) break;
                const float fk = __shfl(f, i + k);
                l += __shfl(li, i + k) * fk;
#pragma unroll
                for (int e = 0; e < N; ++e) o[e] = fmaf(x[k][e], fk, o[e]);
            }
        }
    }
    const RowResult<T> res(p, (int64_t)(from + token) * c.Hq + head, m, l);
    if constexpr (N == 1) {
        float q = o[0] * res.wo;
        const int64_t i = res.at * DH + lane;
        if (res.wp != 0.f) q = fmaf(res.wp, as_float<T>(((const T*)p.prior_out)[i]), q);
        if constexpr (sizeof(T) == 2) ((uint16_t*)p.out)[i] = f32_to_bf16_bits(q);
        else ((float*)p.out)[i] = q;
    } else {
        res.store(p, DH, N * lane, o);
    }
    if (p.lse && lane == 0) p.lse[res.at] = res.lse;
}

// ---- host ---------------------------------------------------------------------------------------
// The scratch array: sums [2 * workgroups][16 rows][dh], references and sums of weights [2 * workgroups][16][2], and what is to be joined [workgroups]
struct CacheAttnScratch {
    int wgs;
    size_t off_ml, off_joins, total;
};
static CacheAttnScratch cache_attn_scratch(const astra_cache_desc& d) {
    CacheAttnScratch s{};
    const bool f32 = d.dtype == ASTRA_F32;
    s.wgs = kCaCus * (d.head_dim == 64    ? f32 ? kCaWgsPerCu<64, float> : kCaWgsPerCu<64, uint16_t>
                      : d.head_dim == 128 ? f32 ? kCaWgsPerCu<128, float> : kCaWgsPerCu<128, uint16_t>
                                          : f32 ? kCaWgsPerCu<256, float> : kCaWgsPerCu<256, uint16_t>);
    // no more than the shares of the smallest size that there can be
    const int64_t blocks = ((int64_t)d.n_tokens * (d.n_q_heads / d.n_kv_heads) / kCaRows + d.n_seqs) * d.n_kv_heads;
    const int64_t tiles = ceil_div((int64_t)d.max_pages * d.page_size, kCaTile);
    const int64_t most = blocks > (int64_t)s.wgs * kCaMinShare ? s.wgs : ceil_div(blocks * tiles, kCaMinShare);
    if (most < s.wgs) s.wgs = (int)(most > 0 ? most : 1);
    const size_t rows = (size_t)2 * s.wgs * kCaRows;
    s.off_ml = align_up(rows * d.head_dim * 4, 256);
    s.off_joins = s.off_ml + align_up(rows * 2 * 4, 256);
    s.total = s.off_joins + align_up((size_t)s.wgs * sizeof(int4), 256);
    return s;
}

template <int DH, typename T>
static int launch_cache_attention(const CacheAttnParams& p, int wgs, hipStream_t s) {
    cache_attn_kernel<DH, T><<<wgs, kCaThreads, 0, s>>>(p);
    const int rc = launch_status();
    if (rc) return rc;
    cache_attn_join_kernel<DH, T><<<dim3(wgs, kCaRows / 4), 256, 0, s>>>(p);
    return launch_status();
}

template <typename T>
static int launch_cache_attention(const CacheAttnParams& p, int dh, int wgs, hipStream_t s) {
    if (dh == 64) return launch_cache_attention<64, T>(p, wgs, s);
    if (dh == 128) return launch_cache_attention<128, T>(p, wgs, s);
    return launch_cache_attention<256, T>(p, wgs, s);
}

}  // namespace astra

using namespace astra;

extern "C" {

size_t astra_cache_attention_workspace_bytes(const astra_cache_desc* desc) {
    if (check_cache_desc(desc) != ASTRA_OK) return 0;
    return cache_attn_scratch(*desc).total;
}

int astra_cache_attention(const astra_cache_desc* desc, const int32_t* page_table, const int32_t* lens, const int32_t* first_row,
                          const void* q, const uint8_t* k_pages, const uint8_t* v_pages, const float* k_scales, const float* v_scales,
                          const void* prior_out, const float* prior_lse, void* out, float* lse_out, void* workspace,
                          size_t workspace_bytes, void* stream) {
    const int rc = check_cache_desc(desc);
    if (rc) return rc;
    if (desc->n_tokens == 0 || desc->n_seqs == 0) return ASTRA_OK;
    if (!page_table || !lens || !first_row || !q || !k_pages || !v_pages || !k_scales || !v_scales || !out || !prior_out != !prior_lse) return ASTRA_ERR_NULL;
    const CacheAttnScratch sc = cache_attn_scratch(*desc);
    if (!workspace || workspace_bytes < sc.total) return ASTRA_ERR_WORKSPACE;
    for (const void* a : {q, (const void*)k_pages, (const void*)v_pages, prior_out, (const void*)out, (const void*)workspace})
        if ((uintptr_t)a % 16 != 0) return ASTRA_ERR_UNSUPPORTED;
    CacheAttnParams p{};
    p.c = cache_step(*desc, page_table, lens, first_row);
    p.q = q; p.k_pages = k_pages; p.v_pages = v_pages; p.k_scales = k_scales; p.v_scales = v_scales;
    p.prior_out = prior_out; p.prior_lse = prior_lse; p.out = out; p.lse = lse_out;
    p.q_stride = desc->q_stride ? desc->q_stride : desc->n_q_heads * desc->head_dim;
    p.scale = desc->scale != 0.f ? desc->scale : 1.f / sqrtf((float)desc->head_dim);
    p.part_o = (float*)workspace;
    p.part_ml = (float*)((char*)workspace + sc.off_ml);
    p.joins = (int4*)((char*)workspace + sc.off_joins);
    if (desc->dtype == ASTRA_BF16) return launch_cache_attention<uint16_t>(p, desc->head_dim, sc.wgs, (hipStream_t)stream);
    return launch_cache_attention<float>(p, desc->head_dim, sc.wgs, (hipStream_t)stream);
}

}  // extern "C"
