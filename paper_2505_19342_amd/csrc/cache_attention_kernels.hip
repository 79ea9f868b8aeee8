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
//
// Bounds (heads of 128, bf16, 32 over 8).  Long contexts: the bytes of the pages, with loads of keys and values a tile ahead of their use.  64 ragged sequences of up to 8192 tokens
// 111 us, 4.84 TB/s (a sum over plain memory reaches 6.1); one of 131072 59 us, 4.5 TB/s.  Vector units are busy for a quarter of that, matrix cores
// for a tenth.  Short ones: one round trip to memory after another (lengths, table, scales and codes) and, where sequences are cut, a second launch: 6.7 + 4.8 us for one
// sequence of 1025 tokens, 8.5 us in one launch for 8 of up to 1021 (12 heads of 64, fp32).  Chunks of prompts: the vector instructions per score (scale, exponential, parts, conversions of
// codes), 30 us for four of up to 256 tokens over up to 2048, 192 TFLOP/s.
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

struct CaJoin;
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
    uint32_t most_blocks;        // row blocks that ascending first rows can make
    int32_t by_block;            // a unit per workgroup, and what is to be joined noted by row block
    // scratch, see CacheAttnPlan
    float* part_o;
    float* part_ml;
    CaJoin* joins;
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
// largest of the four lanes of a column (16 apart)
__device__ __forceinline__ float column_max(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);        // lower halves of both, upper halves of both
    const float w = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(w), __float_as_uint(w), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// 1 in each byte of w that is NaN (all seven bits below the sign set)
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u; }

// What a wavefront knows of its query rows: a block of 16 or 32 rows (new token, head) of one sequence and KV head
struct RowBlock {
    int seq, kv_head;
    int len, n_new, from;        // cached tokens, new tokens, first row of the sequence
    int row0, n_rows;            // first (token, head) row of the block, rows of the sequence in all
    int least, all;              // tokens that the block's first row and its last one attend to
};

// NT: groups of 16 query rows
template <int DH, typename T, int NT>
struct CacheWalk {
    static constexpr int KR = DH < 128 ? DH : 128;                  // bytes of a key row that are in LDS at a time
    static constexpr int KP = KR / 16, KN = 32 * KR / 1024;         // 16-byte pieces of it, and a lane's of the tile
    static constexpr int KC = DH / 32;         // contraction steps of a score
    static constexpr int VCH = DH / 16;        // value channels per lane
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int QP = F32 ? 3 : 1, PP = F32 ? 3 : 2;
    using Piece = std::conditional_t<DH == 256, u32x4, std::conditional_t<DH == 128, u32x2, uint32_t>>;

    // a tile's codes and the scales of its two 16-token halves
    struct Keys {
        u32x4 k[DH / KR][KN];
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

    bf16x8 q[NT][QP][KC];
    f32x4 acc[NT][VCH];
    float m[NT], l[NT];
    int sees[NT];                              // tokens that this lane's rows attend to

    __device__ __forceinline__ void start(const CacheAttnParams& p, const RowBlock& b) {
        const int lane = lane_id(), col = lane & 15, g = lane >> 4;
        const int share = p.c.Hq / p.c.Hkv;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = min(b.row0 + 16 * n + col, b.n_rows - 1), token = row / share, head = b.kv_head * share + row - token * share;
            sees[n] = min(b.len + token + 1, p.c.capacity());
            const gbytes at = (gbytes)p.q + ((int64_t)(b.from + token) * p.q_stride + head * DH + 16 * g) * (int64_t)sizeof(T);
#pragma unroll
            for (int kc = 0; kc < KC; ++kc) {
                const gbytes a = at + (64 * (kc >> 1) + 8 * (kc & 1)) * (int)sizeof(T);
                if constexpr (!F32) {
                    q[n][0][kc] = __builtin_bit_cast(bf16x8, ld_global<u32x4>(a));
                } else {
                    const f32x4 x0 = ld_global<f32x4>(a), x1 = ld_global<f32x4>(a + 16);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float x = e < 4 ? x0[e & 3] : x1[e & 3];
#pragma unroll
                        for (int i = 0; i < QP; ++i) {             // every difference is exact
                            const float part = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
                            q[n][i][kc][e] = (__bf16)part;
                            x -= part;
                        }
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < VCH; ++c) acc[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[n] = -INFINITY;
            l[n] = 0.f;
        }
    }

    __device__ __forceinline__ void nothing() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int c = 0; c < VCH; ++c) acc[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[n] = -INFINITY;
            l[n] = 0.f;
        }
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
        // neighbouring lanes: neighbouring pieces of a row (one row per lane, as the operand has them, costs the first-level cache four times the cycles)
        const uint32_t lane_at = (uint32_t)(lane_id() / KP) * DH + (uint32_t)(lane_id() % KP) * 16u;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int64_t block = pg.block(p.c, hf, b.kv_head);
            x.scale[hf] = ld_global<float>((gbytes)(p.k_scales + block));
            const gbytes kb = (gbytes)p.k_pages + half_at(p, block, t, hf);
#pragma unroll
            for (int c = 0; c < DH / KR; ++c)
#pragma unroll
                for (int i = 0; i < KN / 2; ++i) x.k[c][hf * (KN / 2) + i] = ld_global<u32x4>(kb + lane_at + i * (64 / KP) * DH + c * KR);
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
    // lds: 32 * KR bytes of the wavefront's own; its reads come after its writes, nobody else is waited for.  Pieces are exchanged within a row so that the
    // sixteen rows of an operand's quarter fall into different banks.
    __device__ __forceinline__ void score(const CacheAttnParams& p, const Keys& x, char* lds, float (&s)[NT][8]) const {
        const float sl2 = p.scale * kLog2e;
        const int lane = lane_id(), col = lane & 15, g = lane >> 4;
        auto slot = [](int row, int piece) __attribute__((always_inline)) { return row * KR + (piece ^ (KP == 8 ? (row >> 1) & 7 : (row >> 2) & 3)) * 16; };
        f32x4 d[2][NT] = {};
#pragma unroll
        for (int c = 0; c < DH / KR; ++c) {
#pragma unroll
            for (int i = 0; i < KN; ++i) *reinterpret_cast<u32x4*>(lds + slot(i * (64 / KP) + lane / KP, lane % KP)) = x.k[c][i];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int j = 0; j < KR / 64; ++j) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + slot(16 * hf + col, 4 * j + g));
#pragma unroll
                    for (int a = 0; a < 2; ++a) {
                        const bf16x8 kf = a ? eight_codes(w.z, w.w) : eight_codes(w.x, w.y);
#pragma unroll
                        for (int i = 0; i < QP; ++i)
#pragma unroll
                            for (int n = 0; n < NT; ++n) d[hf][n] = mfma_16x16x32(kf, q[n][i][(c * KR / 64 + j) * 2 + a], d[hf][n]);
                    }
                }
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const float f = sl2 * x.scale[hf];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int v = 0; v < 4; ++v) s[n][4 * hf + v] = d[hf][n][v] * f;
        }
    }

    // scores and values of a tile into the running sums
    __device__ __forceinline__ void absorb(const CacheAttnParams& p, const RowBlock& b, int t, const Pages& pg, float (&s)[NT][8], Values& x) {
        const int g = lane_id() >> 4;
        const bool there[2] = {pg.there(p.c, 0), pg.there(p.c, 1)};
        if (t * kCaTile + kCaTile > b.least || !there[0] || !there[1]) {        // of the whole wavefront
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][e] = there[e >> 2] && t * kCaTile + tok(e, g) < sees[n] ? s[n][e] : -INFINITY;
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
        u32x4 part[NT][PP];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float mx = s[n][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[n][e]);
            // (sums are rescaled with every tile: under a branch for the tiles that raise the reference by much they take a second set of registers)
            const float m_new = fmaxf(m[n], column_max(mx)), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m[n] - ref);
            l[n] *= alpha;
#pragma unroll
            for (int c = 0; c < VCH; ++c) acc[n][c] *= alpha;
            m[n] = m_new;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                float a = __builtin_amdgcn_exp2f(s[n][e] - ref), c = __builtin_amdgcn_exp2f(s[n][e + 1] - ref);
                l[n] += a;
                l[n] += c;
                a *= x.scale[e >> 2];
                c *= x.scale[e >> 2];
#pragma unroll
                for (int i = 0; i < PP; ++i) {                    // the upper halves of both; what is left of them is exact
                    part[n][i][e >> 1] = __builtin_amdgcn_perm(__float_as_uint(c), __float_as_uint(a), 0x07060302u);
                    a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
                    c -= __uint_as_float(__float_as_uint(c) & 0xffff0000u);
                }
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
            for (int i = 0; i < PP; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    acc[n][2 * c2] = mfma_16x16x32(__builtin_bit_cast(bf16x8, lo), __builtin_bit_cast(bf16x8, part[n][i]), acc[n][2 * c2]);
                    acc[n][2 * c2 + 1] = mfma_16x16x32(__builtin_bit_cast(bf16x8, hi), __builtin_bit_cast(bf16x8, part[n][i]), acc[n][2 * c2 + 1]);
                }
        }
    }

    // A tile that hides some token from some row and holds a NaN among its values: zero times NaN would reach rows that do not attend to it.
    // Products of ones (NaN here, token seen there) tell which sums become NaN; the NaN values themselves become zeros.
    __device__ __forceinline__ void careful(int t, Values& x) {
        const int g = lane_id() >> 4;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            u32x4 seen;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const int token = t * kCaTile + tok(e, g);
                seen[e >> 1] = (token < sees[n] ? 0x3f80u : 0u) | (token + 1 < sees[n] ? 0x3f800000u : 0u);          // values that are not there are zeros
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
                    acc[n][2 * c2][v] = a[v] > 0.f ? NAN : acc[n][2 * c2][v];
                    acc[n][2 * c2 + 1][v] = b[v] > 0.f ? NAN : acc[n][2 * c2 + 1][v];
                }
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

    // of the columns, once all tiles are in
    __device__ __forceinline__ void finish_sum() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
        }
    }
};

// ---- the work of a launch, dealt out --------------------------------------------------------------
// A unit is a tile of 32 tokens for one row block.  The units of all row blocks (sequence by sequence, head by head, block by block of rows, the tiles of a
// block in order) are cut into equal shares, one per workgroup: ragged batches keep every workgroup busy equally long, and one long context is
// walked by all of them.  Where there are at least four times as many workgroups as there can be row blocks, a unit is `step` tiles, so many that a unit per workgroup is enough: a workgroup
// that ends one block and begins another starts and joins its wavefronts twice (64 row blocks of up to 250 tiles: 36.7 us in equal shares, 21.6 so; 256 of up to 250: 53.6, 57.2).  Only the device knows the lengths, so every workgroup adds them up itself.  The wavefronts take the tiles
// of a share in turn and are joined in LDS.  Where a share ends inside a row block, the unnormalised sums go to the scratch array:
// a workgroup has at most two such pieces, one that ends a row block begun by others (slot 2w) and one that begins one (slot 2w + 1).
// The workgroup that begins a block notes how many pieces there are, under its own number or, where there are few, the block's, and a second launch joins them in order,
// a workgroup per row where that is no more than kCaJoinWgs (32 rows over 3000 tokens: 45.7 us with four workgroups per block, all of the first launch's numbers among them, 15.9 so).
// Where sequences cannot be long (CUT = false), a row block is one unit and there is no second launch.  WIDE: its workgroup has all the wavefronts of a compute unit, for
// launches of a single round; four, and several workgroups on a unit, where there are more row blocks than units: while one begins or ends its walk, others compute
// (200 sequences of up to 1000 tokens: 78.8 and 50.2 us, 320 blocks of chunks over up to 2000 tokens 30.5 and 24.9; 64 blocks over 1000 16.5 and 17.4).
constexpr int kCaMinShare = 2;        // tiles; 8 where there are enough for every unit: fewer pieces to join (313 tiles of 8 row blocks: 14.3 us, 16.5 with shares of 4)
constexpr int kCaCus = 256;
constexpr int kCaJoinWgs = 16384;
// Tiles of a sequence that is not cut.  A row block that one workgroup walks takes about 5 us and 0.3 us a tile, one after the other where there are more than units; cut ones
// take 11 us with their join and 1.7 ns a tile of them all (heads of 128).  8 row blocks of 33 tiles: 14.3 us whole, 11.9 cut, of 62: 16.2 and 11.4; 64 of 33: 16.5 and 20.0, of 55: 21.5 and 21.1;
// 512 of up to 64: 28.9 and 49, of up to 125: 52 and 66, of up to 256: 117 and 111.  Only the capacity is known here: beyond 128 a sequence is cut whatever there is beside it, or one long one would hold up the others.
static int cache_attn_whole_tiles(int64_t blocks) { return blocks < 24 ? 24 : blocks < 128 ? (int)blocks : 128; }

// how many wavefronts a workgroup has and how many workgroups the registers of a unit leave room for
template <int DH, typename T, int NT, bool WIDE>
struct CaShape {
    static constexpr int per_simd = DH == 256 ? (sizeof(T) == 4 ? 1 : 2) : DH == 128 ? (sizeof(T) == 4 || NT > 1 ? 2 : 3) : (sizeof(T) == 4 || NT > 1 ? 3 : 4);
    static constexpr int waves = WIDE ? 4 * (per_simd > 3 ? 3 : per_simd) : 4, threads = waves * kWave;
    static constexpr int wgs_per_cu = WIDE ? 1 : per_simd;
};

// what joins the pieces of a row block
struct CaJoin {
    int32_t pieces, first, row0, n_rows, kv_head, from, pad[2];      // first: the workgroup that begins the block
};

struct SequencePlan {
    int len, from, n_new;
    __device__ __forceinline__ SequencePlan(int l, int f, int n) : len(l), from(f), n_new(n) {}
    __device__ __forceinline__ SequencePlan(const CacheStep& c, int s) : len(cache_len(c, s)), from(cache_row(c, s)), n_new(max(cache_row(c, s + 1) - from, 0)) {}
    __device__ __forceinline__ uint32_t tiles(const CacheStep& c) const { return (uint32_t)(min(len + n_new, c.capacity()) + kCaTile - 1) / kCaTile; }
    __device__ __forceinline__ uint32_t blocks(const CacheStep& c, int rows) const { return (uint32_t)(n_new * (c.Hq / c.Hkv) + rows - 1) / (uint32_t)rows; }
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
    __device__ __forceinline__ RowResult(const CacheAttnParams& p, bool wanted, int64_t row_head, float m, float l) : at(row_head), wo(0.f), wp(0.f), lse(0.f) {
        if (!wanted) return;
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

template <int DH, typename T, int NT, bool CUT, bool WIDE>
__global__ __launch_bounds__((CaShape<DH, T, NT, WIDE>::threads), (CaShape<DH, T, NT, WIDE>::wgs_per_cu)) void cache_attn_kernel(const CacheAttnParams p) {
    using Walk = CacheWalk<DH, T, NT>;
    constexpr int WAVES = CaShape<DH, T, NT, WIDE>::waves, THREADS = WAVES * kWave, ROWS = 16 * NT;
    constexpr int PASS = 4, STRIDE = 16 * PASS + 4;               // channels per thread and pass when the wavefronts are joined
    __shared__ uint32_t before[kCacheMaxSeqs + 1];                // units before a sequence, where there are more than 64
    __shared__ uint32_t blocks_before[CUT ? kCacheMaxSeqs : 1];
    __shared__ float ml[WAVES][ROWS][2];
    __shared__ __align__(16) float sums[WAVES][16][STRIDE];       // of a wavefront; while it walks, a tile of keys on its way to the operand
    static_assert(sizeof(sums[0]) >= 32 * Walk::KR, "a tile of keys");
    // the arguments arrive together; each use asking for its own is another trip to them
    asm volatile("" ::"s"(p.c.table), "s"(p.c.lens), "s"(p.c.first), "s"(p.q), "s"(p.k_pages), "s"(p.v_pages), "s"(p.k_scales), "s"(p.v_scales), "s"(p.c.n_seqs),
                 "s"(p.c.n_tokens), "s"(p.c.max_pages), "s"(p.c.table_stride), "s"(p.c.n_pages), "s"(p.c.page_shift), "s"(p.c.Hq), "s"(p.c.Hkv), "s"(p.q_stride),
                 "s"(p.scale));
    const CacheStep& c = p.c;
    const int tid = threadIdx.x, lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int share_h = c.Hq / c.Hkv;

    auto scan = [&](uint32_t x) __attribute__((always_inline)) {       // sum of the lanes up to this one
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t up = __shfl_up(x, o);
            if (lane >= o) x += up;
        }
        return x;
    };
    // up to 64 sequences: a lane has one of them
    const bool few = c.n_seqs <= 64;
    SequencePlan lane_plan(0, 0, 0);
    if (few && lane < c.n_seqs) lane_plan = SequencePlan(c, lane);
    uint32_t step = 1, share = 1, blocks = 0, lane_blocks = 0;
    bool nobodys = false;
    if constexpr (CUT) {
        uint32_t tiles = 0;
        auto count = [&](const SequencePlan& sp) __attribute__((always_inline)) {
            const uint32_t b = sp.blocks(c, ROWS) * (uint32_t)c.Hkv;
            blocks += b;
            tiles += b * sp.tiles(c);
        };
        if (few) count(lane_plan);
        else
            for (int s = lane; s < c.n_seqs; s += 64) count(SequencePlan(c, s));
        const uint32_t upto = scan(blocks);
        lane_blocks = upto - blocks;
        blocks = __builtin_amdgcn_readlane(upto, 63);
        tiles = __builtin_amdgcn_readlane(scan(tiles), 63);
        nobodys = blocks > p.most_blocks;        // first rows that do not ascend count rows twice, and the units below would pass 32 bits
        if (nobodys) blocks = tiles = 0;
        const uint32_t least = min(max(tiles / kCaCus, (uint32_t)kCaMinShare), 4u * kCaMinShare);
        if (p.by_block) step = max((tiles + gridDim.x - blocks - 1) / (gridDim.x - blocks), least);
        else share = max((tiles + gridDim.x - 1) / gridDim.x, least);
    }
    auto per_block = [&](const SequencePlan& sp) __attribute__((always_inline)) { return CUT ? (sp.tiles(c) + step - 1) / step : 1u; };
    auto units = [&](const SequencePlan& sp) __attribute__((always_inline)) { return per_block(sp) * sp.blocks(c, ROWS) * (uint32_t)c.Hkv; };
    uint32_t lane_before = 0, all;
    if (few) {
        const uint32_t mine = lane < c.n_seqs ? units(lane_plan) : 0u, upto = scan(mine);
        lane_before = upto - mine;
        all = __builtin_amdgcn_readlane(upto, 63);
    } else {
        if (wave == 0) {
            uint32_t base = 0, base_blocks = 0;
            for (int s0 = 0; s0 < c.n_seqs; s0 += 64) {
                const int s = s0 + lane;
                const uint32_t mine = s < c.n_seqs ? units(SequencePlan(c, s)) : 0u, upto = scan(mine);
                if (s < c.n_seqs) before[s] = base + upto - mine;
                base += __builtin_amdgcn_readlane(upto, 63);
                if constexpr (CUT) {
                    const uint32_t b = s < c.n_seqs ? SequencePlan(c, s).blocks(c, ROWS) * (uint32_t)c.Hkv : 0u, to = scan(b);
                    if (s < c.n_seqs) blocks_before[s] = base_blocks + to - b;
                    base_blocks += __builtin_amdgcn_readlane(to, 63);
                }
            }
            if (lane == 0) before[c.n_seqs] = base;
        }
        __syncthreads();
        all = before[c.n_seqs];
    }
    if (nobodys) all = 0;
    uint32_t u = blockIdx.x < (all + share - 1) / share ? blockIdx.x * share : all;
    const uint32_t end = all - u < share ? all : u + share;
    CaJoin join = {};

    while (u < end) {
        // the last sequence that begins at or before u; those without units are before it
        int s;
        uint32_t in, block0 = 0;                 // units of the sequence before u, row blocks before the sequence
        SequencePlan sp(0, 0, 0);
        if (few) {
            s = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(lane < c.n_seqs && lane_before <= u));
            in = u - (uint32_t)__builtin_amdgcn_readlane(lane_before, s);
            if (CUT) block0 = (uint32_t)__builtin_amdgcn_readlane(lane_blocks, s);      // here, where every lane takes part: from one that does not, there is nothing to read
            sp = SequencePlan(__builtin_amdgcn_readlane(lane_plan.len, s), __builtin_amdgcn_readlane(lane_plan.from, s), __builtin_amdgcn_readlane(lane_plan.n_new, s));
        } else {
            int lo = 0, n = c.n_seqs;
            while (n > 0) {
                const int half = n >> 1;
                if (before[lo + half] <= u) {
                    lo += half + 1;
                    n -= half + 1;
                } else {
                    n = half;
                }
            }
            s = __builtin_amdgcn_readfirstlane(lo - 1);
            in = u - before[s];
            if (CUT) block0 = blocks_before[s];
            sp = SequencePlan(c, s);
        }
        const uint32_t all_tiles = sp.tiles(c), seq_blocks = sp.blocks(c, ROWS), of_block = per_block(sp);
        const uint32_t row = in / of_block;
        const int unit0 = __builtin_amdgcn_readfirstlane((int)(in - row * of_block));
        const int count = __builtin_amdgcn_readfirstlane((int)min(of_block - unit0, end - u));
        const int tile0 = unit0 * (int)step;
        RowBlock b;
        b.seq = s;
        b.kv_head = __builtin_amdgcn_readfirstlane((int)(row / seq_blocks));
        b.len = __builtin_amdgcn_readfirstlane(sp.len);
        b.n_new = __builtin_amdgcn_readfirstlane(sp.n_new);
        b.from = __builtin_amdgcn_readfirstlane(sp.from);
        b.n_rows = b.n_new * share_h;
        b.row0 = __builtin_amdgcn_readfirstlane((int)(row % seq_blocks)) * ROWS;
        b.least = min(b.len + b.row0 / share_h + 1, c.capacity());
        b.all = min(b.len + min(b.row0 + ROWS - 1, b.n_rows - 1) / share_h + 1, c.capacity());

        Walk w;
        // The next tile's keys are asked for as soon as this one's have become scores, its values once this one's are in the sums, the numbers of
        // its pages a tile earlier; beyond the last tile it is asked for again, so that there is one body and no wait covers more than it is for.
        const int stop = min(CUT ? tile0 + count * (int)step : (int)all_tiles, (b.all + kCaTile - 1) / kCaTile);
        int t = tile0 + wave;
        if (t < stop) {
            typename Walk::Keys k;
            typename Walk::Values v;
            typename Walk::Pages now = Walk::pages(p, b, t);
            typename Walk::Pages next = Walk::pages(p, b, min(t + WAVES, stop - 1));
            w.start(p, b);
            Walk::load(p, b, t, now, k);
            // Keys before values, as in the loop: a wait counts loads in their order, and the loop's first wait has to hold for either way into it.
            // Left to the compiler the values came first here and every tile waited for all loads.
            asm volatile("" ::: "memory");
            Walk::load(p, b, t, now, v);
            for (;;) {
                const int then = min(t + WAVES, stop - 1);
                float s[NT][8];
                w.score(p, k, reinterpret_cast<char*>(sums[wave]), s);
                Walk::load(p, b, then, next, k);
                w.absorb(p, b, t, now, s, v);
                Walk::load(p, b, then, next, v);
                t += WAVES;
                if (t >= stop) break;
                now = next;
                next = Walk::pages(p, b, min(t + WAVES, stop - 1));
            }
        } else {
            w.nothing();
        }
        w.finish_sum();

        // the wavefronts' sums, under the largest of their references
        if (g == 0)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                ml[wave][16 * n + col][0] = w.m[n];
                ml[wave][16 * n + col][1] = w.l[n];
            }
        __syncthreads();
        const bool whole = !CUT || count == (int)of_block;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (unit0 == 0 ? 1 : 0);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float m = ml[0][16 * n + col][0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) m = fmaxf(m, ml[i][16 * n + col][0]);
            const float f = w.m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.m[n] - m);
            // from here on a thread of the first 256 has a row and a 16th of its channels
            const int r = (tid >> 4) & 15, piece = tid & 15;
            float mr = ml[0][16 * n + r][0], lr = 0.f;
#pragma unroll
            for (int i = 1; i < WAVES; ++i) mr = fmaxf(mr, ml[i][16 * n + r][0]);
#pragma unroll
            for (int i = 0; i < WAVES; ++i) lr += ml[i][16 * n + r][0] == -INFINITY ? 0.f : ml[i][16 * n + r][1] * __builtin_amdgcn_exp2f(ml[i][16 * n + r][0] - mr);
            const int my_row = b.row0 + 16 * n + r;
            const bool mine = tid < 256 && my_row < b.n_rows;
            const int token = mine ? my_row / share_h : 0, head = b.kv_head * share_h + my_row - token * share_h;
            const RowResult<T> res(p, mine && whole, (int64_t)(b.from + token) * c.Hq + head, mr, lr);
#pragma unroll
            for (int pass = 0; pass < Walk::VCH / PASS; ++pass) {
                if (pass + n > 0) __syncthreads();           // the pass before has been read
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    *reinterpret_cast<f32x4*>(&sums[wave][col][(4 * g + v) * PASS]) =
                        f32x4{w.acc[n][pass * PASS][v] * f, w.acc[n][pass * PASS + 1][v] * f, w.acc[n][pass * PASS + 2][v] * f, w.acc[n][pass * PASS + 3][v] * f};
                __syncthreads();
                if (!mine) continue;
                f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < WAVES; ++i) sum += *reinterpret_cast<const f32x4*>(&sums[i][r][piece * PASS]);
                const int channel = Walk::VCH * piece + pass * PASS;
                if (whole) {
                    float o[PASS] = {sum.x, sum.y, sum.z, sum.w};
                    res.store(p, DH, channel, o);
                } else {
                    *reinterpret_cast<f32x4*>(p.part_o + (slot * ROWS + 16 * n + r) * DH + channel) = sum;
                }
            }
            if (mine && piece == 0) {
                if (whole) {
                    if (p.lse) p.lse[res.at] = res.lse;
                } else {
                    p.part_ml[(slot * ROWS + 16 * n + r) * 2] = mr;
                    p.part_ml[(slot * ROWS + 16 * n + r) * 2 + 1] = lr;
                }
            }
        }
        if (CUT && unit0 == 0 && (p.by_block || !whole)) {
            // up to the workgroup with the block's last tile
            join = CaJoin{whole ? 0 : (int)((u + of_block - 1) / share) - (int)blockIdx.x + 1, (int)blockIdx.x, b.row0, b.n_rows, b.kv_head, b.from, {0, 0}};
            if (p.by_block && tid == 0) p.joins[block0 + row] = join;
        }
        u += count;
        __syncthreads();                         // before the next block's sums
    }
    if (CUT && tid == 0) {
        if (!p.by_block) p.joins[blockIdx.x] = join;
        else
            for (uint32_t i = blocks + blockIdx.x; i < p.most_blocks; i += gridDim.x) p.joins[i] = CaJoin{};
    }
}

// The pieces of a row block that was cut, joined in the order of its tokens: row by row, a wavefront has every fourth piece, all of a wavefront's on their way at once
template <int DH, typename T, int NT>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(const CacheAttnParams p) {
    constexpr int N = DH / 64, ROWS = 16 * NT, U = 8;
    __shared__ float ml[4][2];
    __shared__ __align__(16) float sums[4][DH];
    const CacheStep& c = p.c;
    const CaJoin join = p.joins[blockIdx.x];
    if (join.pieces == 0) return;
    const int share_h = c.Hq / c.Hkv, lane = lane_id(), wave = threadIdx.x >> 6;
    const int rows = min(ROWS, join.n_rows - join.row0);
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        auto slot = [&](int i) { return (2 * (int64_t)(join.first + i) + (i == 0 ? 1 : 0)) * ROWS + r; };
        float m = -INFINITY, l = 0.f, o[N] = {};
        for (int i0 = wave; i0 < join.pieces; i0 += 4 * U) {
            float x[U][N], mi[U], li[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t at = slot(min(i0 + 4 * k, join.pieces - 1));
                mi[k] = p.part_ml[2 * at];
                li[k] = p.part_ml[2 * at + 1];
#pragma unroll
                for (int e = 0; e < N; ++e) x[k][e] = p.part_o[at * DH + N * lane + e];
            }
            float top = m;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (i0 + 4 * k >= join.pieces) mi[k] = -INFINITY;
                top = fmaxf(top, mi[k]);
            }
            const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
            l *= keep;
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] *= keep;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (mi[k] == -INFINITY) continue;            // it saw nothing, or is not there
                const float f = __builtin_amdgcn_exp2f(mi[k] - top);
                l = fmaf(li[k], f, l);
#pragma unroll
                for (int e = 0; e < N; ++e) o[e] = fmaf(x[k][e], f, o[e]);
            }
            m = top;
        }
        __syncthreads();                         // the row before has been read
        if (lane == 0) {
            ml[wave][0] = m;
            ml[wave][1] = l;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sums[wave][N * lane + e] = o[e];
        __syncthreads();
        if (threadIdx.x < DH / 4) {              // of one wavefront: the prior's lse is read by all before any writes in its place
            const int ch = 4 * threadIdx.x;
            float mr = ml[0][0], lr = 0.f, q[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 1; i < 4; ++i) mr = fmaxf(mr, ml[i][0]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (ml[i][0] == -INFINITY) continue;
                const float f = __builtin_amdgcn_exp2f(ml[i][0] - mr);
                lr = fmaf(ml[i][1], f, lr);
#pragma unroll
                for (int e = 0; e < 4; ++e) q[e] = fmaf(sums[i][ch + e], f, q[e]);
            }
            const int row = join.row0 + r, token = row / share_h, head = join.kv_head * share_h + row - token * share_h;
            const RowResult<T> res(p, true, (int64_t)(join.from + token) * c.Hq + head, mr, lr);
            res.store(p, DH, ch, q);
            if (p.lse && threadIdx.x == 0) p.lse[res.at] = res.lse;
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------
// How a call is launched, by its descriptor, and the scratch array of a cut one: sums [2 * workgroups][rows][dh], references and sums of weights
// [2 * workgroups][rows][2], and what is to be joined [workgroups]
struct CacheAttnPlan {
    int nt, wgs;
    uint32_t most_blocks;
    int join_rows;               // workgroups that share the rows of a block when its pieces are joined
    bool cut, wide, by_block;
    size_t off_ml, off_joins, total;
};
template <int DH, typename T>
static int cache_attn_wgs(int nt) {
    return kCaCus * (nt == 1 ? CaShape<DH, T, 1, false>::wgs_per_cu : CaShape<DH, T, 2, false>::wgs_per_cu);
}
static int cache_attn_plan(const astra_cache_desc& d, CacheAttnPlan* pl) {
    CacheAttnPlan s{};
    const bool f32 = d.dtype == ASTRA_F32;
    const int64_t rows = (int64_t)d.n_tokens * (d.n_q_heads / d.n_kv_heads);
    // blocks of 32 rows where sequences have that many on average: half the walks over the cache
    s.nt = !f32 && d.head_dim <= 128 && rows >= 32 * (int64_t)d.n_seqs ? 2 : 1;
    const int64_t tiles = ceil_div((int64_t)d.max_pages * d.page_size, kCaTile);
    const int64_t blocks = (rows / (16 * s.nt) + d.n_seqs) * d.n_kv_heads;               // no more than these
    // rows and units are counted in 32 bits; workgroups have no more than 1024 threads
    if (rows > (1 << 30) || blocks * tiles > 0x7fffffff || blocks * 1024 > kMaxGridThreads) return ASTRA_ERR_UNSUPPORTED;
    s.cut = tiles > cache_attn_whole_tiles(blocks);
    const int64_t n_seqs = d.n_seqs > 0 ? d.n_seqs : 1;
    s.wide = n_seqs * ceil_div(ceil_div(rows, n_seqs), 16 * s.nt) * d.n_kv_heads <= kCaCus;      // row blocks, if every sequence has as many rows as the average
    s.wgs = (int)blocks;
    s.most_blocks = (uint32_t)blocks;
    if (s.cut) {
        int most = d.head_dim == 64    ? f32 ? cache_attn_wgs<64, float>(s.nt) : cache_attn_wgs<64, uint16_t>(s.nt)
                   : d.head_dim == 128 ? f32 ? cache_attn_wgs<128, float>(s.nt) : cache_attn_wgs<128, uint16_t>(s.nt)
                                       : f32 ? cache_attn_wgs<256, float>(s.nt) : cache_attn_wgs<256, uint16_t>(s.nt);
        const int64_t shares = ceil_div(blocks * tiles, kCaMinShare);
        s.wgs = (int)(shares < most ? shares : most);
        s.by_block = 4 * blocks <= s.wgs;
        const int64_t of_block = rows < 16 * s.nt ? rows : 16 * s.nt, joins = s.by_block ? blocks : s.wgs, room = kCaJoinWgs / joins;
        s.join_rows = (int)(of_block < 4 ? of_block : room < 4 ? 4 : room < of_block ? room : of_block);
        const size_t r = (size_t)2 * s.wgs * 16 * s.nt;
        s.off_ml = align_up(r * d.head_dim * 4, 256);
        s.off_joins = s.off_ml + align_up(r * 2 * 4, 256);
        s.total = s.off_joins + align_up((size_t)s.wgs * sizeof(CaJoin), 256);
    }
    if (s.total == 0) s.total = 256;
    *pl = s;
    return ASTRA_OK;
}

template <int DH, typename T, int NT>
static int launch_cache_attention(const CacheAttnParams& p, const CacheAttnPlan& pl, hipStream_t s) {
    using Shape = CaShape<DH, T, NT, false>;
    if (!pl.cut) {
        if constexpr (Shape::per_simd > 1)
            if (pl.wide) {
                cache_attn_kernel<DH, T, NT, false, true><<<pl.wgs, CaShape<DH, T, NT, true>::threads, 0, s>>>(p);
                return launch_status();
            }
        cache_attn_kernel<DH, T, NT, false, false><<<pl.wgs, Shape::threads, 0, s>>>(p);
        return launch_status();
    }
    cache_attn_kernel<DH, T, NT, true, false><<<pl.wgs, Shape::threads, 0, s>>>(p);
    const int rc = launch_status();
    if (rc) return rc;
    cache_attn_join_kernel<DH, T, NT><<<dim3(pl.by_block ? pl.most_blocks : pl.wgs, pl.join_rows), 256, 0, s>>>(p);
    return launch_status();
}

template <int DH, typename T>
static int launch_cache_attention(const CacheAttnParams& p, const CacheAttnPlan& pl, hipStream_t s) {
    if constexpr (sizeof(T) == 2 && DH <= 128)
        if (pl.nt == 2) return launch_cache_attention<DH, T, 2>(p, pl, s);
    return launch_cache_attention<DH, T, 1>(p, pl, s);
}

template <typename T>
static int launch_cache_attention(const CacheAttnParams& p, int dh, const CacheAttnPlan& pl, hipStream_t s) {
    if (dh == 64) return launch_cache_attention<64, T>(p, pl, s);
    if (dh == 128) return launch_cache_attention<128, T>(p, pl, s);
    return launch_cache_attention<256, T>(p, pl, s);
}

}  // namespace astra

using namespace astra;

extern "C" {

size_t astra_cache_attention_workspace_bytes(const astra_cache_desc* desc) {
    CacheAttnPlan pl;
    if (check_cache_desc(desc) != ASTRA_OK || cache_attn_plan(*desc, &pl) != ASTRA_OK) return 0;
    return pl.total;
}

int astra_cache_attention(const astra_cache_desc* desc, const int32_t* page_table, const int32_t* lens, const int32_t* first_row,
                          const void* q, const uint8_t* k_pages, const uint8_t* v_pages, const float* k_scales, const float* v_scales,
                          const void* prior_out, const float* prior_lse, void* out, float* lse_out, void* workspace,
                          size_t workspace_bytes, void* stream) {
    int rc = check_cache_desc(desc);
    if (rc) return rc;
    CacheAttnPlan pl;
    rc = cache_attn_plan(*desc, &pl);
    if (rc) return rc;
    if (desc->n_tokens == 0 || desc->n_seqs == 0) return ASTRA_OK;
    if (!page_table || !lens || !first_row || !q || !k_pages || !v_pages || !k_scales || !v_scales || !out || !prior_out != !prior_lse) return ASTRA_ERR_NULL;
    if (!workspace || workspace_bytes < pl.total) return ASTRA_ERR_WORKSPACE;
    for (const void* a : {q, (const void*)k_pages, (const void*)v_pages, prior_out, (const void*)out, (const void*)workspace})
        if ((uintptr_t)a % 16 != 0) return ASTRA_ERR_UNSUPPORTED;
    CacheAttnParams p{};
    p.c = cache_step(*desc, page_table, lens, first_row);
    p.q = q; p.k_pages = k_pages; p.v_pages = v_pages; p.k_scales = k_scales; p.v_scales = v_scales;
    p.prior_out = prior_out; p.prior_lse = prior_lse; p.out = out; p.lse = lse_out;
    p.q_stride = desc->q_stride ? desc->q_stride : desc->n_q_heads * desc->head_dim;
    p.scale = desc->scale != 0.f ? desc->scale : 1.f / sqrtf((float)desc->head_dim);
    p.most_blocks = pl.most_blocks;
    p.by_block = pl.by_block;
    p.part_o = (float*)workspace;
    p.part_ml = (float*)((char*)workspace + pl.off_ml);
    p.joins = (CaJoin*)((char*)workspace + pl.off_joins);
    if (desc->dtype == ASTRA_BF16) return launch_cache_attention<uint16_t>(p, desc->head_dim, pl, (hipStream_t)stream);
    return launch_cache_attention<float>(p, desc->head_dim, pl, (hipStream_t)stream);
}

}  // extern "C"
