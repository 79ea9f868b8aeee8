// New tokens into the paged cache of 8-bit values (include/astra.h, astra_cache_append): rotary positions, block scales, codes.
#include "cache_common.h"

#include <cfloat>
#include <cmath>

namespace astra {

// ------------------------------------------------------------------------------------------------
// A block (one page, one KV head, keys or values) is the business of one workgroup, which finds the largest of its new values, settles
// the scale and stores the codes; nobody else reads or writes the block.  Scales are powers of two: e4m3 codes are as
// precise relative to their value under any scale but for the subnormal ones at the bottom of 18 binades, so nothing is lost
// by taking the next power, dividing is exact, and a code that is rounded again to a larger scale keeps its value.  An
// angle is formed in fp64 as turns = position * (base^(-2j/dh) / 2 pi) and reduced to an eighth of a turn either side of a
// quarter before it is rounded (positions reach 10^5).
//
// Bounds.  A step of one token per sequence waits for one round trip to memory after another (where the row belongs, the rows, the old scale):
// 4.5 us for one sequence, 5.3 us for 64 (32 + 8 heads of 128, bf16), an empty launch in a row being 3.8 us.  Prompts move bytes: 5700 tokens, 129 MB, 26.1 us,
// 4.9 TB/s, what a copy reaches.  Heads share their angles by four: by two 36.5 us, by eight 34.3 us where by four it was 32.5 us; holding eight pieces
// instead of four 34.4 us; queries before keys and values 42.4 us.
// ------------------------------------------------------------------------------------------------
constexpr int kAppendHold = 4;           // pieces of eight values that a thread holds between the two uses of a block
constexpr int kAppendQHeads = 4;         // query heads per thread; they share their angles
constexpr int kMaxTurnBits = 7;          // pairs of a head of 256: 128

struct AppendParams {
    CacheStep c;
    const int32_t* shift;
    const void* q;
    const void* k;
    const void* v;
    void* q_out;
    uint8_t* pages[2];           // keys, values
    float* scales[2];
    int32_t q_stride, k_stride, v_stride;
    int32_t n_units, rows_per_unit;
    int32_t rotate;
    double turn[kMaxTurnBits];   // base^(-2^(i+1) / dh): turns of pair j are the product over the bits of j
};

// cos and sin of 2 pi * turns.  Taylor polynomials on an eighth of a turn either side: the first terms left out are x^11/11! < 2e-9 and x^12/12! < 2e-10.
__device__ __forceinline__ void cos_sin_turns(double turns, float& cs, float& sn) {
    const double n = rint(4.0 * turns);
    const float x = (float)((turns - 0.25 * n) * 6.283185307179586), x2 = x * x;
    const int quarter = (int)(n - 4.0 * floor(0.25 * n));
    const float s = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
    const float c = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    cs = quarter == 1 || quarter == 2 ? -a : a;
    sn = quarter >= 2 ? -b : b;
}

template <typename T>
struct Eight;                    // eight neighbouring channels as they are loaded
template <>
struct Eight<uint16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ float at(int i) const { return i & 1 ? __uint_as_float(w[i >> 1] & 0xffff0000u) : __uint_as_float(w[i >> 1] << 16); }
};
template <>
struct Eight<float> {
    f32x4 w[2];
    __device__ __forceinline__ void load(const float* p) {
        w[0] = reinterpret_cast<const f32x4*>(p)[0];
        w[1] = reinterpret_cast<const f32x4*>(p)[1];
    }
    __device__ __forceinline__ float at(int i) const { return w[i >> 2][i & 3]; }
};
// STREAM: past the caches.  What a prompt writes is more than they keep for the reader, and in passing would put out what is still to be read;
// 5700 tokens of 32 + 8 + 8 heads of 128: 32.4 us without, 26.1 us with it (streamed loads: 29.9 us).
template <bool STREAM, typename V>
__device__ __forceinline__ void store_piece(void* p, V w) {
    if (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<V*>(p));
    else *reinterpret_cast<V*>(p) = w;
}
template <bool STREAM>
__device__ __forceinline__ void store_eight(uint16_t* p, const float (&x)[8]) {
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    store_piece<STREAM>(p, o);
}
template <bool STREAM>
__device__ __forceinline__ void store_eight(float* p, const float (&x)[8]) {
    store_piece<STREAM>(p, f32x4{x[0], x[1], x[2], x[3]});
    store_piece<STREAM>(p + 4, f32x4{x[4], x[5], x[6], x[7]});
}

// turns per position of the four pairs of piece c8 of a head (pair 4 * c8 + e)
__device__ __forceinline__ void piece_turns(const AppendParams& p, int c8, double (&f)[4]) {
    double t = 0.15915494309189535;                 // 1 / 2 pi
#pragma unroll
    for (int i = 2; i < kMaxTurnBits; ++i) t *= (c8 >> (i - 2)) & 1 ? p.turn[i] : 1.0;
    f[0] = t;
    f[1] = t * p.turn[0];
    f[2] = t * p.turn[1];
    f[3] = f[2] * p.turn[0];
}
__device__ __forceinline__ void turn_piece(float (&x)[8], const float (&cs)[4], const float (&sn)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float a = x[2 * e], b = x[2 * e + 1];
        x[2 * e] = fmaf(a, cs[e], -(b * sn[e]));
        x[2 * e + 1] = fmaf(b, cs[e], a * sn[e]);
    }
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= FLT_MAX; }

// code of v under a scale whose reciprocal is inv
__device__ __forceinline__ float coded(float v, float inv) { return finite(v) ? fminf(fmaxf(v * inv, -kE4m3Max), kE4m3Max) : NAN; }
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}

// the smallest power of two with m <= 448 * scale, within 2^-100 .. 2^110; m finite, not negative
__device__ __forceinline__ float block_scale(float m) {
    const uint32_t bits = __float_as_uint(m);
    // 448 = 1.75 * 2^8
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = min(max(e, -100), 110);
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// the sequence that has row r: the last one that starts at or before it.  Found by halving; whatever the array holds, the result is in range
__device__ __forceinline__ int sequence_of(const CacheStep& c, int r) {
    int lo = 0, n = c.n_seqs;
    while (n > 0) {                      // first s in [0, n_seqs) with first[s] > r
        const int half = n >> 1;
        if (c.first[lo + half] <= r) {
            lo += half + 1;
            n -= half + 1;
        } else {
            n = half;
        }
    }
    return lo - 1;                       // -1: r is before all of them
}

template <typename T, int DH, int THREADS>
__global__ __launch_bounds__(THREADS) void cache_append_kernel(const AppendParams p) {
    constexpr int TPR = DH / 8;                      // threads per row
    constexpr int RPP = THREADS / TPR;               // rows per pass
    constexpr int WAVES = THREADS / kWave;
    constexpr bool STREAM = WAVES > 1;               // prompts
    __shared__ float most[WAVES];
    const CacheStep& c = p.c;
    const int tid = threadIdx.x, lane = lane_id();
    const int c8 = tid % TPR, r_in = tid / TPR;
    double freq[4];
    if (p.rotate) piece_turns(p, c8, freq);

    const int n_kv = p.n_units * 2 * c.Hkv;
    if ((int)blockIdx.x >= n_kv) {
        // ---- queries: a row's piece of four heads per thread
        const uint32_t groups = (uint32_t)(c.Hq + kAppendQHeads - 1) / kAppendQHeads;
        const uint32_t id = (blockIdx.x - (uint32_t)n_kv) * RPP + r_in;
        if (id >= (uint32_t)c.n_tokens * groups) return;
        const int r = (int)(id / groups), h0 = (int)(id - r * groups) * kAppendQHeads;
        const T* src = (const T*)p.q + (int64_t)r * p.q_stride + 8 * c8;             // may be q_out
        T* dst = (T*)p.q_out + (int64_t)r * p.q_stride + 8 * c8;
        Eight<T> in[kAppendQHeads];
#pragma unroll
        for (int j = 0; j < kAppendQHeads; ++j) in[j].load(src + min(h0 + j, c.Hq - 1) * DH);
        const int s = sequence_of(c, r);
        if (s < 0 || r >= c.first[s + 1]) return;
        float cs[4], sn[4];
        if (p.rotate) {
            const double m = (double)((int64_t)cache_len(c, s) + (r - cache_row(c, s)) + (p.shift ? p.shift[s] : 0));
#pragma unroll
            for (int e = 0; e < 4; ++e) cos_sin_turns(m * freq[e], cs[e], sn[e]);
        }
#pragma unroll
        for (int j = 0; j < kAppendQHeads; ++j) {
            if (h0 + j >= c.Hq) break;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = in[j].at(i);
            if (p.rotate) turn_piece(x, cs, sn);
            store_eight<STREAM>(dst + (h0 + j) * DH, x);
        }
        return;
    }

    // ---- keys and values.  A unit is some rows of one head of one matrix; the blocks whose first new row is among them are its own
    const int unit = (int)blockIdx.x / (2 * c.Hkv), y = (int)blockIdx.x - unit * 2 * c.Hkv;
    const int is_v = y >= c.Hkv, h = is_v ? y - c.Hkv : y;
    const bool rotate = p.rotate && !is_v;
    const int page_size = 1 << c.page_shift;
    const T* __restrict__ src = (const T*)(is_v ? p.v : p.k) + h * DH + 8 * c8;
    const int64_t stride = is_v ? p.v_stride : p.k_stride;
    uint8_t* const pages = p.pages[is_v];
    float* const scales = p.scales[is_v];

    const int r0 = unit * p.rows_per_unit;
    int my_row = r0 + lane, my_s = -1, my_t = 0, my_page = -1;
    bool starts = false;
    if (lane < p.rows_per_unit && my_row < c.n_tokens) {
        my_s = sequence_of(c, my_row);
        if (my_s >= 0 && my_row < c.first[my_s + 1]) {
            const int from = cache_row(c, my_s);
            const int64_t t = (int64_t)cache_len(c, my_s) + (my_row - from);
            if (t < c.capacity()) {
                my_t = (int)t;
                if (my_row == from || (my_t & (page_size - 1)) == 0) {
                    my_page = c.table[(int64_t)my_s * c.table_stride + (my_t >> c.page_shift)];
                    starts = my_page >= 0 && my_page < c.n_pages;
                }
            }
        }
    }
    unsigned long long todo = __builtin_amdgcn_ballot_w64(starts);
    for (; todo; todo &= todo - 1) {
        const int at = __builtin_ctzll(todo);
        const int s = __builtin_amdgcn_readlane(my_s, at), t0 = __builtin_amdgcn_readlane(my_t, at), page = __builtin_amdgcn_readlane(my_page, at);
        const int row = r0 + at, off = t0 & (page_size - 1);
        const int rows = min(page_size - off, min(c.first[s + 1], c.n_tokens) - row);
        const int64_t block = (int64_t)page * c.Hkv + h;
        uint8_t* const codes = pages + block * page_size * DH;
        const float old = off ? scales[block] : 0.f;
        const double m0 = (double)((int64_t)t0 + (rotate && p.shift ? p.shift[s] : 0));

        auto get = [&](int i, float(&x)[8]) __attribute__((always_inline)) {
            Eight<T> in;
            in.load(src + (row + i) * stride);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = in.at(e);
            if (rotate) {
                float cs[4], sn[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) cos_sin_turns((m0 + (double)i) * freq[e], cs[e], sn[e]);
                turn_piece(x, cs, sn);
            }
        };
        auto largest = [&](const float(&x)[8], float m) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, finite(x[e]) ? fabsf(x[e]) : 0.f);
            return m;
        };
        float held[kAppendHold][8], mx = 0.f;
#pragma unroll
        for (int j = 0; j < kAppendHold; ++j) {
            const int i = j * RPP + r_in;
            if (i < rows) {
                get(i, held[j]);
                mx = largest(held[j], mx);
            }
        }
        for (int i = kAppendHold * RPP + r_in; i < rows; i += RPP) {
            float x[8];
            get(i, x);
            mx = largest(x, mx);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
        if (WAVES > 1) {
            if (lane == 0) most[tid / kWave] = mx;
            __syncthreads();                       // everybody has read the old scale, too
#pragma unroll
            for (int w = 0; w < WAVES; ++w) mx = fmaxf(mx, most[w]);
            __syncthreads();
        }
        const float scale = fmaxf(old, block_scale(mx)), inv = 1.f / scale;
        auto put = [&](int i, const float(&x)[8]) __attribute__((always_inline)) {
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = coded(x[e], inv);
            u32x2 w;
            w.x = four_codes(z[0], z[1], z[2], z[3]);
            w.y = four_codes(z[4], z[5], z[6], z[7]);
            store_piece<STREAM>(codes + (off + i) * DH + 8 * c8, w);
        };
#pragma unroll
        for (int j = 0; j < kAppendHold; ++j) {
            const int i = j * RPP + r_in;
            if (i < rows) put(i, held[j]);
        }
        for (int i = kAppendHold * RPP + r_in; i < rows; i += RPP) {
            float x[8];
            get(i, x);
            put(i, x);
        }
        if (off && scale > old) {
            const float ratio = old * inv;
            for (int i = tid; i < off * (DH / 8); i += THREADS) {
                u32x2 w = reinterpret_cast<const u32x2*>(codes)[i];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
                    w[k] = four_codes(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
                }
                reinterpret_cast<u32x2*>(codes)[i] = w;
            }
        }
        if (tid == 0) scales[block] = scale;
    }
}

// ---- host ---------------------------------------------------------------------------------------
int check_cache_desc(const astra_cache_desc* d) {
    if (!d) return ASTRA_ERR_NULL;
    if (d->dtype != ASTRA_F32 && d->dtype != ASTRA_BF16) return ASTRA_ERR_DTYPE;
    if (d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->n_q_heads % d->n_kv_heads != 0 || d->n_q_heads > 4096) return ASTRA_ERR_SHAPE;
    if (d->page_size <= 0 || d->n_pages <= 0 || d->max_pages <= 0 || d->n_seqs < 0 || d->n_tokens < 0) return ASTRA_ERR_SHAPE;
    if (d->table_stride != 0 && d->table_stride < d->max_pages) return ASTRA_ERR_SHAPE;
    if (!(d->rope_base >= 0.f) || !(d->scale >= 0.f) || d->rope_base > FLT_MAX || d->scale > FLT_MAX) return ASTRA_ERR_SHAPE;
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return ASTRA_ERR_UNSUPPORTED;
    if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128) return ASTRA_ERR_UNSUPPORTED;
    if (d->n_seqs > kCacheMaxSeqs || d->n_tokens > (1 << 24)) return ASTRA_ERR_UNSUPPORTED;
    if ((int64_t)d->max_pages * d->page_size > (1 << 30)) return ASTRA_ERR_SHAPE;
    const int32_t strides[3] = {d->q_stride, d->k_stride, d->v_stride}, heads[3] = {d->n_q_heads, d->n_kv_heads, d->n_kv_heads};
    for (int i = 0; i < 3; ++i) {
        if (strides[i] == 0) continue;
        if (strides[i] < heads[i] * d->head_dim) return ASTRA_ERR_SHAPE;
        if ((int64_t)strides[i] * elem_bytes(d->dtype) % 16 != 0) return ASTRA_ERR_UNSUPPORTED;
    }
    return ASTRA_OK;
}

CacheStep cache_step(const astra_cache_desc& d, const int32_t* table, const int32_t* lens, const int32_t* first) {
    CacheStep c{};
    c.table = table; c.lens = lens; c.first = first;
    c.n_seqs = d.n_seqs; c.n_tokens = d.n_tokens; c.max_pages = d.max_pages; c.n_pages = d.n_pages;
    c.table_stride = d.table_stride ? d.table_stride : d.max_pages;
    c.page_shift = __builtin_ctz((unsigned)d.page_size);
    c.Hq = d.n_q_heads; c.Hkv = d.n_kv_heads;
    return c;
}

template <typename T, int DH, int THREADS>
static int launch_append(const AppendParams& p, hipStream_t s) {
    constexpr int RPP = THREADS / (DH / 8);
    const int64_t q_rows = p.q ? (int64_t)p.c.n_tokens * ceil_div(p.c.Hq, kAppendQHeads) : 0;
    const int64_t blocks = (int64_t)p.n_units * 2 * p.c.Hkv + ceil_div(q_rows, RPP);
    if (q_rows > (1u << 31) || blocks * THREADS > kMaxGridThreads) return ASTRA_ERR_UNSUPPORTED;
    cache_append_kernel<T, DH, THREADS><<<(unsigned)blocks, THREADS, 0, s>>>(p);
    return launch_status();
}

template <typename T, int THREADS>
static int launch_append(const AppendParams& p, int dh, hipStream_t s) {
    if (dh == 64) return launch_append<T, 64, THREADS>(p, s);
    if (dh == 128) return launch_append<T, 128, THREADS>(p, s);
    return launch_append<T, 256, THREADS>(p, s);
}

template <typename T>
static int launch_append(AppendParams& p, int dh, hipStream_t s) {
    // Rows of a unit: what a sequence has on average, so that a step's tokens are spread over workgroups of one wavefront and a
    // prompt's pages over workgroups of four that hold a page
    int rows = 1;
    while (rows < 64 && rows < (1 << p.c.page_shift) && 2 * rows * p.c.n_seqs <= p.c.n_tokens) rows *= 2;
    p.rows_per_unit = rows;
    p.n_units = (int)ceil_div(p.c.n_tokens, rows);
    return rows >= 16 ? launch_append<T, 256>(p, dh, s) : launch_append<T, 64>(p, dh, s);
}

static bool aligned16(const void* a) { return (uintptr_t)a % 16 == 0; }

}  // namespace astra

using namespace astra;

extern "C" int astra_cache_append(const astra_cache_desc* desc, const int32_t* page_table, const int32_t* lens, const int32_t* first_row,
                                  const int32_t* pos_shift, const void* q, const void* k, const void* v, void* q_out, uint8_t* k_pages,
                                  uint8_t* v_pages, float* k_scales, float* v_scales, void* stream) {
    const int rc = check_cache_desc(desc);
    if (rc) return rc;
    if (desc->n_tokens == 0 || desc->n_seqs == 0) return ASTRA_OK;
    if (!page_table || !lens || !first_row || !k || !v || !k_pages || !v_pages || !k_scales || !v_scales || !q != !q_out) return ASTRA_ERR_NULL;
    for (const void* a : {q, k, v, (const void*)q_out, (const void*)k_pages, (const void*)v_pages})
        if (!aligned16(a)) return ASTRA_ERR_UNSUPPORTED;
    AppendParams p{};
    p.c = cache_step(*desc, page_table, lens, first_row);
    p.shift = pos_shift; p.q = q; p.k = k; p.v = v; p.q_out = q_out;
    p.pages[0] = k_pages; p.pages[1] = v_pages; p.scales[0] = k_scales; p.scales[1] = v_scales;
    const int dh = desc->head_dim;
    p.q_stride = desc->q_stride ? desc->q_stride : desc->n_q_heads * dh;
    p.k_stride = desc->k_stride ? desc->k_stride : desc->n_kv_heads * dh;
    p.v_stride = desc->v_stride ? desc->v_stride : desc->n_kv_heads * dh;
    p.rotate = desc->rope_base > 0.f;
    if (p.rotate) {
        const double per_pair = -2.0 / dh * std::log2((double)desc->rope_base);
        for (int i = 0; i < kMaxTurnBits; ++i) p.turn[i] = std::exp2(per_pair * (1 << i));
    }
    if (desc->dtype == ASTRA_BF16) return launch_append<uint16_t>(p, dh, (hipStream_t)stream);
    return launch_append<float>(p, dh, (hipStream_t)stream);
}
