// Products of a few tokens with weights of 4 bits and a scale per group of columns (include/astra.h, astra_w4_linear).
#include "common.h"

#include <algorithm>
#include <type_traits>

namespace astra {

// ------------------------------------------------------------------------------------------------
// y[t, n] = bias[n] + sum_g scale[n, g] ( sum_{k in g} (16 + code) x  -  (16 + zero) sum_{k in g} x )
// The weights are what has to be read, so the products run on the matrix cores with 16 rows of the weights on the N side and 16 tokens on the M side, and the
// codes reach them in two operations for two: the four bits go to the upper mantissa bits of a bf16 16.0, which makes it 16 + code
// exactly.  One 16x16x32 MFMA sees 32 neighbouring columns of every row, all of one group.  A group's sum stays in fp32 and takes the row's scale there;
// the sum of x over the group comes from another MFMA, against ones.  fp32 tokens are sums of three bf16 parts (8 + 8 + 8 mantissa bits), and their weights
// code - 8, at 20 operations for eight instead of 8: the difference of the two sums above loses three bits, which a bf16 result does not show.
// What a lane loads and what it multiplies are not the same: sixteen neighbouring lanes of an operand belong to sixteen rows, and a load that reaches sixteen
// places takes four times the first-level cache's cycles of one that reaches four.  Lanes load neighbouring pieces of a row (four lanes a row of
// the weights, 16 or 32 lanes a token) and the operands are read from LDS, where x lies already cut into parts and in the order of the weights.
// ------------------------------------------------------------------------------------------------
struct W4Params {
    const void* x;
    const uint8_t* codes;
    const void* scales;
    const uint8_t* zeros;
    const void* bias;
    void* y;
    int64_t n_tokens;
    int32_t x_stride, K, N, group_shift, y_bf16;
};

__device__ __forceinline__ f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

constexpr int kW4MaxTokens = 1 << 19;              // tiles of 16 fit the grid's second side
constexpr float kOffset = 16.f;
// Eight codes as 16 + code, in the order 0 4 1 5 2 6 3 7.  The constants are kept where one instruction can have both (as literals they are two).
struct OffsetConstants {
    uint32_t mask = 0x00780078u, sixteen = 0x41804180u;
    __device__ __forceinline__ OffsetConstants() {
        asm volatile("" : "+s"(mask));
        asm volatile("" : "+v"(sixteen));
    }
};
__device__ __forceinline__ bf16x8 weights_offset(uint32_t w, const OffsetConstants& c) {
    u32x4 o;
    o.x = ((w << 3) & c.mask) | c.sixteen;
    o.y = ((w >> 1) & c.mask) | c.sixteen;
    o.z = ((w >> 5) & c.mask) | c.sixteen;
    o.w = ((w >> 9) & c.mask) | c.sixteen;
    return __builtin_bit_cast(bf16x8, o);
}
// eight codes as (code - 8) / 16, in order
__device__ __forceinline__ bf16x8 weights_exact(uint32_t w) {
    w ^= 0x88888888u;                              // two's complement of code - 8
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (8 * i))), hi = __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (8 * i + 4)));
        o[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, o);
}
// eight neighbouring values of x as they are loaded, and as the operand's bf16 parts in the order of the weights
template <typename T>
struct Tokens;
template <>
struct Tokens<uint16_t> {
    static constexpr int kParts = 1;
    u32x4 w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ void parts(bool there, u32x4 (&a)[1]) const {
        const u32x4 x = there ? w : u32x4{0u, 0u, 0u, 0u};
        a[0].x = __builtin_amdgcn_perm(x.z, x.x, 0x05040100u);
        a[0].y = __builtin_amdgcn_perm(x.z, x.x, 0x07060302u);
        a[0].z = __builtin_amdgcn_perm(x.w, x.y, 0x05040100u);
        a[0].w = __builtin_amdgcn_perm(x.w, x.y, 0x07060302u);
    }
};
template <>
struct Tokens<float> {
    static constexpr int kParts = 3;
    f32x4 w[2];
    __device__ __forceinline__ void load(const float* p) {
        w[0] = reinterpret_cast<const f32x4*>(p)[0];
        w[1] = reinterpret_cast<const f32x4*>(p)[1];
    }
    __device__ __forceinline__ void parts(bool there, u32x4 (&a)[3]) const {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float v0 = there ? w[e >> 2][e & 3] : 0.f, v1 = there ? w[e >> 2][(e & 3) + 1] : 0.f;
#pragma unroll
            for (int i = 0; i < 3; ++i) {                  // every difference is exact
                a[i][e >> 1] = __builtin_amdgcn_perm(__float_as_uint(v1), __float_as_uint(v0), 0x07060302u);
                v0 -= __uint_as_float(__float_as_uint(v0) & 0xffff0000u);
                v1 -= __uint_as_float(__float_as_uint(v1) & 0xffff0000u);
            }
        }
    }
};
// the four lanes of a row each have one value: all four to all of them
__device__ __forceinline__ void spread(uint32_t v, uint32_t (&out)[4]) {
    const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);        // lanes 0 .. 31 twice, lanes 32 .. 63 twice
    const auto a = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false), b = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
    out[0] = a[0];
    out[1] = a[1];
    out[2] = b[0];
    out[3] = b[1];
}

// an element as it lies in memory, converted where it is used: a conversion beside the load is a wait there
template <typename T>
__device__ __forceinline__ uint32_t raw_element(const void* p, int64_t i) {
    if constexpr (sizeof(T) == 2) return ((const uint16_t*)p)[i];
    else return ((const uint32_t*)p)[i];
}
template <typename T>
__device__ __forceinline__ float from_raw(uint32_t w) { return __uint_as_float(sizeof(T) == 2 ? w << 16 : w); }
template <typename T>
__device__ __forceinline__ float element(const void* p, int64_t i) {
    if constexpr (sizeof(T) == 2) return bf16_bits_to_f32(((const uint16_t*)p)[i]);
    else return ((const float*)p)[i];
}

// Sums of the wavefronts in order, and the store: 16 rows of the weights, from n0 on, and 16 tokens, from t0 on; sums: [wavefronts][16][16] floats
template <typename T>
__device__ __forceinline__ void store_sums(const W4Params& p, float* sums, int wave, int waves, int64_t t0, int n0, f32x4 acc) {
    const int lane = lane_id(), col = lane & 15, g = lane >> 4;
#pragma unroll
    for (int v = 0; v < 4; ++v) sums[(wave * 16 + 4 * g + v) * 16 + col] = acc[v];
    __syncthreads();
    for (int e = threadIdx.x; e < 256; e += blockDim.x) {
        const int64_t t = t0 + e / 16;
        const int n = n0 + e % 16;
        if (t >= p.n_tokens || n >= p.N) continue;
        float y = p.bias ? element<T>(p.bias, n) : 0.f;
        for (int k = 0; k < waves; ++k) y += sums[k * 256 + e];
        if (p.y_bf16) ((uint16_t*)p.y)[t * p.N + n] = f32_to_bf16_bits(y);
        else ((float*)p.y)[t * p.N + n] = y;
    }
}

// Scales and zero points of 16 rows for 16 neighbouring groups, on their way through a wavefront's part of LDS: sixteen lanes load the sixteen of a row (a lane per row and
// group would reach sixty-four places at a time), and each lane reads those of its row where a group ends.
struct ScaleSpan {
    static constexpr int kGroups = 16;
    static constexpr int kStride = 18, kZeroStride = 20;      // rows start in different banks
    static constexpr int kScaleBytes = 16 * kStride * 2, kBytes = (kScaleBytes + 16 * kZeroStride + 15) / 16 * 16;
    uint16_t s[4];
    uint8_t z[4];
    // rows n0 .. n0 + 15 (those beyond the last: the last), groups from `first` on (beyond the last: the last)
    __device__ __forceinline__ void load(const W4Params& p, int n0, int groups, int first) {
        const int lane = lane_id(), at = min(first + (lane & 15), groups - 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t j = (int64_t)min(n0 + 4 * i + (lane >> 4), p.N - 1) * groups + at;
            s[i] = ((const uint16_t*)p.scales)[j];
            if (p.zeros) z[i] = p.zeros[j];
        }
    }
    __device__ __forceinline__ void put(const W4Params& p, char* lds) const {
        const int lane = lane_id();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ((uint16_t*)lds)[(4 * i + (lane >> 4)) * kStride + (lane & 15)] = s[i];
            if (p.zeros) ((uint8_t*)lds + kScaleBytes)[(4 * i + (lane >> 4)) * kZeroStride + (lane & 15)] = z[i];
        }
    }
    // of row lane % 16
    __device__ __forceinline__ static float scale(const char* lds, int group) { return bf16_bits_to_f32(((const uint16_t*)lds)[(lane_id() & 15) * kStride + group]); }
    __device__ __forceinline__ static float zero(const W4Params& p, const char* lds, int group) {
        return p.zeros ? (float)(((const uint8_t*)lds + kScaleBytes)[(lane_id() & 15) * kZeroStride + group] & 15) : 8.f;
    }
};

constexpr int kW4RowBytes = 80;                    // of a row's 64 bytes in LDS: sixteen rows' words of one column fall into different banks
template <typename T, int TP, int U>
struct W4Lds {                                     // of a wavefront
    static constexpr int x_stride = U * 256 + 16;  // bytes of a token's part: sixteen tokens' pieces of one column fall into different banks
    static constexpr int x_bytes = Tokens<T>::kParts * TP * x_stride, w_bytes = U * 16 * kW4RowBytes, all = x_bytes + w_bytes;
};

// Few tokens: a workgroup has 16 rows of the weights and TP <= 16 tokens, its wavefronts take U neighbouring blocks of 128 columns in turn; a batch's loads are on
// their way while the one before is worked on.  GS: log2 of the group; blockIdx.y: tile of 16 tokens
template <typename T, int TP, int GS, int U>
__global__ __launch_bounds__(1024) void w4_kernel(const W4Params p) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int PARTS = Tokens<T>::kParts, NG = 128 >> GS, STEPS = 4 / NG;      // groups in a block, products of 32 columns in a group
    constexpr int GROUPS = U * NG, NS = (GROUPS + 3) / 4;                         // groups in a batch, loads for their scales
    constexpr int PIECES = U * 16, NX = (TP * PIECES + 63) / 64;                  // pieces of eight columns of a token in a batch, and of a lane
    using Lds = W4Lds<T, TP, U>;
    extern __shared__ __align__(16) char w4_lds[];
    const int lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16;
    const int64_t t0 = (int64_t)blockIdx.y * 16;
    const int tokens = (int)min(p.n_tokens - t0, (int64_t)TP);
    const int groups = p.K >> GS, batches = (p.K + 128 * U - 1) / (128 * U);
    char* const lds_x = w4_lds + wave * Lds::all;
    char* const lds_w = lds_x + Lds::x_bytes;

    // what this lane loads: a piece of a row (row lane / 4), the scale of group g of a row (row lane % 16), pieces of tokens: offsets from what the workgroup has first
    const uint8_t* const codes = p.codes + (int64_t)n0 * (p.K >> 1);
    const char* const scales = (const char*)p.scales + (int64_t)n0 * groups * (int)sizeof(T);
    const uint8_t* const zeros = p.zeros + (int64_t)n0 * groups;
    const char* const x = (const char*)p.x + t0 * p.x_stride * (int)sizeof(T);
    const int last_row = p.N - 1 - n0;
    const uint32_t w_at = (uint32_t)min(lane >> 2, last_row) * (uint32_t)(p.K >> 1) + 16u * (lane & 3);
    const uint32_t group_at = (uint32_t)min(col, last_row) * (uint32_t)groups;
    uint32_t x_at[NX];
#pragma unroll
    for (int i = 0; i < NX; ++i) {
        const int id = i * 64 + lane;
        x_at[i] = ((uint32_t)min(id / PIECES, tokens - 1) * (uint32_t)p.x_stride + 8u * (id % PIECES)) * (uint32_t)sizeof(T);
    }

    u32x4 raw_w[U];
    uint32_t raw_scale[NS], raw_zero[NS];
    Tokens<T> raw_x[NX];
    auto load = [&](int batch) __attribute__((always_inline)) {
        const int k0 = batch * 128 * U;
        const uint8_t* const wk = codes + (k0 >> 1);
        const char* const xk = x + (int64_t)k0 * (int)sizeof(T);
        // columns beyond the last: read where there is something, counted for nothing (x is 0 there, and so is the scale)
        const bool all = k0 + 128 * U <= p.K;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t at = w_at + 64u * u;
            if (!all) at = (uint32_t)((int)w_at + min(64 * u, ((p.K - 32 - k0) >> 1) - 16 * (lane & 3)));
            raw_w[u] = *reinterpret_cast<const u32x4*>(wk + (all ? (int64_t)at : (int64_t)(int)at));
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const uint32_t at = group_at + (uint32_t)min((k0 >> GS) + 4 * i + g, groups - 1);
            raw_scale[i] = raw_element<T>(scales, at);
            if (p.zeros) raw_zero[i] = zeros[at];
        }
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            int back = 0;
            if (!all) back = max(8 * ((i * 64 + lane) % PIECES) - (p.K - 8 - k0), 0) * (int)sizeof(T);
            raw_x[i].load(reinterpret_cast<const T*>(xk + (int64_t)x_at[i] - back));
        }
    };
    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
    const OffsetConstants constants;
    f32x4 acc = {};
    int batch = wave;
    if (batch < batches) load(batch);
    while (batch < batches) {
        // to LDS, a wavefront's own part: its reads come after its writes, nobody else is waited for
#pragma unroll
        for (int u = 0; u < U; ++u) *reinterpret_cast<u32x4*>(lds_w + (u * 16 + (lane >> 2)) * kW4RowBytes + 16 * (lane & 3)) = raw_w[u];
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int id = i * 64 + lane, token = id / PIECES, piece = id % PIECES;
            u32x4 a[PARTS];
            raw_x[i].parts(batch * 128 * U + 128 * U <= p.K || batch * 128 * U + 8 * piece < p.K, a);
            if (TP * PIECES % 64 == 0 || token < TP)
#pragma unroll
                for (int k = 0; k < PARTS; ++k) *reinterpret_cast<u32x4*>(lds_x + (k * TP + token) * Lds::x_stride + 16 * piece) = a[k];
        }
        float scale[NS][4], zero[NS][4];
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            uint32_t s[4], z[4];
            spread((batch * 128 * U >> GS) + 4 * i + g < groups ? raw_scale[i] : 0u, s);
            if (p.zeros) spread(raw_zero[i], z);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float sc = from_raw<T>(s[j]), zr = p.zeros ? (float)(z[j] & 15u) : 8.f;
                scale[i][j] = F32 ? 16.f * sc : sc;
                zero[i][j] = F32 ? (zr - 8.f) * 0.0625f : zr + kOffset;
            }
        }
        const int next = batch + waves;
        if (next < batches) load(next);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                f32x4 d = {0.f, 0.f, 0.f, 0.f}, sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int a = j * STEPS; a < (j + 1) * STEPS; ++a) {
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(lds_w + (u * 16 + col) * kW4RowBytes + 16 * a + 4 * g);
                    const bf16x8 wf = F32 ? weights_exact(w) : weights_offset(w, constants);
#pragma unroll
                    for (int k = 0; k < PARTS; ++k) {
                        // lanes of tokens that are not there have some other's, or what is left of an earlier call: their rows of the result are dropped
                        const bf16x8 xa = *reinterpret_cast<const bf16x8*>(lds_x + (k * TP + min(col, TP - 1)) * Lds::x_stride + u * 256 + 64 * a + 16 * g);
                        d = mfma_16x16x32(xa, wf, d);
                        if (!F32 || p.zeros) sum = mfma_16x16x32(xa, ones, sum);
                    }
                }
                const int i = (u * NG + j) >> 2, jj = (u * NG + j) & 3;
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[v] = fmaf(scale[i][jj], fmaf(-zero[i][jj], sum[v], d[v]), acc[v]);
            }
        batch = next;
    }
    __syncthreads();                               // everybody is through with its part of LDS
    store_sums<T>(p, (float*)w4_lds, wave, waves, t0, n0, acc);
}

// More tokens (bf16): a workgroup has 16 * RT * WR rows and 16 * TT tokens.  Its wavefronts are WK groups, each with a range of columns, of WR, which have
// 16 * RT rows each and read x from one copy of it in LDS, with the sums of x over the groups beside it.  While a chunk of 128 columns is worked on, the next one goes to the other
// half of LDS and the one after it is on its way from memory.  What bounds it: the operations that make operands of codes and scale the sums (57 % of the vector units' time, the matrix
// cores 19 %, 64 tokens, 4096 x 28672, groups of 64: 34.5 us, 436 TFLOP/s), and x, which passes the second-level caches once for every 16 * RT * WR rows.
// With two row tiles per wavefront (RT) the sums of x over a group are made once, where x is brought, and each result takes (16 + zero) times that.  With one there is room on the matrix
// cores: they multiply x by a second operand that is -(16 + zero) everywhere, which is exact, and half of the groups of wavefronts bring x after their products instead of before, so that
// the two on a SIMD unit want different units.  20 tokens, 14336 x 4096, groups of 32: 40.1 -> 35.1 us (the same with two row tiles: 35.7 -> 37.4).
// The codes have WB copies in LDS.  One is written when its reader is through with it, and waited for at once; but with it two workgroups with one row tile fit a unit, where there
// are that many: 20 tokens, 4096 x 14336, groups of 128: 18.0 -> 14.6 us, where there are not, 4096 x 4096: 9.5 with two copies, 11.2 with one.  Two row tiles: 33.4 -> 31.7 us (100 tokens,
// 4096 x 14336, groups of 64), though 19.7 -> 20.6 with 64 tokens and groups of 128.
template <int TT, int WR, int WK, int RT, int WB, int GS>
struct W4Wide {
    static constexpr int waves = WR * WK, threads = waves * kWave;
    static constexpr int x_bytes = TT * 4 * 1024;                               // [tile][32 columns][lane of the operand] 16 bytes
    static constexpr int sum_bytes = RT > 1 ? (128 >> GS) * TT * 16 * 4 : 0;    // [group][token]
    static constexpr int of_group = x_bytes + sum_bytes;
    static constexpr int w_bytes = RT * 16 * 64, span_bytes = RT * ScaleSpan::kBytes;
    static constexpr int all = 2 * WK * of_group + waves * (WB * w_bytes + span_bytes);
    static constexpr int lds = all > waves * RT * 1024 ? all : waves * RT * 1024;
    static_assert(lds <= 160 * 1024, "LDS of a unit");
};

// sum of eight bf16 values
__device__ __forceinline__ float sum_eight(u32x4 w) {
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t two = w[e];                 // a bit cast of a vector's element itself takes the first one
        s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), one, s, false);
    }
    return s;
}
// v and that of another lane of the sixteen, by the number's bits: 0xB1, 0x4E exchange lanes 1 and 2 apart, 0x141 and 0x140 mirror eight and sixteen
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}

template <int TT, int WR, int WK, int RT, int WB, int GS>
__global__ __launch_bounds__((W4Wide<TT, WR, WK, RT, WB, GS>::threads), (WB * RT == 1 ? 4 : 2)) void w4_wide_kernel(const W4Params p) {
    using Shape = W4Wide<TT, WR, WK, RT, WB, GS>;
    using Span = ScaleSpan;
    constexpr int NG = 128 >> GS, STEPS = 4 / NG, PER_SPAN = Span::kGroups / NG;
    constexpr bool SUMS = RT > 1;                                               // of x over the groups, in LDS
    constexpr int LANES = WR * kWave;                                            // of a group of wavefronts
    constexpr int NX = TT * 16 * 16 / LANES;                                     // pieces of eight columns of a token that a lane brings to LDS
    extern __shared__ __align__(16) char w4_lds[];
    const int lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave / WR, wr = wave % WR;
    const int n0 = (blockIdx.x * WR + wr) * 16 * RT, groups = p.K >> GS;
    const int64_t t0 = (int64_t)blockIdx.y * 16 * TT;
    const int chunks = (p.K + 127) >> 7, rounds = (chunks + WK - 1) / WK, first = wk * rounds;       // every wavefront goes round as often
    char* const lds_x = w4_lds + wk * 2 * Shape::of_group;
    char* const lds_w = w4_lds + WK * 2 * Shape::of_group + wave * (WB * Shape::w_bytes + Shape::span_bytes);
    char* const lds_s = lds_w + WB * Shape::w_bytes;
    const int id = wr * kWave + lane, piece = id & 15, tok = id >> 4;            // lanes of a token are neighbours; the next pieces are LANES / 16 tokens on

    const uint8_t* codes[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) codes[r] = p.codes + (int64_t)min(n0 + 16 * r + (lane >> 2), p.N - 1) * (p.K >> 1) + 16 * (lane & 3);
    const uint16_t* xs[NX];
#pragma unroll
    for (int i = 0; i < NX; ++i) xs[i] = (const uint16_t*)p.x + min(t0 + tok + i * (LANES / 16), p.n_tokens - 1) * p.x_stride + 8 * piece;

    u32x4 raw_w[RT];
    Span span[RT];
    Tokens<uint16_t> raw_x[NX];
    // a chunk beyond the last, and columns beyond the last: read where there is something, counted for nothing (x is 0 there, and so is the scale)
    auto load_w = [&](int chunk) __attribute__((always_inline)) {
        const int wk0 = min(min(chunk, chunks - 1) * 128, p.K - 32 - 32 * (lane & 3)) >> 1;
#pragma unroll
        for (int r = 0; r < RT; ++r) raw_w[r] = *reinterpret_cast<const u32x4*>(codes[r] + wk0);
    };
    auto load_x = [&](int chunk) __attribute__((always_inline)) {
        const int xk0 = min(min(chunk, chunks - 1) * 128, p.K - 8 - 8 * piece);
#pragma unroll
        for (int i = 0; i < NX; ++i) raw_x[i].load(xs[i] + xk0);
    };
    auto stage_x = [&](int chunk, int half) __attribute__((always_inline)) {
        char* const to = lds_x + half * Shape::of_group;
        if (chunk * 128 + 128 > p.K)
#pragma unroll
            for (int i = 0; i < NX; ++i) raw_x[i].w = chunk * 128 + 8 * piece < p.K ? raw_x[i].w : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            u32x4 a[1];
            raw_x[i].parts(true, a);
            const int t = tok + i * (LANES / 16), slot = ((piece & 3) * 16 + ((t & 15) ^ piece)) * 16;       // exchanged within sixteen: a token's pieces in different banks
            *reinterpret_cast<u32x4*>(to + ((t >> 4) * 4 + (piece >> 2)) * 1024 + slot) = a[0];
            if constexpr (SUMS) {
                float sum = add_dpp<0x4E>(add_dpp<0xB1>(sum_eight(a[0])));
                if constexpr (GS > 5) sum = add_dpp<0x141>(sum);
                if constexpr (GS > 6) sum = add_dpp<0x140>(sum);
                if ((piece & ((1 << GS) / 8 - 1)) == 0) ((float*)(to + Shape::x_bytes))[(piece >> (GS - 3)) * TT * 16 + t] = sum;
            }
        }
    };
    // exchanged within a row: sixteen rows' words of one column fall into different banks
    auto stage_w = [&](int half) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < RT; ++r) *reinterpret_cast<u32x4*>(lds_w + half % WB * Shape::w_bytes + (r * 16 + (lane >> 2)) * 64 + 16 * ((lane ^ (lane >> 4)) & 3)) = raw_w[r];
    };
    const OffsetConstants constants;
    f32x4 acc[TT][RT] = {};
#pragma unroll
    for (int r = 0; r < RT; ++r) span[r].load(p, n0 + 16 * r, groups, first * NG);
    load_x(first);
    load_w(first);
    stage_x(first, 0);
    load_x(first + 1);
    stage_w(0);
    load_w(first + 1);
    __syncthreads();
    for (int round = 0; round < rounds; ++round) {
        const int chunk = first + round, half = round & 1, in_span = round % PER_SPAN;
        if (in_span == 0) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                span[r].put(p, lds_s + r * Span::kBytes);
                if (round + PER_SPAN < rounds) span[r].load(p, n0 + 16 * r, groups, (chunk + PER_SPAN) * NG);
            }
        }
        const bool later = !SUMS && wk % 2 == 1, more = round + 1 < rounds;
        if (more && !later) {
            stage_x(chunk + 1, half ^ 1);
            load_x(chunk + 2);
            if (WB > 1) {
                stage_w(half ^ 1);
                load_w(chunk + 2);
            }
        }
        const char* const x = lds_x + half * Shape::of_group;
        const char* const w = lds_w + half % WB * Shape::w_bytes;
        constexpr int kAtOnce = TT * RT * NG > 16 || (WB * RT == 1 && NG == 4) ? 1 : NG;    // groups whose operands there are registers for
#pragma unroll kAtOnce
        for (int j = 0; j < NG; ++j) {
            f32x4 d[TT][RT] = {};
            float s[RT], z[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                s[r] = Span::scale(lds_s + r * Span::kBytes, in_span * NG + j);
                if (chunk * NG + j >= groups) s[r] = 0.f;
                z[r] = Span::zero(p, lds_s + r * Span::kBytes, in_span * NG + j) + kOffset;
            }
            const uint32_t zero = __builtin_amdgcn_perm(__float_as_uint(-z[0]), __float_as_uint(-z[0]), 0x07060706u);
            const bf16x8 zf = __builtin_bit_cast(bf16x8, u32x4{zero, zero, zero, zero});
#pragma unroll
            for (int a = j * STEPS; a < (j + 1) * STEPS; ++a) {
                bf16x8 wf[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) wf[r] = weights_offset(*reinterpret_cast<const uint32_t*>(w + (r * 16 + col) * 64 + 16 * (a ^ (col >> 2)) + 4 * g), constants);
#pragma unroll
                for (int i = 0; i < TT; ++i) {
                    const bf16x8 xa = *reinterpret_cast<const bf16x8*>(x + (i * 4 + a) * 1024 + (g * 16 + (col ^ (4 * a + g))) * 16);
#pragma unroll
                    for (int r = 0; r < RT; ++r) d[i][r] = mfma_16x16x32(xa, wf[r], d[i][r]);
                    if constexpr (!SUMS) d[i][0] = mfma_16x16x32(xa, zf, d[i][0]);
                }
            }
#pragma unroll
            for (int i = 0; i < TT; ++i) {
                f32x4 sum = {0.f, 0.f, 0.f, 0.f};
                if constexpr (SUMS) sum = *reinterpret_cast<const f32x4*>(x + Shape::x_bytes + ((j * TT + i) * 16 + 4 * g) * 4);
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[i][r][v] = fmaf(s[r], SUMS ? fmaf(-z[r], sum[v], d[i][r][v]) : d[i][r][v], acc[i][r][v]);
            }
        }
        if (more && later) {
            stage_x(chunk + 1, half ^ 1);
            load_x(chunk + 2);
        }
        if (more && (later || WB == 1)) {      // this wavefront has read what one copy is written over
            stage_w(half ^ 1);
            load_w(chunk + 2);
        }
        __syncthreads();                       // this half has been read, the other is whole
    }
    // the groups' sums in order, a tile of tokens at a time
    float* const sums = (float*)w4_lds;
    constexpr int ROWS = 16 * RT * WR;
#pragma unroll
    for (int i = 0; i < TT; ++i) {
        if (i > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int v = 0; v < 4; ++v) sums[(wk * 16 + 4 * g + v) * ROWS + (wr * RT + r) * 16 + col] = acc[i][r][v];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * ROWS; e += Shape::threads) {
            const int64_t t = t0 + 16 * i + e / ROWS;
            const int n = blockIdx.x * ROWS + e % ROWS;
            if (t >= p.n_tokens || n >= p.N) continue;
            float y = p.bias ? element<uint16_t>(p.bias, n) : 0.f;
#pragma unroll
            for (int k = 0; k < WK; ++k) y += sums[k * 16 * ROWS + e];
            if (p.y_bf16) ((uint16_t*)p.y)[t * p.N + n] = f32_to_bf16_bits(y);
            else ((float*)p.y)[t * p.N + n] = y;
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------
static int check_w4_desc(const astra_w4_desc* d) {
    if (!d) return ASTRA_ERR_NULL;
    if ((d->dtype != ASTRA_F32 && d->dtype != ASTRA_BF16) || (d->y_dtype != ASTRA_F32 && d->y_dtype != ASTRA_BF16)) return ASTRA_ERR_DTYPE;
    if (d->in_features <= 0 || d->out_features <= 0 || d->group <= 0 || d->in_features % d->group != 0) return ASTRA_ERR_SHAPE;
    if (d->group != 32 && d->group != 64 && d->group != 128) return ASTRA_ERR_UNSUPPORTED;
    if (d->in_features > (1 << 24) || d->out_features > (1 << 24)) return ASTRA_ERR_UNSUPPORTED;
    if (d->x_stride != 0) {
        if (d->x_stride < d->in_features) return ASTRA_ERR_SHAPE;
        if (d->x_stride > (1 << 25)) return ASTRA_ERR_UNSUPPORTED;
        if ((int64_t)d->x_stride * elem_bytes(d->dtype) % 16 != 0) return ASTRA_ERR_UNSUPPORTED;
    }
    return ASTRA_OK;
}

template <typename T, int TP, int GS, int U>
static int launch_w4(const W4Params& p, hipStream_t s) {
    static std::atomic<uint64_t> allowed{0};
    using Lds = W4Lds<T, TP, U>;
    const int batches = (int)ceil_div(p.K, 128 * U), most = TP > 8 ? 8 : 16, waves = batches < most ? batches : most;
    const int64_t nx = ceil_div(p.N, 16), ny = ceil_div(p.n_tokens, 16);
        const int lds = std::max(waves * Lds::all, waves * 256 * (int)sizeof(float));
    if (lds > 64 * 1024) {
        const int rc = allow_dynamic_lds(allowed, reinterpret_cast<const void*>(&w4_kernel<T, TP, GS, U>), most * Lds::all);
        if (rc) return rc;
    }
    w4_kernel<T, TP, GS, U><<<dim3((unsigned)nx, (unsigned)ny), waves * kWave, lds, s>>>(p);
    return launch_status();
}

template <typename T, int TP>
static int launch_w4(const W4Params& p, hipStream_t s) {
    constexpr int U = sizeof(T) == 2 ? 2 : 1;
    if (p.group_shift == 5) return launch_w4<T, TP, 5, U>(p, s);
    if (p.group_shift == 6) return launch_w4<T, TP, 6, U>(p, s);
    return launch_w4<T, TP, 7, U>(p, s);
}

template <int TT, int WR, int WK, int RT, int WB, int GS>
static int launch_w4_wide(const W4Params& p, hipStream_t s) {
    static std::atomic<uint64_t> allowed{0};
    using Shape = W4Wide<TT, WR, WK, RT, WB, GS>;
    const int64_t nx = ceil_div(p.N, 16 * RT * WR), ny = ceil_div(p.n_tokens, 16 * TT);
        if (Shape::lds > 64 * 1024) {
        const int rc = allow_dynamic_lds(allowed, reinterpret_cast<const void*>(&w4_wide_kernel<TT, WR, WK, RT, WB, GS>), Shape::lds);
        if (rc) return rc;
    }
    w4_wide_kernel<TT, WR, WK, RT, WB, GS><<<dim3((unsigned)nx, (unsigned)ny), Shape::threads, Shape::lds, s>>>(p);
    return launch_status();
}

template <int TT, int WR, int WK, int RT, int WB>
static int launch_w4_wide(const W4Params& p, hipStream_t s) {
    if (p.group_shift == 5) return launch_w4_wide<TT, WR, WK, RT, WB, 5>(p, s);
    if (p.group_shift == 6) return launch_w4_wide<TT, WR, WK, RT, WB, 6>(p, s);
    return launch_w4_wide<TT, WR, WK, RT, WB, 7>(p, s);
}

static int launch_w4_wide(const W4Params& p, hipStream_t s) {
    // tiles of 128 rows where those are enough for three quarters of the 256 units; of 32, for 32 tokens, otherwise.  48 tokens, 4096 x 14336 (224 tiles of 128): 20.6 us, in tiles of 32 27.7;
    // 20 tokens (112): 14.6 in tiles of 32
    if (p.n_tokens > 32 && ceil_div(p.N, 128) * ceil_div(p.n_tokens, 64) >= 192) return launch_w4_wide<4, 4, 2, 2, 1>(p, s);
    if (ceil_div(p.N, 128) * ceil_div(p.n_tokens, 32) >= 192) return launch_w4_wide<2, 4, 2, 2, 1>(p, s);
    if (ceil_div(p.N, 32) * ceil_div(p.n_tokens, 32) > 256) return launch_w4_wide<2, 2, 4, 1, 1>(p, s);
    return launch_w4_wide<2, 2, 4, 1, 2>(p, s);
}

template <typename T>
static int launch_w4(const W4Params& p, hipStream_t s) {
    if (p.n_tokens <= 2) return launch_w4<T, 2>(p, s);
    if (p.n_tokens <= 8) return launch_w4<T, 8>(p, s);
    if (sizeof(T) == 2 && p.n_tokens > 16) return launch_w4_wide(p, s);
    return launch_w4<T, 16>(p, s);
}

}  // namespace astra

using namespace astra;

extern "C" int astra_w4_linear(const astra_w4_desc* desc, const void* x, int64_t n_tokens, const uint8_t* codes, const void* scales,
                               const uint8_t* zeros, const void* bias, void* y, void* stream) {
    const int rc = check_w4_desc(desc);
    if (rc) return rc;
    if (n_tokens < 0 || n_tokens > kW4MaxTokens) return ASTRA_ERR_SHAPE;
    if (n_tokens == 0) return ASTRA_OK;
    if (!x || !codes || !scales || !y) return ASTRA_ERR_NULL;
    for (const void* a : {x, (const void*)codes, scales, (const void*)zeros, bias, (const void*)y})
        if ((uintptr_t)a % 16 != 0) return ASTRA_ERR_UNSUPPORTED;
    W4Params p{};
    p.x = x; p.codes = codes; p.scales = scales; p.zeros = zeros; p.bias = bias; p.y = y; p.n_tokens = n_tokens;
    p.K = desc->in_features; p.N = desc->out_features;
    p.x_stride = desc->x_stride ? desc->x_stride : desc->in_features;
    p.group_shift = __builtin_ctz((unsigned)desc->group);
    p.y_bf16 = desc->y_dtype == ASTRA_BF16;
    if (desc->dtype == ASTRA_BF16) return launch_w4<uint16_t>(p, (hipStream_t)stream);
    return launch_w4<float>(p, (hipStream_t)stream);
}
