// Products of a few tokens with weights of 4 bits and a scale per group of columns (include/astra.h, astra_w4_linear).
#include "common.h"

namespace astra {

// ------------------------------------------------------------------------------------------------
// y[t, n] = bias[n] + sum_g scale[n, g] ( sum_{k in g} (16 + code) x  -  (16 + zero) sum_{k in g} x )
// The weights are what has to be read, so the products run on the matrix cores with 16 rows of the weights on the N side and 16 tokens on the M side, and the
// codes reach them in two operations for two: the four bits go to the upper mantissa bits of a bf16 16.0, which makes it 16 + code
// exactly.  A lane loads 16 bytes of a row, 32 columns; the four lanes of a row then trade words (permlane swaps: a 4 x 4 transpose), so that
// one 16x16x32 MFMA sees 32 neighbouring columns of every row, all of one group.  A group's sum stays in fp32 and takes the row's scale there;
// the sum of x over the group comes from another MFMA, against ones.  fp32 tokens are sums of three bf16 parts (8 + 8 + 8 mantissa bits), and their weights
// code - 8, at 20 operations for eight instead of 8: the difference of the two sums above loses three bits, which a bf16 result does not show.
// The wavefronts of a workgroup take blocks of 128 columns in turn, U of them at a time with all their loads on the way, and add up in LDS.
// TT x RT: tiles of 16 tokens and of 16 rows that a workgroup has; more rows for many tokens, whose x otherwise passes the second-level caches more often
// than the weights pass memory.
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

// word i of lane group j <-> word j of lane group i (groups of 16 lanes)
__device__ __forceinline__ u32x4 transpose_words(u32x4 w) {
    auto a = __builtin_amdgcn_permlane32_swap(w.x, w.z, false, false);      // upper half of the first <-> lower half of the second
    auto b = __builtin_amdgcn_permlane32_swap(w.y, w.w, false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);    // odd rows of the first <-> even rows of the second
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return u32x4{(uint32_t)c[0], (uint32_t)c[1], (uint32_t)d[0], (uint32_t)d[1]};
}
constexpr float kOffset = 16.f;
// eight codes as 16 + code, in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ bf16x8 weights_offset(uint32_t w) {
    constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u;
    u32x4 o;
    o.x = ((w << 3) & kMask) | kSixteen;
    o.y = ((w >> 1) & kMask) | kSixteen;
    o.z = ((w >> 5) & kMask) | kSixteen;
    o.w = ((w >> 9) & kMask) | kSixteen;
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
    u32x4 w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ void operand(bf16x8 (&a)[1]) const {
        u32x4 o;
        o.x = __builtin_amdgcn_perm(w.z, w.x, 0x05040100u);
        o.y = __builtin_amdgcn_perm(w.z, w.x, 0x07060302u);
        o.z = __builtin_amdgcn_perm(w.w, w.y, 0x05040100u);
        o.w = __builtin_amdgcn_perm(w.w, w.y, 0x07060302u);
        a[0] = __builtin_bit_cast(bf16x8, o);
    }
};
template <>
struct Tokens<float> {
    f32x4 w[2];
    __device__ __forceinline__ void load(const float* p) {
        w[0] = reinterpret_cast<const f32x4*>(p)[0];
        w[1] = reinterpret_cast<const f32x4*>(p)[1];
    }
    __device__ __forceinline__ void operand(bf16x8 (&a)[3]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = w[e >> 2][e & 3];
#pragma unroll
            for (int i = 0; i < 3; ++i) {                  // every difference is exact
                const float part = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
                a[i][e] = (__bf16)part;
                v -= part;
            }
        }
    }
};

template <typename T>
__device__ __forceinline__ float element(const void* p, int64_t i) {
    if constexpr (sizeof(T) == 2) return bf16_bits_to_f32(((const uint16_t*)p)[i]);
    else return ((const float*)p)[i];
}

// GS: log2 of the group.  blockIdx.x: tile of 16 * RT rows, blockIdx.y: tile of 16 * TT tokens
template <typename T, int TT, int RT, int GS, int U>
__global__ __launch_bounds__(TT * RT > 2 ? 512 : 1024) void w4_kernel(const W4Params p) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int PARTS = F32 ? 3 : 1, NG = 128 >> GS, STEPS = 4 / NG;      // groups in a block, products of 32 columns in a group
    extern __shared__ __align__(16) float sums[];                           // [wavefronts][RT][16][16]
    const int lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16 * RT;
    const int64_t t0 = (int64_t)blockIdx.y * 16 * TT;
    const int groups = p.K >> GS, blocks = (p.K + 127) >> 7;
    const uint8_t* rows[RT];
    int64_t scale_at[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int64_t n = min(n0 + 16 * r + col, p.N - 1);
        rows[r] = p.codes + n * (p.K >> 1) + 16 * g;
        scale_at[r] = n * groups;
    }
    const T* x[TT];
    bool there[TT];
#pragma unroll
    for (int i = 0; i < TT; ++i) {
        there[i] = t0 + 16 * i + col < p.n_tokens;
        x[i] = (const T*)p.x + min(t0 + 16 * i + col, p.n_tokens - 1) * p.x_stride + 8 * g;
    }
    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
    f32x4 acc[TT][RT] = {};

    for (int b0 = wave; b0 < blocks; b0 += waves * U) {
        u32x4 w[U][RT];
        float scale[U][RT][NG], zero[U][RT][NG];
        Tokens<T> xs[U][4][TT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // a block beyond the last, and words and groups beyond the last column: read where there is something, counted for nothing (x is 0, and so is the scale)
            const int k0 = min(b0 + u * waves, blocks - 1) * 128;
#pragma unroll
            for (int r = 0; r < RT; ++r) w[u][r] = *reinterpret_cast<const u32x4*>(rows[r] + (min(k0, p.K - 32 - 32 * g) >> 1));
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int i = 0; i < TT; ++i) {
                    xs[u][a][i] = Tokens<T>{};
                    if (there[i] && b0 + u * waves < blocks && k0 + 32 * a < p.K) xs[u][a][i].load(x[i] + k0 + 32 * a);
                }
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    const int at = (k0 >> GS) + j, in = min(at, groups - 1);
                    scale[u][r][j] = at == in ? element<T>(p.scales, scale_at[r] + in) : 0.f;
                    zero[u][r][j] = p.zeros ? (float)(p.zeros[scale_at[r] + in] & 15) : 8.f;
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int r = 0; r < RT; ++r) w[u][r] = transpose_words(w[u][r]);
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                f32x4 d[TT][RT] = {}, sum[TT] = {};
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    const int a = j * STEPS + st;
                    bf16x8 wf[RT];
#pragma unroll
                    for (int r = 0; r < RT; ++r) wf[r] = F32 ? weights_exact(w[u][r][a]) : weights_offset(w[u][r][a]);
#pragma unroll
                    for (int i = 0; i < TT; ++i) {
                        bf16x8 xa[PARTS];
                        xs[u][a][i].operand(xa);
#pragma unroll
                        for (int k = 0; k < PARTS; ++k) {
#pragma unroll
                            for (int r = 0; r < RT; ++r) d[i][r] = mfma_16x16x32(xa[k], wf[r], d[i][r]);
                            if (!F32 || p.zeros) sum[i] = mfma_16x16x32(xa[k], ones, sum[i]);
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const float s = F32 ? 16.f * scale[u][r][j] : scale[u][r][j];
                    const float z = F32 ? (zero[u][r][j] - 8.f) * 0.0625f : zero[u][r][j] + kOffset;
#pragma unroll
                    for (int i = 0; i < TT; ++i)
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[i][r][v] = fmaf(s, fmaf(-z, sum[i][v], d[i][r][v]), acc[i][r][v]);
                }
            }
        }
    }

    // the wavefronts' sums in order: RT tiles of 16 tokens at a time
#pragma unroll
    for (int i = 0; i < TT; ++i) {
        if (i > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int v = 0; v < 4; ++v) sums[((wave * 16 + 4 * g + v) * RT + r) * 16 + col] = acc[i][r][v];
        __syncthreads();
        for (int e = threadIdx.x; e < 256 * RT; e += blockDim.x) {
            const int64_t t = t0 + 16 * i + e / (16 * RT);
            const int n = n0 + e % (16 * RT);
            if (t >= p.n_tokens || n >= p.N) continue;
            float y = p.bias ? element<T>(p.bias, n) : 0.f;
            for (int k = 0; k < waves; ++k) y += sums[k * 256 * RT + e];
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
        if ((int64_t)d->x_stride * elem_bytes(d->dtype) % 16 != 0) return ASTRA_ERR_UNSUPPORTED;
    }
    return ASTRA_OK;
}

template <typename T, int TT, int RT, int U>
static int launch_w4(const W4Params& p, int waves, hipStream_t s) {
    const int64_t nx = ceil_div(p.N, 16 * RT), ny = ceil_div(p.n_tokens, 16 * TT);
    if (nx > 0x7fffffff || ny > 65535) return ASTRA_ERR_SHAPE;
    const dim3 grid((unsigned)nx, (unsigned)ny);
    const size_t lds = (size_t)waves * RT * 256 * sizeof(float);
    if (p.group_shift == 5) w4_kernel<T, TT, RT, 5, U><<<grid, waves * kWave, lds, s>>>(p);
    else if (p.group_shift == 6) w4_kernel<T, TT, RT, 6, U><<<grid, waves * kWave, lds, s>>>(p);
    else w4_kernel<T, TT, RT, 7, U><<<grid, waves * kWave, lds, s>>>(p);
    return launch_status();
}

template <typename T>
static int launch_w4(const W4Params& p, hipStream_t s) {
    const int blocks = (int)ceil_div(p.K, 128);
    const int waves = blocks <= 4 ? 4 : blocks <= 32 ? 8 : 16;
    if (p.n_tokens <= 16) return launch_w4<T, 1, 1, 2>(p, waves, s);
    if (sizeof(T) == 4 || p.n_tokens <= 32) return launch_w4<T, 2, 1, 1>(p, waves, s);
    return launch_w4<uint16_t, 4, 2, 1>(p, 8, s);
}

}  // namespace astra

using namespace astra;

extern "C" int astra_w4_linear(const astra_w4_desc* desc, const void* x, int64_t n_tokens, const uint8_t* codes, const void* scales,
                               const uint8_t* zeros, const void* bias, void* y, void* stream) {
    const int rc = check_w4_desc(desc);
    if (rc) return rc;
    if (n_tokens < 0 || n_tokens > (1 << 20)) return ASTRA_ERR_SHAPE;
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
