// Products of a few tokens with weights of 4 bits and a scale per group of columns (include/astra.h, astra_w4_linear).
#include "common.h"

namespace astra {

// ------------------------------------------------------------------------------------------------
// y[t, n] = bias[n] + sum_g scale[n, g] ( sum_{k in g} (16 + code) x  -  (16 + zero) sum_{k in g} x )
// The weights are what has to be read, so the products run on the matrix cores with 16 rows of the weights on the N side and the tokens on the M side, and the
// codes reach them in two operations for two: the four bits go to the upper mantissa bits of a bf16 16.0, which makes it 16 + code
// exactly.  A lane loads 16 bytes of a row, 32 columns; the four lanes of a row then trade words (permlane swaps: a 4 x 4 transpose), so that
// one 16x16x32 MFMA sees 32 neighbouring columns of every row, all of one group.  A group's sum stays in fp32 and takes the row's scale there;
// the sum of x over the group comes from another MFMA, against ones.  fp32 tokens are sums of three bf16 parts (8 + 8 + 8 mantissa bits).
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
// eight codes as 16 + code, in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ bf16x8 weights(uint32_t w) {
    constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u;
    u32x4 o;
    o.x = ((w << 3) & kMask) | kSixteen;
    o.y = ((w >> 1) & kMask) | kSixteen;
    o.z = ((w >> 5) & kMask) | kSixteen;
    o.w = ((w >> 9) & kMask) | kSixteen;
    return __builtin_bit_cast(bf16x8, o);
}
// eight neighbouring values of x in that order, as `PARTS` bf16 parts
template <typename T, int PARTS>
__device__ __forceinline__ void tokens(const T* p, bf16x8 (&a)[PARTS]) {
    if constexpr (sizeof(T) == 2) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(p);
        u32x4 o;
        o.x = __builtin_amdgcn_perm(w.z, w.x, 0x05040100u);
        o.y = __builtin_amdgcn_perm(w.z, w.x, 0x07060302u);
        o.z = __builtin_amdgcn_perm(w.w, w.y, 0x05040100u);
        o.w = __builtin_amdgcn_perm(w.w, w.y, 0x07060302u);
        a[0] = __builtin_bit_cast(bf16x8, o);
    } else {
        const f32x4 lo = reinterpret_cast<const f32x4*>(p)[0], hi = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = e & 1 ? hi[e >> 1] : lo[e >> 1];
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {              // every difference is exact
                const float part = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
                a[i][e] = (__bf16)part;
                v -= part;
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ float element(const void* p, int64_t i) {
    if constexpr (sizeof(T) == 2) return bf16_bits_to_f32(((const uint16_t*)p)[i]);
    else return ((const float*)p)[i];
}

// A wavefront per 16 rows of the weights and 16 tokens
template <typename T>
__global__ __launch_bounds__(64) void w4_kernel(const W4Params p) {
    constexpr int PARTS = sizeof(T) == 2 ? 1 : 3;
    const int lane = lane_id(), col = lane & 15, g = lane >> 4;
    const int n = blockIdx.x * 16 + col, n_in = min(n, p.N - 1);
    const int64_t t0 = (int64_t)blockIdx.y * 16, t_in = min(t0 + col, p.n_tokens - 1);
    const T* const x = (const T*)p.x + t_in * p.x_stride + 8 * g;
    const uint8_t* const row = p.codes + (int64_t)n_in * (p.K >> 1);
    const int groups = p.K >> p.group_shift;
    u32x4 ones;
    ones.x = ones.y = ones.z = ones.w = 0x3f803f80u;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f}, d = acc, sum = acc;
    for (int k0 = 0; k0 < p.K; k0 += 128) {
        // columns beyond the last are not there: their words take no part below
        u32x4 w = *reinterpret_cast<const u32x4*>(row + (min(k0 + 32 * g, p.K - 32) >> 1));
        w = transpose_words(w);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int k = k0 + 32 * a;
            if (k >= p.K) break;
            bf16x8 xa[PARTS];
            tokens<T, PARTS>(x + k, xa);
            const bf16x8 wf = weights(w[a]);
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {
                d = mfma_16x16x32(xa[i], wf, d);
                sum = mfma_16x16x32(xa[i], __builtin_bit_cast(bf16x8, ones), sum);
            }
            if (((k + 32) & ((1 << p.group_shift) - 1)) == 0) {
                const int64_t at = (int64_t)n_in * groups + (k >> p.group_shift);
                const float scale = element<T>(p.scales, at), zero = 16.f + (p.zeros ? (float)(p.zeros[at] & 15) : 8.f);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[v] = fmaf(scale, fmaf(-zero, sum[v], d[v]), acc[v]);
                d = f32x4{0.f, 0.f, 0.f, 0.f};
                sum = d;
            }
        }
    }
    if (n >= p.N) return;
    const float bias = p.bias ? element<T>(p.bias, n) : 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int64_t t = t0 + 4 * g + v;
        if (t >= p.n_tokens) break;
        const float y = acc[v] + bias;
        if (p.y_bf16) ((uint16_t*)p.y)[t * p.N + n] = f32_to_bf16_bits(y);
        else ((float*)p.y)[t * p.N + n] = y;
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
    const dim3 grid((unsigned)ceil_div(p.N, 16), (unsigned)ceil_div(n_tokens, 16));
    if (grid.y > 65535) return ASTRA_ERR_SHAPE;
    if (desc->dtype == ASTRA_BF16) w4_kernel<uint16_t><<<grid, 64, 0, (hipStream_t)stream>>>(p);
    else w4_kernel<float><<<grid, 64, 0, (hipStream_t)stream>>>(p);
    return launch_status();
}
