// Products of MXFP4 rows (mx4_device.h has the format): y = a w^T, and the
// gated pair SiLU(a w_gate^T) * (a w_up^T) of a feed-forward block.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 multiplies E2M1 numbers and applies both
// operands' scale bytes itself: lane l holds 32 consecutive codes of row
// l % 32 and the scale byte of that block.  The contraction does not care
// which 32 of a row's values meet in which instruction, as long as both
// operands agree; so with 256 values of k a step, lane l takes the four
// blocks 4 (l / 32) .. + 3 one after the other: 64 consecutive bytes of codes,
// and scale bytes that are one aligned word.
#include "gemm_device.h"
#include "mx4_device.h"
#include "p4q_internal.h"

#include <algorithm>
#include <type_traits>

namespace p4q {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// what becomes of the sums
enum Epilogue { kLinear, kGated, kGatedQuant };

// acc += w a^T over 64 values of k (block I of each lane's four); sw, sa: the
// words of scale bytes
template <int I>
__device__ __forceinline__ void mfma_mx4(v4i w, uint32_t sw, v4i a, uint32_t sa, v16f &acc) {
    const v8i W = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, acc, 4, 4, I, (int)sw, I, (int)sa);
}

__device__ __forceinline__ float silu(float g) { return g / (1.0f + __expf(-g)); }

// 8 consecutive outputs n0 .. n0 + 7 of row m (u: the up sums, gated only).
// Four lanes of a quad hold 32 outputs of one row in order.
template <int EPI, bool BF16>
__device__ __forceinline__ void emit8(const Mx4Product &p, int64_t m, int n0, float (&v)[8], const float (&u)[8]) {
    if constexpr (EPI != kLinear) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = silu(v[i]) * u[i];
    }
    if constexpr (EPI == kGatedQuant) {
        uint32_t byte;
        const uint32_t c = mx4_quantize(v, byte);
        if (m < p.M && n0 < p.N) {
            reinterpret_cast<uint32_t *>(p.codes)[(m * p.N + n0) >> 3] = c;
            if ((n0 & 31) == 0) p.scales[m * p.out_stride + (n0 >> 5)] = (uint8_t)byte;
        }
    } else {
        if (m >= p.M || n0 >= p.N) return;
        uint16_t *dst = static_cast<uint16_t *>(p.y) + m * p.ldy + n0;
        const uint4 w = round16x8<BF16>(v);
        if (p.wide && n0 + 8 <= p.N) {
            *reinterpret_cast<uint4 *>(dst) = w;
        } else {
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (n0 + i < p.N) dst[i] = (uint16_t)(x[i >> 1] >> (16 * (i & 1)));
        }
    }
}

// The 32 codes each of blocks b .. b + 3 of a row, zero past the row's end
__device__ __forceinline__ void load_blocks(const uint8_t *row, int b, int blocks, v4i (&c)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c[i] = v4i{0, 0, 0, 0};
        if (b + i < blocks) c[i] = *reinterpret_cast<const v4i *>(row + 16 * (int64_t)(b + i));
    }
}

// their scale bytes; 0 past the row's end, whatever the padding holds
__device__ __forceinline__ uint32_t load_scales(const uint8_t *row, int b, int blocks) {
    const uint32_t s = *reinterpret_cast<const uint32_t *>(row + b);
    const int left = blocks - b;
    return left >= 4 ? s : left <= 0 ? 0u : s & ((1u << (8 * left)) - 1u);
}

// 32 outputs of MB * 32 rows, the eight wavefronts sharing k in steps of 256;
// their sums meet in LDS in a fixed order.  Operands come straight from memory.
constexpr int kSkinnyWaves = 8;

template <int EPI, bool BF16, int MB>
__global__ __launch_bounds__(64 * kSkinnyWaves) void k_mx4_skinny(const Mx4Product p) {
    constexpr int F = EPI == kLinear ? 1 : 2;
    constexpr int kGroup = 64 * 4 + 4;                     // floats of 8 consecutive outputs, all lanes
    __shared__ float red[kSkinnyWaves][F][MB][4][kGroup];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 31, h = lane >> 5;
    const int n0 = (int)blockIdx.x * 32;
    const int64_t m0 = (int64_t)blockIdx.y * 32 * MB;
    const int blocks = p.K / 32, steps = (blocks + 7) / 8;
    const int64_t kb = p.K / 2;

    const uint8_t *wrow[F], *wsrow[F], *arow[MB], *asrow[MB];
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int64_t n = min(n0 + r, p.N - 1) + (int64_t)f * p.N;
        wrow[f] = p.w + n * kb;
        wsrow[f] = p.ws + n * p.in_stride;
    }
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int64_t m = min(m0 + 32 * b + r, (int64_t)p.M - 1);
        arow[b] = p.a + m * kb;
        asrow[b] = p.as + m * p.in_stride;
    }
    v16f acc[F][MB];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[f][b] = v16f{};

    for (int st = wave; st < steps; st += kSkinnyWaves) {
        const int c0 = 8 * st + 4 * h;
        v4i w[F][4], a[MB][4];
        uint32_t sw[F], sa[MB];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            load_blocks(wrow[f], c0, blocks, w[f]);
            sw[f] = load_scales(wsrow[f], c0, blocks);
        }
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            load_blocks(arow[b], c0, blocks, a[b]);
            sa[b] = load_scales(asrow[b], c0, blocks);
        }
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                mfma_mx4<0>(w[f][0], sw[f], a[b][0], sa[b], acc[f][b]);
                mfma_mx4<1>(w[f][1], sw[f], a[b][1], sa[b], acc[f][b]);
                mfma_mx4<2>(w[f][2], sw[f], a[b][2], sa[b], acc[f][b]);
                mfma_mx4<3>(w[f][3], sw[f], a[b][3], sa[b], acc[f][b]);
            }
    }
    // lane l holds row m0 + l % 32, outputs 8 g + 4 (l / 32) + 0..3 in registers 4 g ..
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4 *>(&red[wave][f][b][g][4 * lane]) =
                    make_float4(acc[f][b][4 * g], acc[f][b][4 * g + 1], acc[f][b][4 * g + 2], acc[f][b][4 * g + 3]);
    __syncthreads();
    for (int t = threadIdx.x; t < 128 * MB; t += 64 * kSkinnyWaves) {
        const int b = t >> 7, mr = (t >> 2) & 31, g = t & 3;
        float v[2][8];
#pragma unroll
        for (int f = 0; f < F; ++f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[f][i] = 0.0f;
#pragma unroll
            for (int w = 0; w < kSkinnyWaves; ++w)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const float4 x = *reinterpret_cast<const float4 *>(&red[w][f][b][g][4 * (mr + 32 * hh)]);
                    v[f][4 * hh + 0] += x.x;
                    v[f][4 * hh + 1] += x.y;
                    v[f][4 * hh + 2] += x.z;
                    v[f][4 * hh + 3] += x.w;
                }
        }
        emit8<EPI, BF16>(p, m0 + 32 * b + mr, n0 + 8 * g, v[0], v[1]);
    }
    if constexpr (EPI == kGatedQuant) {
        // the padding behind a row's last block
        if (n0 + 32 >= p.N && (int)threadIdx.x < 32 * MB && m0 + threadIdx.x < p.M)
            for (int64_t i = p.N / 32; i < p.out_stride; ++i) p.scales[(m0 + threadIdx.x) * p.out_stride + i] = 0;
    }
}

template <int EPI, bool BF16>
hipError_t launch_typed(const Mx4Product &p, hipStream_t stream) {
    const dim3 grid((unsigned)((p.N + 31) / 32), (unsigned)(((int64_t)p.M + 31) / 32));
    hipLaunchKernelGGL((k_mx4_skinny<EPI, BF16, 1>), grid, dim3(64 * kSkinnyWaves), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_linear(p4q_dtype out_dt, Mx4Product p, hipStream_t stream) {
    p.in_stride = mx4_scale_stride(p.K);
    p.wide = p.ldy % 8 == 0 && reinterpret_cast<uintptr_t>(p.y) % 16 == 0;
    return out_dt == P4Q_BF16 ? launch_typed<kLinear, true>(p, stream) : launch_typed<kLinear, false>(p, stream);
}

hipError_t launch_mx4_gated(p4q_dtype out_dt, Mx4Product p, hipStream_t stream) {
    p.in_stride = mx4_scale_stride(p.K);
    p.out_stride = mx4_scale_stride(p.N);
    if (p.codes) return launch_typed<kGatedQuant, false>(p, stream);
    p.wide = p.ldy % 8 == 0 && reinterpret_cast<uintptr_t>(p.y) % 16 == 0;
    return out_dt == P4Q_BF16 ? launch_typed<kGated, true>(p, stream) : launch_typed<kGated, false>(p, stream);
}

}  // namespace p4q
