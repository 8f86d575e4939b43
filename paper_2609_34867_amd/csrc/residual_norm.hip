// What lies between two blocks of a decoder layer, in one pass: the block's
// output, normalized where the model does so and gated, is added to the
// residual, and the next block's RMSNorm of the sum is quantized.
//
//   r' = post ? r / rms(r) * post : r
//   h  = round16(fl32(x + alpha gate r'))            (no r: h = x)
//   int4:  codes = Q4(u; clip), scale = fl32(s / rms(h)),  u = h gamma;
//          values round16(fl32(code scale))
//   MXFP4: codes, scales of fl32(u / rms(h)), 32 values at a time; values exact in fp32
//   rms(z) = sqrt(sum z^2 / d + eps)
//
// The sums of squares, their roots and what is multiplied by them are held in
// 64 bits: an MXFP4 code is decided by a value that 1 / rms scales, and the one
// rounding to fp32 is then that of the definition whatever the order of the
// sum.  The int4 codes need no rms at all: they are those of u, exact in fp32, as
// in the prologue without a residual.
//
// One work-group per row, which stays in registers from the load to the
// codes: x and r are read once, h, the codes and the scales written once.  Bound by
// memory where there are rows enough (11264 of 4096, MXFP4 with its values, 394 MB
// in 69 us = 5.7 TB/s; 60 us again and again on the same rows).  693 rows of 5120,
// normalized before and after, int4 with its values, 11.4 us: a wavefront's 1006 vector
// instructions take about half of it on SIMDs that have three, its loads and two sums over
// the row the rest.  One row of 4096 2.7 us.
#include "mx4_device.h"
#include "p4q_internal.h"
#include "q4_device.h"

namespace p4q {
namespace {

// v of lane ^ M, M < 16 (wave_ops.h)
template <int M>
__device__ __forceinline__ double lane_xor_f64(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)lane_xor<M>((uint32_t)u) | (uint64_t)lane_xor<M>((uint32_t)(u >> 32)) << 32);
}

__device__ __forceinline__ double lane_read_f64(double v, int lane) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)lo | (uint64_t)hi << 32);
}

// Sum over a work-group of WAVES wavefronts, in a fixed order.
template <int WAVES>
__device__ __forceinline__ double block_sum(double s, double *buf) {
    s += lane_xor_f64<1>(s);
    s += lane_xor_f64<2>(s);
    s += lane_xor_f64<4>(s);
    s += lane_xor_f64<8>(s);
    s = (lane_read_f64(s, 0) + lane_read_f64(s, 16)) + (lane_read_f64(s, 32) + lane_read_f64(s, 48));
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = s;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) t += buf[i];
    return t;
}

// 1 / rms of a row; a row of zeros at eps = 0 stays one of zeros.  The hardware's
// estimate (at least 22 bits) and one step of third order, within a few units of
// 2^-53: a twentieth of the instructions of a root and a division.
__device__ __forceinline__ double inverse_rms(double ss, int d, float eps) {
    const double ms = ss * (1.0 / (double)d) + (double)eps;
    double y = __builtin_amdgcn_rsq(ms);
    if (y > 0.0) {                                         // neither infinite nor a NaN
        const double e = __builtin_fma(-ms * y, y, 1.0);
        y = __builtin_fma(y * e, __builtin_fma(0.375, e, 0.5), y);
    }
    return ms == 0.0 ? 0.0 : y;
}

// 16 bytes, as one access (uint4 goes as four where a condition is about it)
__device__ __forceinline__ uint4 load16(const uint16_t *p, int q) {
    const u32x4 v = reinterpret_cast<const u32x4 *>(p)[q];
    return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void store16(uint16_t *p, int q, uint4 v) {
    reinterpret_cast<u32x4 *>(p)[q] = u32x4{v.x, v.y, v.z, v.w};
}

template <bool BF16>
__device__ __forceinline__ void unpack8(uint4 w, float (&v)[8]) {
    const uint32_t xw[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = lo_f32<BF16>(xw[i]);
        v[2 * i + 1] = hi_f32<BF16>(xw[i]);
    }
}

template <int NT, int CH, bool BF16, bool INT4, bool CLIP1>
__global__ __launch_bounds__(NT) void k_residual_rmsnorm_quant(const ResidualNorm a) {
    constexpr int WAVES = NT / 64;
    __shared__ double s_r[WAVES], s_h[WAVES];
    __shared__ uint32_t s_max[WAVES];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    const int chunks = a.d / 8;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    auto row_of = [&](const uint16_t *p, int64_t ld) { return reinterpret_cast<const uint4 *>(p + row * ld); };

    uint4 h[CH], r[CH], g[CH], pg[CH], gt[CH];
    // (lanes past the row's end load its first 16 bytes, and hold zeros for them)
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int q = t + NT * c < chunks ? t + NT * c : 0;
        h[c] = load_nt(row_of(a.x, a.ldx) + q);
        g[c] = load16(a.gamma, q);
        if (a.r) r[c] = load_nt(row_of(a.r, a.ldr) + q);
        if (a.post) pg[c] = load16(a.post, q);
        if (a.gate) gt[c] = load16(a.gate, q);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
        if (t + NT * c >= chunks) h[c] = r[c] = zero;
    if (a.r) {
        double inv = 0.0;
        if (a.post) {
            double ss = 0.0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float v[8];
                unpack8<BF16>(r[c], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)v[i], (double)v[i], ss);
            }
            ss = block_sum<WAVES>(ss, s_r);
            inv = inverse_rms(ss, a.d, a.eps);
        }
        const double f = a.post ? inv * (double)a.alpha : (double)a.alpha;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int q = t + NT * c;
            float x[8], v[8], p[8], e[8], o[8];
            unpack8<BF16>(h[c], x);
            unpack8<BF16>(r[c], v);
            if (a.post) unpack8<BF16>(pg[c], p);
            if (a.gate) unpack8<BF16>(gt[c], e);
            if (!a.post && (!BF16 || !a.gate)) {
                // r, or the product of two fp16 numbers, is exact in fp32 and the fma
                // rounds once
                if (a.gate) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= e[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = __builtin_fmaf(a.alpha, v[i], x[i]);
            } else if constexpr (BF16) {
                // (products of two bfloat16 numbers may leave the range of fp32)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    double w = a.post ? (double)p[i] : 1.0;
                    if (a.gate) w *= (double)e[i];
                    o[i] = (float)__builtin_fma((double)v[i] * f, w, (double)x[i]);
                }
            } else {
                if (a.gate) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) p[i] *= e[i];          // exact
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = (float)__builtin_fma((double)v[i] * f, (double)p[i], (double)x[i]);
            }
            h[c] = round16x8<BF16>(o);
            if (q < chunks) store16(a.h_out + row * a.ldh, q, h[c]);
            else h[c] = zero;                              // (0 times an infinity of post or gate is a NaN)
        }
    }

    double ss = 0.0;
    float am = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        float v[8], w[8];
        unpack8<BF16>(h[c], v);
        if constexpr (INT4) unpack8<BF16>(g[c], w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ss = __builtin_fma((double)v[i], (double)v[i], ss);
            if constexpr (INT4) am = __builtin_fmaxf(am, __builtin_fabsf(v[i] * w[i]));
        }
    }
    if constexpr (INT4) {
        const uint32_t mw = wave_max_u32(__float_as_uint(am));
        if ((t & 63) == 0) s_max[t >> 6] = mw;
    }
    ss = block_sum<WAVES>(ss, s_h);
    const double inv = inverse_rms(ss, a.d, a.eps);

    if constexpr (INT4) {
        uint32_t mw = s_max[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) mw = max(mw, s_max[i]);
        const float top = __uint_as_float(mw);
        const float s = row_scale<CLIP1>(top, a.clip);
        const float scale = s == 0.0f ? 0.0f : (float)((double)s * inv);
        if (t == 0) static_cast<float *>(a.scales)[row] = scale;
        const bool tiny = !(s >= kTinyScale);
        const float rs = tiny ? 0.0f : 1.0f / s;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int q = t + NT * c;
            float u[8], w8[8];
            unpack8<BF16>(h[c], u);
            unpack8<BF16>(g[c], w8);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = u[i] * w8[i];
            uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            uint32_t near = 0;
            if (s != 0.0f) {
                if (!tiny) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) w[k] = q4_fast<CLIP1>(u[k], rs, near);
                }
                if (tiny || __any((int)near)) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float uk = u[k];
                        asm volatile("" : "+v"(uk));
                        w[k] = q4_exact(uk, s);
                    }
                }
            }
            const uint32_t packed = pack_nibbles(w);
            if (q < chunks) {
                reinterpret_cast<uint32_t *>(a.codes)[row * chunks + q] = packed;
                if (a.values) {
                    // (in fp32 first, as the products' epilogue takes them)
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = (float)((int)(packed << (28 - 4 * k)) >> 28) * scale;
                    store16(a.values + row * a.ldv, q, round16x8<BF16>(v));
                }
            }
        }
    } else {
        uint8_t *scales = static_cast<uint8_t *>(a.scales) + row * a.scale_stride;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int q = t + NT * c;
            float u[8], w8[8];
            unpack8<BF16>(h[c], u);
            unpack8<BF16>(g[c], w8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double z = BF16 ? (double)u[i] * (double)w8[i] : (double)(u[i] * w8[i]);
                u[i] = (float)(z * inv);
            }
            uint32_t byte;
            const uint32_t packed = mx4_quantize(u, byte);
            if (q < chunks) {
                if ((t & 3) == 0) scales[q >> 2] = (uint8_t)byte;
                reinterpret_cast<uint32_t *>(a.codes)[row * chunks + q] = packed;
                if (a.values) {
                    mx4_values(packed, byte, u);
                    store16(a.values + row * a.ldv, q, round16x8<BF16>(u));
                }
            }
        }
        const int pad = a.d / 32 + t;                    // the row's padding
        if (pad < (int)a.scale_stride) scales[pad] = 0;
    }
}

template <int NT, int CH, bool BF16>
hipError_t launch_ch(p4q_norm_format fmt, const ResidualNorm &a, hipStream_t stream) {
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(a.M), dim3(NT), 0, stream, a);
        return hipGetLastError();
    };
    if (fmt == P4Q_NORM_MX4) return go(k_residual_rmsnorm_quant<NT, CH, BF16, false, true>);
    return a.clip == 1.0f ? go(k_residual_rmsnorm_quant<NT, CH, BF16, true, true>)
                          : go(k_residual_rmsnorm_quant<NT, CH, BF16, true, false>);
}

// 256 threads a row; where there is at most one row for each CU its latency counts,
// and it gets a thread per 16 bytes, or per 32 (one row of 4096 2.75 against 2.9 us, 256
// rows 3.6 against 3.8; 512 rows of 5120 7.3 against 6.25, 693 normalized before and after
// 14.8 against 11.8).
template <bool BF16>
hipError_t launch_typed(p4q_norm_format fmt, const ResidualNorm &a, hipStream_t stream) {
    const int chunks = a.d / 8;                            // at most 2048
    if (chunks > 256 && a.M <= device_cus()) {
        if (chunks <= 512) return launch_ch<512, 1, BF16>(fmt, a, stream);
        if (chunks <= 1024) return launch_ch<1024, 1, BF16>(fmt, a, stream);
        return launch_ch<1024, 2, BF16>(fmt, a, stream);
    }
    const int per = (chunks + 255) / 256;
    if (per <= 1) return launch_ch<256, 1, BF16>(fmt, a, stream);
    if (per <= 2) return launch_ch<256, 2, BF16>(fmt, a, stream);
    if (per <= 3) return launch_ch<256, 3, BF16>(fmt, a, stream);
    if (per <= 4) return launch_ch<256, 4, BF16>(fmt, a, stream);
    if (per <= 6) return launch_ch<256, 6, BF16>(fmt, a, stream);
    return launch_ch<256, 8, BF16>(fmt, a, stream);
}

}  // namespace

hipError_t launch_residual_rmsnorm_quant(p4q_dtype dt, p4q_norm_format fmt, ResidualNorm a, hipStream_t stream) {
    a.scale_stride = mx4_scale_stride(a.d);
    return dt == P4Q_BF16 ? launch_typed<true>(fmt, a, stream) : launch_typed<false>(fmt, a, stream);
}

}  // namespace p4q
