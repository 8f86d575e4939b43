// MXFP4 quantization of rows (mx4_device.h has the format).
//
// A wavefront takes 512 consecutive values of a row at a time: a lane 8 of
// them (16 bytes), a quad of lanes one block of 32, the wavefront the 16
// scale bytes that a row's padding comes in.  Behind the row's end the lanes
// hold zeros, whose scale byte is the padding's 0.  One pass over memory: 2
// bytes of a value read, 17/32 written, and 2 more where the fake-quantized
// values are asked for (a lane's own 16 bytes, so they may replace x).  Bound by
// it: 11264 rows of 4096 with their values, 209 MB in 33.5 us = 6.2 TB/s; 4 rows
// of 5120 2.6 us.
#include "mx4_device.h"
#include "p4q_internal.h"
#include "q4_device.h"

#include <algorithm>

namespace p4q {
namespace {

constexpr int kThreads = 256;

template <bool BF16>
__global__ __launch_bounds__(kThreads) void k_quant_mx4(const uint8_t *x, int64_t ldx_bytes,
                                                        int64_t items, int groups, int chunks,
                                                        uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                        uint8_t *values, int64_t ldv_bytes) {
    const int lane = threadIdx.x & 63;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t item = block * (kThreads / 64) + (threadIdx.x >> 6);
    if (item >= items) return;
    const int64_t row = item / groups;
    const int q = (int)(item - row * groups) * 64 + lane;
    const bool in = q < chunks;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (in) w = load_nt(reinterpret_cast<const uint4 *>(x + row * ldx_bytes) + q);
    const uint32_t xw[4] = {w.x, w.y, w.z, w.w};
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = lo_f32<BF16>(xw[i]);
        v[2 * i + 1] = hi_f32<BF16>(xw[i]);
    }
    uint32_t byte;
    const uint32_t c = mx4_quantize(v, byte);
    if ((lane & 3) == 0) scales[row * groups * 16 + (q >> 2)] = (uint8_t)byte;
    if (!in) return;
    reinterpret_cast<uint32_t *>(codes)[row * chunks + q] = c;
    if (values) {
        mx4_values(c, byte, v);
        reinterpret_cast<uint4 *>(values + row * ldv_bytes)[q] = round16x8<BF16>(v);
    }
}

}  // namespace

hipError_t launch_quant_mx4(p4q_dtype dt, int M, int K, const void *x, int64_t ldx, uint8_t *codes,
                            uint8_t *scales, void *values, int64_t ldv, hipStream_t stream) {
    const int groups = (int)(mx4_scale_stride(K) / 16);
    const int64_t items = (int64_t)M * groups;
    // (a dimension of a grid holds less than 2^32 threads)
    const unsigned blocks = (unsigned)((items + kThreads / 64 - 1) / (kThreads / 64)), most = 1u << 23;
    const dim3 grid(std::min(blocks, most), (blocks + most - 1) / most);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, stream, static_cast<const uint8_t *>(x), ldx * 2, items, groups,
                           K / 8, codes, scales, static_cast<uint8_t *>(values), ldv * 2);
        return hipGetLastError();
    };
    return dt == P4Q_BF16 ? go(k_quant_mx4<true>) : go(k_quant_mx4<false>);
}

}  // namespace p4q
