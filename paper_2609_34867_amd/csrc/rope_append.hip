// Rotary position embedding of q and k, and the append of k and v to the paged
// cache -- the step between a decoder layer's q|k|v linear and its attention.
//
// Per token t of sequence b (its i-th in the call), with s = cache_lens[b] + i the
// place it takes in the sequence and p = positions[t] (or s):
//     a_j = p theta_j,  theta_j = base^(-2 j / D),  j < D / 2
//     y[j] = x[j] cos a_j - x[j + D/2] sin a_j,  y[j + D/2] = x[j + D/2] cos a_j + x[j] sin a_j
// for every query and key head; the rotated k and v as they are go to row s % P
// of page table[b][s / P].
//
// One wavefront takes a token and a share of its heads.  Angles: lane j makes
// that of pair j once per token.  p theta_j is formed in 64 bits and reduced to a
// fraction of a turn there (in 32 bits an angle of 10^5 rad would be off by 4 10^-3), sine
// and cosine of the fraction in 32.  They pass through LDS to the lanes that need
// them: lane l takes pairs 8 (l % (D/16)) .. + 7 of every head it touches, so it
// reads its 8 sines and cosines once and keeps them in registers.  A step of a
// wavefront covers 1024 / D heads with two 16-byte loads and stores per lane.
// Products and sums are fp32 (one fma), each result rounded once to 16 bits.
// What bounds it: bytes for prompts (16 of 656 to 704 tokens, 32 heads, 10927 in all: 120 us,
// 5.2 TB/s, a plain copy reaches 4.7), the chain of dependent loads (lengths, table, page) for a
// decode step (3.3 us of kernel).
#include "attention_device.h"
#include "gemm_device.h"
#include "kv_cache.h"
#include "p4q_internal.h"

#include <algorithm>
#include <type_traits>

namespace p4q {
namespace {

constexpr int kWaves = 4;               // wavefronts per work-group

template <bool BF16, int D, bool STREAM>
__global__ __launch_bounds__(64 * kWaves) void k_rope_append(RopeAppend a) {
    constexpr int kChunks = D / 16;                 // lanes per head: 8 + 8 values each
    constexpr int kHeads = 64 / kChunks;            // heads per step
    __shared__ float2 s_turn[kWaves][D / 2];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t unit = blockIdx.x * kWaves + wave;
    const int t = (int)(unit / (uint32_t)a.parts), part = (int)(unit - (uint32_t)t * (uint32_t)a.parts);
    if (t >= a.T) return;                           // whole wavefronts; no barrier follows

    // sequence of the token: how many end at or before it
    int b = 0;
    for (int i = 0; i < a.B; i += 64) {
        const int end = i + lane < a.B ? a.cu[i + lane + 1] : 0x7FFFFFFF;
        b += __popcll(__ballot(end <= t));
    }
    if (b >= a.B) return;                           // behind the last sequence: left as it was
    const int first = a.cu[b];
    if (t < first) return;                          // before the first one, or a list that does not ascend
    const int64_t place = (int64_t)(a.cache_lens ? a.cache_lens[b] : 0) + (t - first);
    const int col = page_column(place, a.shift, a.max_pages);
    const int page = col == kNoPage ? kNoPage : valid_page(a.table[(int64_t)b * a.max_pages + col], a.num_pages);
    const double p = a.positions ? (double)a.positions[t] : (double)place;

    const int c = lane & (kChunks - 1), hl = lane / kChunks;
    if (lane < D / 2) {
        const double turns = p * exp2((double)lane * a.log2_ratio) * 0.15915494309189533577;   // 1 / (2 pi)
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        s_turn[wave][lane] = make_float2(cs, sn);
    }
    // the wavefront's own LDS writes, read back by its other lanes
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 w = s_turn[wave][8 * c + j];
        cs[j] = w.x;
        sn[j] = w.y;
    }

    auto load16 = [](const uint16_t *p) __attribute__((always_inline)) {
        // (a head of 64 values lies on one 128-byte line, which both halves read)
        if constexpr (STREAM && D == 128) return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const v4i *>(p)));
        else return *reinterpret_cast<const uint4 *>(p);
    };
    auto store16 = [](uint16_t *p, uint4 x) __attribute__((always_inline)) {
        if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(v4i, x), reinterpret_cast<v4i *>(p));
        else *reinterpret_cast<uint4 *>(p) = x;
    };
    const int heads = a.Hq + 2 * a.Hk;
    const int64_t crow = page == kNoPage ? 0 : page_row(page, a.Hk, 0, a.shift, (int)(place & ((1 << a.shift) - 1)), D);
    const int64_t cstep = (int64_t)D << a.shift;    // from head to head on a page
    for (int h = part * kHeads + hl; h < heads; h += a.parts * kHeads) {
        const uint16_t *src = h < a.Hq ? a.q + (int64_t)t * a.ldq + (int64_t)h * D
                              : h < a.Hq + a.Hk ? a.k + (int64_t)t * a.ldk + (int64_t)(h - a.Hq) * D
                                                : a.v + (int64_t)t * a.ldv + (int64_t)(h - a.Hq - a.Hk) * D;
        const uint4 lo = load16(src + 8 * c), hi = load16(src + 8 * c + D / 2);
        const uint32_t x[4] = {lo.x, lo.y, lo.z, lo.w}, y[4] = {hi.x, hi.y, hi.z, hi.w};
        uint32_t r[4], w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const v2f xf = unpack2<BF16>(x[j]), yf = unpack2<BF16>(y[j]);
            r[j] = pack2<BF16>(__builtin_fmaf(xf[0], cs[2 * j], -(yf[0] * sn[2 * j])),
                               __builtin_fmaf(xf[1], cs[2 * j + 1], -(yf[1] * sn[2 * j + 1])));
            w[j] = pack2<BF16>(__builtin_fmaf(yf[0], cs[2 * j], xf[0] * sn[2 * j]),
                               __builtin_fmaf(yf[1], cs[2 * j + 1], xf[1] * sn[2 * j + 1]));
        }
        const bool is_v = h >= a.Hq + a.Hk;                 // goes through as it is, NaN and all
        const uint4 first8 = is_v ? lo : make_uint4(r[0], r[1], r[2], r[3]);
        const uint4 second8 = is_v ? hi : make_uint4(w[0], w[1], w[2], w[3]);
        auto put = [&](uint16_t *dst) __attribute__((always_inline)) {
            store16(dst + 8 * c, first8);
            store16(dst + 8 * c + D / 2, second8);
        };
        if (h < a.Hq) {
            put(a.q_out + (int64_t)t * a.ldqo + (int64_t)h * D);
        } else {
            const int hk = is_v ? h - a.Hq - a.Hk : h - a.Hq;
            if (!is_v && a.k_out) put(a.k_out + (int64_t)t * a.ldko + (int64_t)hk * D);
            if (page != kNoPage) put((is_v ? a.v_cache : a.k_cache) + crow + hk * cstep);
        }
    }
}

}  // namespace

hipError_t launch_rope_append(p4q_dtype dt, int D, RopeAppend a, float rope_base, hipStream_t stream) {
    const int steps = (a.Hq + 2 * a.Hk + 1024 / D - 1) / (1024 / D);
    // a token's heads are shared among wavefronts while there are few tokens
    // (below four wavefronts per SIMD of the device)
    const int64_t want = (int64_t)device_cus() * 16;
    a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(steps, want / a.T));
    a.log2_ratio = -2.0 / D * __builtin_log2((double)rope_base);
    const int64_t blocks = ((int64_t)a.T * a.parts + kWaves - 1) / kWaves;
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(64 * kWaves), 0, stream, a);
        return hipGetLastError();
    };
    // More than the last-level cache (256 MB) can hand on to the attention that follows
    // is written past it.  Prompts of 704 tokens, 32 heads, with k_out, us past the cache and
    // through it, alone and (in brackets) with attention_packed behind:
    //   D = 128: 1 (23 MB written) 10.9, 10.1 (31.0, 28.0); 4 (92 MB) 32, 37 (72, 71); 8 (185 MB)
    //   63, 71 (131, 131); 16 (369 MB) 123, 131 (249, 244); 32 (738 MB) 244, 254 (478, 473)
    //   D = 64: 4 (46 MB) 18.4, 15.9 (47.4, 43.9); 8 (92 MB) 34, 45 (81, 81); 16 (185 MB) 72, 78
    //   (142, 143); 32 (369 MB) 137, 146 (266, 269)
    // Above the line the append alone is 4 to 11% faster past the cache and both calls are
    // within 2% either way; far below it the attention then pays for the reads.
    const bool stream_out = (int64_t)a.T * (a.Hq + (a.k_out ? 3 : 2) * a.Hk) * D * 2 > (int64_t)128 << 20;
    auto d = [&](auto bf, auto st) {
        return D == 128 ? go(k_rope_append<decltype(bf)::value, 128, decltype(st)::value>)
                        : go(k_rope_append<decltype(bf)::value, 64, decltype(st)::value>);
    };
    auto t = [&](auto bf) { return stream_out ? d(bf, std::true_type{}) : d(bf, std::false_type{}); };
    return dt == P4Q_BF16 ? t(std::true_type{}) : t(std::false_type{});
}

}  // namespace p4q
