// Products of MXFP4 rows (mx4_device.h has the format): y = a w^T, and the
// gated pair SiLU(a w_gate^T) * (a w_up^T) of a feed-forward block.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 multiplies E2M1 numbers and applies both
// operands' scale bytes itself: lane l holds 32 consecutive codes of row
// l % 32 and the scale byte of that block.  The contraction does not care
// which 32 of a row's values meet in which instruction, as long as both
// operands agree; so with 256 values of k a stage, lane l takes the four
// blocks 4 (l / 32) .. + 3 one after the other, whose scale bytes are one
// aligned word.
//
// The weight is the first operand, so a lane of the result holds one row of a
// and runs of 4 consecutive outputs of it: the gate's and the up projection's
// sums of an output meet in one lane, and two lanes hold a block of 32 outputs
// to quantize.
#include "gemm_device.h"
#include "mx4_choice.h"
#include "mx4_device.h"
#include "p4q_internal.h"

#include <algorithm>
#include <type_traits>
#include <utility>

namespace p4q {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

// acc += w a^T over 64 values of k (block I of each lane's four); sw, sa: the
// words of scale bytes
template <int I>
__device__ __forceinline__ void mfma_mx4(v4i w, uint32_t sw, v4i a, uint32_t sa, v16f &acc) {
    const v8i W = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, acc, 4, 4, I, (int)sw, I, (int)sa);
}

// the same over 128 values, 16 x 16
template <int I>
__device__ __forceinline__ void mfma_mx4_16(v4i w, uint32_t sw, v4i a, uint32_t sa, v4f &acc) {
    const v8i W = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(W, A, acc, 4, 4, I, (int)sw, I, (int)sa);
}

// v = SiLU(v) u of N sums, v / (1 + 2^t) u with t = -v log2 e, by the hardware's exp2 and
// reciprocal: one unit in the last place each where the reciprocal is a normal number, but
// a subnormal one comes as 0, and u may bring the product back into range.  So below -87
// u takes what SiLU(v) is of SiLU(-87), v / -87 2^(t(-87) - t), the power as a square since
// it may pass the range before u does.  (u is used up.)  Whether any v is that low: as
// whole numbers, the bits of negative ones rise with their magnitude and lie above those of
// all others.
template <int N>
__device__ __forceinline__ void silu_mul(float (&v)[N], float (&u)[N]) {
    constexpr float kLog2e = 1.44269504088896341f;
    constexpr uint32_t kFar = 0xC2AE0000u;                 // -87
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(v[i]));
    if (__builtin_expect(top > kFar, 0)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (__float_as_uint(v[i]) <= kFar) continue;
            const float root = __builtin_amdgcn_exp2f(0.5f * __builtin_fmaf(kLog2e, v[i], 87.0f * kLog2e));
            // (v of minus infinity: times 0, a NaN as its quotient)
            u[i] = u[i] * root * root * (v[i] * (-1.0f / 87.0f));
            v[i] = -87.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = v[i] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v[i])) * u[i];
}

// 8 consecutive 16-bit outputs n0 .. n0 + 7 of row m, as far as they exist
__device__ __forceinline__ void store8(const Mx4Product &p, int64_t m, int n0, uint4 w) {
    if (m >= p.M || n0 >= p.N) return;
    uint16_t *dst = static_cast<uint16_t *>(p.y) + m * p.ldy + n0;
    if (n0 + 8 <= p.N) {
        __builtin_memcpy(dst, &w, 16);                     // one store, whatever the row's alignment
    } else {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n0 + i < p.N) dst[i] = (uint16_t)(x[i >> 1] >> (16 * (i & 1)));
    }
}

// 8 consecutive outputs n0 .. n0 + 7 of row m (u: the up sums, gated only).
// Four lanes of a quad hold 32 outputs of one row in order.
template <int EPI, bool BF16>
__device__ __forceinline__ void emit8(const Mx4Product &p, int64_t m, int n0, float (&v)[8], float (&u)[8]) {
    if constexpr (EPI != kLinear) silu_mul(v, u);
    if constexpr (EPI == kGatedQuant) {
        uint32_t byte;
        const uint32_t c = mx4_quantize(v, byte);
        if (m < p.M && n0 < p.N) {
            reinterpret_cast<uint32_t *>(p.codes)[(m * p.N + n0) >> 3] = c;
            if ((n0 & 31) == 0) p.scales[m * p.out_stride + (n0 >> 5)] = (uint8_t)byte;
        }
    } else {
        store8(p, m, n0, round16x8<BF16>(v));
    }
}

// ---- tiles through LDS -----------------------------------------------------------
// A work-group of four wavefronts, 2 x 2, computes 64 FM rows by 64 FN weight
// rows, each wavefront FM x FN fragments of 32 x 32.  k runs in stages of 256
// values, four steps each; a ring of RING stages in LDS is filled by DMA and runs
// on across the tiles of a persistent work-group.
//  * A stage's row is 128 bytes, one cache line, loaded by 8 lanes: rows of half a
//    line (stages of 128 values, ring of 4) took 638 us where these took 513 (gate
//    and up of 7B, 11264 rows, before the next points).  Chunk c of 16 bytes (32
//    codes) of row r lies at c ^ (r / 2 % 8), so that 16 rows of a fragment read fall
//    into distinct banks.
//  * Scale bytes come 16 per row, for two stages at once (8 for one: 1024 instead
//    of 768 lines a stage): the rows of a with the odd stage before, those of w
//    with the even one.  An odd number of stages is padded with one that
//    multiplies nothing.  (32 for four stages need the room that the outputs are
//    staged in; stored from registers they took 243 us instead of 234 then, 7B
//    down projection, 11264 rows.)
//  * Operands are read ahead of their step: during steps 2 and 3 those of the next
//    stage's steps 0 to 2, during step 0 those of step 3.  So a slot is read in
//    three steps and has five for its next stage to arrive, whose DMAs are spread
//    over the products of steps 1 to 3 (over four steps, with less time to arrive,
//    2% slower).
//  * KS = 2: two parts of the work-group, of four wavefronts and a ring each, take a
//    half of k each for the same tile, one tile per work-group, and add their sums in
//    LDS.  For long rows and fewer tiles than CUs, where one wavefront per SIMD waits
//    for its barriers and reads, 128 x 5120 x 13824 by 64 x 64 24.7 -> 20.6 us, 292 x
//    5120 x 13824 by 64 x 128 30.3 -> 26.1 (four parts no faster: 20.4).
//  * Past the row's end the DMA's offsets lie outside the buffer and give codes
//    of zero, and the scale bytes there are masked; rows past the last are outside
//    it too.
// Measured, M x N x K = 11264 x 4096 x 11008: 230 us = 4.4 PFLOP/s; gate and up,
// 11264 x 2 * 11008 x 4096: 495 us = 4.1 PFLOP/s.  Of the 230 us (237 when these were
// taken) the products alone take 154, with their reads 177, and the DMA alone 133.  Much
// of the rest is the power limit: the matrix units are busy in 55% of the cycles, at 1.83
// GHz of 2.4, and alone on random codes they reach 6.6 PFLOP/s, on zeros 9.9.
// The sums of a fragment out of the accumulation registers, here and not earlier (left
// to itself the compiler reads them all before the first pass and spills).  It knows
// no hazard of these reads: the caller keeps the distance to the last product.
__device__ __forceinline__ void read_sums(const v16f &acc, float (&v)[16]) {
#pragma unroll
    for (int x = 0; x < 16; ++x) {
        const float a = acc[x];
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[x]) : "a"(a));
    }
}

template <class F, int... I>
__device__ __forceinline__ void unrolled_seq(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
// f(0) .. f(N - 1), the arguments compile-time constants
template <int N, class F>
__device__ __forceinline__ void unrolled(F &&f) {
    unrolled_seq(f, std::make_integer_sequence<int, N>{});
}

// A tile whose k is shared by KS parts of a work-group: the sums of its parts, added in
// LDS in their order, and its outputs
template <bool BF16, int FM, int FN, int KS>
__device__ __forceinline__ void add_parts(const Mx4Product &p, uint8_t *smem, int wave, int lane,
                                          const v16f (&acc)[FN][FM], int64_t m0, int n0) {
    constexpr int X = FM * FN;
    float4 *red = reinterpret_cast<float4 *>(smem);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no DMA into LDS from here on
    __syncthreads();
    // [part][wavefront][fragment][registers 4 g ..][lane], lanes exchanged so that the
    // threads of a quad below read from different banks
    unrolled<X>([&](auto x_c) __attribute__((always_inline)) {
        constexpr int x = decltype(x_c)::value, f = x / FM, j = x % FM;
        float v[16];
        read_sums(acc[f][j], v);
#pragma unroll
        for (int g = 0; g < 4; ++g)
            red[((wave * X + x) * 4 + g) * 64 + (lane ^ (4 * g))] = make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
    });
    __syncthreads();
    // a quad of threads has 32 outputs of a row, 8 each
    for (int t = (int)threadIdx.x; t < 64 * FM * 2 * FN * 4; t += 256 * KS) {
        const int g = t & 3, row = (t >> 2) % (64 * FM), q = (t >> 2) / (64 * FM);
        const int wn = q / FN, f = q % FN, wm = row / (32 * FM), j = row / 32 % FM, r = row & 31;
        float v[8] = {};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const float4 s = red[(((k * 4 + wn * 2 + wm) * X + f * FM + j) * 4 + g) * 64 + ((r + 32 * hh) ^ (4 * g))];
                v[4 * hh + 0] += s.x;
                v[4 * hh + 1] += s.y;
                v[4 * hh + 2] += s.z;
                v[4 * hh + 3] += s.w;
            }
        store8(p, m0 + row, n0 + 32 * q + 8 * g, round16x8<BF16>(v));
    }
}

// What lanes of the wavefront stored to LDS before, its others read behind.  No instruction:
// a wavefront's accesses of LDS keep their order, the compiler has to as well.
__device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

constexpr int kRowBytes = 128;                   // codes of a row in a stage
constexpr int kRowScales = 16;                   // scale bytes of a row, two stages'

template <int EPI, bool BF16, int FM, int FN, int RING, int KS = 1>
__global__ __launch_bounds__(256 * KS, FM * FN > 4 || RING > 2 || KS > 1 ? 1 : 2) void k_mx4_tile(const Mx4Product p, int tiles_m, int tiles_n) {
    constexpr int BM = 64 * FM, BW = 64 * FN;              // rows of a, of w
    constexpr int BN = EPI == kLinear ? BW : BW / 2;       // outputs: half of w's rows are the gate's
    constexpr int FO = EPI == kLinear ? FN : FN / 2;       // fragments of outputs per wavefront
    constexpr int OFF_W = BM * kRowBytes, STAGE = OFF_W + BW * kRowBytes;
    constexpr int OFF_SCALES = RING * STAGE, OFF_SW = BM * kRowScales, SCALES = OFF_SW + BW * kRowScales;
    constexpr int S_RING = RING / 2 + 1, OFF_OUT = OFF_SCALES + S_RING * SCALES;
    // fragments stored together: two, a line of a row, where there is room (192 x 256 tiles, 2881 x 12288 x
    // 4096: 86.7 -> 81.3 us)
    constexpr int EW = FO % 2 == 0 && (FM * FN >= 12 || FM == 1) ? 2 : 1;
    constexpr int OUT_ROW = 64 * EW, OUT_WAVE = EPI == kGatedQuant || KS > 1 ? 0 : 32 * OUT_ROW;
    constexpr int CODE_DMAS = 2 * (FM + FN), DMAS = CODE_DMAS + 1;
    static_assert(EPI == kLinear || FN % 2 == 0, "gate and up fragments");
    static_assert(RING % 2 == 0, "scales of two stages");
    static_assert(FM <= 4 && FN <= 4, "a wavefront's share of the scales is one load");
    static_assert(KS == 1 || (EPI == kLinear && FM * FN * 16384 <= OFF_OUT), "the parts' sums lie where their stages did");
    __shared__ __attribute__((aligned(1024))) uint8_t smem_all[KS * OFF_OUT + 4 * OUT_WAVE];

    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    const int wave_all = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wave = wave_all & 3, part = KS > 1 ? wave_all >> 2 : 0;
    const int wm = wave & 1, wn = wave >> 1;
    uint8_t *smem = smem_all + part * OFF_OUT;
    const int blocks = p.K / 32;
    // this part's stages: KT of them, from the one at k0; an even number, so that scale bytes start 16 bytes apart
    const int KT_all = (blocks + 7) / 8, KT2 = ((KT_all + KS - 1) / KS + 1) & ~1;
    const int KT = KS > 1 ? KT2 : KT_all, k0 = part * KT2;
    const uint32_t kb = (uint32_t)p.K / 2, sb = (uint32_t)p.in_stride;

    // this work-group's tiles: a contiguous share of its XCD's range
    const int T = tiles_m * tiles_n;
    const int xcd = blockIdx.x % kXcds, i0 = blockIdx.x / kXcds;
    const int nb = ((int)gridDim.x - xcd + kXcds - 1) / kXcds;
    const int q = T / kXcds, rr = T % kXcds;
    const int start = (xcd < rr) ? xcd * (q + 1) : rr * (q + 1) + (xcd - rr) * q;
    const int len = q + (xcd < rr ? 1 : 0);
    const int nt = (i0 < len) ? (len - i0 + nb - 1) / nb : 0;
    if (nt == 0) return;                                   // block-uniform
    auto tile_at = [&](int k, int &tm, int &tn) __attribute__((always_inline)) {
        grouped_tile(start + i0 + k * nb, tiles_m, tiles_n, tm, tn);
    };

    // ---- DMA.  A stage is issue_begin(), then issue(i) for i < DMAS: its codes and
    // a quarter per wavefront of the scales of w (even stages, for themselves and the
    // next) or of a (odd ones, for the two stages behind them).  Buffers of the tile
    // of the codes; those of a's scales are a stage ahead.
    const uint32_t lds = lds_addr(smem);
    const uint32_t c_row = (uint32_t)lane >> 3;
    const uint32_t c_chunk[2] = {((uint32_t)lane & 7u) ^ (c_row >> 1), ((uint32_t)lane & 7u) ^ (c_row >> 1) ^ 4u};
    constexpr uint32_t kOutside = 0x80000000u;
    int iss_tile = -1, iss_kt = KT2 - 1, iss_slot = RING - 1, sc_tile = -1, sc_kt = KT2 - 2, sc_slot = S_RING - 1;
    v4i dA = {}, dW = {}, dSA = {}, dSW = {};
    uint32_t iss_v[2] = {}, iss_lds = 0;
    auto rows_of = [](int64_t total, int64_t first, int most) __attribute__((always_inline)) {
        return (uint32_t)min(total - first, (int64_t)most);
    };
    // the place of the next two stages' scales of a
    auto scales_a = [&]() __attribute__((always_inline)) {
        sc_kt += 2;
        if (++sc_slot == S_RING) sc_slot = 0;
        if (sc_kt == KT2) {
            sc_kt = 0;
            ++sc_tile;
            int tm = 0, tn = 0;
            if (sc_tile < nt) tile_at(sc_tile, tm, tn);
            const int64_t m0 = (int64_t)tm * BM;
            dSA = buffer_desc(p.as + m0 * sb, sc_tile < nt ? rows_of(p.M, m0, BM) * sb : 0u);
        }
    };
    auto issue_begin = [&]() __attribute__((always_inline)) {
        if (++iss_kt == KT2) {
            iss_kt = 0;
            ++iss_tile;
            const bool live = iss_tile < nt;               // past the last tile: empty buffers
            int tm = 0, tn = 0;
            if (live) tile_at(iss_tile, tm, tn);
            const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
            // wavefronts 2 and 3 load the second half of w's rows: the up rows
            const int64_t w0 = n0 + (EPI != kLinear && wave >= 2 ? (int64_t)p.N : 0);
            const uint32_t rw = live ? rows_of(p.N, n0, BN) : 0u;
            dA = buffer_desc(p.a + m0 * kb, live ? rows_of(p.M, m0, BM) * kb : 0u);
            dW = buffer_desc(p.w + w0 * kb, rw * kb);
            dSW = buffer_desc(p.ws + w0 * sb, rw * sb);
        }
        if (iss_kt & 1) scales_a();
        iss_slot = (iss_slot + 1) % RING;
        iss_lds = lds + (uint32_t)iss_slot * STAGE;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t c = (uint32_t)(k0 + iss_kt) * 8u + c_chunk[x];
            iss_v[x] = c < (uint32_t)blocks ? c_row * kb + c * 16u : kOutside;
        }
    };
    auto issue = [&](auto i_c) __attribute__((always_inline)) {
        constexpr int i = decltype(i_c)::value;
        if constexpr (i == 0) {
            const uint32_t base = lds + OFF_SCALES + (uint32_t)sc_slot * SCALES;
            if (iss_kt & 1) {
                const uint32_t row = (uint32_t)wave * 16 * FM;
                if (lane < 16 * FM)
                    dma16(dSA, (row + (uint32_t)lane) * sb + (uint32_t)(k0 + sc_kt) * 8u, base + row * kRowScales);
            } else {
                const uint32_t row = (uint32_t)wave * 16 * FN;
                const uint32_t from = EPI == kLinear ? row : (uint32_t)(wave & 1) * 16 * FN;
                if (lane < 16 * FN)
                    dma16(dSW, (from + (uint32_t)lane) * sb + (uint32_t)(k0 + iss_kt) * 8u, base + OFF_SW + row * kRowScales);
            }
        } else if constexpr (i <= 2 * FM) {                // 8 rows of a
            const uint32_t g = (uint32_t)(wave * 2 * FM + i - 1);
            dma16(dA, iss_v[(i - 1) & 1] + g * 8u * kb, iss_lds + g * 1024u);
        } else {                                           // 8 rows of w
            constexpr int j = i - 1 - 2 * FM;
            const uint32_t g = (uint32_t)(wave * 2 * FN + j);
            const uint32_t row = EPI == kLinear ? g : (uint32_t)((wave & 1) * 2 * FN + j);
            dma16(dW, iss_v[j & 1] + row * 8u * kb, iss_lds + OFF_W + g * 1024u);
        }
    };
    // Part x of the stage's DMAs, of `of` parts
    auto issue_part = [&](auto x_c, auto of_c) __attribute__((always_inline)) {
        constexpr int x = decltype(x_c)::value, of = decltype(of_c)::value;
        constexpr int lo = x * DMAS / of, hi = (x + 1) * DMAS / of;
        unrolled<hi - lo>([&](auto d_c) __attribute__((always_inline)) {
            issue(std::integral_constant<int, lo + decltype(d_c)::value>{});
        });
    };

    // ---- operands of a step
    // (gated: a wavefront's first fragments are the gate's, the others the up rows' of the same outputs)
    const int row_w = EPI == kLinear ? wn * 32 * FN : wn * 32 * FO;
    auto w_row = [&](int f) { return EPI == kLinear || f < FO ? 32 * f : BN + 32 * (f - FO); };
    uint32_t xo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) xo[i] = (uint32_t)(r * kRowBytes + (((4 * h + i) ^ ((r >> 1) & 7)) << 4));
    const uint32_t a_at = (uint32_t)(wm * 32 * FM * kRowBytes), w_at = (uint32_t)(OFF_W + row_w * kRowBytes);
    const uint32_t sa_at = (uint32_t)(OFF_SCALES + (wm * 32 * FM + r) * kRowScales + 4 * h);
    const uint32_t sw_at = (uint32_t)(OFF_SCALES + OFF_SW + (row_w + r) * kRowScales + 4 * h);
    v4i a[4][FM], w[4][FN];
    uint32_t ra[FM], rw[FN], sa[FM], sw[FN];
    constexpr int F = FM + FN;
    auto read_one = [&](uint32_t slot, auto i_c, auto k_c) __attribute__((always_inline)) {
        constexpr int i = decltype(i_c)::value, k = decltype(k_c)::value;
        const uint8_t *b = smem + slot * STAGE + xo[i];
        if constexpr (k < FM) a[i][k] = *reinterpret_cast<const v4i *>(b + a_at + 32 * kRowBytes * k);
        else w[i][k - FM] = *reinterpret_cast<const v4i *>(b + w_at + kRowBytes * w_row(k - FM));
    };
    auto read_scale = [&](uint32_t slot, uint32_t half, auto k_c) __attribute__((always_inline)) {
        constexpr int k = decltype(k_c)::value;
        const uint8_t *b = smem + slot * SCALES + half * 8;
        if constexpr (k < FM) ra[k] = *reinterpret_cast<const uint32_t *>(b + sa_at + 32 * kRowScales * k);
        else rw[k - FM] = *reinterpret_cast<const uint32_t *>(b + sw_at + kRowScales * w_row(k - FM));
    };
    typedef std::integral_constant<int, 0> c0;
    typedef std::integral_constant<int, 1> c1;
    typedef std::integral_constant<int, 2> c2;
    typedef std::integral_constant<int, 3> c3;

    // the first stage's scales of a, then what the stages before the first would have issued
    constexpr int X = FM * FN, PARTS = 3 * X, EARLY = X * DMAS / PARTS;
    scales_a();
    if (lane < 16 * FM) {
        const uint32_t row = (uint32_t)wave * 16 * FM;
        dma16(dSA, (row + (uint32_t)lane) * sb + (uint32_t)k0 * 8u, lds + OFF_SCALES + (uint32_t)sc_slot * SCALES + row * kRowScales);
    }
    unrolled<RING>([&](auto) __attribute__((always_inline)) {
        issue_begin();
        unrolled<DMAS>(issue);
    });
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((RING - 1) * DMAS) : "memory");
    uint32_t slot = 0, s_slot = 0;                         // of the stage that is read next
    unrolled<F>([&](auto k) __attribute__((always_inline)) { read_scale(0, 0, k); });
    unrolled<F>([&](auto k) __attribute__((always_inline)) { read_one(0, c0{}, k); });
    unrolled<F>([&](auto k) __attribute__((always_inline)) { read_one(0, c1{}, k); });
    unrolled<F>([&](auto k) __attribute__((always_inline)) { read_one(0, c2{}, k); });

    for (int ck = 0; ck < nt; ++ck) {
        v16f acc[FN][FM];
        // One stage: the first, whose sums begin, one between, or one that pads their
        // number to an even one
        auto stage = [&](int kt, auto kind_c) __attribute__((always_inline)) {
            constexpr bool FIRST = decltype(kind_c)::value == 0, LIVE = decltype(kind_c)::value < 2;
            const int left = blocks - 8 * (k0 + kt) - 4 * h;
            const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
            for (int j = 0; j < FM; ++j) sa[j] = ra[j] & mask;
#pragma unroll
            for (int f = 0; f < FN; ++f) sw[f] = rw[f] & mask;
            auto step = [&](auto i_c) __attribute__((always_inline)) {
                constexpr int i = decltype(i_c)::value;
                if constexpr (i == 1) {
                    // every wavefront holds this stage's operands: its slot is free
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                    issue_begin();
                }
                if constexpr (i == 2) {
                    // the next stage has landed (in order: the ring's others and what step 1 issued
                    // may be outstanding)
                    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((RING - 2) * DMAS + EARLY) : "memory");
                    slot = (slot + 1) % RING;
                    if ((kt & 1) && ++s_slot == S_RING) s_slot = 0;
                }
                __builtin_amdgcn_sched_barrier(0);
                unrolled<FM * FN>([&](auto x_c) __attribute__((always_inline)) {
                    constexpr int x = decltype(x_c)::value, f = x / FM, j = x % FM;
                    if constexpr (FIRST && i == 0) acc[f][j] = v16f{};
                    if constexpr (LIVE) mfma_mx4<i>(w[i][f], sw[f], a[i][j], sa[j], acc[f][j]);
                    // behind each product a share of the reads ahead and of the DMAs: a
                    // wavefront issues in order, and together they would hold up its products
                    if constexpr (i == 0) {
                        // (early, for step 1 waits for them)
                        constexpr int H = X >= 2 ? X / 2 : 1;
                        constexpr int lo = x < H ? x * F / H : F, hi = x < H ? (x + 1) * F / H : F;
                        unrolled<hi - lo>([&](auto k) __attribute__((always_inline)) {
                            read_one(slot, c3{}, std::integral_constant<int, lo + decltype(k)::value>{});
                        });
                    }
                    if constexpr (i >= 2) {
                        constexpr int lo = x * 2 * F / X, hi = (x + 1) * 2 * F / X;
                        unrolled<hi - lo>([&](auto k_c) __attribute__((always_inline)) {
                            constexpr int k = lo + decltype(k_c)::value;
                            typedef std::integral_constant<int, k % F> at;
                            if constexpr (i == 2 && k < F) read_one(slot, c0{}, at{});
                            else if constexpr (i == 2) read_scale(s_slot, (uint32_t)(kt + 1) & 1u, at{});
                            else read_one(slot, std::integral_constant<int, 1 + k / F>{}, at{});
                        });
                    }
                    if constexpr (i > 0)
                        issue_part(std::integral_constant<int, (i - 1) * X + x>{}, std::integral_constant<int, PARTS>{});
                    __builtin_amdgcn_sched_barrier(0);
                });
                __builtin_amdgcn_sched_barrier(0);
            };
            step(c0{});
            step(c1{});
            step(c2{});
            step(c3{});
        };
        stage(0, c0{});
        for (int kt = 1; kt < KT; ++kt) stage(kt, c1{});
        if (KT2 != KT) stage(KT, c2{});

        // ---- lane l holds row l % 32 of a fragment, outputs 8 g + 4 (l / 32) + 0..3 in
        // registers 4 g ..
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");   // the last products before the reads of their sums
        int tm, tn;
        tile_at(ck, tm, tn);
        if constexpr (KS > 1) {
            add_parts<BF16, FM, FN, KS>(p, smem_all, wave_all, lane, acc, (int64_t)tm * BM, tn * BN);
            break;
        }
        const int64_t m0 = (int64_t)tm * BM + wm * 32 * FM;
        const int n0 = tn * BN + wn * 32 * FO;
        const bool full = (int64_t)(tm + 1) * BM <= p.M && (int64_t)(tn + 1) * BN <= p.N;
        uint8_t *out = smem + OFF_OUT + wave * OUT_WAVE;
#pragma unroll
        for (int j = 0; j < FM; ++j) {
#pragma unroll
            for (int f0 = 0; f0 < FO; f0 += EW) {
                float v[EW][16];
#pragma unroll
                for (int e = 0; e < EW; ++e) {
                    read_sums(acc[f0 + e][j], v[e]);
                    if constexpr (EPI != kLinear) {
                        float u[16];
                        read_sums(acc[(f0 + e + FO) % FN][j], u);
                        silu_mul(v[e], u);
                    }
                }
                if constexpr (EPI == kGatedQuant) {
#pragma unroll
                    for (int e = 0; e < EW; ++e) {
                        uint32_t byte;
                        const uint2 c = mx4_quantize_halves(v[e], byte);
                        const int64_t m = m0 + 32 * j + r;
                        const int n = n0 + 32 * (f0 + e);
                        if (m < p.M && n < p.N) {
                            reinterpret_cast<uint2 *>(p.codes)[(m * p.N + n) / 16 + h] = c;
                            if (h == 0) p.scales[m * p.out_stride + n / 32] = (uint8_t)byte;
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < EW; ++e)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const float *o = v[e] + 4 * g;
                            const int chunk = (4 * e + g) ^ (r & (4 * EW - 1));
                            *reinterpret_cast<uint2 *>(out + r * OUT_ROW + chunk * 16 + 8 * h) =
                                make_uint2(round16x2<BF16>(o[0], o[1]), round16x2<BF16>(o[2], o[3]));
                        }
                    lanes_meet();
                    constexpr int LR = 4 * EW;             // lanes per row
#pragma unroll
                    for (int s = 0; s < 32 / (64 / LR); ++s) {
                        const int row = s * (64 / LR) + lane / LR, c = lane % LR;
                        const uint4 val = *reinterpret_cast<const uint4 *>(out + row * OUT_ROW + ((c ^ (row & (LR - 1))) << 4));
                        const int64_t m = m0 + 32 * j + row;
                        const int n = n0 + 32 * f0 + 8 * c;
                        // (rows at halves of lines go past the caches, which hold operands: 2% less time at
                        // 11264 rows, 18.6 -> 16.7 us at 2881 x 4128 x 1120; others would go in smaller
                        // parts: 178 us instead of 164 at 11264 x 5136 x 5120)
                        if (full && p.wide)
                            __builtin_nontemporal_store(v4i{(int)val.x, (int)val.y, (int)val.z, (int)val.w},
                                                        reinterpret_cast<v4i *>(static_cast<uint16_t *>(p.y) + m * p.ldy + n));
                        else store8(p, m, n, val);
                    }
                    lanes_meet();
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (EPI == kGatedQuant) {
            // the padding behind a row's last block
            const int64_t m = (int64_t)tm * BM + threadIdx.x;
            if (tn == tiles_n - 1 && (int)threadIdx.x < BM && m < p.M)
                for (int64_t i = p.N / 32; i < p.out_stride; ++i) p.scales[m * p.out_stride + i] = 0;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no DMA into LDS past the end
}

// ---- few rows: weights streamed past them ------------------------------------------
// A work-group computes 16 FO outputs of 16 MB rows.  Its wavefronts share k in
// contiguous runs of stages of 256 values and need nothing of each other until
// their sums meet in LDS, in a fixed order: each has a ring of two stages of its
// own, filled by DMA, and waits for it alone.
//  * A fragment is 16 rows; a stage's 128 bytes of a row lie as in the tiles above.
//    In a product of 128 values lane l takes the blocks 2 (l / 16) and, in the
//    second, 2 (l / 16) + 1 of row l % 16.
//  * Scale bytes come 32 per row, for four stages at once, into two buffers.
// Bound by memory: 13B down projection (N = 5120, K = 13824), 4 rows, 37.7 MB in 7.7
// us = 4.9 TB/s; 7B gate and up, 16 rows, 48.3 MB in 9.2 us = 5.3 TB/s (12.4 and 16
// with the operands straight from memory to registers: every fragment load touches
// 32 lines there, and each line four times).
constexpr int kRowsRing = 2, kRowsGroup = 4;

template <int EPI, bool BF16, int MB, int NW>
__global__ __launch_bounds__(64 * NW) void k_mx4_rows(const Mx4Product p) {
    constexpr int FO = EPI == kGatedQuant ? 2 : 1;         // fragments of outputs (32: a block to quantize)
    constexpr int F = EPI == kLinear ? FO : 2 * FO;        // of w: the gate's, then the up rows'
    constexpr int FRAG = 16 * kRowBytes, STAGE = (F + MB) * FRAG;
    constexpr int SC_ROW = 8 * kRowsGroup, SC_FRAG = 16 * SC_ROW, GROUP = (F + MB) * SC_FRAG;
    constexpr int OFF_SC = kRowsRing * STAGE, PER_WAVE = OFF_SC + 2 * GROUP;
    constexpr int DMAS = 2 * (F + MB);
    constexpr int RED = NW * F * MB * 1024;
    constexpr int BYTES = NW * PER_WAVE > RED ? NW * PER_WAVE : RED;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[BYTES];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n0 = (int)blockIdx.x * 16 * FO;
    const int64_t m0 = (int64_t)blockIdx.y * 16 * MB;
    const int blocks = p.K / 32, KT = (blocks + 7) / 8;
    // (an even number of stages each, so that their scale bytes start 16 bytes apart)
    const int per = ((KT + NW - 1) / NW + 1) & ~1, first = wave * per, end = min(KT, first + per);
    const uint32_t kb = (uint32_t)p.K / 2, sb = (uint32_t)p.in_stride;

    // one buffer for each operand; a fragment's rows past the last lie outside it
    const uint32_t rm = (uint32_t)min((int64_t)p.M - m0, (int64_t)16 * MB), rn = (uint32_t)min(p.N - n0, 16 * FO);
    const v4i dA = buffer_desc(p.a + m0 * kb, rm * kb), dSA = buffer_desc(p.as + m0 * sb, rm * sb);
    v4i dW[2], dSW[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const int64_t row = n0 + (EPI == kLinear ? 0 : (int64_t)g * p.N);
        dW[g] = buffer_desc(p.w + row * kb, rn * kb);
        dSW[g] = buffer_desc(p.ws + row * sb, rn * sb);
    }
    const uint32_t lds = lds_addr(smem) + (uint32_t)wave * PER_WAVE;
    const uint32_t c_row = (uint32_t)lane >> 3;
    const uint32_t c_chunk[2] = {((uint32_t)lane & 7u) ^ (c_row >> 1), ((uint32_t)lane & 7u) ^ (c_row >> 1) ^ 4u};
    constexpr uint32_t kOutside = 0x80000000u;
    auto issue = [&](int st, int slot) __attribute__((always_inline)) {
        const uint32_t to = lds + (uint32_t)slot * STAGE;
        uint32_t v[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t c = (uint32_t)st * 8u + c_chunk[x];
            v[x] = st < end && c < (uint32_t)blocks ? (c_row + 8 * x) * kb + c * 16u : kOutside;
        }
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int x = 0; x < 2; ++x) dma16(dW[f / FO], v[x] + (uint32_t)(f % FO) * 16u * kb, to + f * FRAG + x * 1024);
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) dma16(dA, v[x] + (uint32_t)b * 16u * kb, to + (F + b) * FRAG + x * 1024);
    };
    // the scale bytes of stages st .. st + 3 (of the last, as far as a row of them goes)
    auto issue_scales = [&](int st, int buf) __attribute__((always_inline)) {
        const uint32_t to = lds + OFF_SC + (uint32_t)buf * GROUP;
        const uint32_t at = (uint32_t)st * 8u + ((uint32_t)lane & 1u) * 16u;
        const uint32_t v = st < end && at < sb ? ((uint32_t)lane >> 1) * sb + at : kOutside;
        if (lane < 32) {
#pragma unroll
            for (int f = 0; f < F; ++f) dma16(dSW[f / FO], v + (uint32_t)(f % FO) * 16u * sb, to + f * SC_FRAG);
#pragma unroll
            for (int b = 0; b < MB; ++b) dma16(dSA, v + (uint32_t)b * 16u * sb, to + (F + b) * SC_FRAG);
        }
    };

    v4f acc[F][MB];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[f][b] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    issue_scales(first, 0);
    issue(first, 0);
    issue(first + 1, 1);
    const uint8_t *mine = smem + wave * PER_WAVE;
    const uint32_t at0 = (uint32_t)(r * kRowBytes + (((2 * q) ^ (r >> 1)) << 4));
    const uint32_t at1 = (uint32_t)(r * kRowBytes + (((2 * q + 1) ^ (r >> 1)) << 4));
    for (int st = first; st < end; ++st) {
        const int i = st - first, slot = i % kRowsRing, group = i / kRowsGroup, in_group = i % kRowsGroup;
        // in order: with the next stage's loads outstanding this one's have landed,
        // and its scale bytes before them
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(DMAS) : "memory");
        v4i x0[F + MB], x1[F + MB];
        uint32_t s[F + MB];
        const int left = blocks - 8 * st - 2 * q;
        const uint32_t mask = left >= 2 ? 0xFFFFu : left == 1 ? 0xFFu : 0u;
#pragma unroll
        for (int f = 0; f < F + MB; ++f) {
            x0[f] = *reinterpret_cast<const v4i *>(mine + slot * STAGE + f * FRAG + at0);
            x1[f] = *reinterpret_cast<const v4i *>(mine + slot * STAGE + f * FRAG + at1);
            s[f] = mask & *reinterpret_cast<const uint16_t *>(mine + OFF_SC + (group & 1) * GROUP + f * SC_FRAG +
                                                              r * SC_ROW + in_group * 8 + 2 * q);
        }
        // held before the slot takes the stage after the next
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        issue(st + kRowsRing, slot);
        if (in_group == 0) issue_scales(st + kRowsGroup, (group + 1) & 1);
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                mfma_mx4_16<0>(x0[f], s[f], x0[F + b], s[F + b], acc[f][b]);
                mfma_mx4_16<1>(x1[f], s[f], x1[F + b], s[F + b], acc[f][b]);
            }
    }
    // lane l holds row m0 + l % 16, outputs 4 (l / 16) + 0..3 of a fragment
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no DMA into LDS from here on
    __syncthreads();
    float4 *red = reinterpret_cast<float4 *>(smem);
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int b = 0; b < MB; ++b)
            red[((wave * F + f) * MB + b) * 64 + lane] = make_float4(acc[f][b][0], acc[f][b][1], acc[f][b][2], acc[f][b][3]);
    __syncthreads();
    constexpr int PER_ROW = 2 * FO;                        // threads of a row, 8 outputs each
    const int t = (int)threadIdx.x;
    if (t < 16 * MB * PER_ROW) {
        const int g = t % PER_ROW, row = t / PER_ROW, b = row >> 4;
        float v[2][8];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[f][e] = 0.0f;
            if (f * FO >= F) continue;
            const int frag = f * FO + (g >> 1);
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const float4 x = red[((w * F + frag) * MB + b) * 64 + (2 * (g & 1) + hh) * 16 + (row & 15)];
                    v[f][4 * hh + 0] += x.x;
                    v[f][4 * hh + 1] += x.y;
                    v[f][4 * hh + 2] += x.z;
                    v[f][4 * hh + 3] += x.w;
                }
        }
        emit8<EPI, BF16>(p, m0 + row, n0 + 8 * g, v[0], v[1]);
    }
    if constexpr (EPI == kGatedQuant) {
        // the padding behind a row's last block
        if (n0 + 32 >= p.N && t < 16 * MB && m0 + t < p.M)
            for (int64_t i = p.N / 32; i < p.out_stride; ++i) p.scales[(m0 + t) * p.out_stride + i] = 0;
    }
}

// ---- launches (mx4_choice.h has which) ---------------------------------------------
// all outputs by tiles of 64 FM x 64 FN (gated: 32 FN)
template <int EPI, bool BF16, int FM, int FN, int RING, int KS = 1>
hipError_t launch_tile(const Mx4Product &p, hipStream_t stream) {
    constexpr int BM = 64 * FM, BN = (EPI == kLinear ? 64 : 32) * FN;
    const int tiles_m = (int)(((int64_t)p.M + BM - 1) / BM), tiles_n = (p.N + BN - 1) / BN;
    const int64_t T = (int64_t)tiles_m * tiles_n;
    // (parts of k: a tile each, their sums lie where the next one's stages would)
    const int64_t grid = KS > 1 ? T : std::min<int64_t>(T, (int64_t)device_cus() * (FM * FN > 4 || RING > 2 ? 1 : 2));
    hipLaunchKernelGGL((k_mx4_tile<EPI, BF16, FM, FN, RING, KS>), dim3((unsigned)grid), dim3(256 * KS), 0, stream, p, tiles_m, tiles_n);
    return hipGetLastError();
}

template <int EPI, bool BF16, int MB>
hipError_t launch_rows(const Mx4Product &p, int cus, hipStream_t stream) {
    constexpr int NO = EPI == kGatedQuant ? 32 : 16;
    const dim3 grid((unsigned)((p.N + NO - 1) / NO), (unsigned)((p.M + 16 * MB - 1) / (16 * MB)));
    if (mx4_rows_waves((int64_t)grid.x * grid.y, cus) == 2)
        hipLaunchKernelGGL((k_mx4_rows<EPI, BF16, MB, 2>), grid, dim3(128), 0, stream, p);
    else
        hipLaunchKernelGGL((k_mx4_rows<EPI, BF16, MB, 4>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

template <int EPI, bool BF16>
hipError_t launch_typed(const Mx4Product &p, hipStream_t stream) {
    const int cus = device_cus();
    const Mx4Kernel which = mx4_kernel((Epilogue)EPI, p.M, p.N, p.K, cus);
    if constexpr (EPI == kLinear) {
        switch (which) {
            case kTile64x64: return launch_tile<EPI, BF16, 1, 1, 4>(p, stream);
            case kTile64x64Parts: return launch_tile<EPI, BF16, 1, 1, 4, 2>(p, stream);
            case kTile64x128Parts: return launch_tile<EPI, BF16, 1, 2, 2, 2>(p, stream);
            case kTile128x192: return launch_tile<EPI, BF16, 2, 3, 2>(p, stream);
            case kTile192x192: return launch_tile<EPI, BF16, 3, 3, 2>(p, stream);
            default: break;
        }
    }
    switch (which) {
        case kRows16: return launch_rows<EPI, BF16, 1>(p, cus, stream);
        case kRows32: return launch_rows<EPI, BF16, 2>(p, cus, stream);
        case kTile64x128: return launch_tile<EPI, BF16, 1, 2, EPI == kLinear ? 2 : 4>(p, stream);
        case kTile128x128: return launch_tile<EPI, BF16, 2, 2, 2>(p, stream);
        case kTile192x256: return launch_tile<EPI, BF16, 3, 4, 2>(p, stream);
        default: return launch_tile<EPI, BF16, 4, 4, 2>(p, stream);
    }
}

// y's rows begin at halves of cache lines
bool half_lines(const Mx4Product &p) { return p.ldy % 32 == 0 && reinterpret_cast<uintptr_t>(p.y) % 64 == 0; }

}  // namespace

hipError_t launch_mx4_linear(p4q_dtype out_dt, Mx4Product p, hipStream_t stream) {
    p.in_stride = mx4_scale_stride(p.K);
    p.wide = half_lines(p);
    return out_dt == P4Q_BF16 ? launch_typed<kLinear, true>(p, stream) : launch_typed<kLinear, false>(p, stream);
}

hipError_t launch_mx4_gated(p4q_dtype out_dt, Mx4Product p, hipStream_t stream) {
    p.in_stride = mx4_scale_stride(p.K);
    p.out_stride = mx4_scale_stride(p.N);
    if (p.codes) return launch_typed<kGatedQuant, false>(p, stream);
    p.wide = half_lines(p);
    return out_dt == P4Q_BF16 ? launch_typed<kGated, true>(p, stream) : launch_typed<kGated, false>(p, stream);
}

}  // namespace p4q
