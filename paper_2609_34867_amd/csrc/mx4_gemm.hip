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
#include <utility>

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

// (the hardware's exp2 and reciprocal, one unit in the last place each)
__device__ __forceinline__ float silu(float g) {
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * g));
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
        store8(p, m, n0, round16x8<BF16>(v));
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

// ---- tiles through LDS -----------------------------------------------------------
// A work-group of four wavefronts, 2 x 2, computes 64 FM rows by 64 FN weight
// rows, each wavefront FM x FN fragments of 32 x 32.  k runs in stages of 256
// values, four steps each; two stages fit in LDS, filled by DMA, and the ring
// runs on across the tiles of a persistent work-group.
//  * A stage's row is 128 bytes, one cache line, loaded by 8 lanes: what the DMA
//    costs is lines touched per instruction, and rows of half a line cost a third
//    more time.  Chunk c of 16 bytes (32 codes) of row r lies at c ^ (r / 2 % 8),
//    so that 16 rows of a fragment read fall into distinct banks.
//  * Scale bytes come 16 per row, for two stages at once: the rows of a with the
//    odd stage before, those of w with the even one.  An odd number of stages is
//    padded with one that multiplies nothing.
//  * Operands are read ahead of their step: during steps 2 and 3 those of the next
//    stage's steps 0 to 2, during step 0 those of step 3.  So a slot is read in
//    three steps and has five for its next stage to arrive, whose DMAs are spread
//    over the products of steps 1 to 3 (over four steps, with less time to arrive,
//    2% slower).
//  * Past the row's end the DMA's offsets lie outside the buffer and give codes
//    of zero, and the scale bytes there are masked; rows past the last are outside
//    it too.
// No instruction: x is taken to change here.
__device__ __forceinline__ void hold(v16f &x) { asm volatile("" : "+a"(x)); }

template <class F, int... I>
__device__ __forceinline__ void unrolled_seq(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
// f(0) .. f(N - 1), the arguments compile-time constants
template <int N, class F>
__device__ __forceinline__ void unrolled(F &&f) {
    unrolled_seq(f, std::make_integer_sequence<int, N>{});
}

constexpr int kRowBytes = 128;                   // codes of a row in a stage
constexpr int kRowScales = 16;                   // scale bytes of a row, two stages'

template <int EPI, bool BF16, int FM, int FN>
__global__ __launch_bounds__(256, FM * FN >= 16 ? 1 : 2) void k_mx4_tile(const Mx4Product p, int tiles_m, int tiles_n) {
    constexpr int BM = 64 * FM, BW = 64 * FN;              // rows of a, of w
    constexpr int BN = EPI == kLinear ? BW : BW / 2;       // outputs: half of w's rows are the gate's
    constexpr int FO = EPI == kLinear ? FN : FN / 2;       // fragments of outputs per wavefront
    constexpr int OFF_W = BM * kRowBytes, STAGE = OFF_W + BW * kRowBytes;
    constexpr int OFF_SCALES = 2 * STAGE, OFF_SW = BM * kRowScales, SCALES = OFF_SW + BW * kRowScales;
    constexpr int OFF_OUT = OFF_SCALES + 2 * SCALES;
    constexpr int EW = FO >= 2 && FM * FN >= 16 ? 2 : 1;   // fragments stored together
    constexpr int OUT_ROW = 64 * EW, OUT_WAVE = EPI == kGatedQuant ? 0 : 32 * OUT_ROW;
    constexpr int CODE_DMAS = 2 * (FM + FN), DMAS = CODE_DMAS + 1;
    static_assert(EPI == kLinear || FN % 2 == 0, "gate and up fragments");
    static_assert(FM <= 4 && FN <= 4, "a wavefront's share of the scales is one load");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[OFF_OUT + 4 * OUT_WAVE];

    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wm = wave & 1, wn = wave >> 1;
    const int blocks = p.K / 32, KT = (blocks + 7) / 8, KT2 = (KT + 1) & ~1;
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
    int iss_tile = -1, iss_kt = KT2 - 1, iss_slot = 1, sc_tile = -1, sc_kt = KT2 - 2, sc_slot = 1;
    v4i dA = {}, dW = {}, dSA = {}, dSW = {};
    uint32_t iss_v[2] = {}, iss_lds = 0;
    auto rows_of = [](int64_t total, int64_t first, int most) __attribute__((always_inline)) {
        return (uint32_t)min(total - first, (int64_t)most);
    };
    // the place of the next two stages' scales of a
    auto scales_a = [&]() __attribute__((always_inline)) {
        sc_kt += 2;
        sc_slot ^= 1;
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
        iss_slot ^= 1;
        iss_lds = lds + (uint32_t)iss_slot * STAGE;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t c = (uint32_t)iss_kt * 8u + c_chunk[x];
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
                    dma16(dSA, (row + (uint32_t)lane) * sb + (uint32_t)sc_kt * 8u, base + row * kRowScales);
            } else {
                const uint32_t row = (uint32_t)wave * 16 * FN;
                const uint32_t from = EPI == kLinear ? row : (uint32_t)(wave & 1) * 16 * FN;
                if (lane < 16 * FN)
                    dma16(dSW, (from + (uint32_t)lane) * sb + (uint32_t)iss_kt * 8u, base + OFF_SW + row * kRowScales);
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

    // the first stage's scales of a, then what two stages before the first would have issued
    constexpr int X = FM * FN, PARTS = 3 * X, EARLY = X * DMAS / PARTS;
    scales_a();
    if (lane < 16 * FM) {
        const uint32_t row = (uint32_t)wave * 16 * FM;
        dma16(dSA, (row + (uint32_t)lane) * sb, lds + OFF_SCALES + (uint32_t)sc_slot * SCALES + row * kRowScales);
    }
    issue_begin();
    unrolled<DMAS>(issue);
    issue_begin();
    unrolled<DMAS>(issue);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(DMAS) : "memory");
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
            const int left = blocks - 8 * kt - 4 * h;
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
                    // the next stage has landed (in order: only what step 1 issued may be outstanding)
                    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(EARLY) : "memory");
                    slot ^= 1;
                    if (kt & 1) s_slot ^= 1;
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
        int tm, tn;
        tile_at(ck, tm, tn);
        const int64_t m0 = (int64_t)tm * BM + wm * 32 * FM;
        const int n0 = tn * BN + wn * 32 * FO;
        const bool full = (int64_t)(tm + 1) * BM <= p.M && (int64_t)(tn + 1) * BN <= p.N;
        uint8_t *out = smem + OFF_OUT + wave * OUT_WAVE;
#pragma unroll
        for (int j = 0; j < FM; ++j) {
#pragma unroll
            for (int f0 = 0; f0 < FO; f0 += EW) {
                // (opaque here, so that no later pass's sums are read before their turn)
#pragma unroll
                for (int e = 0; e < EW; ++e) {
                    hold(acc[f0 + e][j]);
                    if constexpr (EPI != kLinear) hold(acc[f0 + e + FO][j]);
                }
                if constexpr (EPI == kGatedQuant) {
#pragma unroll
                    for (int e = 0; e < EW; ++e) {
                        float v[16];
#pragma unroll
                        for (int x = 0; x < 16; ++x) v[x] = silu(acc[f0 + e][j][x]) * acc[f0 + e + FO][j][x];
                        uint32_t byte;
                        const uint2 c = mx4_quantize_halves(v, byte);
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
                            float o[4];
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                o[x] = acc[f0 + e][j][4 * g + x];
                                if constexpr (EPI == kGated) o[x] = silu(o[x]) * acc[(f0 + e + FO) % FN][j][4 * g + x];
                            }
                            const int chunk = (4 * e + g) ^ (r & (4 * EW - 1));
                            *reinterpret_cast<uint2 *>(out + r * OUT_ROW + chunk * 16 + 8 * h) =
                                make_uint2(round16x2<BF16>(o[0], o[1]), round16x2<BF16>(o[2], o[3]));
                        }
                    constexpr int LR = 4 * EW;             // lanes per row
#pragma unroll
                    for (int s = 0; s < 32 / (64 / LR); ++s) {
                        const int row = s * (64 / LR) + lane / LR, c = lane % LR;
                        const uint4 val = *reinterpret_cast<const uint4 *>(out + row * OUT_ROW + ((c ^ (row & (LR - 1))) << 4));
                        const int64_t m = m0 + 32 * j + row;
                        const int n = n0 + 32 * f0 + 8 * c;
                        if (full) __builtin_memcpy(static_cast<uint16_t *>(p.y) + m * p.ldy + n, &val, 16);
                        else store8(p, m, n, val);
                    }
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

template <int EPI, bool BF16, int FM, int FN>
hipError_t launch_tile(const Mx4Product &p, hipStream_t stream) {
    constexpr int BM = 64 * FM, BN = (EPI == kLinear ? 64 : 32) * FN;
    const int tiles_m = (int)(((int64_t)p.M + BM - 1) / BM), tiles_n = (p.N + BN - 1) / BN;
    const int64_t T = (int64_t)tiles_m * tiles_n;
    const int64_t grid = std::min<int64_t>(T, (int64_t)device_cus() * (FM * FN >= 16 ? 1 : 2));
    hipLaunchKernelGGL((k_mx4_tile<EPI, BF16, FM, FN>), dim3((unsigned)grid), dim3(256), 0, stream, p, tiles_m, tiles_n);
    return hipGetLastError();
}

template <int EPI, bool BF16>
hipError_t launch_typed(const Mx4Product &p, hipStream_t stream) {
    if (p.M > 64) {
        const int64_t tiles = (((int64_t)p.M + 255) / 256) * ((p.N + (EPI == kLinear ? 255 : 127)) / (EPI == kLinear ? 256 : 128));
        return tiles >= device_cus() ? launch_tile<EPI, BF16, 4, 4>(p, stream) : launch_tile<EPI, BF16, 2, 2>(p, stream);
    }
    const dim3 grid((unsigned)((p.N + 31) / 32), (unsigned)(((int64_t)p.M + 31) / 32));
    hipLaunchKernelGGL((k_mx4_skinny<EPI, BF16, 1>), grid, dim3(64 * kSkinnyWaves), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_linear(p4q_dtype out_dt, Mx4Product p, hipStream_t stream) {
    p.in_stride = mx4_scale_stride(p.K);
    return out_dt == P4Q_BF16 ? launch_typed<kLinear, true>(p, stream) : launch_typed<kLinear, false>(p, stream);
}

hipError_t launch_mx4_gated(p4q_dtype out_dt, Mx4Product p, hipStream_t stream) {
    p.in_stride = mx4_scale_stride(p.K);
    p.out_stride = mx4_scale_stride(p.N);
    if (p.codes) return launch_typed<kGatedQuant, false>(p, stream);
    return out_dt == P4Q_BF16 ? launch_typed<kGated, true>(p, stream) : launch_typed<kGated, false>(p, stream);
}

}  // namespace p4q
