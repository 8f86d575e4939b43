// Attention of one new token per sequence over the paged key-value cache:
//     O[b, h] = sum_{j < len_b} softmax_j(<q_bh, k_j> / sqrt(D)) v_j,
// with the Hq / Hk query heads of a group reading the same keys.
//
// Every key and value is used for a handful of queries, so the call is bound by the
// bytes of the cache.  A unit of work is (sequence, key head, up to 16 query heads of its
// group): keys and values are read once per 16 query heads on them (24/1 heads twice, 8
// sequences of 16001 keys 32 us; 16/1 heads once, 27); the four wavefronts of a
// work-group take its tiles of 32 keys in turn, straight from memory to registers, where
// both products run on v_mfma_f32_16x16x32 with the queries as columns -- with one query
// 15 columns are idle, but the matrix instructions still take a small part of the time that
// the bytes do, and no key or value is converted or reduced across lanes:
//  * S^T = K Q^T: row m of matrix tile t is key 8 (m / 4) + 4 t + m % 4 of the 32.
//    Lane l (m = l % 16, g = l / 16) loads 16-byte pieces 4 s + g of its key.
//  * The result then has, in lane l, query l % 16 and keys 8 g + 4 t + r: exactly
//    the eight keys 8 g .. 8 g + 7 that the second product's operand P^T wants there.
//  * O^T += V^T P^T: lane l loads values d = (D/16) m .. + D/16 - 1 of keys 8 g .. 8 g + 7
//    (whole rows, 16 lanes each); matrix instruction j takes d = (D/16) m + j as its row m,
//    whose eight keys are one byte permutation per pair away.
//  * The next tile's keys are loaded under this tile's softmax, its values under
//    the next keys' product; the next unit's first tile under this one's end.  Pages
//    come by scalar loads: a vector load of the table would queue behind the values
//    (one of 131071 keys: 147 us).
// The softmax keeps a running maximum per query, raised only when a tile exceeds it
// by more than 2^8 (exp2 units).  The matrix instructions take weights of the cache's
// type, so each goes in as two such numbers, one from below and the rest: within
// 2^-14 (bf16) and 2^-20 (fp16) of itself, where one alone is off by 2^-8 and 2^-11 and
// makes the outputs' error 1.3 times what rounding them costs.  Their products run under
// the loads (64 ragged sequences 132 us, with one piece 129; one of 131071 keys 91.7 either
// way).  fp16 weights carry 2^7, so that they reach down to 2^-31 of the
// largest.  Scores, maxima, sums and the accumulated values are fp32.
//
// Work is dealt on the device, where the lengths are: all tiles of all units, in
// order, in equal shares to as many work-groups as run at once.  A share begins and
// ends anywhere; a unit's parts, one per work-group, are left in the workspace
// (device-coherent atomic stores, complete before the work-group counts itself in),
// and the one that arrives last adds them up, in a fixed order: results do not
// depend on the order of arrival.  Where a unit is split follows from all lengths of the call,
// so its last bits change with its neighbours.  Chunks of the longest length instead: 64
// sequences of 16 to 16000 keys 270 us, now 130.
// Rows of the cache past a sequence's length are never used: their scores are
// masked and their values replaced by zeros.
//
// One sequence of 131071 keys, 8 key heads: 85 to 92 us (5.8 to 6.3 TB/s; a plain read of as
// much memory 99 us); the 64 ragged sequences 128 to 132 us (5.8 to 6.0 TB/s), 16 sequences of
// 672 to 1217 keys, 32 key heads, 44 to 49 us (5.1 to 5.6 TB/s); one of 371 keys, 40 heads, 8.6
// us: launch, lengths, table, keys, values and the join in LDS one after the other.
#include "attention_device.h"
#include "gemm_device.h"
#include "kv_cache.h"
#include "p4q_internal.h"
#include "wave_ops.h"

#include <algorithm>

namespace p4q {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 32;                       // keys of a tile
constexpr int kRound = kWaves * kKeys;          // keys that a work-group takes at a time
constexpr int kCols = 16;                       // queries of a work-group
constexpr int kUnitCost = 2;                    // tiles that a unit's start and end are worth (us with 1, 2 and 4: 64
                                                // sequences of 16 to 4000 keys, 32/8 heads, 57, 52, 51; one of 700 keys,
                                                // 40 heads, 12.8, 9.9, 11.2)
constexpr int kShort = 16;                      // mean tiles of a unit up to which none is split for its own sake (whole and
                                                // in parts, us: 200 keys, 40 heads 7.8 and 12.2, 371 keys 10.1 and 11.4,
                                                // 700 keys 14.7 and 9.9; 4 x 300 to 600 keys, 32/8 heads, 16.2 and 12.2,
                                                // where it costs most)
constexpr float kRescale = 8.0f;                // raise the running max past this margin (exp2 units)
constexpr int kGroupsPerCu = 2;                 // resident work-groups (250 registers)
constexpr size_t kArrivalBytes = 32768;         // arrival counters at the head of the workspace

// Sums of a softmax over some of the keys, for 4 values of a query
struct Sums {
    float top = -__builtin_huge_valf(), l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    // those over other keys: their maximum m (no key: -inf, with a sum of 0 or NaN), sum and values
    __device__ __forceinline__ void add(float m, float sum, float4 x, float c2) {
        const float t = __builtin_fmaxf(top, m);
        const float f = top == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((top - t) * c2);
        const float e = m == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((m - t) * c2);
        l = l * (top == -__builtin_huge_valf() ? 1.0f : f) + sum * (m == -__builtin_huge_valf() ? 1.0f : e);
        top = t;
        o.x = o.x * f + x.x * e;
        o.y = o.y * f + x.y * e;
        o.z = o.z * f + x.z * e;
        o.w = o.w * f + x.w * e;
    }
};

// x / y for x >= 0, y > 0: in 32 bits where both fit
__device__ __forceinline__ int64_t div_floor(int64_t x, int64_t y) {
    if (((uint64_t)(x | y) >> 32) == 0) return (int64_t)((uint32_t)x / (uint32_t)y);
    return (int64_t)((uint64_t)x / (uint64_t)y);
}

// The tiles of all units, dealt to the work-groups in order: `extra` of them take base
// + 1, the others base.
struct Shares {
    int64_t base, extra;
    __device__ __forceinline__ int64_t start(int64_t group) const { return group * base + min(group, extra); }
    __device__ __forceinline__ int group(int64_t tile) const {
        const int64_t big = extra * (base + 1);
        return (int)(tile < big ? div_floor(tile, base + 1) : extra + div_floor(tile - big, base));
    }
};

template <bool BF16, int D>
__global__ __launch_bounds__(64 * kWaves, 2) void k_decode_attention(DecodeAttention a) {
    constexpr int kSteps = D / 32;              // matrix steps of a key
    constexpr int kV = D / 16;                  // values per lane and key
    constexpr int kRow = D + 4;                 // fp32 of a staged query (its quads spread over the banks)
    constexpr int kPart = kCols * (D + 2);      // a part in the workspace: [kCols][D] sums, [kCols][2] maximum and sum
    constexpr int kQuads = D / 4;
    constexpr int kJoin = D / 32;               // quads per lane of the join at a time
    constexpr int kBatch = 512 / D;             // parts per wavefront of the join at a time
    constexpr int kCoherent = 16;               // sc1: past the caches that other XCDs do not see
    constexpr float kBias = BF16 ? 0.0f : 7.0f;
    __shared__ __attribute__((aligned(16))) float s_acc[kWaves][kCols * kRow];
    __shared__ float s_max[kWaves][kCols], s_sum[kWaves][kCols];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, g = lane >> 4;
    const int qblocks = (a.G + kCols - 1) / kCols, heads = a.Hk * qblocks;
    const int block = (a.G + qblocks - 1) / qblocks;    // query heads of a block, the last one's fewer

    // This work-group's share of all tiles, in the order (sequence, head block, tile),
    // where a unit starts with kUnitCost tiles that stand for its fixed cost.
    auto tiles_of = [&](int len) __attribute__((always_inline)) {
        return kUnitCost + (min(key_count(len), a.max_len) + kKeys - 1) / kKeys;
    };
    int64_t all = 0;
    for (int i = 0; i < a.B; i += 64) {
        const int n = i + lane < a.B ? tiles_of(a.lens[i + lane]) : 0;
        all += (uint32_t)__builtin_amdgcn_readlane((int)wave_inclusive_scan((uint32_t)n), 63);
    }
    all *= heads;
    Shares shares;
    {
        const int64_t units = (int64_t)a.B * heads, mean = div_floor(all, units);
        int64_t groups = units, most = gridDim.x;
        if (mean > kShort) {
            // A unit is split into whole rounds of the wavefronts, fewer and longer ones the
            // more there are to join, and the more queries each part holds (us with half as many
            // rounds, these, and twice as many: 4000 keys, 24/1 heads 17.3, 14.6, 16.6, 30000 keys
            // 30.9, 27.1, 33.0, 4000 keys, 32/8 heads 13.6, 13.5, 14.9; without the 2 for many
            // queries, 24/1 heads, 17.2 and 29.4).
            // With much to read one work-group per CU does best: it has fewer parts to
            // join (us with one and with two: 131071 keys 91 and 101, 32 x 2000 to 2500 keys, 32/8
            // heads, 55.5 and 60.1, 8 x 100 to 30000 35.8 and 39.9; below the line, where two are
            // used, 16000 keys 20.9 and 26.0, 2000 keys 11.8 and 11.8; short units, whose start and
            // end weigh more, keep two: 64 sequences of 30 to 200 keys 34, with one 42).
            const int rounds = max(1, (int)(__builtin_sqrtf((float)mean * (block > 8 ? 2 : 1)) * 0.125f + 0.5f));
            groups = max(units, div_floor(all, kWaves * rounds));
            if (all > 16 * (int64_t)a.cus) most = min(most, (int64_t)a.cus);
        }
        groups = min(groups, most);
        shares.base = div_floor(all, groups);
        shares.extra = all - shares.base * groups;
        if ((int64_t)blockIdx.x >= groups) return;
    }
    int64_t p = shares.start(blockIdx.x);
    const int64_t pend = shares.start((int64_t)blockIdx.x + 1);
    int b = 0, hb = 0, r = 0, tiles = 0;        // the unit (b, hb) and the first of its tiles to do
    {
        const int64_t want = div_floor(p, heads);
        int64_t before = 0;
        for (int i = 0; i < a.B; i += 64) {
            const int n = i + lane < a.B ? tiles_of(a.lens[i + lane]) : 0;
            const uint32_t upto = wave_inclusive_scan((uint32_t)n);
            const int k = __popcll(__ballot(before + upto <= want));
            if (k < 64) {                       // (a sequence: want < all / heads)
                b = i + k;
                tiles = __builtin_amdgcn_readlane(n, k);
                const int64_t at = p - (before + (uint32_t)__builtin_amdgcn_readlane((int)upto, k) - tiles) * heads;
                hb = (int)div_floor(at, tiles);
                r = (int)(at - (int64_t)hb * tiles);
                break;
            }
            before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
    }

    const int64_t page_elems = ((int64_t)a.Hk << a.shift) * D;
    const int pmask = (1 << a.shift) - 1;
    const int krow = 8 * (m >> 2) + (m & 3);    // key of row m, matrix tile 0
    uint4 qf[kSteps], kf[2][kSteps];
    uint32_t vf[8][kV / 2];
    // the two 16-key halves of a tile lie on one page each
    struct Pages {
        int p[2];
    };
    Pages pg, next;
    // the unit's own: length, end of its tiles to do, keys [kt, k1), table, head
    int len, used, rend, kt, k1, h0, cols;
    int64_t head;
    const int32_t *table;
    auto pages_of = [&](int key) __attribute__((always_inline)) {
        Pages x;
#pragma unroll
        for (int e = 0; e < 2; ++e) x.p[e] = uniform_load(table, min(key + 16 * e, used - 1) >> a.shift);   // past the last: its page
        return x;
    };
    // keys and values are read once: nontemporal, so that they do not displace each
    // other in the caches on their way
    auto load16 = [](const uint16_t *src) __attribute__((always_inline)) {
        return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const v4i *>(src)));
    };
    auto load_k = [&](int key, Pages pp) __attribute__((always_inline)) {
        const int page = max(0, valid_page((m >> 3) ? pp.p[1] : pp.p[0], a.num_pages));
        const uint16_t *src = a.k + (int64_t)page * page_elems + head + (int64_t)((key + krow) & pmask) * D + 8 * g;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) kf[t][s] = load16(src + 4 * t * D + 32 * s);
    };
    auto load_v = [&](int key, Pages pp) __attribute__((always_inline)) {
        const int page = max(0, valid_page((g >> 1) ? pp.p[1] : pp.p[0], a.num_pages));
        const uint16_t *src = a.v + (int64_t)page * page_elems + head + (int64_t)((key + 8 * g) & pmask) * D + kV * m;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kV == 8) {
                const uint4 x = load16(src + i * D);
                vf[i][0] = x.x, vf[i][1] = x.y, vf[i][2] = x.z, vf[i][3] = x.w;
            } else {
                const uint2 x = __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const v2i *>(src + i * D)));
                vf[i][0] = x.x, vf[i][1] = x.y;
            }
        }
    };
    // takes up unit (b, hb) from tile r on: its first loads are issued here
    auto begin = [&]() __attribute__((always_inline)) {
        len = key_count(uniform_load(a.lens, b));
        used = min(len, a.max_len);             // max_len keys fit the table
        rend = (int)min((int64_t)tiles, r + (pend - p));
        kt = (max(0, r - kUnitCost) + wave) * kKeys;
        k1 = min(used, max(0, rend - kUnitCost) * kKeys);
        const int hk = hb / qblocks, qb = hb - hk * qblocks;
        cols = min(block, a.G - qb * block);
        h0 = hk * a.G + qb * block;             // first query head
        table = a.table + (int64_t)b * a.max_pages;
        head = ((int64_t)hk << a.shift) * D;
        if (kt < k1) {
            pg = pages_of(kt);
            next = pages_of(kt + kRound);
            load_k(kt, pg);
            const uint16_t *qrow = a.q + (int64_t)b * a.ldq + (int64_t)(h0 + min(m, cols - 1)) * D + 8 * g;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) qf[s] = *reinterpret_cast<const uint4 *>(qrow + 32 * s);
            load_v(kt, pg);
        }
    };

    begin();
    for (;;) {
        v4f acc[kV];
#pragma unroll
        for (int j = 0; j < kV; ++j) acc[j] = v4f{};
        float mx = -__builtin_huge_valf(), sum = 0.0f;      // per query; the sum per lane
        bool bad = len > a.max_len;                         // nobody reads past max_len: NaN
        for (; kt < k1; kt += kRound) {
            bad |= valid_page(pg.p[0], a.num_pages) == kNoPage || valid_page(pg.p[1], a.num_pages) == kNoPage;
            v4f st[2] = {v4f{}, v4f{}};
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) st[t] = mfma16<BF16>(kf[t][s], qf[s], st[t]);
            const bool more = kt + kRound < k1;
            if (more) {
                pg = next;
                load_k(kt + kRound, pg);
                next = pages_of(kt + 2 * kRound);
            }
            if (kt + kKeys > k1) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (kt + 8 * g + i >= k1) {
                        st[i >> 2][i & 3] = -__builtin_huge_valf();
#pragma unroll
                        for (int e = 0; e < kV / 2; ++e) vf[i][e] = 0;
                    }
            }
            float tmax = st[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) tmax = __builtin_fmaxf(tmax, st[i >> 2][i & 3]);
            const bool raise = (tmax - mx) * a.c2 > kRescale || mx == -__builtin_huge_valf();
            if (__any((int)raise)) {                        // for all queries, the same in a query's four lanes
                const float top = __builtin_fmaxf(xmax32(xmax16(tmax)), mx);
                const float alpha = mx == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((mx - top) * a.c2);
                mx = top;
                sum *= alpha;
#pragma unroll
                for (int j = 0; j < kV; ++j) acc[j] *= alpha;
            }
            // The maximum is taken off before the product with c2: rounded after it, it would
            // scale the weights by 2^(up to |mx| c2 2^-24), which overflows or vanishes past 2^28.
            const float off = __builtin_fmaxf(mx, -3.0e38f);    // (no score yet: all of them -inf)
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[i >> 2][i & 3] - off, a.c2, kBias));
                sum += w[i];
            }
            // Each weight as a sum of two 16-bit numbers.  The first is a step below the cut-off
            // weight, so that the second is neither 0 nor negative, which would turn an infinite
            // value into NaN; a weight of 0 stays 0.
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hi[i] = pack2_below<BF16>(w[2 * i], w[2 * i + 1]);
                const v2f h = unpack2<BF16>(hi[i]);
                lo[i] = pack2<BF16>(w[2 * i] - h[0], w[2 * i + 1] - h[1]);
            }
            const uint4 ph = make_uint4(hi[0], hi[1], hi[2], hi[3]), pl = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            // (the second pieces one step behind the first, whose sums they wait for)
            uint4 va, last;
#pragma unroll
            for (int j = 0; j <= kV; ++j) {
                if (j < kV) {
                    const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
                    va = make_uint4(__builtin_amdgcn_perm(vf[1][j >> 1], vf[0][j >> 1], sel),
                                    __builtin_amdgcn_perm(vf[3][j >> 1], vf[2][j >> 1], sel),
                                    __builtin_amdgcn_perm(vf[5][j >> 1], vf[4][j >> 1], sel),
                                    __builtin_amdgcn_perm(vf[7][j >> 1], vf[6][j >> 1], sel));
                    acc[j] = mfma16<BF16>(va, ph, acc[j]);
                }
                if (j > 0) acc[j - 1] = mfma16<BF16>(last, pl, acc[j - 1]);
                last = va;
            }
            if (more) load_v(kt + kRound, pg);
        }
        // what the epilogue needs of this unit; then the next unit's loads are issued under it
        const int c_b = b, c_h0 = h0, c_cols = cols, c_len = len;
        const bool from_start = r == 0, to_end = rend == tiles;
        const int64_t ufirst = p - r, ulast = ufirst + tiles - 1;       // the unit's tiles among all
        p += rend - r;
        const bool again = p < pend;
        if (again) {
            r = 0;
            if (++hb == heads) {
                hb = 0;
                tiles = tiles_of(uniform_load(a.lens, ++b));
            }
            begin();
        }

        sum = xsum32(xsum16(sum));
        if (bad) sum = __builtin_nanf("");
        // the wavefronts' sums, per query: acc[j][e] of lane l is d = kV (4 g + e) + j of query m
        if (g == 0) {
            s_max[wave][m] = mx;
            s_sum[wave][m] = sum;
        }
        if (m < c_cols) {
            float *dst = &s_acc[wave][m * kRow + kV * 4 * g];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < kV; j += 4)
                    *reinterpret_cast<float4 *>(dst + kV * e + j) = make_float4(acc[j][e], acc[j + 1][e], acc[j + 2][e], acc[j + 3][e]);
        }
        __syncthreads();
        uint16_t *const orow = a.out + (int64_t)c_b * a.ldo + (int64_t)c_h0 * D;
        const bool whole = from_start && to_end;
        for (int i = tid; i < c_cols * kQuads; i += 64 * kWaves) {
            const int qi = i / kQuads, d = 4 * (i % kQuads);
            float top = s_max[0][qi];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) top = __builtin_fmaxf(top, s_max[w][qi]);
            float l = 0.0f;
            float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float mw = s_max[w][qi], f = mw == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((mw - top) * a.c2);
                const float4 x = *reinterpret_cast<const float4 *>(&s_acc[w][qi * kRow + d]);
                l = __builtin_fmaf(s_sum[w][qi], mw == -__builtin_huge_valf() ? 1.0f : f, l);   // (no key: 0, or NaN)
                o.x = __builtin_fmaf(x.x, f, o.x);
                o.y = __builtin_fmaf(x.y, f, o.y);
                o.z = __builtin_fmaf(x.z, f, o.z);
                o.w = __builtin_fmaf(x.w, f, o.w);
            }
            if (whole) {
                const float inv = c_len == 0 ? 0.0f : 1.0f / l;
                *reinterpret_cast<uint2 *>(orow + qi * D + d) =
                    make_uint2(pack2_scaled<BF16>(o.x, o.y, inv), pack2_scaled<BF16>(o.z, o.w, inv));
            } else {
                float *dst = a.part + (2 * (int64_t)blockIdx.x + from_start) * kPart;
                const float v[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                for (int e = 0; e < 4; e += 2)
                    __hip_atomic_store(reinterpret_cast<uint64_t *>(dst + qi * D + d + e),
                                       (uint64_t)__float_as_uint(v[e]) | (uint64_t)__float_as_uint(v[e + 1]) << 32,
                                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (d == 0)
                    __hip_atomic_store(reinterpret_cast<uint64_t *>(dst + kCols * D + 2 * qi),
                                       (uint64_t)__float_as_uint(top) | (uint64_t)__float_as_uint(l) << 32,
                                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        if (!whole) {
            // the unit's parts are those of work-groups first .. last
            const int first = shares.group(ufirst), splits = shares.group(ulast) - first + 1;
            // every store of the work-group is complete before it counts itself in
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) {
                const uint32_t before = __hip_atomic_fetch_add(a.arrivals + first, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = before == (uint32_t)(splits - 1);
                if (s_last) __hip_atomic_store(a.arrivals + first, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (s_last) {
                // The last one adds the parts up.  A wavefront takes every kWaves-th part, a
                // lane the quads lane, lane + 64, ..; the wavefronts' sums meet in LDS.  Always
                // in that order, so the result does not depend on who is last.
                const auto parts = __builtin_amdgcn_make_buffer_rsrc(a.part, 0, 0x7FFFFFFF, 0x00020000);
                const int quads = c_cols * kQuads;
                float *const s_join = &s_acc[0][0];         // [kWaves][64 kJoin][6]
                for (int i0 = 0; i0 < quads; i0 += 64 * kJoin) {
                    Sums s[kJoin];
                    uint32_t at[kJoin], ml[kJoin];
#pragma unroll
                    for (int j = 0; j < kJoin; ++j) {
                        const int i = min(i0 + 64 * j + lane, quads - 1);
                        at[j] = (uint32_t)(4 * i);          // [query][D]
                        ml[j] = (uint32_t)(kCols * D + 2 * (i / kQuads));
                    }
                    for (int z0 = wave; z0 < splits; z0 += kBatch * kWaves) {
                        float4 x[kBatch][kJoin];
                        float2 w[kBatch][kJoin];
#pragma unroll
                        for (int u = 0; u < kBatch; ++u) {
                            const int z = z0 + u * kWaves < splits ? z0 + u * kWaves : z0;
                            const uint32_t base = (uint32_t)((2 * (first + z) + (z == 0)) * kPart);
#pragma unroll
                            for (int j = 0; j < kJoin; ++j) {
                                w[u][j] = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(parts, 4 * (base + ml[j]), 0, kCoherent));
                                x[u][j] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(parts, 4 * (base + at[j]), 0, kCoherent));
                            }
                        }
                        __builtin_amdgcn_sched_barrier(0);  // all of them in flight at once
#pragma unroll
                        for (int u = 0; u < kBatch; ++u)
                            if (z0 + u * kWaves < splits)
#pragma unroll
                                for (int j = 0; j < kJoin; ++j) s[j].add(w[u][j].x, w[u][j].y, x[u][j], a.c2);
                    }
                    if (i0 > 0) __syncthreads();
#pragma unroll
                    for (int j = 0; j < kJoin; ++j) {
                        float *dst = s_join + (wave * 64 * kJoin + 64 * j + lane) * 6;
                        dst[0] = s[j].top, dst[1] = s[j].l, dst[2] = s[j].o.x, dst[3] = s[j].o.y, dst[4] = s[j].o.z, dst[5] = s[j].o.w;
                    }
                    __syncthreads();
                    const int i = i0 + tid;                 // 64 kJoin <= 64 kWaves quads
                    if (tid < 64 * kJoin && i < quads) {
                        Sums t;
#pragma unroll
                        for (int w = 0; w < kWaves; ++w) {
                            const float *src = s_join + (w * 64 * kJoin + tid) * 6;
                            t.add(src[0], src[1], make_float4(src[2], src[3], src[4], src[5]), a.c2);
                        }
                        const int qi = i / kQuads, dd = 4 * (i % kQuads);
                        const float inv = c_len == 0 ? 0.0f : 1.0f / t.l;
                        *reinterpret_cast<uint2 *>(orow + qi * D + dd) =
                            make_uint2(pack2_scaled<BF16>(t.o.x, t.o.y, inv), pack2_scaled<BF16>(t.o.z, t.o.w, inv));
                    }
                }
            }
        }
        if (!again) return;
        __syncthreads();                        // the staged sums are read: the next unit's may come
    }
}

// work-groups: as many as the device runs at once, or one per round
int64_t decode_groups(int B, int Hq, int Hk, int max_len) {
    const int64_t heads = (int64_t)Hk * ((Hq / Hk + kCols - 1) / kCols);
    const int64_t rounds = (max_len + kRound - 1) / kRound;
    return std::min<int64_t>(std::min<int64_t>(kGroupsPerCu * device_cus(), kArrivalBytes / 4), B * heads * rounds);
}

}  // namespace

size_t decode_attention_workspace_bytes(int B, int Hq, int Hk, int D, int max_len) {
    return kArrivalBytes + (size_t)(2 * decode_groups(B, Hq, Hk, max_len) * kCols * (D + 2)) * 4;
}

hipError_t launch_decode_attention(p4q_dtype dt, int D, DecodeAttention a, void *ws, hipStream_t stream) {
    a.c2 = 1.4426950408889634f / __builtin_sqrtf((float)D);                 // log2(e) / sqrt(D)
    a.G = a.Hq / a.Hk;
    a.cus = device_cus();
    a.arrivals = static_cast<uint32_t *>(ws);
    a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + kArrivalBytes);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)decode_groups(a.B, a.Hq, a.Hk, a.max_len)), dim3(64 * kWaves), 0, stream, a);
        return hipGetLastError();
    };
    if (dt == P4Q_BF16) return D == 128 ? go(k_decode_attention<true, 128>) : go(k_decode_attention<true, 64>);
    return D == 128 ? go(k_decode_attention<false, 128>) : go(k_decode_attention<false, 64>);
}

}  // namespace p4q
