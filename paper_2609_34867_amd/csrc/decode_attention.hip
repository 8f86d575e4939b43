// Attention of one new token per sequence over the paged key-value cache:
//     O[b, h] = sum_{j < len_b} softmax_j(<q_bh, k_j> / sqrt(D)) v_j,
// with the Hq / Hk query heads of a group reading the same keys.
//
// Every key and value is read once and used for a handful of queries, so the call
// is bound by the bytes of the cache.  A work-group takes (sequence, key head, a
// chunk of the keys); its four wavefronts take the chunk's tiles of 32 keys in
// turn, straight from memory to registers, where both products run on
// v_mfma_f32_16x16x32 with the group's (up to 16) queries as columns -- with one
// query 15 columns are idle, but the matrix instructions still take a tenth of
// the time that the bytes do, and no key or value is converted or reduced across
// lanes:
//  * S^T = K Q^T: row m of matrix tile t is key 8 (m / 4) + 4 t + m % 4 of the 32.
//    Lane l (m = l % 16, g = l / 16) loads 16-byte pieces 4 s + g of its key.
//  * The result then has, in lane l, query l % 16 and keys 8 g + 4 t + r: exactly
//    the eight keys 8 g .. 8 g + 7 that the second product's operand P^T wants there.
//  * O^T += V^T P^T: lane l loads values d = (D/16) m .. + D/16 - 1 of keys 8 g .. 8 g + 7
//    (whole rows, 16 lanes each); matrix instruction j takes d = (D/16) m + j as its row m,
//    whose eight keys are one byte permutation per pair away.
//  * The next tile's keys are loaded under this tile's softmax, its values under
//    the next keys' product.
// The softmax keeps a running maximum per query, raised only when a tile exceeds it
// by more than 2^8 (exp2 units); weights are rounded to the cache's type before they
// multiply v (fp16 with 2^7 on them: from 2^15 down to 2^-24 - 2^-17 of the largest),
// maxima, sums and outputs are fp32.
//
// A chunk's wavefronts are joined in LDS.  Where a sequence takes more than one
// chunk, each work-group leaves its sums in the workspace (device-coherent atomic
// stores, complete before it counts itself in), and the one that arrives last adds
// all of them up, in the order of the chunks: results do not depend on the order of
// arrival.
// Rows of the cache past a sequence's length are never used: their scores are
// masked and their values replaced by zeros.
#include "attention_device.h"
#include "kv_cache.h"
#include "p4q_internal.h"

#include <algorithm>

namespace p4q {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 32;                       // keys of a tile
constexpr int kRound = kWaves * kKeys;          // keys that a work-group takes at a time
constexpr int kCols = 16;                       // queries of a work-group
constexpr float kRescale = 8.0f;                // raise the running max past this margin (exp2 units)
constexpr size_t kArrivalBytes = 32768;         // arrival counters at the head of the workspace

__device__ __forceinline__ uint32_t dword(uint4 x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

template <bool BF16, int D>
__global__ __launch_bounds__(64 * kWaves, 2) void k_decode_attention(DecodeAttention a) {
    constexpr int kSteps = D / 32;              // matrix steps of a key
    constexpr int kV = D / 16;                  // values per lane and key
    constexpr int kRow = D + 4;                 // fp32 of a staged query (its quads spread over the banks)
    constexpr float kBias = BF16 ? 0.0f : 7.0f;
    __shared__ __attribute__((aligned(16))) float s_acc[kWaves][kCols * kRow];
    __shared__ float s_max[kWaves][kCols], s_sum[kWaves][kCols];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, g = lane >> 4;
    const int qblocks = (a.G + kCols - 1) / kCols;
    const int split = (int)blockIdx.x, hk = (int)blockIdx.y / qblocks, qb = (int)blockIdx.y - hk * qblocks;
    const int b = (int)blockIdx.z;
    const int cols = min(kCols, a.G - qb * kCols);
    const int len = key_count(a.lens[b]);
    const int used = min(len, a.max_len);                                  // max_len <= the table
    const int splits = max(1, (used + a.chunk - 1) / a.chunk);
    if (split >= splits) return;
    const int k0 = split * a.chunk, k1 = min(used, k0 + a.chunk);
    bool bad = len > a.max_len;                                            // nobody reads past max_len: NaN

    const int h0 = hk * a.G + qb * kCols;                                  // first query head
    uint4 qf[kSteps];
    const uint16_t *qrow = a.q + (int64_t)b * a.ldq + (int64_t)(h0 + min(m, cols - 1)) * D + 8 * g;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) qf[s] = *reinterpret_cast<const uint4 *>(qrow + 32 * s);

    const int32_t *table = a.table + (int64_t)b * a.max_pages;
    const int64_t head = ((int64_t)hk << a.shift) * D, page_elems = ((int64_t)a.Hk << a.shift) * D;
    const int pmask = (1 << a.shift) - 1;
    // the two 16-key halves of tile kt lie on one page each
    struct Pages {
        int p[2];
    };
    auto pages_of = [&](int kt) __attribute__((always_inline)) {
        Pages r;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int col = min(kt + 16 * e, max(used - 1, 0)) >> a.shift;  // keys past the last: its page
            r.p[e] = table[col];
        }
        return r;
    };
    const int krow = 8 * (m >> 2) + (m & 3);                               // key of row m, tile 0
    uint4 kf[2][kSteps];
    uint32_t vf[8][kV / 2];
    auto load_k = [&](int kt, Pages pg) __attribute__((always_inline)) {
        const int page = max(0, valid_page((m >> 3) ? pg.p[1] : pg.p[0], a.num_pages));
        const uint16_t *p = a.k + (int64_t)page * page_elems + head + (int64_t)((kt + krow) & pmask) * D + 8 * g;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) kf[t][s] = *reinterpret_cast<const uint4 *>(p + 4 * t * D + 32 * s);
    };
    auto load_v = [&](int kt, Pages pg) __attribute__((always_inline)) {
        const int page = max(0, valid_page((g >> 1) ? pg.p[1] : pg.p[0], a.num_pages));
        const uint16_t *p = a.v + (int64_t)page * page_elems + head + (int64_t)((kt + 8 * g) & pmask) * D + kV * m;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kV == 8) {
                const uint4 x = *reinterpret_cast<const uint4 *>(p + i * D);
                vf[i][0] = x.x, vf[i][1] = x.y, vf[i][2] = x.z, vf[i][3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2 *>(p + i * D);
                vf[i][0] = x.x, vf[i][1] = x.y;
            }
        }
    };

    v4f acc[kV];
#pragma unroll
    for (int j = 0; j < kV; ++j) acc[j] = v4f{};
    float mx = -__builtin_huge_valf(), sum = 0.0f;                          // per query; the sum per lane

    int kt = k0 + wave * kKeys;
    if (kt < k1) {
        Pages pg = pages_of(kt);
        load_k(kt, pg);
        load_v(kt, pg);
        Pages next = pages_of(kt + kRound);
        for (; kt < k1; kt += kRound) {
            bad |= valid_page(pg.p[0], a.num_pages) == kNoPage || valid_page(pg.p[1], a.num_pages) == kNoPage;
            v4f st[2] = {v4f{}, v4f{}};
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) st[t] = mfma16<BF16>(kf[t][s], qf[s], st[t]);
            pg = next;
            const bool more = kt + kRound < k1;
            if (more) load_k(kt + kRound, pg);
            next = pages_of(kt + 2 * kRound);
            const bool tail = kt + kKeys > k1;
            if (tail) {
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
            if (__any((int)raise)) {                                        // the same for a query's four lanes
                const float top = __builtin_fmaxf(xmax32(xmax16(tmax)), mx);
                const float alpha = mx == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((mx - top) * a.c2);
                mx = top;
                sum *= alpha;
#pragma unroll
                for (int j = 0; j < kV; ++j) acc[j] *= alpha;
            }
            const float mc = (mx == -__builtin_huge_valf()) ? 0.0f : mx * a.c2 - kBias;
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[i >> 2][i & 3], a.c2, -mc));
                sum += p[i];
            }
            const uint4 pb = make_uint4(pack2<BF16>(p[0], p[1]), pack2<BF16>(p[2], p[3]), pack2<BF16>(p[4], p[5]),
                                        pack2<BF16>(p[6], p[7]));
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
                const uint4 va = make_uint4(__builtin_amdgcn_perm(vf[1][j >> 1], vf[0][j >> 1], sel),
                                            __builtin_amdgcn_perm(vf[3][j >> 1], vf[2][j >> 1], sel),
                                            __builtin_amdgcn_perm(vf[5][j >> 1], vf[4][j >> 1], sel),
                                            __builtin_amdgcn_perm(vf[7][j >> 1], vf[6][j >> 1], sel));
                acc[j] = mfma16<BF16>(va, pb, acc[j]);
            }
            if (more) load_v(kt + kRound, pg);
        }
    }
    sum = xsum32(xsum16(sum));
    if (bad) sum = __builtin_nanf("");

    // the wavefronts' sums, per query: acc[j][r] of lane l is d = kV (4 g + r) + j of query m
    if (g == 0) {
        s_max[wave][m] = mx;
        s_sum[wave][m] = sum;
    }
    if (m < cols) {
        float *dst = &s_acc[wave][m * kRow + kV * 4 * g];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kV; j += 4)
                *reinterpret_cast<float4 *>(dst + kV * r + j) = make_float4(acc[j][r], acc[j + 1][r], acc[j + 2][r], acc[j + 3][r]);
    }
    __syncthreads();
    constexpr int kQuads = D / 4;
    uint16_t *const orow = a.out + (int64_t)b * a.ldo + (int64_t)h0 * D;
    const int unit = b * (int)gridDim.y + (int)blockIdx.y;
    // workspace of a (sequence, head group): per chunk [kCols][D] sums, then [kCols][2] maximum and sum
    constexpr int kPart = kCols * (D + 2);
    float *const parts = a.part + (int64_t)unit * gridDim.x * kPart;
    for (int i = tid; i < cols * kQuads; i += 64 * kWaves) {
        const int qi = i / kQuads, d = 4 * (i % kQuads);
        float top = s_max[0][qi];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = __builtin_fmaxf(top, s_max[w][qi]);
        float l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float mw = s_max[w][qi], f = mw == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((mw - top) * a.c2);
            // (a wavefront without keys has sum 0, or NaN)
            const float4 x = *reinterpret_cast<const float4 *>(&s_acc[w][qi * kRow + d]);
            l = __builtin_fmaf(s_sum[w][qi], mw == -__builtin_huge_valf() ? 1.0f : f, l);
            o.x = __builtin_fmaf(x.x, f, o.x);
            o.y = __builtin_fmaf(x.y, f, o.y);
            o.z = __builtin_fmaf(x.z, f, o.z);
            o.w = __builtin_fmaf(x.w, f, o.w);
        }
        if (splits == 1) {
            const float inv = len == 0 ? 0.0f : 1.0f / l;
            *reinterpret_cast<uint2 *>(orow + qi * D + d) =
                make_uint2(pack2_scaled<BF16>(o.x, o.y, inv), pack2_scaled<BF16>(o.z, o.w, inv));
        } else {
            float *dst = parts + (int64_t)split * kPart;
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
    if (splits == 1) return;
    // every store of the work-group is complete before it counts itself in
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
        const uint32_t before = __hip_atomic_fetch_add(a.arrivals + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = before == (uint32_t)(splits - 1);
        if (s_last) __hip_atomic_store(a.arrivals + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;

    // The last one adds the chunks up.  Its threads take (query, 4 values, a share
    // of the chunks): kShares shares while there are fewer quads than threads, met in LDS.
    auto load2 = [](const float *p) __attribute__((always_inline)) {
        const uint64_t x = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return make_float2(__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)));
    };
    const int quads = cols * kQuads;
    const int shares = quads >= 64 * kWaves ? 1 : 64 * kWaves / quads;       // per pass over the quads
    float *const s_join = &s_acc[0][0];                                     // [shares][quads][6]: fits (6 * 256 words)
    for (int i0 = 0; i0 < quads; i0 += 64 * kWaves) {
        const int i = shares == 1 ? i0 + tid : tid % quads, share = shares == 1 ? 0 : tid / quads;
        const bool mine = i < quads && share < shares;
        float top = -__builtin_huge_valf(), l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (mine) {
            const int qi = i / kQuads, d = 4 * (i % kQuads);
            const int per = (splits + shares - 1) / shares, z0 = share * per, z1 = min(splits, z0 + per);
#pragma unroll 4
            for (int z = z0; z < z1; ++z) {
                const float *src = parts + (int64_t)z * kPart;
                const float2 ml = load2(src + kCols * D + 2 * qi), x = load2(src + qi * D + d), y = load2(src + qi * D + d + 2);
                const float t = __builtin_fmaxf(top, ml.x);
                const float f = top == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((top - t) * a.c2);
                const float e = ml.x == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((ml.x - t) * a.c2);
                top = t;
                l = l * f + ml.y * (ml.x == -__builtin_huge_valf() ? 1.0f : e);
                o.x = o.x * f + x.x * e;
                o.y = o.y * f + x.y * e;
                o.z = o.z * f + y.x * e;
                o.w = o.w * f + y.y * e;
            }
        }
        if (shares > 1) {
            __syncthreads();
            if (mine) {
                float *dst = s_join + (share * quads + i) * 6;
                dst[0] = top, dst[1] = l, dst[2] = o.x, dst[3] = o.y, dst[4] = o.z, dst[5] = o.w;
            }
            __syncthreads();
            if (mine && share == 0) {
                for (int s = 1; s < shares; ++s) {
                    const float *src = s_join + (s * quads + i) * 6;
                    const float t = __builtin_fmaxf(top, src[0]);
                    const float f = top == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((top - t) * a.c2);
                    const float e = src[0] == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((src[0] - t) * a.c2);
                    top = t;
                    l = l * f + src[1] * (src[0] == -__builtin_huge_valf() ? 1.0f : e);
                    o.x = o.x * f + src[2] * e;
                    o.y = o.y * f + src[3] * e;
                    o.z = o.z * f + src[4] * e;
                    o.w = o.w * f + src[5] * e;
                }
            }
        }
        if (mine && share == 0) {
            const int qi = i / kQuads, d = 4 * (i % kQuads);
            const float inv = 1.0f / l;
            *reinterpret_cast<uint2 *>(orow + qi * D + d) =
                make_uint2(pack2_scaled<BF16>(o.x, o.y, inv), pack2_scaled<BF16>(o.z, o.w, inv));
        }
    }
}

// chunk of keys per work-group, a multiple of kRound
int decode_chunk(int B, int Hq, int Hk, int max_len) {
    const int qblocks = (Hq / Hk + kCols - 1) / kCols;
    const int64_t units = (int64_t)B * Hk * qblocks;
    const int64_t want = (int64_t)device_cus() * 4;                         // work-groups
    if (units > (int64_t)(kArrivalBytes / 4)) return (max_len + kRound - 1) / kRound * kRound;   // one counter each
    const int64_t splits = std::min<int64_t>(64, std::max<int64_t>(1, want / units));
    const int64_t keys = (max_len + splits - 1) / splits;
    return (int)((std::max<int64_t>(keys, 2 * kRound) + kRound - 1) / kRound * kRound);
}

}  // namespace

size_t decode_attention_workspace_bytes(int B, int Hq, int Hk, int D, int max_len) {
    const int chunk = decode_chunk(B, Hq, Hk, max_len);
    const int64_t splits = (max_len + chunk - 1) / chunk;
    if (splits <= 1) return 0;
    const int64_t units = (int64_t)B * Hk * ((Hq / Hk + kCols - 1) / kCols);
    return kArrivalBytes + (size_t)(units * splits * kCols * (D + 2)) * 4;
}

hipError_t launch_decode_attention(p4q_dtype dt, int D, DecodeAttention a, void *ws, hipStream_t stream) {
    a.c2 = 1.4426950408889634f / __builtin_sqrtf((float)D);                 // log2(e) / sqrt(D)
    a.chunk = decode_chunk(a.B, a.Hq, a.Hk, a.max_len);
    a.G = a.Hq / a.Hk;
    const int splits = (a.max_len + a.chunk - 1) / a.chunk;
    if (splits > 1) {
        a.arrivals = static_cast<uint32_t *>(ws);
        a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + kArrivalBytes);
    }
    const dim3 grid((unsigned)splits, (unsigned)(a.Hk * ((a.G + kCols - 1) / kCols)), (unsigned)a.B);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid, dim3(64 * kWaves), 0, stream, a);
        return hipGetLastError();
    };
    if (dt == P4Q_BF16) return D == 128 ? go(k_decode_attention<true, 128>) : go(k_decode_attention<true, 64>);
    return D == 128 ? go(k_decode_attention<false, 128>) : go(k_decode_attention<false, 64>);
}

}  // namespace p4q
