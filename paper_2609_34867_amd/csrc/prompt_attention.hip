// Attention of whole prompts or of chunks of them: sequences of different lengths
// packed one behind the other, grouped heads, keys packed likewise or in the paged
// cache.  For sequence b with n tokens and m keys, query head h of key head
// hk = h / G (G = Hq / Hk) and token i:
//     O[i, h] = sum_j softmax_j(<q_ih, k_j,hk> / sqrt(D)) v_j,hk,
//     j <= i + m - n when causal (the last token sees the last key), else j < m;
// a token that sees no key gets zeros.
//
// The rows of a work-group are (token, query head of one group) pairs, 32 per
// wavefront and 128 in all, token by token: the G heads of a group read the same
// keys, so one pass over them serves all G, and short prompts fill the rows.  A
// wavefront's step over a tile of 64 keys is that of the causal prefill kernel
// (attention.hip): S^T = K Q^T on v_mfma_f32_32x32x16 with K from LDS and Q^T in
// registers, the softmax of a row within two lanes, O^T += V^T P^T with the weights
// straight from the S^T registers and V^T by transposing LDS reads; tiles go to
// LDS by DMA, two buffers, one barrier per tile.
//  * The DMA's descriptor is moved to each tile's rows (64 bits), so only a tile's
//    offsets have to fit 32; rows past the sequence's keys read as zeros whatever
//    lies there.  A wavefront fills 16 consecutive rows of a tile, which lie on one
//    page of a paged cache (16 rows or more), so a page costs a wavefront one table
//    entry per tile, fetched a tile ahead.
//  * Weights are rounded to the cache's type before they multiply v, as in the causal prefill
//    kernel; scores, maxima, sums and accumulators are fp32.  The outputs are then 1.2 to 1.4
//    times as far from the exact ones as rounding them alone would leave them (fp16 2.5 to
//    2.9 10^-4 for 2.1, bf16 2.0 to 2.3 10^-3 for 1.6, relative).  Weights in two pieces (as
//    decode attention has them, which waits for memory meanwhile) need half as many matrix
//    instructions again: 8191 tokens 700 us for 510, 16 ragged prompts 184 for 146, 10 x
//    577 at D = 64 46 for 38, 371 tokens 15.6 for 13.6.
//  * fp16 weights carry 2^7, which moves what they can hold (2^-24) that much further
//    below the largest.
// Lengths live on the device: the host launches T G / 128 + B row tiles per key
// head, which is never too few, and each work-group finds its sequence by a prefix
// sum over the lengths (64 at a time; 1024 sequences of 16 tokens, 32/8 heads, 167 us, 4096
// of them 1430).  Row tiles are numbered head by head, longest first, and each
// XCD takes a contiguous eighth of them, so that it reads few heads' keys.  With 8 heads or a
// multiple all XCDs then have as much to do; with others they do not (one prompt of 8191
// tokens: up to 1.5 times the mean at 4 heads, 1.7 at 2, 1.9 at 1, from the mapping).
//
// Few rows over many keys do not fill the device.  Then the keys of a row tile are
// split among work-groups, which leave unnormalized sums in the workspace; a second
// launch joins them in the order of the splits.
//
// One prompt of 8191 tokens, 32/8 heads, bf16: 490 to 530 us from card to card (1.04 to
// 1.12 PFLOP/s; a large library product reaches 1.40), single passes under the profiler 530 to
// 620.  Its MFMAs keep the matrix units busy for 55% of the cycles, vector instructions for 51%,
// and the clock is the power limit's: the same call on zeros takes 387 us.  A form that
// computes the next tile's scores under this tile's softmax needs a fifth fewer cycles and, at
// the lower clock that it is left, as much time.  16 prompts of 9 to 2003 tokens: 139 to 146
// us, 25 per work-group, of it 4 before the first tile (lengths, then
// rows and keys) and 1.8 per tile.  One of 371 tokens, 40 heads: 12.7 to 13.6 us, six tiles one after the
// other at 1.3 each.  Not kept, none faster: three tiles in flight; two key halves per row tile
// in one work-group (371 tokens 14.5 us); sequences in order of length (4 of 300 to 4000
// tokens, D = 64: 102 for 93 us).  D = 64 runs four wavefronts per SIMD (128 registers, 40
// sequences of 577 tokens, 20 heads, 108 us; three of them 117): vector instructions take 71%
// of the cycles, the matrix units 36%; 10 such sequences (33 to 38 us) 43% and 21%.
#include "attention_device.h"
#include "gemm_device.h"
#include "kv_cache.h"
#include "p4q_internal.h"
#include "wave_ops.h"

#include <algorithm>
#include <type_traits>

namespace p4q {
namespace {

constexpr int kNW = 4;                  // wavefronts per work-group
constexpr int kQW = 32;                 // rows per wavefront
constexpr int kQB = kNW * kQW;          // rows per work-group
constexpr int kKT = 64;                 // keys per tile
constexpr float kRescale = 8.0f;        // raise the running max past this margin (exp2 units)
constexpr float kFar = 1024.0f;         // largest maximum (exp2 units) whose rounding costs a weight less than 2^-14
constexpr int kSplitTiles = 4;          // a split has at least this many tiles, if the row tile has (us with 2, 4 and 8 of them:
                                        // 5 tokens over 4000 keys, 32/8 heads, 21.0, 18.4, 20.4; 60 over 1000
                                        // 20.5, 18.8, 22.8)
constexpr int kMaxSplits = 32;

// LDS placement of 16-byte chunk c of row r (D/8 chunks).  K: the rows that a
// fragment read takes together (16 of them, one chunk) fall in distinct banks; V:
// the four keys of a transposing read (64-byte pieces) fall in distinct banks.
template <int D>
__device__ __forceinline__ int k_slot(int r, int c) {
    return D == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int v_slot(int r, int c) {
    return D == 128 ? c ^ ((r & 3) << 2) : c ^ ((r & 2) << 1);
}

// A row tile: which sequence, which rows of it, which keys.
struct RowTile {
    int b;                              // sequence, or -1: nothing to do
    int first, n;                       // its tokens
    int r0, rows;                       // first row of the tile, rows of the sequence (n G)
    int kfirst, m;                      // its keys
    int cap;                            // those that the table can hold (PAGED), else m
    int ntiles;                         // tiles of 64 keys that the row tile sees
    int splits;                         // work-groups that share them
};

template <bool CAUSAL, bool PAGED>
__device__ __forceinline__ RowTile find_tile(const PromptAttention &a, int x, int lane) {
    auto by_g = [&](int r) __attribute__((always_inline)) { return magic_div(r, a.g_magic, a.g_shift); };
    RowTile t;
    t.b = -1;
    int before = 0;                     // row tiles of the sequences before this batch of 64
    for (int i = 0; i < a.B; i += 64) {
        // (lanes past the last sequence look at the last one's lists)
        const int b = min(i + lane, a.B - 1);
        const Span q = packed_span(a.cu_q[b], a.cu_q[b + 1], a.T);
        const Span k = PAGED ? Span{0, key_count(a.lens[b])} : packed_span(a.cu_k[b], a.cu_k[b + 1], a.Tk);
        const int n = i + lane < a.B ? q.last - q.first : 0;
        const int tiles = (int)(((uint32_t)n * (uint32_t)a.G + (uint32_t)(kQB - 1)) / (uint32_t)kQB);
        const int upto = before + (int)wave_inclusive_scan((uint32_t)tiles);
        const int at = __popcll(__ballot(upto <= x));   // sequences that end before tile x (they ascend)
        if (at < 64) {
            t.b = i + at;
            t.first = __builtin_amdgcn_readlane(q.first, at);
            t.n = __builtin_amdgcn_readlane(n, at);
            t.kfirst = __builtin_amdgcn_readlane(k.first, at);
            t.m = __builtin_amdgcn_readlane(k.last, at) - t.kfirst;
            t.cap = PAGED ? min(t.m, a.max_pages << a.shift) : t.m;
            t.rows = t.n * a.G;
            const int mine = __builtin_amdgcn_readlane(tiles, at), j = x - (__builtin_amdgcn_readlane(upto, at) - mine);
            t.r0 = (CAUSAL ? mine - 1 - j : j) * kQB;           // longest (causal) first
            break;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    if (t.b < 0) return t;
    const int last = min(t.r0 + kQB, t.rows) - 1;
    const int keys = CAUSAL ? min(t.cap, max(0, by_g(last) + 1 + (t.m - t.n))) : t.cap;
    t.ntiles = (keys + kKT - 1) / kKT;
    t.splits = max(1, min(min(a.splits, t.ntiles / kSplitTiles), (int)__builtin_sqrtf((float)t.ntiles * a.split_gain)));
    return t;
}

template <bool BF16, int D, bool CAUSAL, bool PAGED>
__global__ __launch_bounds__(64 * kNW, D == 64 ? 4 : 2) void k_prompt_attention(PromptAttention a) {
    constexpr int kRow = 2 * D;             // bytes of a K or V row
    constexpr int kOperand = kKT * kRow;
    constexpr int kTile = 2 * kOperand;     // K, then V
    constexpr int kSteps = D / 16;          // matrix steps of a key
    constexpr int kBlocks = D / 32;         // 32-value blocks of the output
    constexpr int kChunks = D / 8;          // 16-byte chunks of a row
    constexpr int kRpi = 64 / kChunks;      // rows per DMA instruction
    constexpr int NI = 16 / kRpi;           // DMA instructions per operand and wavefront (16 rows)
    constexpr float kBias = BF16 ? 0.0f : 7.0f;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * kTile];
    __shared__ int s_badkey[kNW];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 5, c32 = lane & 31;
    const int total = a.tiles * a.Hk * a.splits;
    const int wg = (int)(blockIdx.y * gridDim.x + blockIdx.x);
    if (wg >= total) return;
    const int logical = xcd_logical(wg, total);
    const int z = logical % a.splits, unit = logical / a.splits;
    const int hk = unit / a.tiles, x = unit - hk * a.tiles;
    const RowTile t = find_tile<CAUSAL, PAGED>(a, x, lane);
    if (t.b < 0 || z >= t.splits) return;
    const int per = (t.ntiles + t.splits - 1) / t.splits;
    const int kt0 = z * per, ktend = min(t.ntiles, kt0 + per);
    const int shift_rows = t.m - t.n;                       // causal: token i sees keys up to i + m - n

    // this wavefront's rows, and this lane's
    auto by_g = [&](int r) __attribute__((always_inline)) { return magic_div(r, a.g_magic, a.g_shift); };
    const int rw0 = t.r0 + kQW * wave;
    const int row = min(rw0 + c32, t.rows - 1);             // rows past the last take its query; not stored
    const int tok = by_g(row), hq = hk * a.G + (row - tok * a.G);
    const int seen = CAUSAL ? min(t.m, tok + 1 + shift_rows) : t.m;     // keys that this row sees (or <= 0)
    // keys that some row, or every row, of the wavefront sees
    const int wlast = min(rw0 + kQW, t.rows) - 1;
    const int most = rw0 >= t.rows ? 0 : CAUSAL ? max(0, min(t.cap, by_g(wlast) + 1 + shift_rows)) : t.cap;
    const int least = CAUSAL ? min(t.m, by_g(min(rw0, t.rows - 1)) + 1 + shift_rows) : t.m;

    // DMA of a tile: instruction n of a wavefront fills rows 16 wave + kRpi n + lane / kChunks of
    // the operand; slot lane % kChunks takes the chunk that k_slot / v_slot place there (both are
    // their own inverses).  Offsets count from the wavefront's first row.
    const int ldk2 = PAGED ? kRow : a.ldk * 2, ldv2 = PAGED ? kRow : a.ldv * 2;
    uint32_t vok[NI], vov[NI];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int r = kRpi * n + lane / kChunks;
        vok[n] = (uint32_t)r * (uint32_t)ldk2 + 16u * (uint32_t)k_slot<D>(16 * wave + r, lane & (kChunks - 1));
        vov[n] = (uint32_t)r * (uint32_t)ldv2 + 16u * (uint32_t)v_slot<D>(16 * wave + r, lane & (kChunks - 1));
    }
    const uint32_t lds0 = lds_addr(smem) + (uint32_t)(wave * NI * 1024);
    const int32_t *table = PAGED ? a.table + (int64_t)t.b * a.max_pages : nullptr;
    // the page of this wavefront's rows of tile kt (PAGED; a tile past the last: the last's)
    auto page_of = [&](int kt) __attribute__((always_inline)) {
        if constexpr (!PAGED) return 0;
        else {
            const int c = fetch_column(kt * kKT + 16 * wave, t.cap, a.shift);
            return c == kNoPage ? kNoPage : uniform_load(table, c);
        }
    };
    // (no tile kt: empty descriptors, nothing is read)
    auto issue = [&](bool isv, int kt, int page) __attribute__((always_inline)) {
        const int key0 = kt * kKT + 16 * wave;
        const int rows = kt < ktend ? min(16, t.m - key0) : 0;
        const int64_t base = PAGED ? page_row(page, a.Hk, hk, a.shift, key0 & ((1 << a.shift) - 1), D)
                                   : (int64_t)(t.kfirst + key0) * (isv ? a.ldv : a.ldk) + (int64_t)hk * D;
        const bool some = rows > 0 && page >= 0;
        const v4i d = buffer_desc((isv ? a.v : a.k) + (some ? base : 0),
                                  some ? (uint32_t)((rows - 1) * (isv ? ldv2 : ldk2) + kRow) : 0u);
#pragma unroll
        for (int n = 0; n < NI; ++n)
            dma16(d, isv ? vov[n] : vok[n], lds0 + (kt & 1) * kTile + (isv ? kOperand : 0) + n * 1024);
    };
    auto usable = [&](int entry) __attribute__((always_inline)) {
        return PAGED ? valid_page(__builtin_amdgcn_readfirstlane(entry), a.num_pages) : 0;
    };

    int page = usable(page_of(kt0));
    int ahead = page_of(kt0 + 1);
    issue(false, kt0, page);
    issue(true, kt0, page);
    // The row's Q^T operands.  The wait for them is placed here, behind the first
    // tile's loads: one that the compiler puts inside the loop would also wait for
    // the next tile's, which it cannot tell apart.
    uint4 qf[kSteps];
    const uint16_t *qrow = a.q + (int64_t)(t.first + tok) * a.ldq + (int64_t)hq * D + 8 * g;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) qf[s] = *reinterpret_cast<const uint4 *>(qrow + 16 * s);
    if constexpr (PAGED) {
        // the first key that lies on no page of the cache (rows that see it are NaN):
        // each wavefront looks at a quarter of the columns, under the first loads
        int bad = 0x7FFFFFFF;
        const int cols = (min(t.cap, ktend * kKT) + (1 << a.shift) - 1) >> a.shift;
        for (int c = ((kt0 * kKT) >> a.shift) + tid; c < cols; c += 64 * kNW)
            if (valid_page(table[c], a.num_pages) == kNoPage) bad = min(bad, max(kt0 * kKT, c << a.shift));
        if (t.m > t.cap) bad = min(bad, t.cap);
        if (__any((int)(bad != 0x7FFFFFFF)))
            for (int i = 1; i < 64; i <<= 1) bad = min(bad, __shfl_xor(bad, i));
        if (lane == 0) s_badkey[wave] = bad;
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(qf[s].x), "+v"(qf[s].y), "+v"(qf[s].z), "+v"(qf[s].w));

    v16f acc[kBlocks];
#pragma unroll
    for (int db = 0; db < kBlocks; ++db) acc[db] = v16f{};
    float mx = -__builtin_huge_valf(), lsum = 0.0f;

    // K fragment addresses: row 32 hf + c32 (its k_slot depends on c32 only)
    const uint32_t kofs = (uint32_t)(c32 * kRow);
    // V^T: lane reads 8 bytes of key 16 s + 8 e + 4 g + (lane % 16) / 4, d =
    // 32 db + 16 ((lane / 16) % 2) + 4 (lane % 4)
    const int vkey = 4 * g + ((lane & 15) >> 2);
    const uint32_t vofs = (uint32_t)(kOperand + vkey * kRow + 8 * (lane & 1));
    const int vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);

    // One tile of 64 keys from LDS buffer kt & 1.  NH = 1: only the first 32 keys
    // are seen by some row of the wavefront; the others are skipped, since weights
    // of 0 would still turn a non-finite row of V into NaN.  The next tile's loads
    // are issued on the way.
    auto tile_keys = [&](int kt, int next_page, auto nh_c) __attribute__((always_inline)) {
        constexpr int NH = decltype(nh_c)::value;
        const uint8_t *sb = smem + (kt & 1) * kTile;
        const int k0 = kt * kKT;
        auto k_read = [&](int hf, int s) __attribute__((always_inline)) {
            return *reinterpret_cast<const uint4 *>(sb + 32 * hf * kRow + kofs + 16u * (uint32_t)k_slot<D>(c32, 2 * s + g));
        };
        auto v_read = [&](int db, int s) __attribute__((always_inline)) {
            const uint8_t *p = sb + vofs + 16 * s * kRow + 16u * (uint32_t)v_slot<D>(vkey, 4 * db + vc);
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t)(p));
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t)(p + 8 * kRow));
            const uint2 u = __builtin_bit_cast(uint2, lo), w = __builtin_bit_cast(uint2, hi);
            return make_uint4(u.x, u.y, w.x, w.y);
        };
        // S^T = K Q^T: lane holds row c32, keys k0 + 32 hf + 8(r/4) + 4g + r%4
        v16f st[NH];
#pragma unroll
        for (int hf = 0; hf < NH; ++hf) st[hf] = v16f{};
        // K steps in batches of two, read two batches ahead
        uint4 kf[2][2][NH];
        auto k_batch = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int hf = 0; hf < NH; ++hf) kf[i & 1][j][hf] = k_read(hf, 2 * i + j);
        };
        k_batch(0);
        k_batch(1);
        issue(false, kt + 1, next_page);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kSteps / 2; ++i) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int hf = 0; hf < NH; ++hf) st[hf] = mfma<BF16>(kf[i & 1][j][hf], qf[2 * i + j], st[hf]);
            if (i + 2 < kSteps / 2) k_batch(i + 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        // V^T of the first 64 values: in flight during the softmax (D = 64: behind it,
        // for the registers that a fourth wavefront per SIMD needs)
        uint4 vf[2][2 * NH];
        auto v_first = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int db = 0; db < 2; ++db)
#pragma unroll
                for (int s = 0; s < 2 * NH; ++s) vf[db][s] = v_read(db, s);
        };
        if constexpr (D == 128) v_first();
        issue(true, kt + 1, next_page);
        __builtin_amdgcn_sched_barrier(0);
        // mask (only where the tile reaches past what every row sees; one
        // wave-uniform branch)
        if (k0 + 32 * NH > least) {
#pragma unroll
            for (int hf = 0; hf < NH; ++hf)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    st[hf][r] = k0 + 32 * hf + 8 * (r >> 2) + 4 * g + (r & 3) < seen ? st[hf][r] : -__builtin_huge_valf();
        }
        float tmax = -__builtin_huge_valf();
#pragma unroll
        for (int hf = 0; hf < NH; ++hf)
#pragma unroll
            for (int r = 0; r < 16; ++r) tmax = __builtin_fmaxf(tmax, st[hf][r]);
        tmax = xmax32(tmax);
        // raise the running max only past the margin (wave-uniform rescale)
        const bool raise = (tmax - mx) * a.c2 > kRescale || mx == -__builtin_huge_valf();
        if (__any((int)raise)) {
            const float mnew = raise ? tmax : mx;
            const float mref = (mnew == -__builtin_huge_valf()) ? 0.0f : mnew;
            const float alpha = (mx == -__builtin_huge_valf()) ? 0.0f : __builtin_amdgcn_exp2f((mx - mref) * a.c2);
            mx = mnew;
            lsum *= alpha;
#pragma unroll
            for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
        }
        // A weight is one fma and exp2: s c2 - mc.  That mc is rounded scales a row's weights
        // by 2^(up to |mc| 2^-24): nothing that shows while |mx| c2 <= kFar, but past 2^28 they
        // overflow, or vanish.  From rows whose maximum is that far off it is taken off first
        // (one wave-uniform branch; without it the call takes the same time, with a
        // subtraction for every score 1 to 8% more).
        const float off = __builtin_fmaxf(mx, -3.0e38f);    // (no score yet: all of them -inf)
        const bool far = __builtin_fabsf(off) * a.c2 > kFar;
        const float rest = far ? off : 0.0f, mc = (off - rest) * a.c2 - kBias;
        if (__any((int)far)) {
#pragma unroll
            for (int hf = 0; hf < NH; ++hf)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[hf][r] -= rest;
        }
        float psum = 0.0f;
        uint4 pb[NH][2];
#pragma unroll
        for (int hf = 0; hf < NH; ++hf) {
            uint32_t pw[8];
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[hf][r], a.c2, -mc));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[hf][r + 1], a.c2, -mc));
                psum += p0 + p1;
                pw[r >> 1] = pack2<BF16>(p0, p1);
            }
            pb[hf][0] = make_uint4(pw[0], pw[1], pw[2], pw[3]);
            pb[hf][1] = make_uint4(pw[4], pw[5], pw[6], pw[7]);
        }
        lsum += psum;                                       // this lane's half; joined at the end
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (D == 64) v_first();
        // O^T += V^T P^T (steps of 16 keys), each block's operands read two
        // blocks ahead
#pragma unroll
        for (int db = 0; db < kBlocks; ++db) {
#pragma unroll
            for (int s = 0; s < 2 * NH; ++s) acc[db] = mfma<BF16>(vf[db & 1][s], pb[s >> 1][s & 1], acc[db]);
            if (db + 2 < kBlocks)
#pragma unroll
                for (int s = 0; s < 2 * NH; ++s) vf[db & 1][s] = v_read(db + 2, s);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // tiles past `most` hold only masked keys: the wavefront loads its share of
    // them and keeps the barriers (one per tile either way)
    const int nlive = min(ktend, (most + kKT - 1) / kKT);
    // tile kt has landed from every wavefront, and every wavefront is done
    // with tile kt - 1, whose buffer the loads of tile kt + 1 overwrite
    auto arrive = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory"); };
    const bool half = nlive * kKT == ((most + kKT - 1) & ~(kKT - 1)) && nlive > kt0 && most - (nlive - 1) * kKT <= 32;
    int kt = kt0;
    for (; kt < nlive - (int)half; ++kt) {
        arrive();
        page = usable(ahead);
        ahead = page_of(kt + 2);
        tile_keys(kt, page, std::integral_constant<int, 2>{});
    }
    if (half) {
        arrive();
        page = usable(ahead);
        ahead = page_of(kt + 2);
        tile_keys(kt, page, std::integral_constant<int, 1>{});
        ++kt;
    }
    for (; kt < ktend; ++kt) {
        arrive();
        page = usable(ahead);
        ahead = page_of(kt + 2);
        issue(false, kt + 1, page);
        issue(true, kt + 1, page);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // every wavefront is done with the tiles
    lsum = xsum32(lsum);
    if (PAGED && seen > min(min(s_badkey[0], s_badkey[1]), min(s_badkey[2], s_badkey[3]))) lsum = __builtin_nanf("");

    if (t.splits > 1) {
        // unnormalized sums, maximum and sum of every row, for the joining launch
        float *part = a.part + (int64_t)(unit * a.splits + z) * kQB * (D + 2);
        float *dst = part + (int64_t)(kQW * wave + c32) * D + 4 * g;
        if (rw0 + c32 >= t.rows) return;
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<float4 *>(dst + 32 * db + 8 * j) =
                    make_float4(acc[db][4 * j], acc[db][4 * j + 1], acc[db][4 * j + 2], acc[db][4 * j + 3]);
        if (g == 0) {
            float2 *ml = reinterpret_cast<float2 *>(part + kQB * D) + kQW * wave + c32;
            *ml = make_float2(mx, lsum);
        }
        return;
    }

    // O[row][d] = acc / lsum; register r of block db holds d = 32 db + 8(r/4) +
    // 4g + r%4.  The wavefront's 32 rows pass through LDS (8-byte unit u of row r at
    // u ^ 2 (r % kChunks)) and leave as whole rows.
    const float inv = 1.0f / lsum;
    uint8_t *stg = smem + wave * (kQW * kRow);
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int u = 8 * db + 2 * j + g;
            uint2 w = make_uint2(pack2_scaled<BF16>(acc[db][4 * j], acc[db][4 * j + 1], inv),
                                 pack2_scaled<BF16>(acc[db][4 * j + 2], acc[db][4 * j + 3], inv));
            if (seen <= 0) w = make_uint2(0, 0);
            *reinterpret_cast<uint2 *>(stg + c32 * kRow + 8 * (u ^ ((c32 & (kChunks - 1)) << 1))) = w;
        }
#pragma unroll
    for (int s = 0; s < kQW / kRpi; ++s) {
        const int r = kRpi * s + lane / kChunks, rr = rw0 + r;
        const uint4 w = *reinterpret_cast<const uint4 *>(stg + r * kRow + 16 * ((lane & (kChunks - 1)) ^ (r & (kChunks - 1))));
        if (rr < t.rows) {
            const int i = by_g(rr), h = hk * a.G + (rr - i * a.G);
            uint16_t *dst = a.out + (int64_t)(t.first + i) * a.ldo + (int64_t)h * D + 8 * (lane & (kChunks - 1));
            __builtin_nontemporal_store(__builtin_bit_cast(v4i, w), reinterpret_cast<v4i *>(dst));
        }
    }
}

// Joins the splits of a row tile: 32 rows per work-group, D / 4 threads per row.
template <bool BF16, int D, bool CAUSAL, bool PAGED>
__global__ __launch_bounds__(256) void k_prompt_join(PromptAttention a) {
    constexpr int kLanes = D / 4;
    const int lane = threadIdx.x & 63;
    const int unit = (int)blockIdx.x, hk = unit / a.tiles;
    const RowTile t = find_tile<CAUSAL, PAGED>(a, unit - hk * a.tiles, lane);
    if (t.b < 0 || t.splits <= 1) return;
    const int d = 4 * ((int)threadIdx.x % kLanes);
    for (int r = (int)blockIdx.y * 32 + (int)threadIdx.x / kLanes; r < ((int)blockIdx.y + 1) * 32; r += 256 / kLanes) {
        const int row = t.r0 + r;
        if (row >= t.rows) return;
        float top = -__builtin_huge_valf(), l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int z = 0; z < t.splits; ++z) {
            const float *part = a.part + (int64_t)(unit * a.splits + z) * kQB * (D + 2);
            const float2 ml = reinterpret_cast<const float2 *>(part + kQB * D)[r];
            const float4 x = *reinterpret_cast<const float4 *>(part + (int64_t)r * D + d);
            const float m = __builtin_fmaxf(top, ml.x);
            const float f = top == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((top - m) * a.c2);
            const float e = ml.x == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f((ml.x - m) * a.c2);
            top = m;
            l = l * f + ml.y * (ml.x == -__builtin_huge_valf() ? 1.0f : e);   // (no key: 0, or NaN)
            o.x = o.x * f + x.x * e;
            o.y = o.y * f + x.y * e;
            o.z = o.z * f + x.z * e;
            o.w = o.w * f + x.w * e;
        }
        const int i = magic_div(row, a.g_magic, a.g_shift), h = hk * a.G + (row - i * a.G);
        const int seen = CAUSAL ? i + 1 + (t.m - t.n) : t.m;
        const float inv = 1.0f / l;
        uint2 w = make_uint2(pack2_scaled<BF16>(o.x, o.y, inv), pack2_scaled<BF16>(o.z, o.w, inv));
        if (seen <= 0) w = make_uint2(0, 0);
        *reinterpret_cast<uint2 *>(a.out + (int64_t)(t.first + i) * a.ldo + (int64_t)h * D + d) = w;
    }
}

// row tiles per key head, never fewer than the sequences have
int64_t row_tiles(int T, int B, int G) { return (int64_t)T * G / kQB + B; }

// What a split saves is the time of the tiles, about 1.3 us each; what it costs is the
// join: 33 ns per row tile and split to write and read the sums.  The sum of both
// is least at sqrt(tiles * gain) splits.  32/8 heads, us with a quarter of this gain, with it,
// with four times as much, and unsplit: 5 tokens over 20000 keys 33.6, 33.6, 33.5, 324; 60 over 4000
// 30.9, 31.1, 34.2, 78; 300 over 4000 57, 45, 44, 82; 300 over 1000 29.0, 29.2, 31.9, 30.0; 1000
// over 1000 earlier ones 46, 55, 46, 47, where it costs most; 1000 over 20000 340, 338, 336, 383.
float split_gain(int T, int Hq) { return 40.0f * kQB / ((float)T * (float)Hq); }

// work-groups that share the keys of a row tile, at most
int prompt_splits(int T, int B, int Hq, int Hk, int64_t most_keys) {
    const int64_t tiles = (most_keys + kKT - 1) / kKT, units = row_tiles(T, B, Hq / Hk) * Hk;
    const int64_t best = (int64_t)__builtin_sqrtf((float)tiles * split_gain(T, Hq));
    return (int)std::max<int64_t>(1, std::min<int64_t>({2 * device_cus() / units, tiles / kSplitTiles, best, (int64_t)kMaxSplits}));
}

}  // namespace

size_t prompt_attention_workspace_bytes(int T, int B, int Hq, int Hk, int D, int64_t most_keys) {
    const int64_t units = row_tiles(T, B, Hq / Hk) * Hk;
    const int splits = prompt_splits(T, B, Hq, Hk, most_keys);
    return splits > 1 ? (size_t)(units * splits * kQB * (D + 2)) * 4 : 0;
}

hipError_t launch_prompt_attention(p4q_dtype dt, int D, PromptAttention a, int causal, int64_t most_keys, void *ws,
                                   size_t ws_bytes, hipStream_t stream) {
    a.c2 = 1.4426950408889634f / __builtin_sqrtf((float)D);                 // log2(e) / sqrt(D)
    a.G = a.Hq / a.Hk;
    const Magic g = magic_of(a.G);
    a.g_magic = g.m, a.g_shift = g.shift;
    const int64_t tiles = row_tiles(a.T, a.B, a.G), units = tiles * a.Hk;
    a.splits = prompt_splits(a.T, a.B, a.Hq, a.Hk, most_keys);
    a.split_gain = split_gain(a.T, a.Hq);
    if (ws_bytes < prompt_attention_workspace_bytes(a.T, a.B, a.Hq, a.Hk, D, most_keys)) a.splits = 1;
    a.part = static_cast<float *>(ws);
    if (units * a.splits > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    a.tiles = (int)tiles;
    const int64_t total = units * a.splits, wrap = 1 << 20;
    auto go = [&](auto dc, auto bf, auto cs, auto pg) {
        constexpr int kDim = decltype(dc)::value;
        constexpr bool kBf = decltype(bf)::value, kCausal = decltype(cs)::value, kPaged = decltype(pg)::value;
        hipLaunchKernelGGL((k_prompt_attention<kBf, kDim, kCausal, kPaged>),
                           dim3((unsigned)std::min(total, wrap), (unsigned)((total + wrap - 1) / wrap)), dim3(64 * kNW),
                           0, stream, a);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && a.splits > 1) {
            hipLaunchKernelGGL((k_prompt_join<kBf, kDim, kCausal, kPaged>), dim3((unsigned)units, kQB / 32), dim3(256), 0,
                               stream, a);
            e = hipGetLastError();
        }
        return e;
    };
    auto d = [&](auto bf, auto cs, auto pg) {
        return D == 128 ? go(std::integral_constant<int, 128>{}, bf, cs, pg) : go(std::integral_constant<int, 64>{}, bf, cs, pg);
    };
    auto c = [&](auto bf, auto pg) { return causal ? d(bf, std::true_type{}, pg) : d(bf, std::false_type{}, pg); };
    auto p = [&](auto bf) { return a.table ? c(bf, std::true_type{}) : c(bf, std::false_type{}); };
    return dt == P4Q_BF16 ? p(std::true_type{}) : p(std::false_type{});
}

}  // namespace p4q
