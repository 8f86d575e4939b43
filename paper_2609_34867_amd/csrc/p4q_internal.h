// Internal launchers behind the C ABI (include/p4q.h).  Arguments have been
// validated by the caller; each launcher only enqueues kernels on `stream`
// and returns the launch status.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

#include "../../include/p4q.h"

namespace p4q {

// ---- per-device constants -----------------------------------------------------
// Launch shapes depend on the device's CU count and on how many blocks of a
// kernel fit on a CU.  Both are fixed for a device, so they are queried once
// per device ordinal and kept in a cache of atomics: concurrent first calls
// from several host threads each store the same value, and no other state
// is shared between calls.
constexpr int kMaxDevices = 64;

inline int current_device() {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) dev = 0;
    return dev;
}

// cached value of query() for the current device; query() returns > 0
template <class Query>
inline int per_device_cached(std::atomic<int> (&cache)[kMaxDevices], Query query) {
    const int dev = current_device();
    if (dev >= kMaxDevices) return query(dev);
    int v = cache[dev].load(std::memory_order_relaxed);
    if (v <= 0) {
        v = query(dev);
        cache[dev].store(v, std::memory_order_relaxed);
    }
    return v;
}

// compute units of the current device (256 on MI355X if the query fails)
inline int device_cus() {
    static std::atomic<int> cache[kMaxDevices];
    return per_device_cached(cache, [](int dev) {
        int cus = 0;
        if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
            cus <= 0)
            cus = 256;
        return cus;
    });
}

// ---- quantize + pack (Q4 per row) ------------------------------------------
hipError_t launch_quant_act(p4q_dtype dt, int M, int K_in, const void *x, int64_t ldx,
                            float clip, uint8_t *codes, float *scales, hipStream_t stream);

// ---- fused prologue: per-token Q4 of RMSNorm(x) * gamma ------------------------
hipError_t launch_rmsnorm_quant(p4q_dtype dt, int M, int d, const void *x, int64_t ldx,
                                const void *gamma, float eps, float clip, uint8_t *codes,
                                float *scales, hipStream_t stream);

// ---- MXFP4: rows of 4-bit floats with one power of two per 32 ------------------
// (mx4_device.h has the format.)  Fields behind `set by the launcher` are the
// kernels' own.
hipError_t launch_quant_mx4(p4q_dtype dt, int M, int K, const void *x, int64_t ldx, uint8_t *codes,
                            uint8_t *scales, void *values, int64_t ldv, hipStream_t stream);

// bytes of a row of scales: one byte per 32 values, padded to 16 bytes so that
// rows start aligned and 512 values of a product find their 16 bytes
__host__ __device__ inline int64_t mx4_scale_stride(int64_t K) { return (K + 511) / 512 * 16; }

struct ResidualNorm {
    int M, d;
    const uint16_t *x, *r, *post, *gate, *gamma;     // r, post and gate may be null
    int64_t ldx, ldr;
    float alpha, eps, clip;
    uint16_t *h_out;                                 // given iff r is
    int64_t ldh;
    uint8_t *codes;
    void *scales;                                    // fp32 [M], or bytes [M, stride]
    uint16_t *values;                                // may be null
    int64_t ldv;
    // set by the launcher
    int64_t scale_stride;
};
hipError_t launch_residual_rmsnorm_quant(p4q_dtype dt, p4q_norm_format fmt, ResidualNorm a, hipStream_t stream);

struct Mx4Product {
    int M, N, K;                                     // N: outputs (gated: half the weight's rows)
    const uint8_t *a, *as, *w, *ws;                  // codes and scale bytes
    void *y;
    int64_t ldy;
    uint8_t *codes, *scales;                         // gated and quantized: instead of y
    // set by the launcher
    int64_t in_stride, out_stride;                   // bytes of a row of scales
    bool wide;                                       // y's rows begin at halves of cache lines
};
hipError_t launch_mx4_linear(p4q_dtype out_dt, Mx4Product p, hipStream_t stream);
hipError_t launch_mx4_gated(p4q_dtype out_dt, Mx4Product p, hipStream_t stream);

// ---- attention prefill (FP16 / BF16 Q, K, V; head dimension 128) -------------
hipError_t launch_attention(p4q_dtype dt, int B, int L, int H, const void *q, const void *k,
                            const void *v, int64_t ld, void *o, int64_t ldo, int causal,
                            hipStream_t stream);

// ---- serving: the paged key-value cache and the attention that reads it --------
// (kv_cache.h has the layout; `shift` is log2 of the page size.)  Fields behind
// `set by the launcher` are the kernels' own.
struct RopeAppend {
    int T, B, Hq, Hk;
    const uint16_t *q, *k, *v;
    int64_t ldq, ldk, ldv;
    const int32_t *cu, *cache_lens, *positions;      // the last two may be null
    uint16_t *q_out, *k_out;                         // k_out may be null
    int64_t ldqo, ldko;
    uint16_t *k_cache, *v_cache;
    int num_pages, shift, max_pages;
    const int32_t *table;
    // set by the launcher
    int parts;                                       // wavefronts per token
    double log2_ratio;                               // log2(theta_1 / theta_0)
};
hipError_t launch_rope_append(p4q_dtype dt, int D, RopeAppend a, float rope_base, hipStream_t stream);

struct PromptAttention {
    int T, Tk, B, Hq, Hk;
    const uint16_t *q, *k, *v;                       // k and v: packed rows, or the caches
    int64_t ldq, ldo;
    int ldk, ldv;                                    // packed
    const int32_t *cu_q, *cu_k;                      // cu_k: packed
    const int32_t *lens, *table;                     // the cache's (table null: packed)
    int num_pages, shift, max_pages;
    uint16_t *out;
    // set by the launcher
    int G, tiles, splits;
    uint32_t g_magic;                                // division by G (kv_cache.h)
    int g_shift;
    float c2, split_gain;
    float *part;
};
// most_keys: a bound of the keys of a sequence
size_t prompt_attention_workspace_bytes(int T, int B, int Hq, int Hk, int D, int64_t most_keys);
hipError_t launch_prompt_attention(p4q_dtype dt, int D, PromptAttention a, int causal, int64_t most_keys, void *ws,
                                   size_t ws_bytes, hipStream_t stream);

struct DecodeAttention {
    int B, Hq, Hk, max_len;
    const uint16_t *q, *k, *v;                       // k and v: the caches
    int64_t ldq, ldo;
    const int32_t *lens, *table;
    int num_pages, shift, max_pages;
    uint16_t *out;
    // set by the launcher
    int G, cus;
    float c2;
    uint32_t *arrivals;
    float *part;
};
size_t decode_attention_workspace_bytes(int B, int Hq, int Hk, int D, int max_len);
hipError_t launch_decode_attention(p4q_dtype dt, int D, DecodeAttention a, void *ws, hipStream_t stream);

// ---- selector ---------------------------------------------------------------
struct SelectWorkspace {
    int32_t *stats;      // [B][N][J+1]: D_0..D_{J-1}, Nv   (documented)
    int64_t *keys;       // [B][J][N]: exact order keys (internal)
    uint32_t *vcodes = nullptr;   // [B][N][d/8] packed visual codes, or none
};

// the three-stage selector's workspace: the above, then
struct SelectFullWorkspace {
    SelectWorkspace sel;    // vcodes set
    int32_t *gram;          // [B][N][N] code Gram matrices (exact int32)
    int64_t *mp;            // [kDivInitPlanes][B][N] partial maxima over the kept
    int32_t *mq;            //        set, as pairs (p, q) (see diversity.hip)
    int32_t *stages;        // [B][K] stage picks when the caller gives none
};
size_t select_full_workspace_bytes(int B, int N, int d, int J, int K);
SelectFullWorkspace select_full_workspace_carve(void *ws, int B, int N, int d, int J, int K);
size_t select_workspace_bytes(int B, int N, int d, int J);
SelectWorkspace select_workspace_carve(void *ws, int B, int N, int d, int J);

hipError_t launch_select(p4q_dtype dt, int B, int N, int d, const void *vis,
                         const void *concepts, int J, const void *text, int T, int K,
                         float clip, int32_t *idx_out, void *tokens_out,
                         const SelectWorkspace &ws, hipStream_t stream);

hipError_t launch_select_full(p4q_dtype dt, int B, int N, int d, const void *vis,
                              const void *concepts, int J, const float *cls_attn,
                              const void *text, int T, int K, int kq, int ks, float clip,
                              int32_t *idx_out, int32_t *stages_out, void *tokens_out,
                              const SelectFullWorkspace &ws, hipStream_t stream);

constexpr int kDivInitPlanes = 8;

// Visual Diversity completion (diversity.hip): n0 = kq + ks tokens already
// in stages[b][0, n0); kd greedy picks appended there in pick order;
// idx_out[b][0, K) = all K kept tokens, ascending.
hipError_t launch_diversity(int B, int N, int K, int n0, int kd, const int32_t *gram,
                            const float *cls_attn, int64_t *mp, int32_t *mq, int32_t *stages,
                            int32_t *idx_out, hipStream_t stream);

// ---- calibration mechanics (calib.hip) ---------------------------------------
hipError_t launch_quant_scaled(p4q_dtype dt, int R, int K, const void *z, int64_t ldz,
                               const float *sigma, int divide, float clip, const float *clip_rows,
                               uint8_t *codes, float *scales, float *absmax, int32_t *kstar,
                               hipStream_t stream);
size_t calib_linear_workspace_bytes(int M, int N, int K);
hipError_t launch_calib_linear(p4q_dtype dt, int M, int N, int K, const void *x, int64_t ldx,
                               const void *w, int64_t ldw, const float *target, int64_t ldt,
                               const float *sigma, float clip_a, const float *clip_w,
                               float *loss, float *grad_sigma, float *grad_clip_a,
                               float *grad_clip_w, void *ws, hipStream_t stream);

size_t calib_block_workspace_bytes(int M, int d, int f, int H);
hipError_t launch_calib_block(int M, int d, int f, int H, const void *x, const float *target,
                              int64_t ldt, const void *w_qkv, const void *w_o, const void *w_gu,
                              const void *w_down, const void *gamma1, const void *gamma2,
                              float eps, float rope_base, const float *sigma, const float *clip_a,
                              const float *clip_w, float *loss, float *grad_sigma,
                              float *grad_clip_a, float *grad_clip_w, void *ws,
                              hipStream_t stream);

// ---- W4A4 GEMM ---------------------------------------------------------------
// G_b = C_b C_b^T for b < B, C_b = codes + b * n * (k/2) packed [n, k/2];
// G int32 [B][n][n].
hipError_t launch_code_gram(int B, int n, int k, const uint8_t *codes, int32_t *G,
                            hipStream_t stream);
size_t gemm_workspace_bytes(int M, int N, int K);
// Zeroes the arrival counters at the head of a GEMM workspace (a fill kernel
// on the stream; the GEMM calls leave them zero, so this is needed once per
// workspace whose contents are not known to be zero).
hipError_t gemm_workspace_clear(void *ws, size_t ws_bytes, hipStream_t stream);
hipError_t launch_w4a4_gemm(int M, int N, int K, const uint8_t *a, const float *sa,
                            const uint8_t *w, const float *sw, p4q_dtype out_dt, void *y,
                            int64_t ldy, int32_t *acc_out, void *ws, size_t ws_bytes,
                            hipStream_t stream);

// The same on the 6-bit matrix instructions (w4a4_f6.hip): ws holds
// gemm_f6_bytes(M, N, K) bytes, 16-byte aligned.
size_t gemm_f6_bytes(int M, int N, int K);
hipError_t launch_w4a4_gemm_f6(int M, int N, int K, const uint8_t *a, const float *sa,
                               const uint8_t *w, const float *sw, p4q_dtype out_dt, void *y,
                               int64_t ldy, int32_t *acc_out, void *ws, hipStream_t stream);

// ---- diagnostics (diag.hip) ----------------------------------------------------
hipError_t launch_diag_mfma_i8(int blocks, int iters, int32_t *out, hipStream_t stream);
hipError_t launch_diag_read(const void *src, size_t bytes, int blocks, uint32_t *out,
                            hipStream_t stream);

}  // namespace p4q
