// C ABI of libp4q (declared in include/p4q.h): argument validation, workspace
// sizing and dispatch.  Every check runs on the host before any HIP call, so a
// rejected call enqueues nothing; launch failures map to P4Q_ERR_HIP.
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "kv_cache.h"
#include "overlap.h"
#include "p4q_internal.h"

namespace {

thread_local char g_last_error[512] = "";

int fail(int status, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return status;
}

int ok() {
    g_last_error[0] = '\0';
    return P4Q_OK;
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

bool valid_dtype(int dt) { return dt == P4Q_FP16 || dt == P4Q_BF16; }

// clip in [2^-16, 1]; NaN fails both comparisons
bool valid_clip(float c) { return c >= 0x1p-16f && c <= 1.0f; }

int hip_status(hipError_t e, const char *what) {
    if (e != hipSuccess)
        return fail(P4Q_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

}  // namespace

extern "C" {

const char *p4q_version(void) { return "p4q 0.1.0 gfx950"; }

const char *p4q_status_string(int status) {
    switch (status) {
        case P4Q_OK: return "P4Q_OK";
        case P4Q_ERR_INVALID_ARG: return "P4Q_ERR_INVALID_ARG";
        case P4Q_ERR_UNSUPPORTED: return "P4Q_ERR_UNSUPPORTED";
        case P4Q_ERR_WORKSPACE: return "P4Q_ERR_WORKSPACE";
        case P4Q_ERR_HIP: return "P4Q_ERR_HIP";
        default: return "P4Q_ERR_UNKNOWN";
    }
}

const char *p4q_last_error(void) { return g_last_error; }

// the selector's size limits (outside them p4q_select rejects the call)
static bool select_shape_ok(int B, int N, int d, int J) {
    return B > 0 && N > 0 && N <= 8192 && d >= 32 && d <= 16384 && d % 32 == 0 && J > 0 &&
           J <= 8 && !(J > 4 && d > 8192);
}

size_t p4q_select_workspace_bytes(int B, int N, int d, int J) {
    if (!select_shape_ok(B, N, d, J)) return 0;
    return p4q::select_workspace_bytes(B, N, d, J);
}

// Checks shared by p4q_select and p4q_select_noalloc: everything but the
// workspace.  Returns P4Q_OK or the failing status (message recorded).
static int check_select_args(const char *who, p4q_dtype dt, int B, int N, int d,
                             const void *vis, const void *concepts, int J, const void *text,
                             int T, int K, float clip, const int32_t *idx_out,
                             const void *tokens_out) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "%s: dtype %d", who, (int)dt);
    if (B <= 0 || N <= 0 || d <= 0 || J <= 0 || K <= 0 || T < 0)
        return fail(P4Q_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d N=%d d=%d J=%d K=%d T=%d)",
                    who, B, N, d, J, K, T);
    if (K > N) return fail(P4Q_ERR_INVALID_ARG, "%s: K=%d > N=%d", who, K, N);
    if (!vis || !concepts || !idx_out || !tokens_out)
        return fail(P4Q_ERR_INVALID_ARG, "%s: null pointer", who);
    if ((T > 0) != (text != nullptr))
        return fail(P4Q_ERR_INVALID_ARG, "%s: text must be given iff T > 0", who);
    if (!valid_clip(clip)) return fail(P4Q_ERR_INVALID_ARG, "%s: clip %g outside [2^-16, 1]", who, clip);
    if (d % 32 != 0) return fail(P4Q_ERR_INVALID_ARG, "%s: d=%d not a multiple of 32", who, d);
    if (!aligned(vis, 16) || !aligned(concepts, 16) || !aligned(tokens_out, 16) ||
        (text && !aligned(text, 16)) || !aligned(idx_out, 4))
        return fail(P4Q_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    if (N > 8192) return fail(P4Q_ERR_UNSUPPORTED, "%s: N=%d > 8192", who, N);
    if (J > 8) return fail(P4Q_ERR_UNSUPPORTED, "%s: J=%d > 8", who, J);
    if (d > 16384) return fail(P4Q_ERR_UNSUPPORTED, "%s: d=%d > 16384", who, d);
    if (J > 4 && d > 8192) return fail(P4Q_ERR_UNSUPPORTED, "%s: J > 4 needs d <= 8192", who);
    return P4Q_OK;
}

int p4q_select(p4q_dtype dt, int B, int N, int d, const void *vis, const void *concepts, int J,
               const void *text, int T, int K, float clip, int32_t *idx_out, void *tokens_out,
               void *ws, size_t ws_bytes, hipStream_t stream) {
    if (const int st = check_select_args("p4q_select", dt, B, N, d, vis, concepts, J, text, T, K,
                                         clip, idx_out, tokens_out))
        return st;
    const size_t need = p4q::select_workspace_bytes(B, N, d, J);
    if (!ws || ws_bytes < need)
        return fail(P4Q_ERR_WORKSPACE, "p4q_select: workspace %zu < %zu bytes", ws_bytes, need);
    if (!aligned(ws, 256)) return fail(P4Q_ERR_INVALID_ARG, "p4q_select: workspace not 256-byte aligned");
    const p4q::SelectWorkspace w = p4q::select_workspace_carve(ws, B, N, d, J);
    return hip_status(p4q::launch_select(dt, B, N, d, vis, concepts, J, text, T, K, clip, idx_out,
                                         tokens_out, w, stream),
                      "p4q_select");
}

}  // extern "C"

// ---- the selector without a caller-supplied workspace ------------------------
// Its workspace lives in `scratch`, one array per device in the library's
// device image.  In host code the name `scratch` is only a stand-in for the
// symbol: its device address is looked up (hipGetSymbolAddress) once per
// device, with that device current, and only that address is ever passed on.
static __device__ __align__(256) uint8_t scratch[P4Q_SELECT_SCRATCH_BYTES];

namespace {

std::atomic<uintptr_t> g_scratch_addr[p4q::kMaxDevices];

// Device address of `scratch` on the device `stream` belongs to (the
// caller's current device for the null stream).  Returns P4Q_OK or an error
// status with the message recorded.
int scratch_address(hipStream_t stream, void **addr, const char *who) {
    int dev = 0, cur = 0;
    hipError_t e = hipGetDevice(&cur);
    if (e == hipSuccess) {
        dev = cur;
        if (stream) e = hipStreamGetDevice(stream, &dev);
    }
    if (e != hipSuccess) return fail(P4Q_ERR_HIP, "%s: device of the stream: %s", who, hipGetErrorString(e));
    if (dev < 0 || dev >= p4q::kMaxDevices)
        return fail(P4Q_ERR_UNSUPPORTED, "%s: device %d beyond the %d supported", who, dev, p4q::kMaxDevices);
    uintptr_t a = g_scratch_addr[dev].load(std::memory_order_acquire);
    if (a == 0) {
        // with that device current: each device holds its own copy of the array
        if (dev != cur && (e = hipSetDevice(dev)) != hipSuccess)
            return fail(P4Q_ERR_HIP, "%s: hipSetDevice(%d): %s", who, dev, hipGetErrorString(e));
        void *p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        const hipError_t e2 = (dev != cur) ? hipSetDevice(cur) : hipSuccess;
        if (e != hipSuccess || p == nullptr)
            return fail(P4Q_ERR_HIP, "%s: hipGetSymbolAddress(scratch): %s", who,
                        hipGetErrorString(e != hipSuccess ? e : hipErrorInvalidSymbol));
        if (e2 != hipSuccess)
            return fail(P4Q_ERR_HIP, "%s: hipSetDevice(%d): %s", who, cur, hipGetErrorString(e2));
        a = reinterpret_cast<uintptr_t>(p);
        g_scratch_addr[dev].store(a, std::memory_order_release);   // racing first calls store the same
    }
    *addr = reinterpret_cast<void *>(a);
    return P4Q_OK;
}

}  // namespace

extern "C" {

int p4q_select_noalloc(p4q_dtype dt, int B, int N, int d, const void *vis, const void *concepts,
                       int J, const void *text, int T, int K, float clip, int32_t *idx_out,
                       void *tokens_out, hipStream_t stream) {
    if (const int st = check_select_args("p4q_select_noalloc", dt, B, N, d, vis, concepts, J, text,
                                         T, K, clip, idx_out, tokens_out))
        return st;
    const size_t need = p4q::select_workspace_bytes(B, N, d, J);
    if (need > (size_t)P4Q_SELECT_SCRATCH_BYTES)
        return fail(P4Q_ERR_WORKSPACE,
                    "p4q_select_noalloc: B=%d N=%d d=%d J=%d needs %zu bytes of scratch, more than "
                    "the %zu the library holds per device (use p4q_select with a workspace)",
                    B, N, d, J, need, (size_t)P4Q_SELECT_SCRATCH_BYTES);
    void *ws = nullptr;
    if (const int st = scratch_address(stream, &ws, "p4q_select_noalloc")) return st;
    const p4q::SelectWorkspace w = p4q::select_workspace_carve(ws, B, N, d, J);
    return hip_status(p4q::launch_select(dt, B, N, d, vis, concepts, J, text, T, K, clip, idx_out,
                                         tokens_out, w, stream),
                      "p4q_select_noalloc");
}

size_t p4q_select_full_workspace_bytes(int B, int N, int d, int J, int K) {
    if (!select_shape_ok(B, N, d, J) || d > 8192 || K <= 0 || K > N) return 0;
    return p4q::select_full_workspace_bytes(B, N, d, J, K);
}

int p4q_select_budgets(int K, int *kq, int *ks, int *kd) {
    if (K < 0 || !kq || !ks || !kd) return fail(P4Q_ERR_INVALID_ARG, "p4q_select_budgets: K=%d or null output", K);
    *kq = (int)((int64_t)K * 3 / 10);
    *ks = (int)((int64_t)K * 2 / 10);
    *kd = K - *kq - *ks;
    return ok();
}

int p4q_select_full(p4q_dtype dt, int B, int N, int d, const void *vis, const void *concepts, int J,
                    const float *cls_attn, const void *text, int T, int K, int kq, int ks, float clip,
                    int32_t *idx_out, int32_t *stages_out, void *tokens_out, void *ws, size_t ws_bytes,
                    hipStream_t stream) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "p4q_select_full: dtype %d", (int)dt);
    if (B <= 0 || N <= 0 || d <= 0 || J <= 0 || K <= 0 || T < 0)
        return fail(P4Q_ERR_INVALID_ARG,
                    "p4q_select_full: sizes must be positive (B=%d N=%d d=%d J=%d K=%d T=%d)", B, N, d, J, K, T);
    if (K > N) return fail(P4Q_ERR_INVALID_ARG, "p4q_select_full: K=%d > N=%d", K, N);
    if (kq < 0 || ks < 0 || (int64_t)kq + ks > K)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_select_full: budgets kq=%d ks=%d do not fit K=%d", kq, ks, K);
    if (!vis || !concepts || !cls_attn || !idx_out || !tokens_out)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_select_full: null pointer");
    if ((T > 0) != (text != nullptr))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_select_full: text must be given iff T > 0");
    if (!valid_clip(clip))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_select_full: clip %g outside [2^-16, 1]", clip);
    if (d % 32 != 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_select_full: d=%d not a multiple of 32", d);
    if (!aligned(vis, 16) || !aligned(concepts, 16) || !aligned(tokens_out, 16) ||
        (text && !aligned(text, 16)) || !aligned(idx_out, 4) || !aligned(cls_attn, 4) ||
        (stages_out && !aligned(stages_out, 4)))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_select_full: misaligned pointer");
    if (N > 8192) return fail(P4Q_ERR_UNSUPPORTED, "p4q_select_full: N=%d > 8192", N);
    if (J > 8) return fail(P4Q_ERR_UNSUPPORTED, "p4q_select_full: J=%d > 8", J);
    if (d > 8192) return fail(P4Q_ERR_UNSUPPORTED, "p4q_select_full: d=%d > 8192", d);
    if (B > 65535) return fail(P4Q_ERR_UNSUPPORTED, "p4q_select_full: B=%d > 65535", B);
    const size_t need = p4q::select_full_workspace_bytes(B, N, d, J, K);
    if (!ws || ws_bytes < need)
        return fail(P4Q_ERR_WORKSPACE, "p4q_select_full: workspace %zu < %zu bytes", ws_bytes, need);
    if (!aligned(ws, 256)) return fail(P4Q_ERR_INVALID_ARG, "p4q_select_full: workspace not 256-byte aligned");
    const p4q::SelectFullWorkspace w = p4q::select_full_workspace_carve(ws, B, N, d, J, K);
    return hip_status(p4q::launch_select_full(dt, B, N, d, vis, concepts, J, cls_attn, text, T, K, kq, ks,
                                              clip, idx_out, stages_out, tokens_out, w, stream),
                      "p4q_select_full");
}

int p4q_quant_act(p4q_dtype dt, int M, int K_in, const void *x, int64_t ldx, float clip,
                  uint8_t *codes, float *scales, hipStream_t stream) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "p4q_quant_act: dtype %d", (int)dt);
    if (M <= 0 || K_in <= 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_act: M=%d K_in=%d", M, K_in);
    if (K_in % 32 != 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_act: K_in=%d not a multiple of 32", K_in);
    if (K_in > 65536) return fail(P4Q_ERR_UNSUPPORTED, "p4q_quant_act: K_in=%d > 65536", K_in);
    if (ldx < K_in || ldx % 8 != 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_act: ldx=%lld (need >= K_in, multiple of 8)", (long long)ldx);
    if (!x || !codes || !scales) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_act: null pointer");
    if (!aligned(x, 16) || !aligned(codes, 16) || !aligned(scales, 4))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_act: misaligned pointer");
    if (!valid_clip(clip)) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_act: clip %g outside [2^-16, 1]", clip);
    return hip_status(p4q::launch_quant_act(dt, M, K_in, x, ldx, clip, codes, scales, stream),
                      "p4q_quant_act");
}

int p4q_rmsnorm_quant(p4q_dtype dt, int M, int d, const void *x, int64_t ldx, const void *gamma,
                      float eps, float clip, uint8_t *codes, float *scales, hipStream_t stream) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "p4q_rmsnorm_quant: dtype %d", (int)dt);
    if (M <= 0 || d <= 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_rmsnorm_quant: M=%d d=%d", M, d);
    if (d % 32 != 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_rmsnorm_quant: d=%d not a multiple of 32", d);
    if (d > 16384) return fail(P4Q_ERR_UNSUPPORTED, "p4q_rmsnorm_quant: d=%d > 16384", d);
    if (ldx < d || ldx % 8 != 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_rmsnorm_quant: ldx=%lld (need >= d, multiple of 8)", (long long)ldx);
    if (!x || !gamma || !codes || !scales) return fail(P4Q_ERR_INVALID_ARG, "p4q_rmsnorm_quant: null pointer");
    if (!aligned(x, 16) || !aligned(gamma, 16) || !aligned(codes, 16) || !aligned(scales, 4))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_rmsnorm_quant: misaligned pointer");
    if (!(eps >= 0.0f && eps <= 1.0f)) return fail(P4Q_ERR_INVALID_ARG, "p4q_rmsnorm_quant: eps %g outside [0, 1]", eps);
    if (!valid_clip(clip)) return fail(P4Q_ERR_INVALID_ARG, "p4q_rmsnorm_quant: clip %g outside [2^-16, 1]", clip);
    return hip_status(p4q::launch_rmsnorm_quant(dt, M, d, x, ldx, gamma, eps, clip, codes, scales, stream),
                      "p4q_rmsnorm_quant");
}

int p4q_attention_prefill(p4q_dtype dt, int B, int L, int H, int D, const void *q, const void *k,
                          const void *v, int64_t ld, void *out, int64_t ld_out, int causal,
                          hipStream_t stream) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "p4q_attention_prefill: dtype %d", (int)dt);
    if (B <= 0 || L <= 0 || H <= 0 || D <= 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_attention_prefill: B=%d L=%d H=%d D=%d", B, L, H, D);
    if (D != 128) return fail(P4Q_ERR_UNSUPPORTED, "p4q_attention_prefill: head dimension %d (128 only)", D);
    if (causal != 0 && causal != 1) return fail(P4Q_ERR_INVALID_ARG, "p4q_attention_prefill: causal=%d", causal);
    if (ld < (int64_t)H * D || ld % 8 != 0 || ld_out < (int64_t)H * D || ld_out % 4 != 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_attention_prefill: ld=%lld ld_out=%lld (need >= H*D; multiples of 8 / 4)",
                    (long long)ld, (long long)ld_out);
    if (!q || !k || !v || !out) return fail(P4Q_ERR_INVALID_ARG, "p4q_attention_prefill: null pointer");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 8))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_attention_prefill: misaligned pointer");
    if (B > 65535 || H > 65535 || (int64_t)L * ld * 2 >= (1LL << 31))
        return fail(P4Q_ERR_UNSUPPORTED, "p4q_attention_prefill: B=%d H=%d L=%d ld=%lld too large (L*ld*2 < 2^31)",
                    B, H, L, (long long)ld);
    return hip_status(p4q::launch_attention(dt, B, L, H, q, k, v, ld, out, ld_out, causal, stream),
                      "p4q_attention_prefill");
}

// ---- serving: the paged cache and its attention ---------------------------------
// Limits that the calls share.  Returns P4Q_OK or the failing status (message
// recorded).
static int check_heads(const char *who, p4q_dtype dt, int T, int B, int Hq, int Hk, int D) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "%s: dtype %d", who, (int)dt);
    if (T <= 0 || B <= 0 || Hq <= 0 || Hk <= 0 || D <= 0 || Hq % Hk != 0)
        return fail(P4Q_ERR_INVALID_ARG, "%s: T=%d B=%d Hq=%d Hk=%d D=%d (positive, Hq a multiple of Hk)", who, T, B,
                    Hq, Hk, D);
    if (D != 64 && D != 128) return fail(P4Q_ERR_UNSUPPORTED, "%s: head dimension %d (64 or 128)", who, D);
    if (T > (1 << 24) || B > 65535 || Hq > 1024 || (int64_t)T * (Hq / Hk) >= (1LL << 31) ||
        (int64_t)T * Hq / 128 + (int64_t)B * Hk >= (1LL << 26))
        return fail(P4Q_ERR_UNSUPPORTED, "%s: T=%d B=%d Hq=%d Hk=%d too large", who, T, B, Hq, Hk);
    return P4Q_OK;
}

static int check_stride(const char *who, const char *name, int64_t ld, int heads, int D) {
    if (ld < (int64_t)heads * D || ld % 8 != 0)
        return fail(P4Q_ERR_INVALID_ARG, "%s: row stride %lld of %s (need >= %lld, multiple of 8)", who, (long long)ld,
                    name, (long long)heads * D);
    if (ld >= (1 << 24)) return fail(P4Q_ERR_UNSUPPORTED, "%s: row stride %lld of %s >= 2^24", who, (long long)ld, name);
    return P4Q_OK;
}

static int check_cache(const char *who, const void *k_cache, const void *v_cache, int num_pages, int page_size,
                       const int32_t *table, int max_pages) {
    if (!k_cache || !v_cache || !table) return fail(P4Q_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(table, 4))
        return fail(P4Q_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    if (num_pages <= 0 || max_pages <= 0)
        return fail(P4Q_ERR_INVALID_ARG, "%s: num_pages=%d max_pages=%d", who, num_pages, max_pages);
    if (p4q::page_shift(page_size) < 0)
        return fail(P4Q_ERR_UNSUPPORTED, "%s: page size %d (a power of two from 16 to 4096)", who, page_size);
    if ((int64_t)max_pages * page_size >= (1LL << 30))
        return fail(P4Q_ERR_UNSUPPORTED, "%s: max_pages=%d of %d rows: 2^30 keys or more", who, max_pages, page_size);
    return P4Q_OK;
}

int p4q_rope_append(p4q_dtype dt, int T, int B, int Hq, int Hk, int D, const void *q, int64_t ldq, const void *k,
                    int64_t ldk, const void *v, int64_t ldv, const int32_t *cu_seqlens, const int32_t *cache_lens,
                    const int32_t *positions, float rope_base, void *q_out, int64_t ldq_out, void *k_out,
                    int64_t ldk_out, void *k_cache, void *v_cache, int num_pages, int page_size,
                    const int32_t *block_table, int max_pages, hipStream_t stream) {
    const char *who = "p4q_rope_append";
    if (const int st = check_heads(who, dt, T, B, Hq, Hk, D)) return st;
    if (!q || !k || !v || !q_out || !cu_seqlens) return fail(P4Q_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(k_out, 16) ||
        !aligned(cu_seqlens, 4) || !aligned(cache_lens, 4) || !aligned(positions, 4))
        return fail(P4Q_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    if (const int st = check_stride(who, "q", ldq, Hq, D)) return st;
    if (const int st = check_stride(who, "k", ldk, Hk, D)) return st;
    if (const int st = check_stride(who, "v", ldv, Hk, D)) return st;
    if (const int st = check_stride(who, "q_out", ldq_out, Hq, D)) return st;
    if (k_out)
        if (const int st = check_stride(who, "k_out", ldk_out, Hk, D)) return st;
    if ((q_out == q && ldq_out != ldq) || (k_out == k && ldk_out != ldk))
        return fail(P4Q_ERR_INVALID_ARG, "%s: an output in place needs its input's row stride", who);
    if (!(rope_base > 1.0f) || !(rope_base < __builtin_huge_valf()))
        return fail(P4Q_ERR_INVALID_ARG, "%s: rope_base=%g", who, (double)rope_base);
    if (const int st = check_cache(who, k_cache, v_cache, num_pages, page_size, block_table, max_pages)) return st;
    p4q::RopeAppend a{};
    a.T = T, a.B = B, a.Hq = Hq, a.Hk = Hk;
    a.q = static_cast<const uint16_t *>(q), a.k = static_cast<const uint16_t *>(k), a.v = static_cast<const uint16_t *>(v);
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
    a.cu = cu_seqlens, a.cache_lens = cache_lens, a.positions = positions;
    a.q_out = static_cast<uint16_t *>(q_out), a.k_out = static_cast<uint16_t *>(k_out);
    a.ldqo = ldq_out, a.ldko = ldk_out;
    a.k_cache = static_cast<uint16_t *>(k_cache), a.v_cache = static_cast<uint16_t *>(v_cache);
    a.num_pages = num_pages, a.shift = p4q::page_shift(page_size), a.max_pages = max_pages, a.table = block_table;
    return hip_status(p4q::launch_rope_append(dt, D, a, rope_base, stream), who);
}

size_t p4q_attention_prompt_workspace_bytes(int T, int B, int Hq, int Hk, int D, int64_t most_keys) {
    if (check_heads("", P4Q_FP16, T, B, Hq, Hk, D) != P4Q_OK || most_keys < 0 || most_keys >= (1LL << 31)) return 0;
    return p4q::prompt_attention_workspace_bytes(T, B, Hq, Hk, D, most_keys);
}

int p4q_attention_packed(p4q_dtype dt, int T, int Tk, int B, int Hq, int Hk, int D, const void *q, int64_t ldq,
                         const void *k, int64_t ldk, const void *v, int64_t ldv, const int32_t *cu_seqlens,
                         const int32_t *cu_seqlens_k, void *out, int64_t ld_out, int causal, void *ws,
                         size_t ws_bytes, hipStream_t stream) {
    const char *who = "p4q_attention_packed";
    if (const int st = check_heads(who, dt, T, B, Hq, Hk, D)) return st;
    if (Tk < 0) return fail(P4Q_ERR_INVALID_ARG, "%s: Tk=%d", who, Tk);
    if (Tk > (1 << 24)) return fail(P4Q_ERR_UNSUPPORTED, "%s: Tk=%d > 2^24", who, Tk);
    if (causal != 0 && causal != 1) return fail(P4Q_ERR_INVALID_ARG, "%s: causal=%d", who, causal);
    if (!q || !out || !cu_seqlens || (Tk > 0 && (!k || !v))) return fail(P4Q_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!cu_seqlens_k && Tk != T)
        return fail(P4Q_ERR_INVALID_ARG, "%s: %d key rows for %d tokens need cu_seqlens_k", who, Tk, T);
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(cu_seqlens, 4) ||
        !aligned(cu_seqlens_k, 4))
        return fail(P4Q_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    if (const int st = check_stride(who, "q", ldq, Hq, D)) return st;
    if (const int st = check_stride(who, "k", ldk, Hk, D)) return st;
    if (const int st = check_stride(who, "v", ldv, Hk, D)) return st;
    if (const int st = check_stride(who, "out", ld_out, Hq, D)) return st;
    p4q::PromptAttention a{};
    a.T = T, a.Tk = Tk, a.B = B, a.Hq = Hq, a.Hk = Hk;
    a.q = static_cast<const uint16_t *>(q), a.k = static_cast<const uint16_t *>(k), a.v = static_cast<const uint16_t *>(v);
    a.ldq = ldq, a.ldk = (int)ldk, a.ldv = (int)ldv, a.ldo = ld_out;
    a.cu_q = cu_seqlens, a.cu_k = cu_seqlens_k ? cu_seqlens_k : cu_seqlens;
    a.out = static_cast<uint16_t *>(out);
    return hip_status(p4q::launch_prompt_attention(dt, D, a, causal, Tk, aligned(ws, 16) ? ws : nullptr,
                                                   ws && aligned(ws, 16) ? ws_bytes : 0, stream), who);
}

int p4q_attention_prefill_paged(p4q_dtype dt, int T, int B, int Hq, int Hk, int D, const void *q, int64_t ldq,
                                const void *k_cache, const void *v_cache, int num_pages, int page_size,
                                const int32_t *block_table, int max_pages, const int32_t *cu_seqlens,
                                const int32_t *seq_lens, void *out, int64_t ld_out, int causal, void *ws,
                                size_t ws_bytes, hipStream_t stream) {
    const char *who = "p4q_attention_prefill_paged";
    if (const int st = check_heads(who, dt, T, B, Hq, Hk, D)) return st;
    if (causal != 0 && causal != 1) return fail(P4Q_ERR_INVALID_ARG, "%s: causal=%d", who, causal);
    if (!q || !out || !cu_seqlens || !seq_lens) return fail(P4Q_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(cu_seqlens, 4) || !aligned(seq_lens, 4))
        return fail(P4Q_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    if (const int st = check_stride(who, "q", ldq, Hq, D)) return st;
    if (const int st = check_stride(who, "out", ld_out, Hq, D)) return st;
    if (const int st = check_cache(who, k_cache, v_cache, num_pages, page_size, block_table, max_pages)) return st;
    p4q::PromptAttention a{};
    a.T = T, a.B = B, a.Hq = Hq, a.Hk = Hk;
    a.q = static_cast<const uint16_t *>(q), a.k = static_cast<const uint16_t *>(k_cache);
    a.v = static_cast<const uint16_t *>(v_cache);
    a.ldq = ldq, a.ldo = ld_out, a.cu_q = cu_seqlens, a.lens = seq_lens, a.table = block_table;
    a.num_pages = num_pages, a.shift = p4q::page_shift(page_size), a.max_pages = max_pages;
    a.out = static_cast<uint16_t *>(out);
    return hip_status(p4q::launch_prompt_attention(dt, D, a, causal, (int64_t)max_pages * page_size,
                                                   aligned(ws, 16) ? ws : nullptr,
                                                   ws && aligned(ws, 16) ? ws_bytes : 0, stream), who);
}

size_t p4q_attention_decode_workspace_bytes(int B, int Hq, int Hk, int D, int max_len) {
    if (check_heads("", P4Q_FP16, B, B, Hq, Hk, D) != P4Q_OK || max_len <= 0 || max_len >= (1 << 30)) return 0;
    return p4q::decode_attention_workspace_bytes(B, Hq, Hk, D, max_len);
}

int p4q_attention_decode(p4q_dtype dt, int B, int Hq, int Hk, int D, const void *q, int64_t ldq, const void *k_cache,
                         const void *v_cache, int num_pages, int page_size, const int32_t *block_table, int max_pages,
                         const int32_t *seq_lens, int max_len, void *out, int64_t ld_out, void *ws, size_t ws_bytes,
                         hipStream_t stream) {
    const char *who = "p4q_attention_decode";
    if (const int st = check_heads(who, dt, B, B, Hq, Hk, D)) return st;
    if (!q || !out || !seq_lens) return fail(P4Q_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(seq_lens, 4))
        return fail(P4Q_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    if (const int st = check_stride(who, "q", ldq, Hq, D)) return st;
    if (const int st = check_stride(who, "out", ld_out, Hq, D)) return st;
    if (const int st = check_cache(who, k_cache, v_cache, num_pages, page_size, block_table, max_pages)) return st;
    if (max_len < 1 || max_len > (int64_t)max_pages * page_size)
        return fail(P4Q_ERR_INVALID_ARG, "%s: max_len=%d outside [1, %lld]", who, max_len,
                    (long long)max_pages * page_size);
    const size_t need = p4q::decode_attention_workspace_bytes(B, Hq, Hk, D, max_len);
    if (!ws || ws_bytes < need)
        return fail(P4Q_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, ws_bytes, need);
    if (!aligned(ws, 16)) return fail(P4Q_ERR_INVALID_ARG, "%s: workspace not 16-byte aligned", who);
    p4q::DecodeAttention a{};
    a.B = B, a.Hq = Hq, a.Hk = Hk, a.max_len = max_len;
    a.q = static_cast<const uint16_t *>(q), a.k = static_cast<const uint16_t *>(k_cache);
    a.v = static_cast<const uint16_t *>(v_cache);
    a.ldq = ldq, a.ldo = ld_out, a.lens = seq_lens, a.table = block_table;
    a.num_pages = num_pages, a.shift = p4q::page_shift(page_size), a.max_pages = max_pages;
    a.out = static_cast<uint16_t *>(out);
    return hip_status(p4q::launch_decode_attention(dt, D, a, ws, stream), who);
}

static int calib_block_shape_error(int M, int d, int f, int H) {
    if (M <= 0 || d <= 0 || f <= 0 || H <= 0) return P4Q_ERR_INVALID_ARG;
    if (d % 128 != 0 || f % 128 != 0 || d % H != 0 || (d / H) % 2 != 0) return P4Q_ERR_INVALID_ARG;
    if (M > 4096 || d > 16384 || f > 16384 || (int64_t)M * 2 * f >= (1LL << 31) ||
        (int64_t)3 * d * d >= (1LL << 31) || (int64_t)2 * f * d >= (1LL << 31))
        return P4Q_ERR_UNSUPPORTED;
    return P4Q_OK;
}

size_t p4q_calib_block_workspace_bytes(int M, int d, int f, int H) {
    if (calib_block_shape_error(M, d, f, H) != P4Q_OK) return 0;
    return p4q::calib_block_workspace_bytes(M, d, f, H);
}

int p4q_calib_block_grad(p4q_dtype dt, int M, int d, int f, int H, const void *x,
                         const float *target, int64_t ldt, const void *w_qkv, const void *w_o,
                         const void *w_gu, const void *w_down, const void *gamma1,
                         const void *gamma2, float eps, float rope_base, const float *sigma,
                         const float *clip_a, const float *clip_w, float *loss,
                         float *grad_sigma, float *grad_clip_a, float *grad_clip_w, void *ws,
                         size_t ws_bytes, hipStream_t stream) {
    if (dt != P4Q_FP16) return fail(P4Q_ERR_UNSUPPORTED, "p4q_calib_block_grad: only fp16 blocks");
    if (const int st = calib_block_shape_error(M, d, f, H))
        return fail(st, "p4q_calib_block_grad: M=%d d=%d f=%d H=%d outside the limits", M, d, f, H);
    if (ldt < d) return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_block_grad: ldt=%lld < d", (long long)ldt);
    if (!(eps >= 0.0f && eps <= 1.0f) || !(rope_base > 1.0f))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_block_grad: eps=%g rope_base=%g", (double)eps,
                    (double)rope_base);
    if (!x || !target || !w_qkv || !w_o || !w_gu || !w_down || !gamma1 || !gamma2 || !sigma ||
        !clip_a || !clip_w || !loss || !grad_sigma || !grad_clip_a || !grad_clip_w)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_block_grad: null pointer");
    for (int g = 0; g < 4; ++g)
        if (!(clip_a[g] > 0.0f && clip_a[g] <= 1.0f))
            return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_block_grad: clip_a[%d]=%g outside (0, 1]", g,
                        (double)clip_a[g]);
    const void *ptrs[] = {x, target, w_qkv, w_o, w_gu, w_down, gamma1, gamma2, sigma, clip_w,
                          loss, grad_sigma, grad_clip_a, grad_clip_w};
    for (const void *q : ptrs)
        if (!aligned(q, 16)) return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_block_grad: misaligned pointer");
    if (ldt % 4 != 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_block_grad: ldt not a multiple of 4");
    const size_t need = p4q::calib_block_workspace_bytes(M, d, f, H);
    if (!ws || ws_bytes < need)
        return fail(P4Q_ERR_WORKSPACE, "p4q_calib_block_grad: workspace %zu < %zu bytes", ws_bytes, need);
    if (!aligned(ws, 256)) return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_block_grad: workspace not 256-byte aligned");
    return hip_status(p4q::launch_calib_block(M, d, f, H, x, target, ldt, w_qkv, w_o, w_gu, w_down,
                                              gamma1, gamma2, eps, rope_base, sigma, clip_a, clip_w,
                                              loss, grad_sigma, grad_clip_a, grad_clip_w, ws, stream),
                      "p4q_calib_block_grad");
}

size_t p4q_w4a4_linear_workspace_bytes(int M, int N_out, int K_in) {
    if (M <= 0 || N_out <= 0 || K_in <= 0 || K_in % 32 != 0 || K_in > 131072 ||
        (int64_t)M > 65535LL * 128)
        return 0;
    return p4q::gemm_workspace_bytes(M, N_out, K_in);
}

int p4q_w4a4_linear(int M, int N_out, int K_in, const uint8_t *a_codes, const float *a_scales,
                    const uint8_t *w_codes, const float *w_scales, p4q_dtype out_dt, void *y,
                    int64_t ldy, int32_t *acc_out, void *ws, size_t ws_bytes, hipStream_t stream) {
    if (!valid_dtype(out_dt)) return fail(P4Q_ERR_UNSUPPORTED, "p4q_w4a4_linear: dtype %d", (int)out_dt);
    if (M <= 0 || N_out <= 0 || K_in <= 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_w4a4_linear: M=%d N_out=%d K_in=%d", M, N_out, K_in);
    if (K_in % 32 != 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_w4a4_linear: K_in=%d not a multiple of 32", K_in);
    if (K_in > 131072) return fail(P4Q_ERR_UNSUPPORTED, "p4q_w4a4_linear: K_in=%d > 131072", K_in);
    if (ldy < N_out) return fail(P4Q_ERR_INVALID_ARG, "p4q_w4a4_linear: ldy=%lld < N_out", (long long)ldy);
    if (!a_codes || !a_scales || !w_codes || !w_scales || !y)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_w4a4_linear: null pointer");
    if (!aligned(a_codes, 16) || !aligned(w_codes, 16) || !aligned(y, 4) || !aligned(a_scales, 4) ||
        !aligned(w_scales, 4) || (acc_out && !aligned(acc_out, 4)))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_w4a4_linear: misaligned pointer");
    if ((int64_t)M > 65535LL * 128) return fail(P4Q_ERR_UNSUPPORTED, "p4q_w4a4_linear: M too large");
    return hip_status(p4q::launch_w4a4_gemm(M, N_out, K_in, a_codes, a_scales, w_codes, w_scales,
                                            out_dt, y, ldy, acc_out, ws, ws_bytes, stream),
                      "p4q_w4a4_linear");
}

// ---- MXFP4 -------------------------------------------------------------------
size_t p4q_mx4_scale_stride(int K) {
    if (K < 32 || K > 131072 || K % 32 != 0) return 0;
    return (size_t)p4q::mx4_scale_stride(K);
}

using p4q::Rows;
using p4q::rows_at;
using p4q::share_memory;
// (a stride that no operand goes with may be any number)
static Rows rows16_at(const void *p, int64_t rows, int64_t ld, int64_t cols) {
    return p ? rows_at(p, rows, 2 * ld, 2 * cols) : Rows{};
}
static Rows mx4_codes_at(const uint8_t *p, int64_t rows, int K) { return rows_at(p, rows, K / 2, K / 2); }
static Rows mx4_scales_at(const uint8_t *p, int64_t rows, int K) {
    return rows_at(p, rows, p4q::mx4_scale_stride(K), p4q::mx4_scale_stride(K));
}

// A 16-bit operand's rows: 16-byte aligned and at least `width` apart.
static bool rows_ok(const void *p, int64_t ld, int width) { return aligned(p, 16) && ld >= width && ld % 8 == 0; }

int p4q_quant_mx4(p4q_dtype dt, int M, int K, const void *x, int64_t ldx, uint8_t *codes,
                  uint8_t *scales, void *values, int64_t ldv, hipStream_t stream) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "p4q_quant_mx4: dtype %d", (int)dt);
    if (M <= 0 || K <= 0 || K % 32 != 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_mx4: M=%d K=%d (K a multiple of 32)", M, K);
    if (K > 131072 || M * ((K + 511LL) / 512) >= (1LL << 26))
        return fail(P4Q_ERR_UNSUPPORTED, "p4q_quant_mx4: M=%d K=%d too large", M, K);
    if (!x || !codes || !scales) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_mx4: null pointer");
    if (!rows_ok(x, ldx, K) || (values && !rows_ok(values, ldv, K)))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_mx4: ldx=%lld ldv=%lld (need >= K, multiples of 8; 16-byte aligned rows)",
                    (long long)ldx, (long long)ldv);
    if (values == x && ldv != ldx)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_mx4: values in place need the same row stride");
    if (!aligned(codes, 16) || !aligned(scales, 16)) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_mx4: misaligned pointer");
    const Rows in = rows16_at(x, M, ldx, K), held = rows16_at(values, M, ldv, K);
    const Rows c = mx4_codes_at(codes, M, K), sc = mx4_scales_at(scales, M, K);
    if ((values != x && share_memory(held, in)) || share_memory(c, sc) || share_memory(c, in) || share_memory(c, held) ||
        share_memory(sc, in) || share_memory(sc, held))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_mx4: operands overlap");
    return hip_status(p4q::launch_quant_mx4(dt, M, K, x, ldx, codes, scales, values, ldv, stream), "p4q_quant_mx4");
}

static int check_mx4_product(const char *who, int M, int N_out, int K, const uint8_t *a_codes,
                             const uint8_t *a_scales, const uint8_t *w_codes, const uint8_t *w_scales) {
    if (M <= 0 || N_out <= 0 || K <= 0 || K % 32 != 0)
        return fail(P4Q_ERR_INVALID_ARG, "%s: M=%d N_out=%d K=%d (K a multiple of 32)", who, M, N_out, K);
    if (M > (1 << 20) || N_out > (1 << 22) || K > 131072)
        return fail(P4Q_ERR_UNSUPPORTED, "%s: M=%d N_out=%d K=%d too large", who, M, N_out, K);
    if (!a_codes || !a_scales || !w_codes || !w_scales) return fail(P4Q_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned(a_codes, 16) || !aligned(a_scales, 16) || !aligned(w_codes, 16) || !aligned(w_scales, 16))
        return fail(P4Q_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    return P4Q_OK;
}

static int check_mx4_output(const char *who, p4q_dtype out_dt, const void *y, int64_t ldy, int N_out) {
    if (!valid_dtype(out_dt)) return fail(P4Q_ERR_UNSUPPORTED, "%s: dtype %d", who, (int)out_dt);
    if (!y || !aligned(y, 4)) return fail(P4Q_ERR_INVALID_ARG, "%s: y null or misaligned", who);
    if (ldy < N_out) return fail(P4Q_ERR_INVALID_ARG, "%s: ldy=%lld < N_out", who, (long long)ldy);
    return P4Q_OK;
}

// `out`, a result, shares memory with an operand of the product (pair: rows of the weight for each output)
static bool over_mx4_operand(const Rows &out, const p4q::Mx4Product &p, int pair) {
    return share_memory(out, mx4_codes_at(p.a, p.M, p.K)) || share_memory(out, mx4_scales_at(p.as, p.M, p.K)) ||
           share_memory(out, mx4_codes_at(p.w, (int64_t)pair * p.N, p.K)) ||
           share_memory(out, mx4_scales_at(p.ws, (int64_t)pair * p.N, p.K));
}

static p4q::Mx4Product mx4_product(int M, int N_out, int K, const uint8_t *a_codes, const uint8_t *a_scales,
                                   const uint8_t *w_codes, const uint8_t *w_scales) {
    p4q::Mx4Product p = {};
    p.M = M, p.N = N_out, p.K = K;
    p.a = a_codes, p.as = a_scales, p.w = w_codes, p.ws = w_scales;
    return p;
}

int p4q_mx4_linear(int M, int N_out, int K, const uint8_t *a_codes, const uint8_t *a_scales,
                   const uint8_t *w_codes, const uint8_t *w_scales, p4q_dtype out_dt, void *y,
                   int64_t ldy, hipStream_t stream) {
    const char *who = "p4q_mx4_linear";
    if (const int st = check_mx4_product(who, M, N_out, K, a_codes, a_scales, w_codes, w_scales)) return st;
    if (const int st = check_mx4_output(who, out_dt, y, ldy, N_out)) return st;
    p4q::Mx4Product p = mx4_product(M, N_out, K, a_codes, a_scales, w_codes, w_scales);
    p.y = y, p.ldy = ldy;
    if (over_mx4_operand(rows16_at(y, M, ldy, N_out), p, 1))
        return fail(P4Q_ERR_INVALID_ARG, "%s: y overlaps an operand", who);
    return hip_status(p4q::launch_mx4_linear(out_dt, p, stream), who);
}

int p4q_mx4_gated_linear(int M, int N_out, int K, const uint8_t *a_codes, const uint8_t *a_scales,
                         const uint8_t *w_codes, const uint8_t *w_scales, p4q_dtype out_dt, void *y,
                         int64_t ldy, hipStream_t stream) {
    const char *who = "p4q_mx4_gated_linear";
    if (const int st = check_mx4_product(who, M, N_out, K, a_codes, a_scales, w_codes, w_scales)) return st;
    if (const int st = check_mx4_output(who, out_dt, y, ldy, N_out)) return st;
    p4q::Mx4Product p = mx4_product(M, N_out, K, a_codes, a_scales, w_codes, w_scales);
    p.y = y, p.ldy = ldy;
    if (over_mx4_operand(rows16_at(y, M, ldy, N_out), p, 2))
        return fail(P4Q_ERR_INVALID_ARG, "%s: y overlaps an operand", who);
    return hip_status(p4q::launch_mx4_gated(out_dt, p, stream), who);
}

int p4q_mx4_gated_linear_quant(int M, int N_out, int K, const uint8_t *a_codes,
                               const uint8_t *a_scales, const uint8_t *w_codes,
                               const uint8_t *w_scales, uint8_t *codes, uint8_t *scales,
                               hipStream_t stream) {
    const char *who = "p4q_mx4_gated_linear_quant";
    if (const int st = check_mx4_product(who, M, N_out, K, a_codes, a_scales, w_codes, w_scales)) return st;
    if (N_out % 32 != 0) return fail(P4Q_ERR_INVALID_ARG, "%s: N_out=%d not a multiple of 32", who, N_out);
    if (!codes || !scales || !aligned(codes, 16) || !aligned(scales, 16))
        return fail(P4Q_ERR_INVALID_ARG, "%s: codes or scales null or misaligned", who);
    if (codes == a_codes || scales == a_scales)
        return fail(P4Q_ERR_INVALID_ARG, "%s: the result cannot replace the activations", who);
    p4q::Mx4Product p = mx4_product(M, N_out, K, a_codes, a_scales, w_codes, w_scales);
    p.codes = codes, p.scales = scales;
    const Rows c = mx4_codes_at(codes, M, N_out), sc = mx4_scales_at(scales, M, N_out);
    if (share_memory(c, sc) || over_mx4_operand(c, p, 2) || over_mx4_operand(sc, p, 2))
        return fail(P4Q_ERR_INVALID_ARG, "%s: codes or scales overlap another operand", who);
    return hip_status(p4q::launch_mx4_gated(P4Q_BF16, p, stream), who);
}

int p4q_residual_rmsnorm_quant(p4q_dtype dt, p4q_norm_format fmt, int M, int d, const void *x,
                               int64_t ldx, const void *r, int64_t ldr, const void *post_gamma,
                               const void *gate, float alpha, const void *gamma, float eps,
                               float clip, void *h_out, int64_t ldh, uint8_t *codes, void *scales,
                               void *values, int64_t ldv, hipStream_t stream) {
    const char *who = "p4q_residual_rmsnorm_quant";
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "%s: dtype %d", who, (int)dt);
    if (fmt != P4Q_NORM_INT4 && fmt != P4Q_NORM_MX4) return fail(P4Q_ERR_UNSUPPORTED, "%s: format %d", who, (int)fmt);
    if (M <= 0 || d <= 0 || d % 32 != 0) return fail(P4Q_ERR_INVALID_ARG, "%s: M=%d d=%d (d a multiple of 32)", who, M, d);
    if (d > 16384 || M >= (1 << 23)) return fail(P4Q_ERR_UNSUPPORTED, "%s: M=%d d=%d too large", who, M, d);
    if (!x || !gamma || !codes || !scales) return fail(P4Q_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!r && (h_out || gate || post_gamma || alpha != 1.0f))
        return fail(P4Q_ERR_INVALID_ARG, "%s: h_out, gate, post_gamma and alpha need r", who);
    if (r && !h_out) return fail(P4Q_ERR_INVALID_ARG, "%s: r needs h_out", who);
    if (!rows_ok(x, ldx, d) || (r && (!rows_ok(r, ldr, d) || !rows_ok(h_out, ldh, d))) ||
        (values && !rows_ok(values, ldv, d)))
        return fail(P4Q_ERR_INVALID_ARG, "%s: row strides %lld %lld %lld %lld (need >= d, multiples of 8; 16-byte aligned rows)",
                    who, (long long)ldx, (long long)ldr, (long long)ldh, (long long)ldv);
    if (r && ((h_out == x && ldh != ldx) || (h_out == r && ldh != ldr)))
        return fail(P4Q_ERR_INVALID_ARG, "%s: h_out in place needs the same row stride", who);
    if (!aligned(gamma, 16) || !aligned(codes, 16) || (post_gamma && !aligned(post_gamma, 16)) ||
        (gate && !aligned(gate, 16)) || !aligned(scales, fmt == P4Q_NORM_MX4 ? 16 : 4))
        return fail(P4Q_ERR_INVALID_ARG, "%s: misaligned pointer", who);
    if (!(eps >= 0.0f && eps <= 1.0f)) return fail(P4Q_ERR_INVALID_ARG, "%s: eps %g outside [0, 1]", who, eps);
    if (!(alpha - alpha == 0.0f)) return fail(P4Q_ERR_INVALID_ARG, "%s: alpha %g", who, alpha);
    if (!valid_clip(clip) || (fmt == P4Q_NORM_MX4 && clip != 1.0f))
        return fail(P4Q_ERR_INVALID_ARG, "%s: clip %g (int4: in [2^-16, 1]; MXFP4: 1)", who, clip);
    // h_out may be x or r; nothing else that is written shares memory
    const Rows in[5] = {rows16_at(x, M, ldx, d), rows16_at(r, M, ldr, d), rows16_at(gamma, 1, d, d),
                        rows16_at(post_gamma, 1, d, d), rows16_at(gate, 1, d, d)};
    const Rows out[4] = {rows16_at(h_out, M, ldh, d), rows16_at(values, M, ldv, d), mx4_codes_at(codes, M, d),
                         fmt == P4Q_NORM_MX4 ? mx4_scales_at(static_cast<uint8_t *>(scales), M, d) : rows_at(scales, M, 4, 4)};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < i; ++j)
            if (share_memory(out[i], out[j])) return fail(P4Q_ERR_INVALID_ARG, "%s: two results overlap", who);
        for (int j = 0; j < 5; ++j)
            if (share_memory(out[i], in[j]) && !(i == 0 && j < 2 && h_out == (j == 0 ? x : r)))
                return fail(P4Q_ERR_INVALID_ARG, "%s: a result overlaps an operand (h_out may be x or r)", who);
    }
    p4q::ResidualNorm a = {};
    a.M = M, a.d = d;
    a.x = static_cast<const uint16_t *>(x), a.ldx = ldx;
    a.r = static_cast<const uint16_t *>(r), a.ldr = ldr;
    a.post = static_cast<const uint16_t *>(post_gamma);
    a.gate = static_cast<const uint16_t *>(gate);
    a.gamma = static_cast<const uint16_t *>(gamma);
    a.alpha = alpha, a.eps = eps, a.clip = clip;
    a.h_out = static_cast<uint16_t *>(h_out), a.ldh = ldh;
    a.codes = codes, a.scales = scales;
    a.values = static_cast<uint16_t *>(values), a.ldv = ldv;
    return hip_status(p4q::launch_residual_rmsnorm_quant(dt, fmt, a, stream), who);
}

int p4q_quant_scaled(p4q_dtype dt, int R, int K, const void *z, int64_t ldz, const float *sigma,
                     int divide, float clip, const float *clip_rows, uint8_t *codes,
                     float *scales, float *absmax, int32_t *kstar, hipStream_t stream) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "p4q_quant_scaled: dtype %d", (int)dt);
    if (R <= 0 || K <= 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_scaled: R=%d K=%d", R, K);
    if (K % 32 != 0) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_scaled: K=%d not a multiple of 32", K);
    if (K > 16384) return fail(P4Q_ERR_UNSUPPORTED, "p4q_quant_scaled: K=%d > 16384", K);
    if (ldz < K || ldz % 8 != 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_scaled: ldz=%lld (need >= K, multiple of 8)", (long long)ldz);
    if (divide != 0 && divide != 1) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_scaled: divide=%d", divide);
    if (!clip_rows && !(clip > 0.0f && clip <= 1.0f))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_scaled: clip=%g outside (0, 1]", (double)clip);
    if (!z || !sigma || !codes || !scales) return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_scaled: null pointer");
    if (!aligned(z, 16) || !aligned(sigma, 16) || !aligned(codes, 16) || !aligned(scales, 4) ||
        (clip_rows && !aligned(clip_rows, 4)) || (absmax && !aligned(absmax, 4)) || (kstar && !aligned(kstar, 4)))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_quant_scaled: misaligned pointer");
    return hip_status(p4q::launch_quant_scaled(dt, R, K, z, ldz, sigma, divide, clip, clip_rows, codes,
                                               scales, absmax, kstar, stream),
                      "p4q_quant_scaled");
}

static int calib_shape_error(int M, int N, int K) {
    if (M <= 0 || N <= 0 || K <= 0) return P4Q_ERR_INVALID_ARG;
    if (N % 64 != 0 || K % 128 != 0) return P4Q_ERR_INVALID_ARG;
    if (K > 16384 || M > (1 << 20) || N > (1 << 20) || (int64_t)M * N >= (1LL << 31) ||
        (int64_t)N * K >= (1LL << 31))
        return P4Q_ERR_UNSUPPORTED;
    return P4Q_OK;
}

size_t p4q_calib_linear_workspace_bytes(int M, int N, int K) {
    if (calib_shape_error(M, N, K) != P4Q_OK) return 0;
    return p4q::calib_linear_workspace_bytes(M, N, K);
}

int p4q_calib_linear_grad(p4q_dtype dt, int M, int N, int K, const void *x, int64_t ldx,
                          const void *w, int64_t ldw, const float *target, int64_t ldt,
                          const float *sigma, float clip_a, const float *clip_w, float *loss,
                          float *grad_sigma, float *grad_clip_a, float *grad_clip_w, void *ws,
                          size_t ws_bytes, hipStream_t stream) {
    if (!valid_dtype(dt)) return fail(P4Q_ERR_UNSUPPORTED, "p4q_calib_linear_grad: dtype %d", (int)dt);
    const int se = calib_shape_error(M, N, K);
    if (se != P4Q_OK)
        return fail(se, "p4q_calib_linear_grad: M=%d N=%d K=%d (need N %% 64 == 0, K %% 128 == 0, "
                    "K <= 16384, M*N and N*K < 2^31)", M, N, K);
    if (ldx < K || ldx % 8 != 0 || ldw < K || ldw % 8 != 0 || ldt < N || ldt % 4 != 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_linear_grad: ldx=%lld ldw=%lld ldt=%lld",
                    (long long)ldx, (long long)ldw, (long long)ldt);
    if (!(clip_a > 0.0f && clip_a <= 1.0f))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_linear_grad: clip_a=%g outside (0, 1]", (double)clip_a);
    if (!x || !w || !target || !sigma || !clip_w || !loss || !grad_sigma || !grad_clip_a || !grad_clip_w)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_linear_grad: null pointer");
    if (!aligned(x, 16) || !aligned(w, 16) || !aligned(target, 16) || !aligned(sigma, 16) ||
        !aligned(clip_w, 4) || !aligned(loss, 4) || !aligned(grad_sigma, 4) ||
        !aligned(grad_clip_a, 4) || !aligned(grad_clip_w, 4) || (ws && !aligned(ws, 256)))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_calib_linear_grad: misaligned pointer");
    const size_t need = p4q::calib_linear_workspace_bytes(M, N, K);
    if (!ws || ws_bytes < need)
        return fail(P4Q_ERR_WORKSPACE, "p4q_calib_linear_grad: workspace %zu < %zu bytes", ws_bytes, need);
    return hip_status(p4q::launch_calib_linear(dt, M, N, K, x, ldx, w, ldw, target, ldt, sigma, clip_a,
                                               clip_w, loss, grad_sigma, grad_clip_a, grad_clip_w, ws,
                                               stream),
                      "p4q_calib_linear_grad");
}

int p4q_diag_mfma_i8(int blocks, int iters, int32_t *out, hipStream_t stream) {
    if (blocks < 1 || blocks > (1 << 20) || iters < 1 || iters > (1 << 20))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_diag_mfma_i8: blocks=%d iters=%d", blocks, iters);
    if (!out || !aligned(out, 4)) return fail(P4Q_ERR_INVALID_ARG, "p4q_diag_mfma_i8: out");
    return hip_status(p4q::launch_diag_mfma_i8(blocks, iters, out, stream), "p4q_diag_mfma_i8");
}

int p4q_diag_stream_read(const void *src, size_t bytes, int blocks, uint32_t *out,
                         hipStream_t stream) {
    if (blocks < 1 || blocks > (1 << 20) || bytes % 16 != 0 || bytes == 0)
        return fail(P4Q_ERR_INVALID_ARG, "p4q_diag_stream_read: blocks=%d bytes=%zu", blocks, bytes);
    if (!src || !out || !aligned(src, 16) || !aligned(out, 4))
        return fail(P4Q_ERR_INVALID_ARG, "p4q_diag_stream_read: pointer");
    return hip_status(p4q::launch_diag_read(src, bytes, blocks, out, stream), "p4q_diag_stream_read");
}

}  // extern "C"
