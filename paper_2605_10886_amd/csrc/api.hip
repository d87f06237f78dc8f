// C ABI of the library: argument validation (host only, before any HIP call) and
// forwarding to the kernel launchers.  See include/loka.h for the contract.
#include "common.h"
#include "experts.h"

#include <algorithm>
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <mutex>

namespace loka {
// quantize.hip
size_t quantize_workspace_bytes(loka_scale_mode, int64_t, int64_t);
loka_status quantize_launch(const void*, int64_t, int64_t, int64_t, loka_scale_mode, int, uint8_t*, float*, void*,
                            hipStream_t);
loka_status e4m3_from_f32_launch(const float*, uint8_t*, int64_t, hipStream_t);
// gemm.hip
int variant_count();
const char* variant_name(int);
bool variant_supports(const loka_gemm_desc*, int);
size_t variant_workspace(const loka_gemm_desc*, int, bool fp8out = false);
loka_status fp8_gemm_norm_launch(const loka_gemm_desc*, int, const uint8_t*, const float*, const uint8_t*, const float*,
                                 const void*, const void*, void*, float*, uint8_t*, float*, void*, hipStream_t);
bool variant_supports_fp8out(const loka_gemm_desc*, int);
int variant_fp8out_default(const loka_gemm_desc*);
bool variant_supports_fused(const loka_gemm_desc*, int);
bool variant_supports_xq(const loka_gemm_desc*, int);
int variant_xq_default(const loka_gemm_desc*);
loka_status fp8_linear_norm_xq_launch(const loka_gemm_desc*, int, const void*, uint8_t*, float*, const uint8_t*, const float*,
                                      const void*, const void*, void*, float*, hipStream_t);
int variant_fused_default(const loka_gemm_desc*);
loka_status fp8_linear_norm_launch(const loka_gemm_desc*, int, const void*, const uint8_t*, const float*, const void*,
                                   const void*, void*, float*, float*, hipStream_t);
bool variant_has_wait_flag(const loka_gemm_desc*, int, bool fp8out = false);
void test_set_spin_limit(long long);
// ceiling.hip
loka_status machine_ceiling(int, double, void*, size_t, double*, hipStream_t);
size_t bf16_gemm_workspace_bytes(const loka_gemm_desc*);
size_t bf16_gemm_min_workspace_bytes(const loka_gemm_desc*);
loka_status bf16_gemm_launch(const loka_gemm_desc*, const void*, const void*, float*, void*, size_t, hipStream_t, bool weights_ready = false);
// probe.hip
size_t probe_workspace_bytes();
loka_status probe_launch(const float*, const float*, int64_t, int64_t, int64_t, loka_probe_stats*, float*, void*,
                         hipStream_t);
// dispatch.hip
int default_variant(const loka_gemm_desc*);
// tracker.hip
size_t tracker_workspace_bytes(int64_t, int64_t);
loka_status tracker_update_launch(const void*, int64_t, int64_t, int64_t, int64_t, float*, float*, void*, hipStream_t);
// mxfp4.hip
loka_status mxfp4_quantize_launch(const void*, int64_t, int64_t, int64_t, int, uint8_t*, uint8_t*, hipStream_t);
loka_status mxfp4_dequantize_launch(const uint8_t*, const uint8_t*, int64_t, int64_t, void*, int64_t, hipStream_t);
// mxfp4_gemm.hip
int mxfp4_gemm_form(const loka_gemm_desc*);
size_t mxfp4_gemm_workspace_bytes(const loka_gemm_desc*);
loka_status mxfp4_gemm_launch(const loka_gemm_desc*, const uint8_t*, const uint8_t*, const uint8_t*, const uint8_t*, void*, float*, void*,
                              size_t, hipStream_t);
bool mxfp4_linear_fused(const loka_gemm_desc*);
loka_status mxfp4_linear_fused_launch(const loka_gemm_desc*, const void*, int64_t, const uint8_t*, const uint8_t*, void*, float*, hipStream_t);
// rmsnorm.hip
loka_status add_rmsnorm_launch(const loka_rms_desc*, const void*, const void*, const void*, void*, void*, void*, uint8_t*, float*, float*,
                               hipStream_t);
size_t rmsnorm_backward_workspace_bytes(int64_t, int64_t);
loka_status rmsnorm_backward_launch(const loka_rms_desc*, const void*, const uint8_t*, const float*, const float*, const void*, const void*,
                                    void*, float*, void*, hipStream_t);

static bool mode_ok(int m) { return m >= LOKA_SCALE_TENSOR && m <= LOKA_SCALE_BLOCK_128x128_POW2; }       // modes a GEMM operand can have
static bool quant_mode_ok(int m) { return m >= LOKA_SCALE_TENSOR && m <= LOKA_SCALE_BLOCK_128x1; }
static bool is_block_x(int m) { return m == LOKA_SCALE_BLOCK_1x128 || m == LOKA_SCALE_BLOCK_1x128_POW2; }
static bool is_block_w(int m) { return m == LOKA_SCALE_BLOCK_128x128 || m == LOKA_SCALE_BLOCK_128x128_POW2; }

// Shape / enum validation shared by the GEMM entry points; does not look at pointers.
loka_status validate_desc(const loka_gemm_desc* d, bool fp8) {
    if (!d) return LOKA_ERR_NULL;
    if (d->M <= 0 || d->N <= 0 || d->K <= 0 || d->batch <= 0) return LOKA_ERR_SHAPE;
    if (d->M > INT32_MAX || d->N > INT32_MAX || d->K > INT32_MAX / 2 || d->batch > INT32_MAX) return LOKA_ERR_SHAPE;
    if (d->N % 16) return LOKA_ERR_SHAPE;
    if (fp8 ? (d->K % 16) : (d->K % 8)) return LOKA_ERR_SHAPE;
    if (d->strideX < 0 || d->strideW < 0 || d->strideO < 0) return LOKA_ERR_SHAPE;
    if (d->batch > 1 && d->strideO < d->M * d->N) return LOKA_ERR_SHAPE;
    if ((d->strideX % 16) || (d->strideW % 16) || (d->strideO % 8)) return LOKA_ERR_ALIGN;
    if (!fp8) return LOKA_OK;
    if (!mode_ok(d->x_mode) || !mode_ok(d->w_mode)) return LOKA_ERR_UNSUPPORTED;
    if (d->norm < LOKA_NORM_NONE || d->norm > LOKA_NORM_BLOCKNORM) return LOKA_ERR_UNSUPPORTED;
    if (d->act < LOKA_ACT_NONE || d->act > LOKA_ACT_HARDSWISH) return LOKA_ERR_UNSUPPORTED;
    if (d->act != LOKA_ACT_NONE && d->norm != LOKA_NORM_BLOCKNORM) return LOKA_ERR_UNSUPPORTED;
    if (d->norm == LOKA_NORM_BLOCKNORM) {
        if (d->block_n <= 0 || d->N % d->block_n) return LOKA_ERR_SHAPE;
        if (d->block_n != 256) return LOKA_ERR_UNSUPPORTED;
    }
    const bool xb = is_block_x(d->x_mode), wb = is_block_w(d->w_mode);
    if (xb != wb) return LOKA_ERR_UNSUPPORTED;
    // (power-of-two scales on both operands or on neither: the scaled matrix instruction takes both)
    if ((d->x_mode == LOKA_SCALE_BLOCK_1x128_POW2) != (d->w_mode == LOKA_SCALE_BLOCK_128x128_POW2)) return LOKA_ERR_UNSUPPORTED;
    if (xb && (d->N % 128 || d->K % 128)) return LOKA_ERR_SHAPE;
    if (!xb) {
        if (!(d->x_mode == LOKA_SCALE_TENSOR || d->x_mode == LOKA_SCALE_ROW)) return LOKA_ERR_UNSUPPORTED;
        if (!(d->w_mode == LOKA_SCALE_TENSOR || d->w_mode == LOKA_SCALE_COL)) return LOKA_ERR_UNSUPPORTED;
    }
    if (!(d->eps >= 0.f)) return LOKA_ERR_UNSUPPORTED;
    return LOKA_OK;
}

int variant_cheapest(const loka_gemm_desc* d, size_t max_ws);

int resolve_variant(const loka_gemm_desc* d) {
    if (d->variant >= 0) return variant_supports(d, d->variant) ? d->variant : -1;
    return default_variant(d);
}

// The library's choice when it may use `ws_bytes` of scratch: the usual one where that fits, else the best of those that do
// (-1: none, or the caller named the variant).
static int variant_within(const loka_gemm_desc* d, int v, size_t ws_bytes) {
    if (v < 0 || variant_workspace(d, v) <= ws_bytes) return v;
    return d->variant >= 0 || d->norm == LOKA_NORM_BLOCKNORM ? -1 : variant_cheapest(d, ws_bytes);
}

// Layers that always run without scratch (loka.h): the kernels whose tile spans the row, or no row norm at all, unless few
// output tiles meet a long K (split K, whose partial sums need room).
static bool scratch_optional(const loka_gemm_desc* d) {
    const int64_t t128 = ((d->M + 127) / 128) * ((d->N + 127) / 128) * d->batch;
    return (d->N <= 1024 || d->norm == LOKA_NORM_NONE) && !(t128 <= 128 && d->K >= 2048);
}

// What loka_fp8_gemm_norm runs with this workspace (the workspace may still be too small for it).
static int resolve_for_scratch(const loka_gemm_desc* d, const void* workspace, size_t ws_bytes) {
    const int v = resolve_variant(d);
    if (v < 0 || d->variant >= 0 || !scratch_optional(d)) return v;
    const int fit = variant_within(d, v, workspace ? ws_bytes : 0);
    return fit >= 0 ? fit : v;
}

}  // namespace loka

using namespace loka;

extern "C" {

const char* loka_status_string(loka_status s) {
    switch (s) {
        case LOKA_OK: return "ok";
        case LOKA_ERR_NULL: return "null pointer";
        case LOKA_ERR_SHAPE: return "bad shape";
        case LOKA_ERR_ALIGN: return "misaligned pointer or stride";
        case LOKA_ERR_UNSUPPORTED: return "unsupported combination";
        case LOKA_ERR_WORKSPACE: return "workspace missing or too small";
        case LOKA_ERR_HIP: return "HIP runtime error";
        case LOKA_ERR_NO_CANDIDATE: return "no FP8 candidate within the error budget";
        case LOKA_ERR_TIMEOUT: return "a bounded wait inside the launch ran out";
    }
    return "unknown status";
}

int64_t loka_scale_count(loka_scale_mode mode, int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0) return -1;
    switch (mode) {
        case LOKA_SCALE_TENSOR: return 1;
        case LOKA_SCALE_ROW: return rows;
        case LOKA_SCALE_COL: return cols;
        case LOKA_SCALE_BLOCK_1x128:
        case LOKA_SCALE_BLOCK_1x128_POW2: return (cols % 128) ? -1 : rows * (cols / 128);
        case LOKA_SCALE_BLOCK_128x128:
        case LOKA_SCALE_BLOCK_128x128_POW2: return (cols % 128 || rows % 128) ? -1 : (rows / 128) * (cols / 128);
        case LOKA_SCALE_BLOCK_128x1: return (rows % 128) ? -1 : (rows / 128) * cols;
    }
    return -1;
}

size_t loka_quantize_workspace(loka_scale_mode mode, int64_t rows, int64_t cols, int transpose_out) {
    if (!transpose_out && (mode == LOKA_SCALE_ROW || is_block_x(mode))) return 0;
    if (is_block_w(mode) || mode == LOKA_SCALE_BLOCK_128x1) return 0;      // groups that fit a workgroup: one pass
    if (loka_scale_count(mode, rows, cols) < 0) return 0;
    return quantize_workspace_bytes(mode, rows, cols);       // partial maxima
}

loka_status loka_quantize(const void* x_bf16, int64_t rows, int64_t cols, int64_t ld, loka_scale_mode mode,
                          int transpose_out, uint8_t* q, float* scales, void* workspace, size_t ws_bytes,
                          void* hip_stream) {
    if (!x_bf16 || !q || !scales) return LOKA_ERR_NULL;
    if (!quant_mode_ok(mode)) return LOKA_ERR_UNSUPPORTED;
    if (rows <= 0 || cols <= 0 || ld < cols) return LOKA_ERR_SHAPE;
    if (cols % 16 || (transpose_out && rows % 16)) return LOKA_ERR_SHAPE;
    if (loka_scale_count(mode, rows, cols) < 0) return LOKA_ERR_SHAPE;
    if (ld % 8) return LOKA_ERR_ALIGN;
    if (!aligned16(x_bf16) || !aligned16(q) || (reinterpret_cast<uintptr_t>(scales) & 3u)) return LOKA_ERR_ALIGN;
    if (transpose_out && (mode == LOKA_SCALE_ROW || is_block_x(mode))) return LOKA_ERR_UNSUPPORTED;
    if (!transpose_out && mode == LOKA_SCALE_BLOCK_128x1) return LOKA_ERR_UNSUPPORTED;
    const size_t need = loka_quantize_workspace(mode, rows, cols, transpose_out);
    if (need && (!workspace || ws_bytes < need)) return LOKA_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return LOKA_ERR_ALIGN;
    return quantize_launch(x_bf16, rows, cols, ld, mode, transpose_out, q, scales, workspace,
                           static_cast<hipStream_t>(hip_stream));
}

loka_status loka_e4m3_from_f32(const float* t, uint8_t* codes, int64_t n, void* hip_stream) {
    if (!t || !codes) return LOKA_ERR_NULL;
    if (n <= 0) return LOKA_ERR_SHAPE;
    return e4m3_from_f32_launch(t, codes, n, static_cast<hipStream_t>(hip_stream));
}

int loka_variant_count(void) { return variant_count(); }
const char* loka_variant_name(int variant) { return variant_name(variant); }

int loka_variant_supports(const loka_gemm_desc* desc, int variant) {
    if (validate_desc(desc, true) != LOKA_OK) return 0;
    return variant_supports(desc, variant) ? 1 : 0;
}

// ---- loka_fp8_gemm_norm_static: the scratch of loka_fp8_gemm_norm in library-owned device memory.
// `static_scratch` is a host-side stand-in for a device array: its device address is asked from the runtime once per
// device (with that device current) and only that address is ever handed to kernels or copies.
constexpr size_t kStaticScratchBytes = LOKA_STATIC_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char static_scratch[kStaticScratchBytes];
namespace {
constexpr int kScratchMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kScratchMaxDevices] = {};
}  // namespace

// Device address of the current device's copy of the array (set-up on the first call per device).
static loka_status static_scratch_address(void** ptr) {
    int dev = 0;
    LOKA_HIP_TRY(hipGetDevice(&dev));
    if (dev < 0 || dev >= kScratchMaxDevices) return LOKA_ERR_HIP;
    std::lock_guard<std::mutex> lk(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        LOKA_HIP_TRY(hipGetSymbolAddress(&p, HIP_SYMBOL(static_scratch)));
        if (!p) return LOKA_ERR_HIP;
        g_scratch_ptr[dev] = p;
    }
    *ptr = g_scratch_ptr[dev];
    return LOKA_OK;
}

loka_status loka_fp8_gemm_norm_static(const loka_gemm_desc* desc, const uint8_t* xq, const float* sx, const uint8_t* wq,
                                      const float* sw, const void* gamma_bf16, const void* beta_bf16, void* out_bf16,
                                      float* y_fp32, void* hip_stream) {
    if (!desc || !xq || !sx || !wq || !sw || !out_bf16) return LOKA_ERR_NULL;
    const loka_status st = validate_desc(desc, true);
    if (st != LOKA_OK) return st;
    if (!aligned16(xq) || !aligned16(wq) || !aligned16(sx) || !aligned16(sw) || !aligned16(out_bf16) ||
        !aligned16(y_fp32) || !aligned16(gamma_bf16) || !aligned16(beta_bf16))
        return LOKA_ERR_ALIGN;
    int v = resolve_variant(desc);
    if (v < 0) return LOKA_ERR_UNSUPPORTED;
    v = variant_within(desc, v, kStaticScratchBytes);
    if (v < 0) return LOKA_ERR_WORKSPACE;                           // beyond the array: use loka_fp8_gemm_norm with a workspace
    const size_t need = variant_workspace(desc, v);
    void* ws = nullptr;
    if (need) {
        const loka_status sa = static_scratch_address(&ws);
        if (sa != LOKA_OK) return sa;
    }
    return fp8_gemm_norm_launch(desc, v, xq, sx, wq, sw, gamma_bf16, beta_bf16, out_bf16, y_fp32, nullptr, nullptr, ws,
                                static_cast<hipStream_t>(hip_stream));
}

size_t loka_fp8_gemm_norm_workspace(const loka_gemm_desc* desc) {
    if (validate_desc(desc, true) != LOKA_OK) return 0;
    const int v = resolve_variant(desc);
    return v < 0 ? 0 : variant_workspace(desc, v);
}

loka_status loka_fp8_gemm_norm(const loka_gemm_desc* desc, const uint8_t* xq, const float* sx, const uint8_t* wq,
                               const float* sw, const void* gamma_bf16, const void* beta_bf16, void* out_bf16,
                               float* y_fp32, void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!desc || !xq || !sx || !wq || !sw || !out_bf16) return LOKA_ERR_NULL;
    const loka_status st = validate_desc(desc, true);
    if (st != LOKA_OK) return st;
    if (!aligned16(xq) || !aligned16(wq) || !aligned16(sx) || !aligned16(sw) || !aligned16(out_bf16) ||
        !aligned16(y_fp32) || !aligned16(gamma_bf16) || !aligned16(beta_bf16))
        return LOKA_ERR_ALIGN;
    const int v = resolve_for_scratch(desc, workspace, ws_bytes);
    if (v < 0) return LOKA_ERR_UNSUPPORTED;
    const size_t need = variant_workspace(desc, v);
    if (need && (!workspace || ws_bytes < need)) return LOKA_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return LOKA_ERR_ALIGN;
    return fp8_gemm_norm_launch(desc, v, xq, sx, wq, sw, gamma_bf16, beta_bf16, out_bf16, y_fp32, nullptr, nullptr,
                                workspace, static_cast<hipStream_t>(hip_stream));
}

loka_status loka_fp8_linear_norm(const loka_gemm_desc* desc, const void* x_bf16, const uint8_t* wq, const float* sw,
                                 const void* gamma_bf16, const void* beta_bf16, void* out_bf16, float* y_fp32,
                                 float* sx_out, void* hip_stream) {
    if (!desc || !x_bf16 || !wq || !sw || !out_bf16) return LOKA_ERR_NULL;
    const loka_status st = validate_desc(desc, true);
    if (st != LOKA_OK) return st;
    if (desc->x_mode != LOKA_SCALE_ROW) return LOKA_ERR_UNSUPPORTED;
    if (!aligned16(x_bf16) || !aligned16(wq) || !aligned16(sw) || !aligned16(out_bf16) || !aligned16(y_fp32) ||
        !aligned16(gamma_bf16) || !aligned16(beta_bf16) || !aligned16(sx_out))
        return LOKA_ERR_ALIGN;
    // kernels that keep whole rows of X in one workgroup (strip32, wreg32): the row amax needs no second pass
    const int v = desc->variant >= 0 ? desc->variant : variant_fused_default(desc);
    if (v < 0 || !variant_supports_fused(desc, v)) return LOKA_ERR_UNSUPPORTED;
    return fp8_linear_norm_launch(desc, v, x_bf16, wq, sw, gamma_bf16, beta_bf16, out_bf16, y_fp32, sx_out,
                                  static_cast<hipStream_t>(hip_stream));
}

loka_status loka_fp8_linear_norm_xq(const loka_gemm_desc* desc, const void* x_bf16, uint8_t* xq_out, float* sx_out,
                                    const uint8_t* wq, const float* sw, const void* gamma_bf16, const void* beta_bf16,
                                    void* out_bf16, float* y_fp32, void* hip_stream) {
    if (!desc || !x_bf16 || !xq_out || !sx_out || !wq || !sw || !out_bf16) return LOKA_ERR_NULL;
    const loka_status st = validate_desc(desc, true);
    if (st != LOKA_OK) return st;
    if (desc->x_mode != LOKA_SCALE_ROW) return LOKA_ERR_UNSUPPORTED;
    if (!aligned16(x_bf16) || !aligned16(xq_out) || !aligned16(sx_out) || !aligned16(wq) || !aligned16(sw) ||
        !aligned16(out_bf16) || !aligned16(y_fp32) || !aligned16(gamma_bf16) || !aligned16(beta_bf16))
        return LOKA_ERR_ALIGN;
    const int v = desc->variant >= 0 ? desc->variant : variant_xq_default(desc);
    if (v < 0 || !variant_supports_xq(desc, v)) return LOKA_ERR_UNSUPPORTED;
    return fp8_linear_norm_xq_launch(desc, v, x_bf16, xq_out, sx_out, wq, sw, gamma_bf16, beta_bf16, out_bf16, y_fp32,
                                     static_cast<hipStream_t>(hip_stream));
}

// -1 when the named variant has no FP8-output epilogue or cannot run the shape.
static int fp8out_variant(const loka_gemm_desc* desc) {
    if (desc->variant >= 0) return variant_supports_fp8out(desc, desc->variant) ? desc->variant : -1;
    return variant_fp8out_default(desc);
}

loka_status loka_fp8_gemm_norm_check(const loka_gemm_desc* desc, const void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!desc) return LOKA_ERR_NULL;
    const loka_status st = validate_desc(desc, true);
    if (st != LOKA_OK) return st;
    // `workspace` may belong to a loka_fp8_gemm_norm call or to a loka_fp8_gemm_norm_fp8out call, whose kernels (with
    // desc->variant < 0) and sizes can differ either way: enough for one of the two that wait is enough.  Every workspace
    // with a bounded wait begins with the same header.
    const int v = resolve_for_scratch(desc, workspace, ws_bytes), vq = fp8out_variant(desc);
    size_t need = SIZE_MAX;
    if (v >= 0 && variant_has_wait_flag(desc, v)) need = variant_workspace(desc, v);
    if (vq >= 0 && variant_has_wait_flag(desc, vq, true)) need = std::min(need, variant_workspace(desc, vq, true));
    if (need == SIZE_MAX) return v < 0 ? LOKA_ERR_UNSUPPORTED : LOKA_OK;
    if (!workspace || ws_bytes < need) return LOKA_ERR_WORKSPACE;
    // header of the workspace: [0] the nonce of the last launch that used it, [1] the nonce of the last launch in
    // which a wait ran out (0 in both: never used)
    unsigned long long hdr[2] = {0, 0};
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    LOKA_HIP_TRY(hipMemcpyAsync(hdr, workspace, sizeof(hdr), hipMemcpyDeviceToHost, s));
    LOKA_HIP_TRY(hipStreamSynchronize(s));
    return (hdr[0] != 0 && hdr[0] == hdr[1]) ? LOKA_ERR_TIMEOUT : LOKA_OK;
}

void loka_test_set_spin_limit(int64_t polls) { test_set_spin_limit(polls); }

loka_status loka_machine_ceiling(int kind, double millis, void* scratch, size_t scratch_bytes, double* value_host,
                                 void* hip_stream) {
    if (!scratch || !value_host) return LOKA_ERR_NULL;
    if (kind < 0 || kind > 7 || !(millis > 0.0)) return LOKA_ERR_UNSUPPORTED;
    if (!aligned16(scratch)) return LOKA_ERR_ALIGN;
    if (scratch_bytes < (size_t(1) << 22) || (kind == 2 && scratch_bytes < (size_t(1) << 26))) return LOKA_ERR_WORKSPACE;
    return machine_ceiling(kind, millis, scratch, scratch_bytes, value_host, static_cast<hipStream_t>(hip_stream));
}

size_t loka_fp8_gemm_norm_fp8out_workspace(const loka_gemm_desc* desc) {
    if (validate_desc(desc, true) != LOKA_OK) return 0;
    const int v = fp8out_variant(desc);
    return v < 0 ? 0 : variant_workspace(desc, v, true);
}

loka_status loka_fp8_gemm_norm_fp8out(const loka_gemm_desc* desc, const uint8_t* xq, const float* sx, const uint8_t* wq,
                                      const float* sw, const void* gamma_bf16, const void* beta_bf16, uint8_t* oq,
                                      float* so, float* y_fp32, void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!desc || !xq || !sx || !wq || !sw || !oq || !so) return LOKA_ERR_NULL;
    const loka_status st = validate_desc(desc, true);
    if (st != LOKA_OK) return st;
    if (!aligned16(xq) || !aligned16(wq) || !aligned16(sx) || !aligned16(sw) || !aligned16(oq) || !aligned16(so) ||
        !aligned16(y_fp32) || !aligned16(gamma_bf16) || !aligned16(beta_bf16))
        return LOKA_ERR_ALIGN;
    const int v = fp8out_variant(desc);
    if (v < 0) return LOKA_ERR_UNSUPPORTED;
    const size_t need = variant_workspace(desc, v, true);
    if (need && (!workspace || ws_bytes < need)) return LOKA_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return LOKA_ERR_ALIGN;
    return fp8_gemm_norm_launch(desc, v, xq, sx, wq, sw, gamma_bf16, beta_bf16, nullptr, y_fp32, oq, so, workspace,
                                static_cast<hipStream_t>(hip_stream));
}

size_t loka_bf16_gemm_workspace(const loka_gemm_desc* desc) {
    if (validate_desc(desc, false) != LOKA_OK) return 0;
    return bf16_gemm_workspace_bytes(desc);
}

loka_status loka_bf16_gemm(const loka_gemm_desc* desc, const void* x_bf16, const void* w_bf16, float* yref_fp32,
                           void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!desc || !x_bf16 || !w_bf16 || !yref_fp32) return LOKA_ERR_NULL;
    const loka_status st = validate_desc(desc, false);
    if (st != LOKA_OK) return st;
    if (!aligned16(x_bf16) || !aligned16(w_bf16) || !aligned16(yref_fp32)) return LOKA_ERR_ALIGN;
    if (!workspace || ws_bytes < bf16_gemm_min_workspace_bytes(desc)) return LOKA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return LOKA_ERR_ALIGN;
    return bf16_gemm_launch(desc, x_bf16, w_bf16, yref_fp32, workspace, ws_bytes, static_cast<hipStream_t>(hip_stream));
}

size_t loka_probe_error_workspace(int64_t M, int64_t N) {
    (void)M; (void)N;
    return probe_workspace_bytes();
}

loka_status loka_probe_error(const float* y, const float* yref, int64_t M, int64_t N, int64_t ld,
                             loka_probe_stats* stats_device, float* rowmax_device, void* workspace, size_t ws_bytes,
                             void* hip_stream) {
    if (!y || !yref || !stats_device) return LOKA_ERR_NULL;
    if (M <= 0 || N <= 0 || ld < N) return LOKA_ERR_SHAPE;
    if (N % 4 || ld % 4) return LOKA_ERR_SHAPE;
    if (!aligned16(y) || !aligned16(yref) || (reinterpret_cast<uintptr_t>(stats_device) & 7u)) return LOKA_ERR_ALIGN;
    if (!workspace || ws_bytes < probe_workspace_bytes()) return LOKA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return LOKA_ERR_ALIGN;
    return probe_launch(y, yref, M, N, ld, stats_device, rowmax_device, workspace,
                        static_cast<hipStream_t>(hip_stream));
}

// Shape rules of the tracker, shared by the workspace query and the call.
static loka_status validate_tracker(int64_t B, int64_t K, int64_t ld, int64_t n_old) {
    if (B <= 0 || K <= 0 || ld < K || n_old < 0) return LOKA_ERR_SHAPE;
    if (K % 8 || ld % 8) return LOKA_ERR_SHAPE;
    if (K > 32768 || B > (INT64_C(1) << 40) || n_old > (INT64_C(1) << 52)) return LOKA_ERR_SHAPE;
    return LOKA_OK;
}

size_t loka_tracker_update_workspace(int64_t B, int64_t K) {
    if (validate_tracker(B, K, K, 0) != LOKA_OK) return 0;
    return tracker_workspace_bytes(B, K);
}

loka_status loka_tracker_update(const void* x_bf16, int64_t B, int64_t K, int64_t ld, int64_t n_old, float* mu,
                                float* sigma, void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!x_bf16 || !mu || !sigma) return LOKA_ERR_NULL;
    const loka_status st = validate_tracker(B, K, ld, n_old);
    if (st != LOKA_OK) return st;
    if (!aligned16(x_bf16) || !aligned16(mu) || !aligned16(sigma)) return LOKA_ERR_ALIGN;
    if (!workspace || ws_bytes < tracker_workspace_bytes(B, K)) return LOKA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return LOKA_ERR_ALIGN;
    return tracker_update_launch(x_bf16, B, K, ld, n_old, mu, sigma, workspace, static_cast<hipStream_t>(hip_stream));
}

// ---- MXFP4
int64_t loka_mxfp4_padded(int64_t cols) { return cols <= 0 || cols > INT64_MAX - 127 ? -1 : (cols + 127) / 128 * 128; }

// More elements than any memory holds: refused before sizes are multiplied further.
static bool too_many(int64_t batch, int64_t rows, int64_t cols) {
    return static_cast<double>(batch) * static_cast<double>(rows) * static_cast<double>(cols) > 281474976710656.0;      // 2^48
}
static bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

loka_status loka_mxfp4_quantize(const void* x_bf16, int64_t rows, int64_t cols, int64_t ld, int transpose_out, uint8_t* q,
                                uint8_t* scales, void* hip_stream) {
    if (!x_bf16 || !q || !scales) return LOKA_ERR_NULL;
    if (rows <= 0 || cols <= 0 || ld < cols || rows > INT32_MAX || cols > INT32_MAX || too_many(1, rows, cols)) return LOKA_ERR_SHAPE;
    if (!aligned_to(x_bf16, 2) || !aligned16(q) || !aligned_to(scales, 4)) return LOKA_ERR_ALIGN;
    return mxfp4_quantize_launch(x_bf16, rows, cols, ld, transpose_out, q, scales, static_cast<hipStream_t>(hip_stream));
}

loka_status loka_mxfp4_dequantize(const uint8_t* q, const uint8_t* scales, int64_t rows, int64_t cols, void* out_bf16, int64_t ld,
                                  void* hip_stream) {
    if (!q || !scales || !out_bf16) return LOKA_ERR_NULL;
    if (rows <= 0 || cols <= 0 || ld < cols || rows > INT32_MAX || cols > INT32_MAX || too_many(1, rows, cols)) return LOKA_ERR_SHAPE;
    if (!aligned_to(out_bf16, 2) || !aligned16(q) || !aligned_to(scales, 4)) return LOKA_ERR_ALIGN;
    return mxfp4_dequantize_launch(q, scales, rows, cols, out_bf16, ld, static_cast<hipStream_t>(hip_stream));
}

// Shape rules of the products, shared by the workspace queries and the calls (linear: strides and batch are not read).
static loka_status validate_mxfp4(const loka_gemm_desc* d, bool linear) {
    if (!d) return LOKA_ERR_NULL;
    if (d->M <= 0 || d->N <= 0 || d->K <= 0 || d->batch <= 0) return LOKA_ERR_SHAPE;
    if (d->M > INT32_MAX || d->N > INT32_MAX || d->K > INT32_MAX || d->batch > INT32_MAX) return LOKA_ERR_SHAPE;
    if (too_many(1, d->M, d->K) || too_many(1, d->N, d->K) || too_many(d->batch, d->M, d->N)) return LOKA_ERR_SHAPE;
    if (d->norm != LOKA_NORM_NONE || d->act != LOKA_ACT_NONE || d->variant != -1) return LOKA_ERR_UNSUPPORTED;
    if (linear) return d->batch == 1 ? LOKA_OK : LOKA_ERR_UNSUPPORTED;
    if (d->batch > 1) {
        const int64_t Kp = loka_mxfp4_padded(d->K);
        if (d->strideX < 0 || d->strideW < 0 || d->strideO < d->M * d->N) return LOKA_ERR_SHAPE;
        if ((d->strideX && d->strideX < d->M * Kp) || (d->strideW && d->strideW < d->N * Kp)) return LOKA_ERR_SHAPE;
        if (d->strideX % 128 || d->strideW % 128) return LOKA_ERR_ALIGN;
    }
    return LOKA_OK;
}

int loka_test_mxfp4_form(const loka_gemm_desc* desc) { return validate_mxfp4(desc, false) != LOKA_OK ? -1 : mxfp4_gemm_form(desc); }

size_t loka_mxfp4_gemm_workspace(const loka_gemm_desc* desc) {
    return validate_mxfp4(desc, false) != LOKA_OK ? 0 : mxfp4_gemm_workspace_bytes(desc);
}

loka_status loka_mxfp4_gemm(const loka_gemm_desc* desc, const uint8_t* xq, const uint8_t* sx, const uint8_t* wq, const uint8_t* sw,
                            void* out_bf16, float* y_fp32, void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!desc || !xq || !sx || !wq || !sw || (!out_bf16 && !y_fp32)) return LOKA_ERR_NULL;
    const loka_status st = validate_mxfp4(desc, false);
    if (st != LOKA_OK) return st;
    if (!aligned16(xq) || !aligned16(wq) || !aligned_to(sx, 4) || !aligned_to(sw, 4) || !aligned16(out_bf16) || !aligned16(y_fp32) ||
        !aligned16(workspace))
        return LOKA_ERR_ALIGN;
    return mxfp4_gemm_launch(desc, xq, sx, wq, sw, out_bf16, y_fp32, workspace, workspace ? ws_bytes : 0,
                             static_cast<hipStream_t>(hip_stream));
}

// The workspace of the layer: codes of x, then their scales, then the product's own.
static size_t linear_codes_bytes(const loka_gemm_desc* d) {
    const size_t n = static_cast<size_t>(d->M) * static_cast<size_t>(loka_mxfp4_padded(d->K));
    return n / 2 + (n / 32 + 15) / 16 * 16;
}
size_t loka_mxfp4_linear_workspace(const loka_gemm_desc* desc) {
    if (validate_mxfp4(desc, true) != LOKA_OK || mxfp4_linear_fused(desc)) return 0;
    return linear_codes_bytes(desc) + mxfp4_gemm_workspace_bytes(desc);
}

loka_status loka_mxfp4_linear(const loka_gemm_desc* desc, const void* x_bf16, int64_t ld, const uint8_t* wq, const uint8_t* sw,
                              void* out_bf16, float* y_fp32, void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!desc || !x_bf16 || !wq || !sw || (!out_bf16 && !y_fp32)) return LOKA_ERR_NULL;
    const loka_status st = validate_mxfp4(desc, true);
    if (st != LOKA_OK) return st;
    if (ld < desc->K) return LOKA_ERR_SHAPE;
    if (!aligned_to(x_bf16, 2) || !aligned16(wq) || !aligned_to(sw, 4) || !aligned16(out_bf16) || !aligned16(y_fp32)) return LOKA_ERR_ALIGN;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (mxfp4_linear_fused(desc)) return mxfp4_linear_fused_launch(desc, x_bf16, ld, wq, sw, out_bf16, y_fp32, stream);
    const size_t need = loka_mxfp4_linear_workspace(desc);
    if (!workspace || ws_bytes < need) return LOKA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return LOKA_ERR_ALIGN;
    uint8_t* const xq = static_cast<uint8_t*>(workspace);
    uint8_t* const sx = xq + static_cast<size_t>(desc->M) * static_cast<size_t>(loka_mxfp4_padded(desc->K)) / 2;
    const size_t used = linear_codes_bytes(desc);
    const loka_status sq = mxfp4_quantize_launch(x_bf16, desc->M, desc->K, ld, 0, xq, sx, stream);
    if (sq != LOKA_OK) return sq;
    return mxfp4_gemm_launch(desc, xq, sx, wq, sw, out_bf16, y_fp32, xq + used, ws_bytes - used, stream);
}

// ---- residual addition + RMSNorm
static bool rms_mode_ok(int m) { return m == LOKA_SCALE_ROW || is_block_x(m); }

// Shape rules shared by the forward pass, the backward pass and its workspace query.
static loka_status validate_rms(const loka_rms_desc* d) {
    if (!d) return LOKA_ERR_NULL;
    if (d->rows <= 0 || d->cols <= 0 || d->cols % 16) return LOKA_ERR_SHAPE;
    if (d->rows > INT32_MAX || d->cols > 32768) return LOKA_ERR_SHAPE;
    return LOKA_OK;
}
// An output over an input (contiguous rows over rows `ld` apart) has to have its row stride: each element is then read before it is written.
static bool rms_in_place_ok(const loka_rms_desc* d, const void* out, const void* in, int64_t ld) {
    return out == nullptr || out != in || d->rows == 1 || ld == d->cols;
}
// ... and those of a matrix with scales in `mode`
static loka_status validate_rms_mode(const loka_rms_desc* d, int mode) {
    if (!rms_mode_ok(mode)) return LOKA_ERR_UNSUPPORTED;
    return is_block_x(mode) && d->cols % 128 ? LOKA_ERR_SHAPE : LOKA_OK;
}

loka_status loka_add_rmsnorm(const loka_rms_desc* desc, const void* x_bf16, const void* residual_bf16, const void* gamma_bf16,
                             void* h_out_bf16, void* y_out, void* y_scales, uint8_t* hq, float* hs, float* rstd, void* hip_stream) {
    if (!desc || !x_bf16 || !y_out) return LOKA_ERR_NULL;
    loka_status st = validate_rms(desc);
    if (st != LOKA_OK) return st;
    if (desc->out < LOKA_RMS_OUT_BF16 || desc->out > LOKA_RMS_OUT_MXFP4 || !(desc->eps >= 0.f)) return LOKA_ERR_UNSUPPORTED;
    if ((desc->out != LOKA_RMS_OUT_BF16 && !y_scales) || (hq != nullptr) != (hs != nullptr)) return LOKA_ERR_NULL;
    if (desc->out == LOKA_RMS_OUT_E4M3 && (st = validate_rms_mode(desc, desc->out_mode)) != LOKA_OK) return st;
    if (hq && (st = validate_rms_mode(desc, desc->ckpt_mode)) != LOKA_OK) return st;
    if (desc->ld_x < desc->cols || (residual_bf16 && desc->ld_r < desc->cols)) return LOKA_ERR_SHAPE;
    if (desc->ld_x % 8 || (residual_bf16 && desc->ld_r % 8)) return LOKA_ERR_ALIGN;
    if (!aligned16(x_bf16) || !aligned16(residual_bf16) || !aligned16(gamma_bf16) || !aligned16(h_out_bf16) || !aligned16(y_out) ||
        !aligned16(hq) || !aligned_to(y_scales, 4) || !aligned_to(hs, 4) || !aligned_to(rstd, 4))
        return LOKA_ERR_ALIGN;
    if (!rms_in_place_ok(desc, h_out_bf16, x_bf16, desc->ld_x) || !rms_in_place_ok(desc, h_out_bf16, residual_bf16, desc->ld_r)) return LOKA_ERR_SHAPE;
    return add_rmsnorm_launch(desc, x_bf16, residual_bf16, gamma_bf16, h_out_bf16, y_out, y_scales, hq, hs, rstd,
                              static_cast<hipStream_t>(hip_stream));
}

size_t loka_rmsnorm_backward_workspace(const loka_rms_desc* desc) {
    return validate_rms(desc) != LOKA_OK ? 0 : rmsnorm_backward_workspace_bytes(desc->rows, desc->cols);
}

loka_status loka_rmsnorm_backward(const loka_rms_desc* desc, const void* dy_bf16, const uint8_t* hq, const float* hs, const float* rstd,
                                  const void* gamma_bf16, const void* dh_bf16, void* dx_bf16, float* dgamma, void* workspace,
                                  size_t ws_bytes, void* hip_stream) {
    if (!desc || !dy_bf16 || !hq || !hs || !rstd || !dx_bf16) return LOKA_ERR_NULL;
    loka_status st = validate_rms(desc);
    if (st != LOKA_OK) return st;
    if ((st = validate_rms_mode(desc, desc->ckpt_mode)) != LOKA_OK) return st;
    if (desc->ld_x < desc->cols || (dh_bf16 && desc->ld_r < desc->cols)) return LOKA_ERR_SHAPE;
    if (desc->ld_x % 8 || (dh_bf16 && desc->ld_r % 8)) return LOKA_ERR_ALIGN;
    if (!aligned16(dy_bf16) || !aligned16(hq) || !aligned16(gamma_bf16) || !aligned16(dh_bf16) || !aligned16(dx_bf16) ||
        !aligned_to(hs, 4) || !aligned_to(rstd, 4) || !aligned_to(dgamma, 4))
        return LOKA_ERR_ALIGN;
    if (!rms_in_place_ok(desc, dx_bf16, dy_bf16, desc->ld_x) || !rms_in_place_ok(desc, dx_bf16, dh_bf16, desc->ld_r)) return LOKA_ERR_SHAPE;
    if (dgamma) {
        if (!workspace || ws_bytes < rmsnorm_backward_workspace_bytes(desc->rows, desc->cols)) return LOKA_ERR_WORKSPACE;
        if (!aligned16(workspace)) return LOKA_ERR_ALIGN;
    }
    return rmsnorm_backward_launch(desc, dy_bf16, hq, hs, rstd, gamma_bf16, dh_bf16, dx_bf16, dgamma, workspace,
                                   static_cast<hipStream_t>(hip_stream));
}

// ---- a layer of experts
static loka_status validate_route(const loka_route_desc* d) {
    if (!d) return LOKA_ERR_NULL;
    if (d->tokens <= 0 || d->tokens > (INT64_C(1) << 25) || d->experts <= 0 || d->experts > 1024 || d->top_k <= 0 || d->top_k > 16 || d->top_k > d->experts ||
        d->ld < d->experts || too_many(1, d->tokens, d->ld))
        return LOKA_ERR_SHAPE;
    return d->score == LOKA_SCORE_SOFTMAX || d->score == LOKA_SCORE_SIGMOID ? LOKA_OK : LOKA_ERR_UNSUPPORTED;
}

size_t loka_route_workspace(const loka_route_desc* desc) { return validate_route(desc) != LOKA_OK ? 0 : route_workspace_bytes(desc); }

loka_status loka_route(const loka_route_desc* desc, const void* logits, int32_t* expert, float* weight, int32_t* slot, int32_t* row,
                       int32_t* offsets, void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!desc || !logits || !expert || !weight || !slot || !row || !offsets) return LOKA_ERR_NULL;
    const loka_status st = validate_route(desc);
    if (st != LOKA_OK) return st;
    if (!aligned_to(logits, desc->bf16 ? 2 : 4) || !aligned_to(expert, 4) || !aligned_to(weight, 4) || !aligned_to(slot, 4) || !aligned_to(row, 4) ||
        !aligned_to(offsets, 4))
        return LOKA_ERR_ALIGN;
    const size_t need = route_workspace_bytes(desc);
    if (need && (!workspace || ws_bytes < need)) return LOKA_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return LOKA_ERR_ALIGN;
    return route_launch(desc, logits, expert, weight, slot, row, offsets, workspace, static_cast<hipStream_t>(hip_stream));
}

loka_status loka_route_backward(const loka_route_desc* desc, const void* logits, const int32_t* expert, const float* dweight, void* dlogits,
                                void* hip_stream) {
    if (!desc || !logits || !expert || !dweight || !dlogits) return LOKA_ERR_NULL;
    const loka_status st = validate_route(desc);
    if (st != LOKA_OK) return st;
    const uintptr_t size = desc->bf16 ? 2 : 4;
    if (!aligned_to(logits, size) || !aligned_to(dlogits, size) || !aligned_to(expert, 4) || !aligned_to(dweight, 4)) return LOKA_ERR_ALIGN;
    return route_backward_launch(desc, logits, expert, dweight, dlogits, static_cast<hipStream_t>(hip_stream));
}

constexpr int64_t kMostWidth = INT64_C(1) << 20;       // of a layer of experts, so that a tile's rows lie within 32-bit offsets

int64_t loka_grouped_blocks(int64_t rows, int64_t groups) {
    if (rows <= 0 || rows > INT32_MAX || groups <= 0 || groups > kMostGroups) return -1;
    return (rows + (kGroupBlock - 1) * std::min(rows, groups)) / kGroupBlock;
}

static loka_status grouped_quantize_checked(const loka_grouped_quantize_desc* d, const void* x, const int32_t* index, const int32_t* offsets, uint8_t* q,
                                            float* scales, uint8_t* qt, float* st, void* hip_stream) {
    if (d->rows <= 0 || d->rows > INT32_MAX || d->cols <= 0 || d->cols > kMostWidth || d->ld < d->cols || d->groups <= 0 || d->groups > kMostGroups) return LOKA_ERR_SHAPE;
    if (index && (d->x_rows <= 0 || d->x_rows > INT32_MAX)) return LOKA_ERR_SHAPE;
    if (too_many(1, d->rows, d->cols) || too_many(1, index ? d->x_rows : d->rows, d->ld)) return LOKA_ERR_SHAPE;
    if (!offsets && d->rows % d->groups) return LOKA_ERR_SHAPE;
    if (!aligned_to(x, 2) || !aligned_to(index, 4) || !aligned_to(offsets, 4) || !aligned16(q) || !aligned16(qt) || !aligned_to(scales, 4) || !aligned_to(st, 4))
        return LOKA_ERR_ALIGN;
    return grouped_quantize_launch(d, x, index, offsets, q, scales, qt, st, static_cast<hipStream_t>(hip_stream));
}

loka_status loka_grouped_quantize(const loka_grouped_quantize_desc* desc, const void* x_bf16, const int32_t* index, const int32_t* offsets,
                                  uint8_t* q, float* scales, uint8_t* qt, float* st, void* hip_stream) {
    if (!desc || !x_bf16 || (q != nullptr) != (scales != nullptr) || (qt != nullptr) != (st != nullptr) || (!q && !qt)) return LOKA_ERR_NULL;
    return grouped_quantize_checked(desc, x_bf16, index, offsets, q, scales, qt, st, hip_stream);
}

static loka_status validate_grouped(const loka_grouped_desc* d, bool gathered) {
    if (!d) return LOKA_ERR_NULL;
    if (d->rows <= 0 || d->rows > INT32_MAX || d->N <= 0 || d->N > kMostWidth || d->K <= 0 || d->K > kMostWidth || d->groups <= 0 || d->groups > kMostGroups)
        return LOKA_ERR_SHAPE;
    if (gathered && (d->x_rows <= 0 || d->x_rows > INT32_MAX)) return LOKA_ERR_SHAPE;
    if (too_many(256, d->rows, d->N) || too_many(256, d->rows, d->K)) return LOKA_ERR_SHAPE;       // 2^40
    return LOKA_OK;
}
static bool grouped_wgrad_ok(const loka_grouped_desc* d) { return !too_many(256 * static_cast<int64_t>(d->groups), d->K, d->N) && grouped_wgrad_fits(d); }
static loka_status validate_grouped_gemm(const loka_grouped_desc* d, bool gathered) {
    const loka_status st = validate_grouped(d, gathered);
    if (st != LOKA_OK) return st;
    if (!grouped_gemm_fits(d)) return LOKA_ERR_SHAPE;
    return d->w_form == LOKA_W_TURNED || d->w_form == LOKA_W_ALONG ? LOKA_OK : LOKA_ERR_UNSUPPORTED;
}

loka_status loka_grouped_gemm(const loka_grouped_desc* desc, const uint8_t* xq, const float* sx, const int32_t* index, const int32_t* offsets,
                              const uint8_t* wq, const float* sw, void* out_bf16, float* y_fp32, void* hip_stream) {
    if (!desc || !xq || !sx || !offsets || !wq || !sw || (!out_bf16 && !y_fp32)) return LOKA_ERR_NULL;
    const loka_status st = validate_grouped_gemm(desc, index != nullptr);
    if (st != LOKA_OK) return st;
    if (!aligned16(xq) || !aligned_to(sx, 4) || !aligned_to(index, 4) || !aligned_to(offsets, 4) || !aligned16(wq) || !aligned_to(sw, 4) ||
        !aligned16(out_bf16) || !aligned16(y_fp32))
        return LOKA_ERR_ALIGN;
    return grouped_gemm_launch(desc, xq, sx, index, offsets, wq, sw, out_bf16, y_fp32, static_cast<hipStream_t>(hip_stream));
}

// The workspace of the layer: codes of x, then their scales.
size_t loka_grouped_linear_workspace(const loka_grouped_desc* desc, int with_index) {
    if (validate_grouped_gemm(desc, with_index != 0) != LOKA_OK || grouped_linear_fused(desc)) return 0;
    const size_t n = static_cast<size_t>(with_index ? desc->x_rows : desc->rows) * static_cast<size_t>(group_blocks(desc->K));
    return n * kGroupBlock + (n * 4 + 15) / 16 * 16;
}

loka_status loka_grouped_linear(const loka_grouped_desc* desc, const void* x_bf16, int64_t ld, const int32_t* index, const int32_t* offsets,
                                const uint8_t* wq, const float* sw, void* out_bf16, float* y_fp32, void* workspace, size_t ws_bytes,
                                void* hip_stream) {
    if (!desc || !x_bf16 || !offsets || !wq || !sw || (!out_bf16 && !y_fp32)) return LOKA_ERR_NULL;
    const loka_status st = validate_grouped_gemm(desc, index != nullptr);
    if (st != LOKA_OK) return st;
    if (ld < desc->K) return LOKA_ERR_SHAPE;
    if (!aligned_to(x_bf16, 2) || !aligned_to(index, 4) || !aligned_to(offsets, 4) || !aligned16(wq) || !aligned_to(sw, 4) || !aligned16(out_bf16) ||
        !aligned16(y_fp32))
        return LOKA_ERR_ALIGN;
    if (grouped_linear_fused(desc))
        return grouped_linear_fused_launch(desc, x_bf16, ld, index, offsets, wq, sw, out_bf16, y_fp32, static_cast<hipStream_t>(hip_stream));
    const size_t need = loka_grouped_linear_workspace(desc, index != nullptr);
    if (need && (!workspace || ws_bytes < need)) return LOKA_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return LOKA_ERR_ALIGN;
    const int64_t rows = index ? desc->x_rows : desc->rows;
    uint8_t* const xq = static_cast<uint8_t*>(workspace);
    float* const sx = reinterpret_cast<float*>(xq + static_cast<size_t>(rows) * static_cast<size_t>(group_blocks(desc->K)) * kGroupBlock);
    const loka_grouped_quantize_desc qd{rows, desc->K, ld, rows, 1};
    const loka_status sq = grouped_quantize_checked(&qd, x_bf16, nullptr, nullptr, xq, sx, nullptr, nullptr, hip_stream);
    if (sq != LOKA_OK) return sq;
    return grouped_gemm_launch(desc, xq, sx, index, offsets, wq, sw, out_bf16, y_fp32, static_cast<hipStream_t>(hip_stream));
}

size_t loka_grouped_wgrad_workspace(const loka_grouped_desc* desc) {
    return validate_grouped(desc, false) != LOKA_OK || !grouped_wgrad_ok(desc) ? 0 : grouped_wgrad_workspace_bytes(desc);
}

loka_status loka_grouped_wgrad(const loka_grouped_desc* desc, const uint8_t* xt, const float* sxt, const uint8_t* dyt, const float* sdyt,
                               const int32_t* offsets, void* dw_bf16, float* dw_fp32, void* workspace, size_t ws_bytes, void* hip_stream) {
    if (!desc || !xt || !sxt || !dyt || !sdyt || !offsets || (!dw_bf16 && !dw_fp32)) return LOKA_ERR_NULL;
    const loka_status st = validate_grouped(desc, false);
    if (st != LOKA_OK) return st;
    if (!grouped_wgrad_ok(desc)) return LOKA_ERR_SHAPE;
    if (!aligned16(xt) || !aligned_to(sxt, 4) || !aligned16(dyt) || !aligned_to(sdyt, 4) || !aligned_to(offsets, 4) || !aligned16(dw_bf16) || !aligned16(dw_fp32))
        return LOKA_ERR_ALIGN;
    const size_t need = grouped_wgrad_workspace_bytes(desc);
    if (need && (!workspace || ws_bytes < need)) return LOKA_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return LOKA_ERR_ALIGN;
    return grouped_wgrad_launch(desc, xt, sxt, dyt, sdyt, offsets, dw_bf16, dw_fp32, workspace, static_cast<hipStream_t>(hip_stream));
}

static loka_status validate_combine(const loka_combine_desc* d) {
    if (!d) return LOKA_ERR_NULL;
    if (d->tokens <= 0 || d->top_k <= 0 || d->top_k > 16 || d->tokens > (INT64_C(1) << 30) / d->top_k || d->cols <= 0 || d->cols > kMostWidth || d->rows <= 0 ||
        d->rows > INT32_MAX || too_many(1, d->rows, d->cols) || too_many(1, d->tokens, d->cols))
        return LOKA_ERR_SHAPE;
    return LOKA_OK;
}

loka_status loka_combine(const loka_combine_desc* desc, const void* y_bf16, const int32_t* slot, const float* weight,
                         const void* residual_bf16, void* out_bf16, void* hip_stream) {
    if (!desc || !y_bf16 || !slot || !out_bf16) return LOKA_ERR_NULL;
    const loka_status st = validate_combine(desc);
    if (st != LOKA_OK) return st;
    if (!aligned_to(y_bf16, 2) || !aligned_to(slot, 4) || !aligned_to(weight, 4) || !aligned_to(residual_bf16, 2) || !aligned_to(out_bf16, 2)) return LOKA_ERR_ALIGN;
    return combine_launch(desc, y_bf16, slot, weight, residual_bf16, out_bf16, static_cast<hipStream_t>(hip_stream));
}

loka_status loka_combine_backward(const loka_combine_desc* desc, const void* dout_bf16, const void* y_bf16, const int32_t* slot,
                                  const float* weight, void* dy_bf16, float* dweight, void* hip_stream) {
    if (!desc || !dout_bf16 || !slot || (!dy_bf16 && !dweight) || (dweight && !y_bf16)) return LOKA_ERR_NULL;
    const loka_status st = validate_combine(desc);
    if (st != LOKA_OK) return st;
    if (!aligned_to(dout_bf16, 2) || !aligned_to(y_bf16, 2) || !aligned_to(slot, 4) || !aligned_to(weight, 4) || !aligned_to(dy_bf16, 2) || !aligned_to(dweight, 4))
        return LOKA_ERR_ALIGN;
    return combine_backward_launch(desc, dout_bf16, y_bf16, slot, weight, dy_bf16, dweight, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
