// C ABI of libsemanticache: argument validation on the host, then the kernel launchers.
// Everything that can be rejected without touching the device is rejected before any HIP call.
#include "../../include/semanticache.h"

#include <string.h>

#include "sc_host.h"
#include "sc_paged.h"
#include "sc_rows_meet.h"
#include <algorithm>
#include <vector>

namespace sc {

Tuning &tuning() {
    static Tuning t;
    return t;
}

static thread_local char g_last_error[256] = "";

static sc_status runtime_status(hipError_t e) {
    if (e == hipSuccess) return SC_OK;
    strncpy(g_last_error, hipGetErrorString(e), sizeof(g_last_error) - 1);
    g_last_error[sizeof(g_last_error) - 1] = 0;
    return SC_ERR_RUNTIME;
}

static bool dtype_ok(int t) { return t == SC_F32 || t == SC_BF16; }
static size_t elem_size(int t) { return t == SC_BF16 ? 2 : 4; }
static bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace sc

using namespace sc;

extern "C" {

const char *sc_status_string(sc_status status) {
    switch (status) {
        case SC_OK: return "SC_OK";
        case SC_ERR_INVALID_ARG: return "SC_ERR_INVALID_ARG";
        case SC_ERR_UNSUPPORTED: return "SC_ERR_UNSUPPORTED";
        case SC_ERR_CAPACITY: return "SC_ERR_CAPACITY";
        case SC_ERR_WORKSPACE: return "SC_ERR_WORKSPACE";
        case SC_ERR_RUNTIME: return "SC_ERR_RUNTIME";
    }
    return "SC_ERR_UNKNOWN";
}

const char *sc_last_runtime_error(void) { return g_last_error; }

const char *sc_version(void) { return "0.1.0"; }

int sc_tune_set(const char *key, int value) {
    if (!key) return -1;
    Tuning &t = tuning();
    if (!strcmp(key, "decode_max_splits")) t.decode_max_splits = value;
    else if (!strcmp(key, "decode_min_rows")) t.decode_min_rows = value;
    else if (!strcmp(key, "decode_mfma_min_group")) t.decode_mfma_min_group = value;
    else if (!strcmp(key, "decode_local_handover")) t.decode_local_handover = value;
    else if (!strcmp(key, "decode_poll_budget")) t.decode_poll_budget = value;
    else if (!strcmp(key, "gsc_chunks_per_item")) t.gsc_chunks_per_item = value;
    else if (!strcmp(key, "gsc_grid_x")) t.gsc_grid_x = value;
    else if (!strcmp(key, "gsc_fast_path")) t.gsc_fast_path = value;
    else if (!strcmp(key, "gsc_chunks_per_task")) t.gsc_chunks_per_task = value;
    else if (!strcmp(key, "gsc_polls")) t.gsc_polls = value;
    else if (!strcmp(key, "multi_block_rows")) t.multi_block_rows = value;
    else if (!strcmp(key, "global_polls")) t.global_polls = value;
    else if (!strcmp(key, "multi_target_wgs")) t.multi_target_wgs = value;
    else return -1;
    return 0;
}

int sc_tune_get(const char *key) {
    if (!key) return -1;
    const Tuning &t = tuning();
    if (!strcmp(key, "decode_max_splits")) return t.decode_max_splits;
    if (!strcmp(key, "decode_min_rows")) return t.decode_min_rows;
    if (!strcmp(key, "decode_mfma_min_group")) return t.decode_mfma_min_group;
    if (!strcmp(key, "decode_local_handover")) return t.decode_local_handover;
    if (!strcmp(key, "decode_poll_budget")) return t.decode_poll_budget;
    if (!strcmp(key, "gsc_chunks_per_item")) return t.gsc_chunks_per_item;
    if (!strcmp(key, "gsc_grid_x")) return t.gsc_grid_x;
    if (!strcmp(key, "gsc_fast_path")) return t.gsc_fast_path;
    if (!strcmp(key, "gsc_chunks_per_task")) return t.gsc_chunks_per_task;
    if (!strcmp(key, "gsc_polls")) return t.gsc_polls;
    if (!strcmp(key, "multi_block_rows")) return t.multi_block_rows;
    if (!strcmp(key, "global_polls")) return t.global_polls;
    if (!strcmp(key, "multi_target_wgs")) return t.multi_target_wgs;
    return -1;
}

// ------------------------------------------------------------------------------------------------
sc_status sc_check_lengths(const int32_t *lengths, int count, int *first_bad, void *stream) {
    if (!lengths || count <= 0 || !aligned4(lengths)) return SC_ERR_INVALID_ARG;
    if (first_bad) *first_bad = -1;
    std::vector<int32_t> host((size_t)count);
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e = hipMemcpyAsync(host.data(), lengths, (size_t)count * sizeof(int32_t), hipMemcpyDeviceToHost, st);
    if (e == hipSuccess) e = hipStreamSynchronize(st);
    if (e != hipSuccess) return runtime_status(e);
    for (int i = 0; i < count; ++i)
        if (host[i] < 0) {
            if (first_bad) *first_bad = i;
            return SC_ERR_CAPACITY;
        }
    return SC_OK;
}

// ------------------------------------------------------------------------------------------------
sc_status sc_stream_read_probe(const void *src, size_t bytes, void *sink, void *stream) {
    if (!src || !sink || bytes < 16 || !aligned16(src) || !aligned4(sink)) return SC_ERR_INVALID_ARG;
    return runtime_status(launch_stream_read_probe(src, bytes, sink, static_cast<hipStream_t>(stream)));
}

// ------------------------------------------------------------------------------------------------
size_t sc_segment_workspace_bytes(int B, int N_max) {
    (void)B; (void)N_max;
    return 0;
}

sc_status sc_segment(const uint8_t *mask, int64_t mask_stride_b, const int32_t *seq_lens, int B, int N_max,
                     int32_t *offsets, int64_t offsets_stride_b, int offsets_cap, int32_t *num_chunks,
                     void *ws, size_t ws_bytes, void *stream) {
    (void)ws; (void)ws_bytes;
    if (!mask || !offsets || !num_chunks) return SC_ERR_INVALID_ARG;
    if (B <= 0 || N_max <= 0) return SC_ERR_INVALID_ARG;
    if (offsets_cap < 2) return SC_ERR_CAPACITY;
    if (mask_stride_b < N_max || offsets_stride_b < offsets_cap) return SC_ERR_INVALID_ARG;
    if (!aligned4(offsets) || !aligned4(num_chunks) || (seq_lens && !aligned4(seq_lens))) return SC_ERR_INVALID_ARG;
    if (B > 65535 * 32 || (N_max + 32767) / 32768 > 65535) return SC_ERR_UNSUPPORTED;   // grid sizes
    return runtime_status(launch_segment(mask, mask_stride_b, seq_lens, B, N_max, offsets, offsets_stride_b,
                                         offsets_cap, num_chunks, static_cast<hipStream_t>(stream)));
}

// ------------------------------------------------------------------------------------------------
size_t sc_gsc_merge_workspace_bytes(int B, int Hkv, int N_max, int d) {
    if (B <= 0 || Hkv <= 0 || N_max <= 0) return 0;
    return gsc_merge_workspace_bytes(B, Hkv, N_max, d);
}
size_t sc_gsc_merge_workspace_bytes_for(int B, int Hkv, int N_max, int d, sc_dtype out_dtype) {
    if (B <= 0 || Hkv <= 0 || N_max <= 0 || !dtype_ok(out_dtype)) return 0;
    return gsc_merge_workspace_bytes(B, Hkv, N_max, d, (int)elem_size(out_dtype));
}

static sc_status gsc_check_and_fill(const void *K, const void *V, sc_dtype in_dtype, int64_t stride_b, int64_t stride_h,
                                    int64_t stride_n, const int32_t *seq_lens, const int32_t *offsets,
                                    int64_t offsets_stride_b, const int32_t *num_chunks, int B, int Hkv, int N_max, int d,
                                    float tau, void *Kc, void *Vc, sc_dtype out_dtype, int cap, int32_t *counts,
                                    const int32_t *base_lens, bool append, int32_t *comp_lens, int32_t *cluster_id,
                                    void *ws, size_t ws_bytes, GscMergeArgs &a) {
    if (!K || !V || !offsets || !num_chunks || !Kc || !Vc || !counts || !comp_lens) return SC_ERR_INVALID_ARG;
    // every workgroup reads the old length while one of them files the new one
    if (append && (!base_lens || base_lens == comp_lens || !aligned4(base_lens))) return SC_ERR_INVALID_ARG;
    if (B <= 0 || Hkv <= 0 || N_max <= 0) return SC_ERR_INVALID_ARG;
    if (cap <= 0) return SC_ERR_CAPACITY;
    if (!dtype_ok(in_dtype) || !dtype_ok(out_dtype)) return SC_ERR_UNSUPPORTED;
    if (d != 64 && d != 128) return SC_ERR_UNSUPPORTED;
    if (Hkv > 65535 || B > 65535 || (long long)B * Hkv > (1 << 24)) return SC_ERR_UNSUPPORTED;   // grid sizes
    const size_t es = elem_size(in_dtype);
    if (stride_n < d || stride_h < 0 || stride_b < 0) return SC_ERR_INVALID_ARG;
    if ((stride_n * es) % 16 || (stride_h * es) % 16 || (stride_b * es) % 16) return SC_ERR_INVALID_ARG;
    if (!aligned16(K) || !aligned16(V) || !aligned16(Kc) || !aligned16(Vc)) return SC_ERR_INVALID_ARG;
    if (!aligned4(counts) || !aligned4(comp_lens) || !aligned4(offsets) || !aligned4(num_chunks)) return SC_ERR_INVALID_ARG;
    if (offsets_stride_b < 2) return SC_ERR_INVALID_ARG;
    if (tau != tau) return SC_ERR_INVALID_ARG;
    const size_t need = gsc_merge_workspace_bytes(B, Hkv, N_max, d, (int)elem_size(out_dtype));
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SC_ERR_WORKSPACE;

    a.K = K; a.V = V; a.in_dtype = static_cast<DType>(in_dtype);
    a.stride_b = stride_b; a.stride_h = stride_h; a.stride_n = stride_n;
    a.seq_lens = seq_lens; a.offsets = offsets; a.offsets_stride_b = offsets_stride_b; a.num_chunks = num_chunks;
    a.B = B; a.Hkv = Hkv; a.N_max = N_max; a.d = d; a.tau = tau;
    a.Kc = Kc; a.Vc = Vc; a.out_dtype = static_cast<DType>(out_dtype); a.cap = cap;
    a.counts = counts; a.comp_lens = comp_lens; a.cluster_id = cluster_id; a.ws = ws;
    a.base_lens = append ? base_lens : nullptr;
    a.tune = tuning();
    return SC_OK;
}

static sc_status gsc_common(const void *K, const void *V, sc_dtype in_dtype, int64_t stride_b, int64_t stride_h,
                            int64_t stride_n, const int32_t *seq_lens, const int32_t *offsets, int64_t offsets_stride_b,
                            const int32_t *num_chunks, int B, int Hkv, int N_max, int d, float tau, void *Kc, void *Vc,
                            sc_dtype out_dtype, int cap, int32_t *counts, const int32_t *base_lens, bool append,
                            int32_t *comp_lens, int32_t *cluster_id, void *ws, size_t ws_bytes, void *stream) {
    GscMergeArgs a;
    const sc_status st = gsc_check_and_fill(K, V, in_dtype, stride_b, stride_h, stride_n, seq_lens, offsets, offsets_stride_b,
                                            num_chunks, B, Hkv, N_max, d, tau, Kc, Vc, out_dtype, cap, counts, base_lens,
                                            append, comp_lens, cluster_id, ws, ws_bytes, a);
    if (st != SC_OK) return st;
    return runtime_status(launch_gsc_merge(a, static_cast<hipStream_t>(stream)));
}

sc_status sc_gsc_merge(const void *K, const void *V, sc_dtype in_dtype, int64_t stride_b, int64_t stride_h,
                       int64_t stride_n, const int32_t *seq_lens, const int32_t *offsets, int64_t offsets_stride_b,
                       const int32_t *num_chunks, int B, int Hkv, int N_max, int d, float tau, void *Kc, void *Vc,
                       sc_dtype out_dtype, int cap, int32_t *counts, int32_t *comp_lens, int32_t *cluster_id,
                       void *ws, size_t ws_bytes, void *stream) {
    return gsc_common(K, V, in_dtype, stride_b, stride_h, stride_n, seq_lens, offsets, offsets_stride_b, num_chunks, B, Hkv,
                      N_max, d, tau, Kc, Vc, out_dtype, cap, counts, nullptr, false, comp_lens, cluster_id, ws, ws_bytes,
                      stream);
}

sc_status sc_gsc_merge_append(const void *K, const void *V, sc_dtype in_dtype, int64_t stride_b, int64_t stride_h,
                              int64_t stride_n, const int32_t *seq_lens, const int32_t *offsets,
                              int64_t offsets_stride_b, const int32_t *num_chunks, int B, int Hkv, int N_max, int d,
                              float tau, void *Kc, void *Vc, sc_dtype out_dtype, int cap, int32_t *counts,
                              const int32_t *base_lens, int32_t *comp_lens, int32_t *cluster_id, void *ws,
                              size_t ws_bytes, void *stream) {
    return gsc_common(K, V, in_dtype, stride_b, stride_h, stride_n, seq_lens, offsets, offsets_stride_b, num_chunks, B, Hkv,
                      N_max, d, tau, Kc, Vc, out_dtype, cap, counts, base_lens, true, comp_lens, cluster_id, ws, ws_bytes,
                      stream);
}

size_t sc_gsc_merge_global_workspace_bytes(int B, int Hkv, int N_max, int d) {
    if (B <= 0 || Hkv <= 0 || N_max <= 0) return 0;
    return gsc_global_workspace_bytes(B, Hkv, N_max, d);
}

sc_status sc_gsc_merge_global(const void *K, const void *V, sc_dtype in_dtype, int64_t stride_b, int64_t stride_h,
                              int64_t stride_n, const int32_t *seq_lens, int B, int Hkv, int N_max, int d, float tau,
                              void *Kc, void *Vc, sc_dtype out_dtype, int cap, int32_t *counts, int32_t *comp_lens,
                              int32_t *cluster_id, void *ws, size_t ws_bytes, void *stream) {
    if (B <= 0 || Hkv <= 0 || N_max <= 0) return SC_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SC_ERR_WORKSPACE;
    // the start of the workspace takes the one-chunk offsets; everything else is checked as for sc_gsc_merge
    int32_t *offsets = reinterpret_cast<int32_t *>(ws), *num_chunks = offsets + 2 * B;
    GscMergeArgs a;
    const sc_status st = gsc_check_and_fill(K, V, in_dtype, stride_b, stride_h, stride_n, seq_lens, offsets, 2, num_chunks, B, Hkv,
                                            N_max, d, tau, Kc, Vc, out_dtype, cap, counts, nullptr, false, comp_lens, cluster_id,
                                            ws, ws_bytes, a);
    if (st != SC_OK) return st;
    if (ws_bytes < gsc_global_workspace_bytes(B, Hkv, N_max, d)) return SC_ERR_WORKSPACE;
    return runtime_status(launch_gsc_global(a, static_cast<hipStream_t>(stream)));
}

size_t sc_gsc_merge_budget_workspace_bytes(int B, int Hkv, int N_max, int d) {
    if (B <= 0 || Hkv <= 0 || N_max <= 0) return 0;
    return align_up(gsc_merge_workspace_bytes(B, Hkv, N_max, d), 256) + gsc_budget_state_bytes();
}

sc_status sc_gsc_merge_budget(const void *K, const void *V, sc_dtype in_dtype, int64_t stride_b, int64_t stride_h,
                              int64_t stride_n, const int32_t *seq_lens, const int32_t *offsets,
                              int64_t offsets_stride_b, const int32_t *num_chunks, int B, int Hkv, int N_max, int d,
                              int64_t budget_rows, float tau_lo, float tau_hi, int iterations, void *Kc, void *Vc,
                              sc_dtype out_dtype, int cap, int32_t *counts, int32_t *comp_lens, int32_t *cluster_id,
                              float *tau_out, int64_t *rows_out, void *ws, size_t ws_bytes, void *stream) {
    if (!tau_out || !aligned4(tau_out) || (rows_out && (reinterpret_cast<uintptr_t>(rows_out) & 7u))) return SC_ERR_INVALID_ARG;
    if (iterations < 0 || iterations > 32 || budget_rows < 0) return SC_ERR_INVALID_ARG;
    if (tau_lo != tau_lo || tau_hi != tau_hi || tau_lo > tau_hi) return SC_ERR_INVALID_ARG;
    if (B <= 0 || Hkv <= 0 || N_max <= 0) return SC_ERR_INVALID_ARG;
    // everything else is checked exactly as for sc_gsc_merge (no launch happens on a failed check)
    GscMergeArgs a;
    const sc_status st = gsc_check_and_fill(K, V, in_dtype, stride_b, stride_h, stride_n, seq_lens, offsets, offsets_stride_b,
                                            num_chunks, B, Hkv, N_max, d, tau_lo, Kc, Vc, out_dtype, cap, counts, nullptr,
                                            false, comp_lens, cluster_id, ws, ws_bytes, a);
    if (st != SC_OK) return st;
    const size_t gsc_bytes = align_up(gsc_merge_workspace_bytes(B, Hkv, N_max, d), 256);
    if (ws_bytes < gsc_bytes + gsc_budget_state_bytes()) return SC_ERR_WORKSPACE;
    return runtime_status(launch_gsc_budget(a, (long long)budget_rows, tau_lo, tau_hi, iterations, tau_out,
                                            reinterpret_cast<long long *>(rows_out),
                                            reinterpret_cast<char *>(ws) + gsc_bytes, static_cast<hipStream_t>(stream)));
}

// ------------------------------------------------------------------------------------------------
size_t sc_decode_attn_workspace_bytes(int B, int Hq, int Hkv, int cap, int d) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || cap <= 0 || Hq % Hkv) return 0;
    return decode_workspace_bytes(B, Hq, Hkv, cap, d);
}

sc_status sc_decode_attn_init_workspace(void *ws, size_t ws_bytes, int B, int Hkv, void *stream) {
    if (B <= 0 || Hkv <= 0) return SC_ERR_INVALID_ARG;
    const size_t state = decode_workspace_state_bytes(B, Hkv);
    if (!ws || ws_bytes < state || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SC_ERR_WORKSPACE;
    return runtime_status(launch_decode_init_workspace(ws, state, static_cast<hipStream_t>(stream)));
}

static sc_status decode_common(const void *Q, sc_dtype q_dtype, const void *Kc, const void *Vc, sc_dtype kv_dtype, int cap,
                               const int32_t *counts, const int32_t *comp_lens, const void *Kt, const void *Vt,
                               int tail_cap, const int32_t *tail_lens, bool with_tail, int B, int Hq, int Hkv, int d,
                               float scale, void *O, sc_dtype o_dtype, float *lse, void *ws, size_t ws_bytes,
                               void *stream, size_t state_bytes = 0) {
    if (!Q || !Kc || !Vc || !counts || !comp_lens || !O) return SC_ERR_INVALID_ARG;
    if (with_tail && (!Kt || !Vt || !tail_lens)) return SC_ERR_INVALID_ARG;
    if (B <= 0 || Hq <= 0 || Hkv <= 0) return SC_ERR_INVALID_ARG;
    if (cap <= 0 || (with_tail && tail_cap <= 0)) return SC_ERR_CAPACITY;
    if (with_tail && (int64_t)cap + tail_cap > INT32_MAX) return SC_ERR_CAPACITY;
    if (!dtype_ok(q_dtype) || !dtype_ok(kv_dtype) || !dtype_ok(o_dtype)) return SC_ERR_UNSUPPORTED;
    if (d != 64 && d != 128) return SC_ERR_UNSUPPORTED;
    if (Hq % Hkv) return SC_ERR_UNSUPPORTED;
    if (Hq / Hkv > 8) return SC_ERR_UNSUPPORTED;
    if (Hkv > 65535 || B > 65535) return SC_ERR_UNSUPPORTED;
    if (!aligned16(Q) || !aligned16(Kc) || !aligned16(Vc) || !aligned16(O)) return SC_ERR_INVALID_ARG;
    if (with_tail && (!aligned16(Kt) || !aligned16(Vt) || !aligned4(tail_lens))) return SC_ERR_INVALID_ARG;
    if (!aligned4(counts) || !aligned4(comp_lens) || (lse && !aligned4(lse))) return SC_ERR_INVALID_ARG;
    if (scale != scale) return SC_ERR_INVALID_ARG;
    size_t need = decode_workspace_bytes(B, Hq, Hkv, cap, d);
    if (state_bytes) need = need - decode_workspace_state_bytes(B, Hkv) + state_bytes;
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SC_ERR_WORKSPACE;

    DecodeArgs a;
    a.state_bytes = state_bytes;
    a.Q = Q; a.q_dtype = static_cast<DType>(q_dtype);
    a.Kc = Kc; a.Vc = Vc; a.kv_dtype = static_cast<DType>(kv_dtype); a.cap = cap;
    a.counts = counts; a.comp_lens = comp_lens;
    if (with_tail) { a.Kt = Kt; a.Vt = Vt; a.tail_lens = tail_lens; a.tail_cap = tail_cap; }
    a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.d = d;
    a.scale = (scale == 0.f) ? 1.0f / sqrtf((float)d) : scale;
    a.O = O; a.o_dtype = static_cast<DType>(o_dtype); a.lse = lse; a.ws = ws;
    return runtime_status(launch_decode(a, static_cast<hipStream_t>(stream)));
}

sc_status sc_decode_attn(const void *Q, sc_dtype q_dtype, const void *Kc, const void *Vc, sc_dtype kv_dtype, int cap,
                         const int32_t *counts, const int32_t *comp_lens, int B, int Hq, int Hkv, int d, float scale,
                         void *O, sc_dtype o_dtype, float *lse, void *ws, size_t ws_bytes, void *stream) {
    return decode_common(Q, q_dtype, Kc, Vc, kv_dtype, cap, counts, comp_lens, nullptr, nullptr, 0, nullptr, false, B, Hq,
                         Hkv, d, scale, O, o_dtype, lse, ws, ws_bytes, stream);
}

sc_status sc_decode_attn_static(const void *Q, sc_dtype q_dtype, const void *Kc, const void *Vc, sc_dtype kv_dtype,
                                int cap, const int32_t *counts, const int32_t *comp_lens, int B, int Hq, int Hkv, int d,
                                float scale, void *O, sc_dtype o_dtype, float *lse, void *stream) {
    // the size check comes first: nothing below may depend on a scratch that is too small
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv) return SC_ERR_INVALID_ARG;
    if (cap <= 0) return SC_ERR_CAPACITY;
    if (d != 64 && d != 128) return SC_ERR_UNSUPPORTED;
    if (decode_workspace_bytes(B, Hq, Hkv, cap, d) > kDecodeStaticScratchBytes) return SC_ERR_WORKSPACE;
    if ((long long)B * Hkv > kDecodeStaticMaxHeads) return SC_ERR_WORKSPACE;
    if (!Q || !Kc || !Vc || !counts || !comp_lens || !O) return SC_ERR_INVALID_ARG;
    void *ws = nullptr;
    const hipError_t e = decode_static_scratch(&ws);
    if (e != hipSuccess) return runtime_status(e);
    // The array is shared by calls of every shape, so its state region (epochs and flags of the split
    // hand-over) has ONE layout, for kDecodeStaticMaxHeads heads: a call of one shape never writes partials
    // over the state a call of another shape relies on.  The partials follow behind it.
    return decode_common(Q, q_dtype, Kc, Vc, kv_dtype, cap, counts, comp_lens, nullptr, nullptr, 0, nullptr, false, B, Hq,
                         Hkv, d, scale, O, o_dtype, lse, ws, kDecodeStaticArrayBytes, stream, kDecodeStaticStateBytes);
}

sc_status sc_decode_attn_tail(const void *Q, sc_dtype q_dtype, const void *Kc, const void *Vc, sc_dtype kv_dtype, int cap,
                              const int32_t *counts, const int32_t *comp_lens, const void *Kt, const void *Vt,
                              int tail_cap, const int32_t *tail_lens, int B, int Hq, int Hkv, int d, float scale,
                              void *O, sc_dtype o_dtype, float *lse, void *ws, size_t ws_bytes, void *stream) {
    return decode_common(Q, q_dtype, Kc, Vc, kv_dtype, cap, counts, comp_lens, Kt, Vt, tail_cap, tail_lens, true, B, Hq,
                         Hkv, d, scale, O, o_dtype, lse, ws, ws_bytes, stream);
}

size_t sc_multi_attn_workspace_bytes(int B, int Hq, int Hkv, int nq, int cap, int d) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || nq <= 0 || cap <= 0 || Hq % Hkv) return 0;
    return multi_workspace_bytes(B, Hq, Hkv, nq, cap, d);
}

static sc_status multi_common(const void *Q, sc_dtype q_dtype, int nq, const void *Kc, const void *Vc, sc_dtype kv_dtype,
                              int cap, const int32_t *counts, const int32_t *comp_lens, const void *Kt, const void *Vt,
                              int tail_cap, const int32_t *tail_lens, int causal, bool with_tail, int B, int Hq, int Hkv,
                              int d, float scale, void *O, sc_dtype o_dtype, float *lse, void *ws, size_t ws_bytes,
                              void *stream) {
    if (!Q || !Kc || !Vc || !counts || !comp_lens || !O) return SC_ERR_INVALID_ARG;
    if (with_tail && (!Kt || !Vt || !tail_lens || !aligned16(Kt) || !aligned16(Vt) || !aligned4(tail_lens))) return SC_ERR_INVALID_ARG;
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || nq <= 0) return SC_ERR_INVALID_ARG;
    if (cap <= 0 || (with_tail && tail_cap <= 0)) return SC_ERR_CAPACITY;
    if (with_tail && (int64_t)cap + tail_cap > (1 << 30)) return SC_ERR_CAPACITY;
    // the mask between the query rows exists on the matrix-core path only
    if (with_tail && causal && !(d == 128 && q_dtype == SC_BF16 && kv_dtype == SC_BF16)) return SC_ERR_UNSUPPORTED;
    if (!dtype_ok(q_dtype) || !dtype_ok(kv_dtype) || !dtype_ok(o_dtype)) return SC_ERR_UNSUPPORTED;
    if (d != 64 && d != 128) return SC_ERR_UNSUPPORTED;
    if (Hq % Hkv) return SC_ERR_UNSUPPORTED;
    if (Hq / Hkv > 8) return SC_ERR_UNSUPPORTED;
    if (Hkv > 65535 || B > 65535 || nq > 4096) return SC_ERR_UNSUPPORTED;   // grid sizes
    if (!aligned16(Q) || !aligned16(Kc) || !aligned16(Vc) || !aligned4(O)) return SC_ERR_INVALID_ARG;
    if (!aligned4(counts) || !aligned4(comp_lens) || (lse && !aligned4(lse))) return SC_ERR_INVALID_ARG;
    if (scale != scale) return SC_ERR_INVALID_ARG;
    const size_t need = multi_workspace_bytes(B, Hq, Hkv, nq, cap + (with_tail ? tail_cap : 0), d);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SC_ERR_WORKSPACE;

    MultiArgs a;
    a.Q = Q; a.q_dtype = static_cast<DType>(q_dtype); a.nq = nq;
    a.Kc = Kc; a.Vc = Vc; a.kv_dtype = static_cast<DType>(kv_dtype); a.cap = cap;
    a.counts = counts; a.comp_lens = comp_lens;
    if (with_tail) { a.Kt = Kt; a.Vt = Vt; a.tail_lens = tail_lens; a.tail_cap = tail_cap; a.causal = causal ? 1 : 0; }
    a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.d = d;
    a.scale = (scale == 0.f) ? 1.0f / sqrtf((float)d) : scale;
    a.O = O; a.o_dtype = static_cast<DType>(o_dtype); a.lse = lse; a.ws = ws;
    return runtime_status(launch_multi(a, static_cast<hipStream_t>(stream)));
}

sc_status sc_multi_attn(const void *Q, sc_dtype q_dtype, int nq, const void *Kc, const void *Vc, sc_dtype kv_dtype,
                        int cap, const int32_t *counts, const int32_t *comp_lens, int B, int Hq, int Hkv, int d,
                        float scale, void *O, sc_dtype o_dtype, float *lse, void *ws, size_t ws_bytes, void *stream) {
    return multi_common(Q, q_dtype, nq, Kc, Vc, kv_dtype, cap, counts, comp_lens, nullptr, nullptr, 0, nullptr, 0, false, B,
                        Hq, Hkv, d, scale, O, o_dtype, lse, ws, ws_bytes, stream);
}

sc_status sc_multi_attn_tail(const void *Q, sc_dtype q_dtype, int nq, const void *Kc, const void *Vc, sc_dtype kv_dtype,
                             int cap, const int32_t *counts, const int32_t *comp_lens, const void *Kt, const void *Vt,
                             int tail_cap, const int32_t *tail_lens, int causal, int B, int Hq, int Hkv, int d,
                             float scale, void *O, sc_dtype o_dtype, float *lse, void *ws, size_t ws_bytes, void *stream) {
    return multi_common(Q, q_dtype, nq, Kc, Vc, kv_dtype, cap, counts, comp_lens, Kt, Vt, tail_cap, tail_lens, causal, true,
                        B, Hq, Hkv, d, scale, O, o_dtype, lse, ws, ws_bytes, stream);
}


// ------------------------------------------------------------------------------------------------
// Whether the rows of d elements of a three-dimensional array have no element in common: from the smallest stride on, each has to reach beyond what lies within it.
// (The stride of a dimension of one means nothing.)
static bool rows_apart(const int64_t (&size)[3], const int64_t (&stride)[3], int64_t d) {
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
    int64_t span = d;
    for (int i : order) {
        if (size[i] <= 1) continue;
        if (stride[i] < span || stride[i] > INT64_MAX / 4 / size[i]) return false;
        span += (size[i] - 1) * stride[i];
    }
    return true;
}

// the cache of the sc_paged_* calls: everything about it that the host can see
static sc_status paged_check(const sc_paged_cache *c, PagedView &v, int64_t code_bytes = 0) {
    if (!c || !c->K || !c->V || !c->table) return SC_ERR_INVALID_ARG;
    if (c->B <= 0 || c->Hkv <= 0 || c->num_pages <= 0 || c->table_len <= 0) return SC_ERR_INVALID_ARG;
    if (!code_bytes && !dtype_ok(c->dtype)) return SC_ERR_UNSUPPORTED;
    if (c->d != 64 && c->d != 128) return SC_ERR_UNSUPPORTED;
    if (c->B > 65535 || c->Hkv > 65535 || (int64_t)c->B * c->Hkv > (1 << 20)) return SC_ERR_UNSUPPORTED;
    const int R = c->page_rows;
    if (R < 16 || R > 1024 || (R & (R - 1))) return SC_ERR_INVALID_ARG;
    if (c->page_heads != (c->table_per_head ? 1 : c->Hkv)) return SC_ERR_INVALID_ARG;
    if ((int64_t)c->table_len * R > INT32_MAX) return SC_ERR_UNSUPPORTED;
    const int64_t es = code_bytes ? code_bytes : (int64_t)elem_size(c->dtype);
    // in any order of pages, heads and rows
    const int64_t size[3] = {c->num_pages, c->page_heads, R}, stride[3] = {c->stride_page, c->stride_head, c->stride_row};
    for (int i = 0; i < 3; ++i)
        if (size[i] > 1 && (stride[i] < 0 || (stride[i] * es) % 16)) return SC_ERR_INVALID_ARG;
    if (c->stride_row < c->d || c->stride_row > INT32_MAX / (R * es)) return SC_ERR_INVALID_ARG;      // offsets inside the rows of a head are 32-bit
    if (!rows_apart(size, stride, c->d)) return SC_ERR_INVALID_ARG;
    if (!aligned16(c->K) || !aligned16(c->V) || !aligned4(c->table)) return SC_ERR_INVALID_ARG;
    if (c->counts && !aligned16(c->counts)) return SC_ERR_INVALID_ARG;      // read four at a time
    if (!c->k_min != !c->k_max) return SC_ERR_INVALID_ARG;
    if (!aligned16(c->k_min) || !aligned16(c->k_max)) return SC_ERR_INVALID_ARG;
    v.K = static_cast<char *>(c->K); v.V = static_cast<char *>(c->V);
    v.counts = c->counts;
    v.k_min = static_cast<char *>(c->k_min); v.k_max = static_cast<char *>(c->k_max);
    v.table = c->table;
    v.page_bytes = c->stride_page * es; v.head_bytes = c->stride_head * es; v.row_bytes = (int)(c->stride_row * es);
    v.num_pages = c->num_pages; v.page_heads = c->page_heads;
    v.R = R; v.log2_R = __builtin_ctz((unsigned)R);
    v.P = c->table_len; v.table_per_head = c->table_per_head != 0;
    v.B = c->B; v.H = c->Hkv; v.d = c->d; v.dtype = static_cast<DType>(c->dtype);
    return SC_OK;
}

// whether two arrays have no element in common (b may be NULL)
static bool apart(const int32_t *a, int64_t na, const int32_t *b, int64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return !b || x + na * sizeof(int32_t) <= y || y + nb * sizeof(int32_t) <= x;
}

// the same for the cache of the sc_paged8_* calls
static sc_status paged8_check(const sc_paged8_cache *c, PagedView &v, Paged8View &w) {
    if (!c) return SC_ERR_INVALID_ARG;
    const sc_paged_cache plain = {c->K, c->V, c->counts, nullptr, nullptr, c->table, c->stride_page, c->stride_head, c->stride_row, SC_F32,
                                  c->num_pages, c->page_heads, c->page_rows, c->table_len, c->table_per_head, c->B, c->Hkv, c->d};
    const sc_status st = paged_check(&plain, v, 1);
    if (st != SC_OK) return st;
    if (c->code != SC_E4M3 && c->code != SC_I8) return SC_ERR_UNSUPPORTED;
    const int E = c->block_rows;
    if (E < 16 || E > 128 || (E & (E - 1)) || E > c->page_rows) return SC_ERR_INVALID_ARG;
    if (!c->k_scale || !c->v_scale || !aligned4(c->k_scale) || !aligned4(c->v_scale)) return SC_ERR_INVALID_ARG;
    const int64_t scales = (int64_t)c->num_pages * c->page_heads * (c->page_rows / E);
    if (!apart(reinterpret_cast<const int32_t *>(c->k_scale), scales, reinterpret_cast<const int32_t *>(c->v_scale), scales)) return SC_ERR_INVALID_ARG;
    w.k_scale = c->k_scale; w.v_scale = c->v_scale;
    w.log2_block = __builtin_ctz((unsigned)E);
    w.code = c->code == SC_E4M3 ? 1 : 2;
    return SC_OK;
}

// Rows [B, heads, N, d]: aligned, and, where the call writes them, none with a stride of less than a row.
static bool rows_ok(const void *p, int64_t B, int64_t H, int64_t N, int64_t sb, int64_t sh, int64_t sn, int64_t d, int64_t es, bool written) {
    const int64_t size[3] = {B, H, N}, stride[3] = {sb, sh, sn};
    for (int i = 0; i < 3; ++i)
        if (size[i] > 1 && (stride[i] < 0 || (stride[i] * es) % 16 || (written && stride[i] < d))) return false;
    return aligned16(p);
}

// the rows of sc_paged_append and sc_paged8_append (a.c is there already): K and V of elements of `es` bytes; a page, or a block, of `rows` rows is one workgroup's at most
static sc_status append_check(const sc_paged_rows *r, int64_t es, int rows, PagedAppendArgs &a) {
    const PagedView &c = a.c;
    if (!r || !r->K || !r->V || !r->base_lens || !r->lens || r->N <= 0) return SC_ERR_INVALID_ARG;
    if (!aligned4(r->base_lens) || !aligned4(r->lens) || !aligned4(r->new_lens) || !aligned4(r->positions) || !aligned4(r->counts)) return SC_ERR_INVALID_ARG;
    if (!r->counts != !c.counts) return SC_ERR_INVALID_ARG;
    if (!rows_ok(r->K, c.B, c.H, r->N, r->k_stride_b, r->k_stride_h, r->k_stride_n, c.d, es, false)) return SC_ERR_INVALID_ARG;
    if (!rows_ok(r->V, c.B, c.H, r->N, r->v_stride_b, r->v_stride_h, r->v_stride_n, c.d, es, false)) return SC_ERR_INVALID_ARG;
    if (r->cos_sin) {
        if (r->rot <= 0 || r->rot > c.d || r->rot % 16 || r->max_position <= 0 || !aligned16(r->cos_sin)) return SC_ERR_INVALID_ARG;
        if (!r->positions && r->per_head) return SC_ERR_INVALID_ARG;      // a token has one position
    } else if (r->rot != 0 || r->Q) {
        return SC_ERR_INVALID_ARG;
    }
    if (!r->Q != !r->Q_out) return SC_ERR_INVALID_ARG;
    int64_t qs = 2;
    if (r->Q) {
        if (!dtype_ok(r->q_dtype)) return SC_ERR_UNSUPPORTED;
        if (r->Hq <= 0) return SC_ERR_INVALID_ARG;
        qs = (int64_t)elem_size(r->q_dtype);
        if (!rows_ok(r->Q, c.B, r->Hq, r->N, r->q_stride_b, r->q_stride_h, r->q_stride_n, c.d, qs, false)) return SC_ERR_INVALID_ARG;
        if (!rows_ok(r->Q_out, c.B, r->Hq, r->N, r->o_stride_b, r->o_stride_h, r->o_stride_n, c.d, qs, true)) return SC_ERR_INVALID_ARG;
        if (r->Hq > 65535) return SC_ERR_UNSUPPORTED;
    }
    if (!paged_append_fits(c.B, c.H, rows, r->N, r->Q ? r->Hq : 0)) return SC_ERR_UNSUPPORTED;      // grid size
    const int64_t q_size[3] = {c.B, r->Hq, r->N}, o_stride[3] = {r->o_stride_b, r->o_stride_h, r->o_stride_n};
    if (r->Q && !rows_apart(q_size, o_stride, c.d)) return SC_ERR_INVALID_ARG;
    // every workgroup reads the old lengths and the positions while one of them files the new lengths
    const int64_t n = (int64_t)c.B * (r->per_head ? c.H : 1);
    if (!apart(r->lens, n, r->base_lens, n) || !apart(r->lens, n, r->new_lens, n) || !apart(r->lens, n, r->positions, c.B)) return SC_ERR_INVALID_ARG;
    a.K = static_cast<const char *>(r->K); a.V = static_cast<const char *>(r->V);
    a.k_b = r->k_stride_b * es; a.k_h = r->k_stride_h * es; a.k_n = r->k_stride_n * es;
    a.v_b = r->v_stride_b * es; a.v_h = r->v_stride_h * es; a.v_n = r->v_stride_n * es;
    a.counts = r->counts;
    a.N = r->N; a.per_head = r->per_head != 0;
    a.base_lens = r->base_lens; a.new_lens = r->new_lens; a.lens = r->lens;
    a.cos_sin = r->cos_sin; a.max_position = r->max_position; a.rot = r->cos_sin ? r->rot : 0; a.interleaved = r->interleaved != 0;
    a.Hq = r->Hq; a.positions = r->positions;
    a.Q = static_cast<const char *>(r->Q); a.Q_out = static_cast<char *>(r->Q_out);
    a.q_b = r->q_stride_b * qs; a.q_h = r->q_stride_h * qs; a.q_n = r->q_stride_n * qs;
    a.o_b = r->o_stride_b * qs; a.o_h = r->o_stride_h * qs; a.o_n = r->o_stride_n * qs;
    a.q_dtype = r->Q ? static_cast<DType>(r->q_dtype) : a.c.dtype;
    return SC_OK;
}

sc_status sc_paged_append(const sc_paged_cache *cache, const sc_paged_rows *r, void *stream) {
    PagedAppendArgs a;
    sc_status st = paged_check(cache, a.c);
    if (st == SC_OK) st = append_check(r, (int64_t)elem_size(cache->dtype), cache->page_rows, a);
    if (st != SC_OK) return st;
    return runtime_status(launch_paged_append(a, static_cast<hipStream_t>(stream)));
}

sc_status sc_paged8_append(const sc_paged8_cache *cache, const sc_paged_rows *r, sc_dtype kv_dtype, void *stream) {
    PagedAppendArgs a;
    Paged8View w;
    sc_status st = paged8_check(cache, a.c, w);
    if (st == SC_OK && !dtype_ok(kv_dtype)) st = SC_ERR_UNSUPPORTED;
    if (st != SC_OK) return st;
    a.c.dtype = static_cast<DType>(kv_dtype);
    st = append_check(r, (int64_t)elem_size(kv_dtype), cache->block_rows, a);
    if (st != SC_OK) return st;
    return runtime_status(launch_paged8_append(a, w, static_cast<hipStream_t>(stream)));
}

size_t sc_paged_workspace_bytes(int B, int Hq, int Hkv, int d, int table_len) {
    if (B <= 0 || Hkv <= 0 || Hq <= 0 || table_len <= 0 || Hq % Hkv || (d != 64 && d != 128)) return 0;
    const size_t attend = paged_decode_bytes(Hq / Hkv, d), select = paged_select_bytes(B, Hkv, table_len);
    return paged_state_bytes() + (attend > select ? attend : select);
}

sc_status sc_paged_init_workspace(void *ws, size_t ws_bytes, void *stream) {
    const size_t state = paged_state_bytes();
    if (!ws || ws_bytes < state || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SC_ERR_WORKSPACE;
    return runtime_status(launch_decode_init_workspace(ws, state, static_cast<hipStream_t>(stream)));
}

// what the calls with a query have in common
static sc_status paged_query_check(sc_status st, const PagedView &v, const void *Q, sc_dtype q_dtype, int Hq, const int32_t *lens, const void *ws) {
    if (st != SC_OK) return st;
    if (!Q || !lens || Hq <= 0 || !aligned16(Q) || !aligned4(lens)) return SC_ERR_INVALID_ARG;
    if (!dtype_ok(q_dtype) || Hq % v.H || Hq / v.H > 16) return SC_ERR_UNSUPPORTED;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SC_ERR_WORKSPACE;
    return SC_OK;
}
// ... and those that attend (a.c, a.sel, a.sel_lens, a.keep, a.window and a.sinks are there already)
static sc_status paged_attend(sc_status st, PagedDecodeArgs &a, const void *Q, sc_dtype q_dtype, int Hq, const int32_t *lens, int lens_per_head, float scale,
                              void *O, sc_dtype o_dtype, float *lse, void *ws, size_t ws_bytes, void *stream) {
    st = paged_query_check(st, a.c, Q, q_dtype, Hq, lens, ws);
    if (st != SC_OK) return st;
    if (!O || !aligned16(O) || !aligned4(lse) || !a.sel != !a.sel_lens || !aligned4(a.sel) || !aligned4(a.sel_lens)) return SC_ERR_INVALID_ARG;
    if (!dtype_ok(o_dtype)) return SC_ERR_UNSUPPORTED;
    if (scale != scale) return SC_ERR_INVALID_ARG;
    if (a.sel && a.keep <= 0) return SC_ERR_CAPACITY;
    if (a.sel && a.keep > (1 << 20)) return SC_ERR_UNSUPPORTED;
    if (a.window < 0 || a.sinks < 0) return SC_ERR_INVALID_ARG;
    const int64_t most = (int64_t)(a.sel ? a.keep : a.c.P) * a.c.R;
    if ((most / 64 + 1) * a.c.B * a.c.H > (1 << 30)) return SC_ERR_UNSUPPORTED;      // the kernel counts stretches of 64 rows and more in 32 bits
    if (ws_bytes < paged_state_bytes() + paged_decode_bytes(Hq / a.c.H, a.c.d)) return SC_ERR_WORKSPACE;
    a.Q = Q; a.q_dtype = static_cast<DType>(q_dtype); a.Hq = Hq;
    a.lens = lens; a.lens_per_head = lens_per_head != 0;
    a.scale = (scale == 0.f) ? 1.0f / sqrtf((float)a.c.d) : scale;
    a.O = O; a.o_dtype = static_cast<DType>(o_dtype); a.lse = lse; a.ws = ws;
    return runtime_status(launch_paged_decode(a, static_cast<hipStream_t>(stream)));
}

sc_status sc_paged_decode_attn(const sc_paged_cache *cache, const void *Q, sc_dtype q_dtype, int Hq, const int32_t *lens,
                               int lens_per_head, const int32_t *sel, const int32_t *sel_lens, int keep, float scale, void *O,
                               sc_dtype o_dtype, float *lse, void *ws, size_t ws_bytes, void *stream) {
    PagedDecodeArgs a;
    const sc_status st = paged_check(cache, a.c);
    a.sel = sel; a.sel_lens = sel_lens; a.keep = sel ? keep : 0;
    return paged_attend(st, a, Q, q_dtype, Hq, lens, lens_per_head, scale, O, o_dtype, lse, ws, ws_bytes, stream);
}

sc_status sc_paged_window_attn(const sc_paged_cache *cache, const void *Q, sc_dtype q_dtype, int Hq, const int32_t *lens,
                               int lens_per_head, int window, int sinks, float scale, void *O, sc_dtype o_dtype, float *lse,
                               void *ws, size_t ws_bytes, void *stream) {
    PagedDecodeArgs a;
    const sc_status st = paged_check(cache, a.c);
    a.sel = a.sel_lens = nullptr; a.keep = 0;
    a.window = window; a.sinks = sinks;
    return paged_attend(st, a, Q, q_dtype, Hq, lens, lens_per_head, scale, O, o_dtype, lse, ws, ws_bytes, stream);
}

sc_status sc_paged8_decode_attn(const sc_paged8_cache *cache, const void *Q, sc_dtype q_dtype, int Hq, const int32_t *lens,
                                int lens_per_head, int window, int sinks, float scale, void *O, sc_dtype o_dtype, float *lse,
                                void *ws, size_t ws_bytes, void *stream) {
    PagedDecodeArgs a;
    Paged8View w;
    const sc_status st = paged8_check(cache, a.c, w);
    a.sel = a.sel_lens = nullptr; a.keep = 0;
    a.window = window; a.sinks = sinks;
    if (st == SC_OK) {
        a.code = w.code; a.log2_block = w.log2_block;
        a.k_scale = w.k_scale; a.v_scale = w.v_scale;
    }
    return paged_attend(st, a, Q, q_dtype, Hq, lens, lens_per_head, scale, O, o_dtype, lse, ws, ws_bytes, stream);
}

sc_status sc_paged_select(const sc_paged_cache *cache, const void *Q, sc_dtype q_dtype, int Hq, const int32_t *lens, int lens_per_head,
                          int keep, int first, int recent, int32_t *sel, int32_t *sel_lens, void *ws, size_t ws_bytes, void *stream) {
    PagedSelectArgs a;
    const sc_status st = paged_query_check(paged_check(cache, a.c), a.c, Q, q_dtype, Hq, lens, ws);
    if (st != SC_OK) return st;
    if (!cache->k_min || !sel || !sel_lens || !aligned4(sel) || !aligned4(sel_lens) || first < 0 || recent < 0) return SC_ERR_INVALID_ARG;
    if (keep <= 0 || (int64_t)first + recent > keep) return SC_ERR_CAPACITY;
    if (keep > (1 << 20)) return SC_ERR_UNSUPPORTED;
    if ((int64_t)(cache->table_len / 16 + 1) * cache->B * cache->Hkv > INT32_MAX) return SC_ERR_UNSUPPORTED;      // grid size
    if (ws_bytes < paged_state_bytes() + paged_select_bytes(cache->B, cache->Hkv, cache->table_len)) return SC_ERR_WORKSPACE;
    a.Q = Q; a.q_dtype = static_cast<DType>(q_dtype); a.Hq = Hq;
    a.lens = lens; a.lens_per_head = lens_per_head != 0;
    a.keep = keep; a.first = first; a.recent = recent;
    a.sel = sel; a.sel_lens = sel_lens; a.ws = ws;
    return runtime_status(launch_paged_select(a, static_cast<hipStream_t>(stream)));
}

size_t sc_prompt_attn_workspace_bytes(int B, int Hq, int Hkv, int N, int M, int d) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || N <= 0 || M <= 0 || Hq % Hkv || (d != 64 && d != 128)) return 0;
    return prompt_workspace_bytes(B, Hq, Hkv, N, M, d);
}

sc_status sc_prompt_attn(const sc_prompt *x, void *ws, size_t ws_bytes, void *stream) {
    if (!x || !x->Q || !x->K || !x->V || !x->O) return SC_ERR_INVALID_ARG;
    if (x->B <= 0 || x->Hq <= 0 || x->Hkv <= 0 || x->N <= 0 || x->M <= 0 || x->window < 0 || x->sinks < 0 || x->scale != x->scale) return SC_ERR_INVALID_ARG;
    if (!dtype_ok(x->dtype) || (x->d != 64 && x->d != 128) || x->Hq % x->Hkv) return SC_ERR_UNSUPPORTED;
    if (x->B > 65535 || x->Hq > 65535 || (int64_t)x->N * (x->Hq / x->Hkv) > (1 << 30) || x->M > (1 << 30)) return SC_ERR_UNSUPPORTED;      // counted in 32 bits
    if (!aligned4(x->lse) || !aligned4(x->q_lens) || !aligned4(x->kv_lens)) return SC_ERR_INVALID_ARG;
    const int64_t es = (int64_t)elem_size(x->dtype);
    if (!rows_ok(x->Q, x->B, x->Hq, x->N, x->q_stride_b, x->q_stride_h, x->q_stride_n, x->d, es, false)) return SC_ERR_INVALID_ARG;
    if (!rows_ok(x->K, x->B, x->Hkv, x->M, x->k_stride_b, x->k_stride_h, x->k_stride_n, x->d, es, false)) return SC_ERR_INVALID_ARG;
    if (!rows_ok(x->V, x->B, x->Hkv, x->M, x->v_stride_b, x->v_stride_h, x->v_stride_n, x->d, es, false)) return SC_ERR_INVALID_ARG;
    if (!rows_ok(x->O, x->B, x->Hq, x->N, x->o_stride_b, x->o_stride_h, x->o_stride_n, x->d, es, true)) return SC_ERR_INVALID_ARG;
    const int64_t size[3] = {x->B, x->Hq, x->N}, stride[3] = {x->o_stride_b, x->o_stride_h, x->o_stride_n};
    if (!rows_apart(size, stride, x->d)) return SC_ERR_INVALID_ARG;
    if (x->M > 1 && (x->k_stride_n * es > INT32_MAX / 64 || x->v_stride_n * es > INT32_MAX / 64)) return SC_ERR_UNSUPPORTED;      // offsets inside a tile of keys are 32-bit
    if (!prompt_fits(x->B, x->Hq, x->Hkv, x->N, x->M, x->d, x->dtype == SC_BF16)) return SC_ERR_UNSUPPORTED;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < prompt_workspace_bytes(x->B, x->Hq, x->Hkv, x->N, x->M, x->d)) return SC_ERR_WORKSPACE;
    // O and lse are nothing else (a workgroup reads queries, keys and values while others write)
    auto rows = [&](const void *p, int heads, int n, int64_t sb, int64_t sh, int64_t sn) { return RowsAt{(uint64_t)(uintptr_t)p, {x->B, heads, n}, {sb * es, sh * es, sn * es}, x->d * es}; };
    auto array = [](const void *p, int64_t bytes) { return RowsAt{(uint64_t)(uintptr_t)p, {1, 1, 1}, {0, 0, 0}, bytes}; };
    const RowsAt O = rows(x->O, x->Hq, x->N, x->o_stride_b, x->o_stride_h, x->o_stride_n), lse = array(x->lse, (int64_t)x->B * x->Hq * x->N * 4);
    const RowsAt inputs[5] = {rows(x->Q, x->Hq, x->N, x->q_stride_b, x->q_stride_h, x->q_stride_n), rows(x->K, x->Hkv, x->M, x->k_stride_b, x->k_stride_h, x->k_stride_n),
                              rows(x->V, x->Hkv, x->M, x->v_stride_b, x->v_stride_h, x->v_stride_n), array(x->q_lens, (int64_t)x->B * 4), array(x->kv_lens, (int64_t)x->B * 4)};
    if (x->lse && rows_meet(O, lse)) return SC_ERR_INVALID_ARG;
    for (const RowsAt &i : inputs)
        if (i.at && (rows_meet(O, i) || (x->lse && rows_meet(lse, i)))) return SC_ERR_INVALID_ARG;
    PromptArgs a;
    a.Q = static_cast<const char *>(x->Q); a.K = static_cast<const char *>(x->K); a.V = static_cast<const char *>(x->V);
    a.O = static_cast<char *>(x->O); a.lse = x->lse;
    a.q_b = x->q_stride_b * es; a.q_h = x->q_stride_h * es; a.q_n = x->q_stride_n * es;
    a.k_b = x->k_stride_b * es; a.k_h = x->k_stride_h * es; a.k_n = x->M > 1 ? x->k_stride_n * es : 0;
    a.v_b = x->v_stride_b * es; a.v_h = x->v_stride_h * es; a.v_n = x->M > 1 ? x->v_stride_n * es : 0;
    a.o_b = x->o_stride_b * es; a.o_h = x->o_stride_h * es; a.o_n = x->o_stride_n * es;
    a.q_lens = x->q_lens; a.kv_lens = x->kv_lens;
    a.dtype = static_cast<DType>(x->dtype);
    a.B = x->B; a.Hq = x->Hq; a.Hkv = x->Hkv; a.N = x->N; a.M = x->M; a.d = x->d; a.window = x->window; a.sinks = x->sinks;
    a.scale = (x->scale == 0.f) ? 1.0f / sqrtf((float)x->d) : x->scale;
    a.ws = ws;
    return runtime_status(launch_prompt(a, static_cast<hipStream_t>(stream)));
}

size_t sc_paged_reserve_workspace_bytes(int sequences, int table_len) {
    if (sequences <= 0 || table_len <= 0 || sequences > (1 << 20) || (int64_t)sequences * table_len > (1 << 28)) return 0;
    return paged_reserve_bytes(sequences, table_len);
}

sc_status sc_paged_reserve(int32_t *table, int sequences, int table_len, int num_pages, int page_rows, const int32_t *base_lens, const int32_t *new_lens, int N,
                           int window, int sinks, int32_t *free_pages, int32_t *num_free, int32_t *lens, int32_t *slots, void *ws, size_t ws_bytes, void *stream) {
    if (!table || !base_lens || !free_pages || !num_free || !lens) return SC_ERR_INVALID_ARG;
    if (sequences <= 0 || table_len <= 0 || num_pages <= 0 || N < 0 || window < 0 || sinks < 0) return SC_ERR_INVALID_ARG;
    if (!aligned4(table) || !aligned4(base_lens) || !aligned4(new_lens) || !aligned4(free_pages) || !aligned4(num_free) || !aligned4(lens) || !aligned4(slots)) return SC_ERR_INVALID_ARG;
    if (page_rows < 16 || page_rows > 1024 || (page_rows & (page_rows - 1))) return SC_ERR_INVALID_ARG;
    if (sequences > (1 << 20) || (int64_t)sequences * table_len > (1 << 28)) return SC_ERR_UNSUPPORTED;      // counted in 32 bits
    if ((int64_t)table_len * page_rows > INT32_MAX || (int64_t)num_pages * page_rows > INT32_MAX) return SC_ERR_UNSUPPORTED;      // rows and slots are 32-bit
    // what is written is nothing else (the second of two launches reads the lengths again)
    const int64_t S = sequences;
    const int32_t *array[7] = {table, lens, free_pages, num_free, N > 0 ? slots : nullptr, base_lens, new_lens};
    const int64_t size[7] = {S * table_len, S, num_pages, 1, S * N, S, S};
    for (int i = 0; i < 5; ++i)
        for (int k = i + 1; k < 7; ++k)
            if (array[i] && !apart(array[i], size[i], array[k], size[k])) return SC_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < paged_reserve_bytes(sequences, table_len)) return SC_ERR_WORKSPACE;
    const PagedReserveArgs a = {table, sequences, table_len, num_pages, page_rows, base_lens, new_lens, N, window, sinks, free_pages, num_free, lens, N > 0 ? slots : nullptr};
    return runtime_status(launch_paged_reserve(a, ws, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
