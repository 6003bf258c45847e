// C ABI of the library: argument checks, launch geometry, error reporting.
#include <cfloat>
#include <vector>

#include "common.cuh"

namespace moesched {

static thread_local int g_last_cuda_error = 0;
int& last_cuda_error_slot() { return g_last_cuda_error; }

Geometry plan_geometry(int N) {
  Geometry ge;
  // Every number of words has kernels of its own: the work of a step grows with it (squared in a search level), and rounded
  // up to 1, 2, 4 or 8 (60 to 100 matrices, Birkhoff / greedy) N = 72 took 3.3 / 43 us a matching in place of 2.7 / 37, N = 160
  // 10.7 / 230 in place of 6.7 / 144, N = 224 11.7 / 382 in place of 10.3 / 327.
  ge.cpl = (N + 31) / 32;
  ge.S = N;
  ge.cluster = false;
  ge.wpb = 1;
  ge.smem = 0;
  return ge;
}

int sm_count() {
  static int cached[64] = {0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if (cached[dev] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
    cached[dev] = n;
  }
  return cached[dev];
}

static int fail_cuda(cudaError_t e) {
  g_last_cuda_error = (int)e;
  return MOESCHED_ECUDA;
}

bool model_in_range(const moesched_model_t& m) {
  const int64_t lim20 = 1LL << 20, lim30 = 1LL << 30, lim40 = 1LL << 40;
  return m.bytes_per_token >= 1 && m.bytes_per_token <= lim20 && m.link_gbps >= 1 && m.link_gbps <= lim20 &&
         m.reconfig_ns >= 0 && m.reconfig_ns <= lim40 && m.expert_fixed_ns >= 0 && m.expert_fixed_ns <= lim40 &&
         m.expert_ps_per_token >= 0 && m.expert_ps_per_token <= lim30 && m.expert_knee_tokens >= 0 &&
         m.expert_knee_tokens <= 2147483647LL;
}

#ifdef MOESCHED_CHECKED
static std::vector<FaultReader>& fault_readers() {
  static std::vector<FaultReader> readers;   // built on first use: the files register during static initialisation
  return readers;
}
void register_fault_reader(FaultReader reader) { fault_readers().push_back(reader); }
#endif

static bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
static bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0; }

// The argument checks of the entry points that moesched_path_run is made of.
static bool size_ok(int B, int N, int k) { return B >= 0 && N >= 1 && N <= MOESCHED_MAX_N && k >= 1; }
static bool mw_pointers_ok(const void* demand, const void* perm, const void* dur, const void* count, const void* residual,
                           const void* status, const void* work) {
  return demand && perm && dur && count && status && aligned4(demand) && aligned4(dur) && aligned4(count) &&
         aligned4(status) && aligned4(residual) && aligned8(work);
}
static bool bvn_pointers_ok(const void* demand, const void* perm, const void* coef, const void* count, const void* aug,
                            const void* scratch, const void* status, const void* work) {
  return demand && perm && coef && count && status && aligned4(demand) && aligned4(coef) && aligned4(count) &&
         aligned4(status) && aligned4(aug) && aligned8(work) && (reinterpret_cast<uintptr_t>(scratch) & 31) == 0;
}
static bool eval_pointers_ok(const void* demand, const void* perm, const void* dur, const void* count, const void* status) {
  return demand && perm && dur && count && status && aligned4(demand) && aligned4(dur) && aligned4(count) && aligned4(status);
}

static bool expert_sizes_ok(int R, int E, int groups, int dtype, int act) {
  return R >= 0 && R <= MOESCHED_MAX_ROWS && E >= 1 && E <= MOESCHED_MAX_EXPERTS && groups >= E && groups % E == 0 && groups <= MOESCHED_MAX_GROUPS &&
         (dtype == MOESCHED_BF16 || dtype == MOESCHED_FP16) && (act == MOESCHED_ACT_SILU || act == MOESCHED_ACT_GELU);
}
static bool ffn_width_ok(int v) { return v >= 8 && v <= 65536 && v % 8 == 0; }

static bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
static bool token_type_ok(int dtype) { return dtype == MOESCHED_BF16 || dtype == MOESCHED_FP16 || dtype == MOESCHED_FP32; }
static bool token_sizes_ok(int rows, int D, int dtype) {
  return rows >= 0 && rows <= MOESCHED_MAX_ROWS && ffn_width_ok(D) && token_type_ok(dtype);
}
static bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
static bool choose_sizes_ok(int rows, int E, int k, int dtype, int score, float factor) {
  return rows >= 0 && rows <= MOESCHED_MAX_ROWS && E >= 1 && E <= MOESCHED_MAX_EXPERTS && k >= 1 && k <= E && k <= MOESCHED_MAX_TOP_K &&
         token_type_ok(dtype) && (score == MOESCHED_SCORE_SOFTMAX || score == MOESCHED_SCORE_SIGMOID) && factor >= -FLT_MAX && factor <= FLT_MAX;
}
static bool rows_sizes_ok(int G, int T, int k) {
  return G >= 0 && T >= 0 && (int64_t)G * T <= MOESCHED_MAX_ROWS && k >= 1 && k <= MOESCHED_MAX_TOP_K && (int64_t)T * k <= 0x7fffffff;
}

}  // namespace moesched

using namespace moesched;

extern "C" {

int moesched_mw_decompose(int B, int N, const int32_t* d_demand, int k_max, uint8_t* d_perm, int32_t* d_dur,
                          int32_t* d_count, int32_t* d_residual, int32_t* d_status, int64_t* d_work,
                          void* stream) {
  if (!size_ok(B, N, k_max)) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!mw_pointers_ok(d_demand, d_perm, d_dur, d_count, d_residual, d_status, d_work)) return MOESCHED_EINVAL;
  cudaError_t e = run_mw(B, N, d_demand, k_max, d_perm, d_dur, d_count, d_residual, d_status,
                         reinterpret_cast<long long*>(d_work), static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

size_t moesched_bvn_scratch_bytes(int B, int N) {
  if (B < 0 || N < 1 || N > MOESCHED_MAX_N) return 0;
  return (size_t)B * N * bvn_scratch_stride(N) * sizeof(int32_t);
}

size_t moesched_workspace_bytes(int B, int N, int k_max) {
  if (k_max < 1) return 0;
  return moesched_bvn_scratch_bytes(B, N);
}

int moesched_bvn_decompose(int B, int N, const int32_t* d_demand, int k_max, uint8_t* d_perm, int32_t* d_coef,
                           int32_t* d_count, int32_t* d_aug, int32_t* d_scratch, int32_t* d_status,
                           int64_t* d_work, void* stream) {
  if (!size_ok(B, N, k_max)) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!bvn_pointers_ok(d_demand, d_perm, d_coef, d_count, d_aug, d_scratch, d_status, d_work)) return MOESCHED_EINVAL;
  cudaError_t e = run_bvn(B, N, d_demand, k_max, d_perm, d_coef, d_count, d_aug, d_scratch, d_status,
                          reinterpret_cast<long long*>(d_work), static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

static int schedule_eval_impl(int B, int N, const int32_t* d_demand, int k_stride, const uint8_t* d_perm,
                              const int32_t* d_dur, const int32_t* d_count, const moesched_model_t* h_model,
                              int64_t* d_makespan_overlap_ns, int64_t* d_makespan_serial_ns,
                              int64_t* d_compute_idle_ns, int64_t* d_link_idle_tokens, int64_t* d_unserved_tokens,
                              int32_t* d_status, int64_t* d_prefix_overlap_ns, int64_t* d_prefix_unserved_tokens,
                              void* stream) {
  if (!size_ok(B, N, k_stride)) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!eval_pointers_ok(d_demand, d_perm, d_dur, d_count, d_status) || !h_model || !d_makespan_overlap_ns ||
      !d_makespan_serial_ns || !d_compute_idle_ns || !d_link_idle_tokens || !d_unserved_tokens)
    return MOESCHED_EINVAL;
  if (!aligned8(d_makespan_overlap_ns) || !aligned8(d_makespan_serial_ns) || !aligned8(d_compute_idle_ns) ||
      !aligned8(d_link_idle_tokens) || !aligned8(d_unserved_tokens) || !aligned8(d_prefix_overlap_ns) ||
      !aligned8(d_prefix_unserved_tokens))
    return MOESCHED_EINVAL;
  const moesched_model_t m = *h_model;
  if (!model_in_range(m)) return MOESCHED_EINVAL;
  cudaError_t e = run_eval(B, N, d_demand, k_stride, d_perm, d_dur, d_count, m,
                           reinterpret_cast<long long*>(d_makespan_overlap_ns),
                           reinterpret_cast<long long*>(d_makespan_serial_ns),
                           reinterpret_cast<long long*>(d_compute_idle_ns),
                           reinterpret_cast<long long*>(d_link_idle_tokens),
                           reinterpret_cast<long long*>(d_unserved_tokens), d_status,
                           reinterpret_cast<long long*>(d_prefix_overlap_ns),
                           reinterpret_cast<long long*>(d_prefix_unserved_tokens),
                           static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_schedule_eval(int B, int N, const int32_t* d_demand, int k_stride, const uint8_t* d_perm,
                           const int32_t* d_dur, const int32_t* d_count, const moesched_model_t* h_model,
                           int64_t* d_makespan_overlap_ns, int64_t* d_makespan_serial_ns,
                           int64_t* d_compute_idle_ns, int64_t* d_link_idle_tokens, int64_t* d_unserved_tokens,
                           int32_t* d_status, void* stream) {
  return schedule_eval_impl(B, N, d_demand, k_stride, d_perm, d_dur, d_count, h_model, d_makespan_overlap_ns,
                            d_makespan_serial_ns, d_compute_idle_ns, d_link_idle_tokens, d_unserved_tokens,
                            d_status, nullptr, nullptr, stream);
}

int moesched_schedule_prefix_eval(int B, int N, const int32_t* d_demand, int k_stride, const uint8_t* d_perm,
                                  const int32_t* d_dur, const int32_t* d_count, const moesched_model_t* h_model,
                                  int64_t* d_makespan_overlap_ns, int64_t* d_makespan_serial_ns,
                                  int64_t* d_compute_idle_ns, int64_t* d_link_idle_tokens,
                                  int64_t* d_unserved_tokens, int32_t* d_status, int64_t* d_prefix_overlap_ns,
                                  int64_t* d_prefix_unserved_tokens, void* stream) {
  if (B > 0 && (!d_prefix_overlap_ns || !d_prefix_unserved_tokens)) return MOESCHED_EINVAL;
  return schedule_eval_impl(B, N, d_demand, k_stride, d_perm, d_dur, d_count, h_model, d_makespan_overlap_ns,
                            d_makespan_serial_ns, d_compute_idle_ns, d_link_idle_tokens, d_unserved_tokens,
                            d_status, d_prefix_overlap_ns, d_prefix_unserved_tokens, stream);
}

int moesched_path_run(const moesched_path_t* p, int B, int N, const int32_t* d_demand, const moesched_model_t* h_model,
                      int overlap, void* stream) {
  // everything is checked before anything is enqueued
  if (p == nullptr || p->k_mw > 0x7fffffff || p->k_bvn > 0x7fffffff || p->k_mw < 1 || p->k_bvn < 1 || !size_ok(B, N, 1) ||
      p->score_stride < B)
    return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  const bool fork = overlap != 0 && p->side_stream != nullptr;
  if (fork && (!p->fork_event || !p->join_event)) return MOESCHED_EINVAL;
  if (!bvn_pointers_ok(d_demand, p->d_bvn_perm, p->d_bvn_coef, p->d_bvn_count, nullptr, p->d_bvn_scratch, p->d_bvn_status,
                       p->d_bvn_work) ||
      !mw_pointers_ok(d_demand, p->d_mw_perm, p->d_mw_dur, p->d_mw_count, nullptr, p->d_mw_status, p->d_mw_work) ||
      !eval_pointers_ok(d_demand, p->d_bvn_perm, p->d_bvn_coef, p->d_bvn_count, p->d_bvn_eval_status) ||
      !eval_pointers_ok(d_demand, p->d_mw_perm, p->d_mw_dur, p->d_mw_count, p->d_mw_eval_status) ||
      !p->d_mw_scores || !p->d_bvn_scores || !aligned8(p->d_mw_scores) || !aligned8(p->d_bvn_scores))
    return MOESCHED_EINVAL;
  if (h_model == nullptr || !model_in_range(*h_model)) return MOESCHED_EINVAL;
  const cudaStream_t main = static_cast<cudaStream_t>(stream);
  const cudaStream_t side = fork ? static_cast<cudaStream_t>(p->side_stream) : main;
  // The Birkhoff part runs on the caller's stream, which need not be the one of the last call with these buffers.
  // (An event from outside a capture must not be waited for inside, nor one from inside outside.)
  cudaEvent_t done = static_cast<cudaEvent_t>(p->done_event);
  if (done != nullptr) {
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(main, &capturing);
    if (e == cudaSuccess && capturing != cudaStreamCaptureStatusNone) done = nullptr;
    else if (e == cudaSuccess) e = cudaStreamWaitEvent(main, done, 0);
    if (e != cudaSuccess) return fail_cuda(e);
  }
  if (fork) {
    cudaError_t e = cudaEventRecord(static_cast<cudaEvent_t>(p->fork_event), main);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(side, static_cast<cudaEvent_t>(p->fork_event), 0);
    if (e != cudaSuccess) return fail_cuda(e);
  }
  // the Birkhoff decomposition is the longer one: it goes first, and on the caller's stream, so that no event stands
  // between it and what comes before and after
  const size_t st = (size_t)p->score_stride;
  int64_t *sb = p->d_bvn_scores, *sm = p->d_mw_scores;
  int rc = moesched_bvn_decompose(B, N, d_demand, (int)p->k_bvn, p->d_bvn_perm, p->d_bvn_coef, p->d_bvn_count, nullptr,
                                  p->d_bvn_scratch, p->d_bvn_status, p->d_bvn_work, main);
  if (rc == MOESCHED_OK)
    rc = moesched_mw_decompose(B, N, d_demand, (int)p->k_mw, p->d_mw_perm, p->d_mw_dur, p->d_mw_count, nullptr,
                               p->d_mw_status, p->d_mw_work, side);
  if (rc == MOESCHED_OK)
    rc = moesched_schedule_eval(B, N, d_demand, (int)p->k_mw, p->d_mw_perm, p->d_mw_dur, p->d_mw_count, h_model, sm, sm + st,
                                sm + 2 * st, sm + 3 * st, sm + 4 * st, p->d_mw_eval_status, side);
  if (rc == MOESCHED_OK)
    rc = moesched_schedule_eval(B, N, d_demand, (int)p->k_bvn, p->d_bvn_perm, p->d_bvn_coef, p->d_bvn_count, h_model, sb,
                                sb + st, sb + 2 * st, sb + 3 * st, sb + 4 * st, p->d_bvn_eval_status, main);
  if (fork) {   // also after an error: what was enqueued on the side stream is joined
    cudaError_t e = cudaEventRecord(static_cast<cudaEvent_t>(p->join_event), side);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(main, static_cast<cudaEvent_t>(p->join_event), 0);
    if (e != cudaSuccess && rc == MOESCHED_OK) rc = fail_cuda(e);
  }
  if (done != nullptr) {
    cudaError_t e = cudaEventRecord(done, main);
    if (e != cudaSuccess && rc == MOESCHED_OK) rc = fail_cuda(e);
  }
  return rc;
}

size_t moesched_order_scratch_bytes(int B, int k_stride) {
  if (B < 0 || k_stride < 1 || k_stride > MOESCHED_ORDER_MAX_K) return 0;
  return (size_t)B * (2 * (size_t)k_stride + 5) * sizeof(int64_t) + (((size_t)B * sizeof(int32_t) + 7) & ~(size_t)7);
}

int moesched_schedule_order(int B, int N, const int32_t* d_demand, int k_stride, const uint8_t* d_perm,
                            const int32_t* d_dur, const int32_t* d_count, const moesched_model_t* h_model,
                            int32_t* d_order, int64_t* d_makespan_ns, int64_t* d_emission_ns, int32_t* d_rule,
                            int32_t* d_status, void* d_scratch, void* stream) {
  if (B < 0 || N < 1 || N > MOESCHED_MAX_N || k_stride < 1 || k_stride > MOESCHED_ORDER_MAX_K) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!d_demand || !d_perm || !d_dur || !d_count || !h_model || !d_order || !d_makespan_ns || !d_emission_ns ||
      !d_rule || !d_status || !d_scratch)
    return MOESCHED_EINVAL;
  if (!aligned4(d_demand) || !aligned4(d_dur) || !aligned4(d_count) || !aligned4(d_order) || !aligned4(d_rule) ||
      !aligned4(d_status) || !aligned8(d_makespan_ns) || !aligned8(d_emission_ns) || !aligned8(d_scratch))
    return MOESCHED_EINVAL;
  const moesched_model_t m = *h_model;
  if (!model_in_range(m)) return MOESCHED_EINVAL;
  // scratch: job times [B][k_stride] x 2, five score arrays [B], the scoring status [B]
  long long* leg = static_cast<long long*>(d_scratch);
  long long* comp = leg + (size_t)B * k_stride;
  long long* scores = comp + (size_t)B * k_stride;
  int32_t* eval_status = reinterpret_cast<int32_t*>(scores + (size_t)5 * B);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = run_eval(B, N, d_demand, k_stride, d_perm, d_dur, d_count, m, scores, scores + B, scores + 2 * (size_t)B,
                           scores + 3 * (size_t)B, scores + 4 * (size_t)B, eval_status, leg, comp, st, true);
  if (e == cudaSuccess)
    e = run_order(B, k_stride, leg, comp, d_count, eval_status, d_order, reinterpret_cast<long long*>(d_makespan_ns),
                  reinterpret_cast<long long*>(d_emission_ns), d_rule, d_status, st);
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_schedule_permute(int B, int N, int k_stride, const uint8_t* d_perm, const int32_t* d_dur,
                              const int32_t* d_order, uint8_t* d_perm_out, int32_t* d_dur_out, void* stream) {
  if (B < 0 || N < 1 || N > MOESCHED_MAX_N || k_stride < 1) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!d_perm || !d_dur || !d_order || !d_perm_out || !d_dur_out) return MOESCHED_EINVAL;
  if (!aligned4(d_dur) || !aligned4(d_order) || !aligned4(d_dur_out) || d_perm == d_perm_out || d_dur == d_dur_out)
    return MOESCHED_EINVAL;
  cudaError_t e = run_permute(B, N, k_stride, d_perm, d_dur, d_order, d_perm_out, d_dur_out,
                              static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_best_budget(int B, int k_stride, const int32_t* d_count, const int64_t* d_prefix_overlap_ns,
                         const int64_t* d_prefix_unserved_tokens, int64_t ns_per_unserved_token,
                         int32_t* d_best_k, int64_t* d_best_cost, void* stream) {
  if (B < 0 || k_stride < 1 || ns_per_unserved_token < 0 || ns_per_unserved_token > (1LL << 15)) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!d_count || !d_prefix_overlap_ns || !d_prefix_unserved_tokens || !d_best_k || !d_best_cost) return MOESCHED_EINVAL;
  if (!aligned4(d_count) || !aligned4(d_best_k) || !aligned8(d_prefix_overlap_ns) ||
      !aligned8(d_prefix_unserved_tokens) || !aligned8(d_best_cost))
    return MOESCHED_EINVAL;
  cudaError_t e = run_best_budget(B, k_stride, d_count, reinterpret_cast<const long long*>(d_prefix_overlap_ns),
                                  reinterpret_cast<const long long*>(d_prefix_unserved_tokens),
                                  (long long)ns_per_unserved_token, d_best_k,
                                  reinterpret_cast<long long*>(d_best_cost), static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_ideal_a2a(int B, int N, const int32_t* d_demand, const moesched_model_t* h_model, int64_t* d_comm_ns,
                       int64_t* d_makespan_ns, int32_t* d_status, void* stream) {
  if (B < 0 || N < 1 || N > MOESCHED_MAX_N) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!d_demand || !h_model || !d_comm_ns || !d_makespan_ns || !d_status) return MOESCHED_EINVAL;
  if (!aligned4(d_demand) || !aligned4(d_status) || !aligned8(d_comm_ns) || !aligned8(d_makespan_ns))
    return MOESCHED_EINVAL;
  const moesched_model_t m = *h_model;
  if (!model_in_range(m)) return MOESCHED_EINVAL;
  cudaError_t e = run_ideal_a2a(B, N, d_demand, m, reinterpret_cast<long long*>(d_comm_ns),
                                reinterpret_cast<long long*>(d_makespan_ns), d_status,
                                static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_sinkhorn_scale(int B, int N, const int32_t* d_demand, int iters, double smooth, int scale_bits,
                            double* d_scaled, int32_t* d_fixed, double* d_stretch, double* d_row_err,
                            int32_t* d_status, void* stream) {
  if (B < 0 || N < 1 || N > MOESCHED_MAX_N || iters < 1 || !(smooth >= 0.0) || scale_bits < 1 || scale_bits > 24)
    return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!d_demand || !d_scaled || !d_fixed || !d_stretch || !d_row_err || !d_status) return MOESCHED_EINVAL;
  if (!aligned4(d_demand) || !aligned4(d_fixed) || !aligned4(d_status) || !aligned8(d_scaled) ||
      !aligned8(d_stretch) || !aligned8(d_row_err))
    return MOESCHED_EINVAL;
  cudaError_t e = run_sinkhorn(B, N, d_demand, iters, smooth, scale_bits, d_scaled, d_fixed, d_stretch, d_row_err,
                               d_status, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_sinkhorn_durations(int B, int k_stride, const int32_t* d_coef, const int32_t* d_count,
                                const double* d_stretch, int scale_bits, int32_t* d_dur, void* stream) {
  if (B < 0 || k_stride < 1 || scale_bits < 1 || scale_bits > 24) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!d_coef || !d_count || !d_stretch || !d_dur) return MOESCHED_EINVAL;
  if (!aligned4(d_coef) || !aligned4(d_count) || !aligned4(d_dur) || !aligned8(d_stretch)) return MOESCHED_EINVAL;
  cudaError_t e = run_sinkhorn_durations(B, k_stride, d_coef, d_count, d_stretch, scale_bits, d_dur,
                                         static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_bvn_real_decompose(int B, int N, const double* d_matrix, double tol, int k_max, uint8_t* d_perm,
                                double* d_lambda, int32_t* d_count, double* d_sum_lambda, double* d_max_left,
                                double* d_scratch, int32_t* d_status, void* stream) {
  if (B < 0 || N < 1 || N > MOESCHED_MAX_N || k_max < 1 || !(tol >= 0.0)) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!d_matrix || !d_perm || !d_lambda || !d_count || !d_sum_lambda || !d_max_left || !d_scratch || !d_status)
    return MOESCHED_EINVAL;
  if (!aligned8(d_matrix) || !aligned8(d_lambda) || !aligned8(d_sum_lambda) || !aligned8(d_max_left) ||
      !aligned8(d_scratch) || !aligned4(d_count) || !aligned4(d_status))
    return MOESCHED_EINVAL;
  cudaError_t e = run_bvn_real(B, N, d_matrix, tol, k_max, d_perm, d_lambda, d_count, d_sum_lambda, d_max_left,
                               d_scratch, d_status, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_route_demand(int B, int N, int S, int E, const int32_t* d_experts, int32_t* d_demand, int32_t* d_counts,
                          int32_t* d_slot, int32_t* d_status, void* stream) {
  if (!size_ok(B, N, 1) || S < 0 || E < N || E > MOESCHED_MAX_EXPERTS || E % N != 0 || (int64_t)B * N > 0x7fffffff)
    return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if ((S > 0 && (!d_experts || !d_slot)) || !d_demand || !d_counts || !d_status || !aligned4(d_experts) || !aligned4(d_demand) ||
      !aligned4(d_counts) || !aligned4(d_slot) || !aligned4(d_status))
    return MOESCHED_EINVAL;
  cudaError_t e = run_route(B, N, S, E, d_experts, d_demand, d_counts, d_slot, d_status, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

size_t moesched_slots_scratch_bytes(int B, int N, int k_stride) {
  return size_ok(B, N, k_stride) ? slots_scratch_bytes(B, N, k_stride) : 0;
}

int moesched_schedule_slots(int B, int N, const int32_t* d_demand, int k_stride, const uint8_t* d_perm, const int32_t* d_dur,
                            const int32_t* d_count, int experts_per_rank, const int32_t* d_counts, int32_t* d_start,
                            int32_t* d_length, int32_t* d_row, int32_t* d_rows, int32_t* d_offsets, int32_t* d_scratch,
                            int32_t* d_status, void* stream) {
  if (!size_ok(B, N, k_stride)) return MOESCHED_EINVAL;
  if ((d_counts == nullptr) != (d_offsets == nullptr)) return MOESCHED_EINVAL;
  if (d_counts != nullptr && (experts_per_rank < 1 || experts_per_rank > MOESCHED_MAX_EXPERTS / N)) return MOESCHED_EINVAL;
  if (B == 0) return MOESCHED_OK;
  if (!eval_pointers_ok(d_demand, d_perm, d_dur, d_count, d_status) || !d_start || !d_length || !d_row || !d_rows ||
      !aligned4(d_start) || !aligned4(d_length) || !aligned4(d_row) || !aligned4(d_rows) || !aligned4(d_counts) ||
      !aligned4(d_offsets) || !aligned4(d_scratch))
    return MOESCHED_EINVAL;
  cudaError_t e = run_slots(B, N, d_demand, k_stride, d_perm, d_dur, d_count, experts_per_rank, d_counts, d_start, d_length, d_row,
                            d_rows, d_offsets, d_scratch, d_status, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

size_t moesched_expert_scratch_bytes(int R, int I, int groups, int backward) {
  if (R < 0 || R > MOESCHED_MAX_ROWS || !ffn_width_ok(I) || groups < 1 || groups > MOESCHED_MAX_GROUPS) return 0;
  return expert_scratch(R, I, groups, backward != 0).bytes;
}

int moesched_expert_ffn(int R, int D, int I, int E, int groups, int dtype, int act, const void* d_x, const void* d_w_gate,
                        const void* d_w_up, const void* d_w_down, const int32_t* d_offsets, void* d_y, float* d_gate,
                        float* d_up, void* d_scratch, int32_t* d_status, void* stream) {
  if (!expert_sizes_ok(R, E, groups, dtype, act) || !ffn_width_ok(D) || !ffn_width_ok(I)) return MOESCHED_EINVAL;
  if ((d_gate == nullptr) != (d_up == nullptr) || !d_offsets || !aligned4(d_offsets) || !d_status || !aligned4(d_status))
    return MOESCHED_EINVAL;
  const void* pointers[] = {d_x, d_w_gate, d_w_up, d_w_down, d_y, d_scratch};
  for (const void* p : pointers)
    if ((R > 0 && p == nullptr) || !aligned16(p)) return MOESCHED_EINVAL;
  if (!aligned16(d_gate) || !aligned16(d_up) || (reinterpret_cast<uintptr_t>(d_scratch) & 255) != 0) return MOESCHED_EINVAL;
  cudaError_t e = run_expert_ffn(R, D, I, E, groups, dtype, act, d_x, d_w_gate, d_w_up, d_w_down, d_offsets, d_y, d_gate, d_up,
                                 d_scratch, d_status, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_expert_ffn_backward(int R, int D, int I, int E, int groups, int dtype, int act, const void* d_dy, const void* d_x,
                                 const void* d_w_gate, const void* d_w_up, const void* d_w_down, const int32_t* d_offsets,
                                 const float* d_gate, const float* d_up, void* d_dx, void* d_dw_gate, void* d_dw_up,
                                 void* d_dw_down, void* d_scratch, int32_t* d_status, void* stream) {
  if (!expert_sizes_ok(R, E, groups, dtype, act) || !ffn_width_ok(D) || !ffn_width_ok(I)) return MOESCHED_EINVAL;
  if (!d_offsets || !aligned4(d_offsets) || !d_status || !aligned4(d_status) || !d_dw_gate || !d_dw_up || !d_dw_down ||
      !d_scratch || (reinterpret_cast<uintptr_t>(d_scratch) & 255) != 0)
    return MOESCHED_EINVAL;
  const void* pointers[] = {d_dy, d_x, d_w_gate, d_w_up, d_w_down, d_gate, d_up, d_dx, d_dw_gate, d_dw_up, d_dw_down};
  for (const void* p : pointers)
    if ((R > 0 && p == nullptr) || !aligned16(p)) return MOESCHED_EINVAL;
  cudaError_t e = run_expert_backward(R, D, I, E, groups, dtype, act, d_dy, d_x, d_w_gate, d_w_up, d_w_down, d_offsets, d_gate, d_up,
                                      d_dx, d_dw_gate, d_dw_up, d_dw_down, d_scratch, d_status, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_expert_matvec4(int R, int K, int N, int E, int groups, int group, int dtype, int act, const void* d_x,
                            const uint8_t* d_w, const void* d_scale, const uint8_t* d_w_up, const void* d_scale_up,
                            const int32_t* d_offsets, void* d_y, int32_t* d_status, void* stream) {
  if (d_w_up == nullptr) act = MOESCHED_ACT_SILU;   // (not looked at)
  if (!expert_sizes_ok(R, E, groups, dtype, act) || K < 1 || N < 1 || (group != 32 && group != 64 && group != 128) ||
      K % group != 0 || K > (1 << 24) || N > (1 << 24))
    return MOESCHED_EINVAL;
  if ((d_w_up == nullptr) != (d_scale_up == nullptr) || !d_offsets || !aligned4(d_offsets) || !d_status || !aligned4(d_status))
    return MOESCHED_EINVAL;
  const void* pointers[] = {d_x, d_w, d_scale, d_y};
  for (const void* p : pointers)
    if ((R > 0 && p == nullptr) || !aligned16(p)) return MOESCHED_EINVAL;
  if (!aligned16(d_w_up) || !aligned16(d_scale_up)) return MOESCHED_EINVAL;
  cudaError_t e = run_few(R, K, N, E, groups, group, dtype, act, d_x, d_w, d_scale, d_w_up, d_scale_up, d_offsets, d_y, nullptr,
                          nullptr, d_status, false, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_rms_norm(int rows, int D, int dtype, float eps, int group, const void* d_x, const void* d_residual,
                      const void* d_weight, void* d_sum, void* d_y, uint8_t* d_q, float* d_scale, float* d_rstd, void* stream) {
  if (!token_sizes_ok(rows, D, dtype) || !(eps >= 0.0f && eps <= FLT_MAX)) return MOESCHED_EINVAL;
  if (d_q != nullptr && !group_ok(group)) return MOESCHED_EINVAL;
  if (rows == 0) return MOESCHED_OK;
  if (!d_x || !d_weight || (!d_y && !d_q) || (d_residual == nullptr) != (d_sum == nullptr) || (d_q == nullptr) != (d_scale == nullptr))
    return MOESCHED_EINVAL;
  const void* pointers[] = {d_x, d_residual, d_weight, d_sum, d_y, d_q, d_scale};
  for (const void* p : pointers)
    if (!aligned16(p)) return MOESCHED_EINVAL;
  if (!aligned4(d_rstd)) return MOESCHED_EINVAL;
  cudaError_t e = run_norm(rows, D, dtype, eps, group, d_x, d_residual, d_weight, d_sum, d_y, d_q, d_scale, d_rstd,
                           static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

size_t moesched_norm_scratch_bytes(int rows, int D) { return token_sizes_ok(rows, D, MOESCHED_FP32) ? norm_scratch_bytes(rows, D) : 0; }

int moesched_rms_norm_backward(int rows, int D, int dtype, const void* d_dy, const void* d_h, const void* d_weight,
                               const float* d_rstd, const void* d_dsum, void* d_dx, void* d_dweight, float* d_scratch, void* stream) {
  if (!token_sizes_ok(rows, D, dtype) || !d_dweight || !aligned16(d_dweight)) return MOESCHED_EINVAL;
  const void* pointers[] = {d_dy, d_h, d_weight, d_dx, d_scratch};
  for (const void* p : pointers)
    if ((rows > 0 && p == nullptr) || !aligned16(p)) return MOESCHED_EINVAL;
  if ((rows > 0 && !d_rstd) || !aligned4(d_rstd) || !aligned16(d_dsum)) return MOESCHED_EINVAL;
  cudaError_t e = run_norm_backward(rows, D, dtype, d_dy, d_h, d_weight, d_rstd, d_dsum, d_dx, d_dweight, d_scratch,
                                    static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_route_choose(int rows, int E, int k, int dtype, int score, int normalise, float factor, const void* d_logits,
                          const float* d_bias, int32_t* d_experts, float* d_weights, void* stream) {
  if (!choose_sizes_ok(rows, E, k, dtype, score, factor)) return MOESCHED_EINVAL;
  if (rows == 0) return MOESCHED_OK;
  if (!d_logits || !d_experts || !d_weights || !aligned_to(d_logits, dtype == MOESCHED_FP32 ? 4 : 2) || !aligned4(d_bias) ||
      !aligned4(d_experts) || !aligned4(d_weights))
    return MOESCHED_EINVAL;
  cudaError_t e = run_choose(rows, E, k, dtype, score, normalise != 0, factor, d_logits, d_bias, d_experts, d_weights,
                             static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_route_choose_backward(int rows, int E, int k, int dtype, int score, int normalise, float factor,
                                   const float* d_dweights, const void* d_logits, const int32_t* d_experts, void* d_dlogits,
                                   void* stream) {
  if (!choose_sizes_ok(rows, E, k, dtype, score, factor)) return MOESCHED_EINVAL;
  if (rows == 0) return MOESCHED_OK;
  const size_t size = dtype == MOESCHED_FP32 ? 4 : 2;
  if (!d_dweights || !d_logits || !d_experts || !d_dlogits || !aligned_to(d_logits, size) || !aligned_to(d_dlogits, size) ||
      !aligned4(d_dweights) || !aligned4(d_experts))
    return MOESCHED_EINVAL;
  cudaError_t e = run_choose_backward(rows, E, k, dtype, score, normalise != 0, factor, d_dweights, d_logits, d_experts, d_dlogits,
                                      static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_tokens_to_rows(int G, int T, int k, int row_bytes, int scales, const void* d_x, const float* d_scale,
                            const int32_t* d_slot, void* d_rows, float* d_row_scale, void* stream) {
  if (!rows_sizes_ok(G, T, k) || row_bytes < 8 || row_bytes > (1 << 18) || row_bytes % 8 != 0 || scales < 0 || scales > 65536)
    return MOESCHED_EINVAL;
  if (G == 0 || T == 0) return MOESCHED_OK;
  if (!d_x || !d_slot || !d_rows || (scales == 0) != (d_scale == nullptr) || (scales == 0) != (d_row_scale == nullptr))
    return MOESCHED_EINVAL;
  const void* pointers[] = {d_x, d_scale, d_rows, d_row_scale};
  for (const void* p : pointers)
    if (!aligned16(p)) return MOESCHED_EINVAL;
  if (!aligned4(d_slot)) return MOESCHED_EINVAL;
  cudaError_t e = run_tokens_to_rows(G, T, k, row_bytes, scales, d_x, d_scale, d_slot, d_rows, d_row_scale,
                                     static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_rows_to_tokens(int G, int T, int k, int D, int dtype, const void* d_rows, const int32_t* d_slot,
                            const float* d_weights, const void* d_add, void* d_y, void* stream) {
  if (!rows_sizes_ok(G, T, k) || !token_sizes_ok(0, D, dtype)) return MOESCHED_EINVAL;
  if (G == 0 || T == 0) return MOESCHED_OK;
  if (!d_rows || !d_slot || !d_y || !aligned16(d_rows) || !aligned16(d_add) || !aligned16(d_y) || !aligned4(d_slot) || !aligned4(d_weights))
    return MOESCHED_EINVAL;
  cudaError_t e = run_rows_to_tokens(G, T, k, D, dtype, d_rows, d_slot, d_weights, d_add, d_y, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_rows_to_tokens_backward(int G, int T, int k, int D, int dtype, const void* d_dy, const void* d_rows,
                                     const int32_t* d_slot, const float* d_weights, void* d_drows, float* d_dweights, void* stream) {
  if (!rows_sizes_ok(G, T, k) || !token_sizes_ok(0, D, dtype)) return MOESCHED_EINVAL;
  if (G == 0 || T == 0) return MOESCHED_OK;
  if (!d_dy || !d_rows || !d_slot || !d_weights || !d_drows || !d_dweights || !aligned16(d_dy) || !aligned16(d_rows) ||
      !aligned16(d_drows) || !aligned4(d_slot) || !aligned4(d_weights) || !aligned4(d_dweights))
    return MOESCHED_EINVAL;
  cudaError_t e = run_rows_to_tokens_backward(G, T, k, D, dtype, d_dy, d_rows, d_slot, d_weights, d_drows, d_dweights,
                                              static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

int moesched_rows_widen(int R, int D, int group, int dtype, const uint8_t* d_q, const float* d_scale, void* d_y, void* stream) {
  if (!token_sizes_ok(R, D, dtype) || !group_ok(group)) return MOESCHED_EINVAL;
  if (R == 0) return MOESCHED_OK;
  if (!d_q || !d_scale || !d_y || !aligned16(d_q) || !aligned16(d_scale) || !aligned16(d_y)) return MOESCHED_EINVAL;
  cudaError_t e = run_rows_widen(R, D, group, dtype, d_q, d_scale, d_y, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MOESCHED_OK : fail_cuda(e);
}

long long moesched_debug_index_faults(void) {
#ifdef MOESCHED_CHECKED
  if (cudaDeviceSynchronize() != cudaSuccess) return -2;
  long long total = 0;
  for (FaultReader read : fault_readers()) {
    const unsigned v = read();
    if (v == 0xffffffffu) return -2;
    total += v;
  }
  return total;
#else
  return -1;
#endif
}

int moesched_last_cuda_error(void) { return g_last_cuda_error; }

const char* moesched_strerror(int code) {
  switch (code) {
    case MOESCHED_OK: return "ok";
    case MOESCHED_EINVAL: return "invalid argument: null or misaligned pointer, or a size out of range";
    case MOESCHED_ECUDA: return "a CUDA call failed (see moesched_last_cuda_error)";
    case MOESCHED_ETOOBIG: return "batch too large for the library's built-in scratch array";
    default: return "unknown moesched return code";
  }
}

const char* moesched_status_str(int status) {
  switch (status) {
    case MOESCHED_ST_OK: return "ok: complete result";
    case MOESCHED_ST_TRUNCATED: return "truncated: the matching budget ran out before the matrix did";
    case MOESCHED_ST_BAD_INPUT: return "bad input: the matrix or schedule violates the documented range";
    case MOESCHED_ST_INTERNAL: return "internal: an iteration limit was hit (a bug in the library)";
    default: return "unknown moesched status";
  }
}

}  // extern "C"
