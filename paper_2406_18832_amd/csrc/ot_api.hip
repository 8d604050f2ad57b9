// C ABI of libot (declared in include/ot.h): argument checks on the host,
// then kernel launches on the caller's stream.  Nothing here allocates
// device memory; the only state between calls is a block of status words.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <atomic>
#include <mutex>
#include <vector>

#include "ot_kv8.h"
#include "ot_mx4.h"

namespace {

// Largest K the kernels' 32-bit in-tile offsets cover (a tile of at most
// 320 K-byte rows must stay below 2^31 bytes).
constexpr int64_t kMaxK = int64_t(1) << 22;
constexpr int64_t kMaxLnK = int64_t(1) << 16;  // LayerNorm width (exact sums, one workgroup per row)
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;
// Calls of so many tokens and channels that not even 128 x 256 tiles of them
// are a 32-bit count are refused (the launcher leaves a smaller tile out where
// its own grid does not fit).
bool grid_ok(int64_t M, int64_t N) { return (M + 127) / 128 * ((N + 255) / 256) <= kMaxRows; }

// MX4: the largest LayerNorm and linear whose workgroups fit a launch (fewer than
// 2^32 work-items, 1024 of them to a row or to 16 channels).
constexpr int64_t kMaxLnMx4Rows = (int64_t(1) << 22) - 1;
constexpr int64_t kMaxMx4N = (int64_t(1) << 26) - 1;
bool mx4_k_ok(int64_t K) { return K >= 32 && K % 32 == 0 && K <= ot::kMx4MaxK; }

// KV8: heads, sequences, tokens of a call and pages of a sequence (positions stay
// below 2^30, rows of all query heads of a key head below 2^30).
constexpr int64_t kMaxKv8Heads = 1024, kMaxKv8Queries = 16384, kMaxKv8Batch = 65535;
constexpr int64_t kMaxKv8Tokens = int64_t(1) << 24, kMaxKv8Pages = int64_t(1) << 24;
// Rows of H D elements so far apart, 16-byte aligned each; the last one's offset fits.
bool kv8_ld_ok(int64_t ld, int64_t width) {
  return ld >= width && ld % 8 == 0 && ld < (int64_t(1) << 32);
}

bool bits_ok(int bits) { return bits >= 2 && bits <= 8; }
int qmax(int bits) { return (1 << (bits - 1)) - 1; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

ot_status hip_status(hipError_t e) { return e == hipSuccess ? OT_OK : OT_EHIP; }

// A word of pinned host memory that a kernel of one synchronous call raises
// and the call reads after its stream synchronization, instead of copying
// the call's outputs back to look at them (two copies through the runtime's
// staging buffer: 50 us after a fold of 20480 channels).  The words
// come from one 4 KiB block, allocated on first use and kept until the
// process ends; a call holds its word only while it runs.  Without one (every
// word taken, no pinned memory, or a stream under capture, on which the call
// is going to fail: its word could not be given back) word() is nullptr and the
// caller reads its outputs back.
class StatusWord {
 public:
  explicit StatusWord(hipStream_t st) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &capture) != hipSuccess) {
      (void)hipGetLastError();
      return;
    }
    if (capture != hipStreamCaptureStatusNone) return;
    int *block = words();
    if (block == nullptr) return;
    uint64_t used = used_.load(std::memory_order_relaxed);
    while (~used != 0) {
      const int i = __builtin_ctzll(~used);
      if (used_.compare_exchange_weak(used, used | (uint64_t(1) << i),
                                      std::memory_order_acquire, std::memory_order_relaxed)) {
        index_ = i;
        word_ = block + i * kStride;
        __atomic_store_n(word_, 0, __ATOMIC_RELEASE);
        return;
      }
    }
  }
  // Only when no kernel that may write it still runs (its stream has been
  // synchronized): any other word is never handed out again.
  void release() {
    if (word_ != nullptr) used_.fetch_and(~(uint64_t(1) << index_), std::memory_order_release);
    word_ = nullptr;
  }
  // After a launch that reported an error.  The error may be an older one of
  // this thread and the kernel running all the same: the word goes back only
  // once the stream is known to be idle.
  void release_after_error(hipStream_t st) {
    if (word_ != nullptr && hipStreamSynchronize(st) == hipSuccess) release();
  }
  int *word() const { return word_; }
  bool raised() const { return __atomic_load_n(word_, __ATOMIC_ACQUIRE) != 0; }

 private:
  static constexpr int kStride = 16;  // a 64-byte line each, 64 of them
  static int *words() {
    static std::once_flag once;
    std::call_once(once, [] {
      // another thread may be capturing a graph: this allocation is no part of it
      hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
      (void)hipThreadExchangeStreamCaptureMode(&mode);
      void *p = nullptr;
      if (hipHostMalloc(&p, 64 * kStride * sizeof(int),
                        hipHostMallocPortable | hipHostMallocMapped | hipHostMallocCoherent) ==
          hipSuccess)
        block_ = static_cast<int *>(p);
      else
        (void)hipGetLastError();
      (void)hipThreadExchangeStreamCaptureMode(&mode);
    });
    return block_;
  }
  static int *block_;
  static std::atomic<uint64_t> used_;
  int *word_ = nullptr;
  int index_ = 0;
};
int *StatusWord::block_ = nullptr;
std::atomic<uint64_t> StatusWord::used_{0};

bool all_finite(const std::vector<float> &v) {
  for (float f : v)
    if (!isfinite(f)) return false;
  return true;
}

}  // namespace

extern "C" {

const char *ot_strerror(int status) {
  switch (status) {
    case OT_OK: return "ok";
    case OT_EINVAL: return "invalid argument (null or misaligned pointer, bits outside [2, 8], negative size)";
    case OT_ESHAPE: return "unsupported shape (K must be a positive multiple of 16 within limits; sizes must be nonzero where required)";
    case OT_ERANGE: return "K * qa * qw >= 2^31: the int32 accumulator could overflow";
    case OT_ENONFINITE: return "non-finite value (NaN or infinity) in calibration data or weights";
    case OT_EHIP: return "HIP runtime error";
    case OT_ENOSCRATCH: return "these sizes need more scratch than ot_qlinear_noalloc's fixed array holds (use ot_qlinear with a workspace)";
    default: return "unknown status";
  }
}

int ot_abi_version(void) { return 1; }

#ifndef OT_SOURCES_SHA256
#define OT_SOURCES_SHA256 "unknown"
#endif
#ifndef OT_HEADER_SHA256
#define OT_HEADER_SHA256 "unknown"
#endif
#define OT_STR2(x) #x
#define OT_STR(x) OT_STR2(x)

const char *ot_build_info(void) {
  return "sources_sha256=" OT_SOURCES_SHA256 ";arch=gfx950;hip=" OT_STR(HIP_VERSION_MAJOR) "." OT_STR(
      HIP_VERSION_MINOR) "." OT_STR(HIP_VERSION_PATCH) ";header_sha256=" OT_HEADER_SHA256;
}

ot_status ot_calibrate(const uint16_t *x, int64_t rows, int64_t K, int a_bits, int first,
                       float *minmax, float *z, float *s, float *inv_s, void *stream) {
  if (!x || !minmax || !z || !s || !inv_s) return OT_EINVAL;
  if (!bits_ok(a_bits) || rows < 0 || K < 0) return OT_EINVAL;
  if (rows == 0 || K == 0 || rows > kMaxRows || K > kMaxRows) return OT_ESHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  ot_status rc;
  if (first && (rc = hip_status(ot::launch_calib_reset(minmax, K, st))) != OT_OK) return rc;
  if ((rc = hip_status(ot::launch_calib_minmax(x, rows, K, minmax, st))) != OT_OK) return rc;
  if (ot::calib_finish_ok(K)) {
    StatusWord status(st);
    if (status.word() != nullptr) {
      if (ot::launch_calib_finish(minmax, K, qmax(a_bits), z, s, inv_s, status.word(), st) !=
          hipSuccess) {
        status.release_after_error(st);
        return OT_EHIP;
      }
      if (hipStreamSynchronize(st) != hipSuccess) return OT_EHIP;
      const bool bad = status.raised();
      status.release();
      return bad ? OT_ENONFINITE : OT_OK;
    }
  }
  std::vector<float> state((size_t)(2 * K));
  if ((rc = hip_status(hipMemcpyAsync(state.data(), minmax, sizeof(float) * 2 * K,
                                      hipMemcpyDeviceToHost, st))) != OT_OK)
    return rc;
  if ((rc = hip_status(hipStreamSynchronize(st))) != OT_OK) return rc;
  if (!all_finite(state)) return OT_ENONFINITE;
  if ((rc = hip_status(ot::launch_calib_finalize(minmax, K, qmax(a_bits), 1, z, s, inv_s, st))) !=
      OT_OK)
    return rc;
  return hip_status(hipStreamSynchronize(st));
}

ot_status ot_scales_from_minmax(const float *minmax, int64_t K, int a_bits, int symmetrize,
                                float *z, float *s, float *inv_s, void *stream) {
  if (!bits_ok(a_bits) || K < 0) return OT_EINVAL;
  if (K == 0 || K > kMaxRows) return OT_ESHAPE;
  if (!minmax || !z || !s || !inv_s) return OT_EINVAL;
  return hip_status(ot::launch_calib_finalize(minmax, K, qmax(a_bits), symmetrize ? 1 : 0, z, s,
                                              inv_s, static_cast<hipStream_t>(stream)));
}

// After a fold's launch (its status e): waits for it and tells whether every
// scale and bias is finite (a NaN scale marks non-finite weights), from the
// kernel's status word or, without one, from sW and b' read back.
static ot_status fold_result(hipError_t e, StatusWord &status, const float *sW,
                             const float *bprime, int64_t N, hipStream_t st) {
  if (e != hipSuccess) {
    status.release_after_error(st);
    return OT_EHIP;
  }
  if (status.word() != nullptr) {
    if (hipStreamSynchronize(st) != hipSuccess) return OT_EHIP;
    const bool bad = status.raised();
    status.release();
    return bad ? OT_ENONFINITE : OT_OK;
  }
  ot_status rc;
  std::vector<float> scale((size_t)N), bias((size_t)N);
  if ((rc = hip_status(hipMemcpyAsync(scale.data(), sW, sizeof(float) * N, hipMemcpyDeviceToHost,
                                      st))) != OT_OK ||
      (rc = hip_status(hipMemcpyAsync(bias.data(), bprime, sizeof(float) * N,
                                      hipMemcpyDeviceToHost, st))) != OT_OK)
    return rc;
  if ((rc = hip_status(hipStreamSynchronize(st))) != OT_OK) return rc;
  if (!all_finite(scale) || !all_finite(bias)) return OT_ENONFINITE;
  return OT_OK;
}

ot_status ot_fold_weights(const uint16_t *W, const uint16_t *b, int64_t N, int64_t K, int w_bits,
                          const float *z, const float *s, int8_t *Wq, float *sW, float *bprime,
                          void *stream) {
  if (!W || !z || !s || !Wq || !sW || !bprime) return OT_EINVAL;
  if (!bits_ok(w_bits) || N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || K == 0 || N > kMaxRows || K > kMaxRows) return OT_ESHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  StatusWord status(st);
  const hipError_t e =
      ot::launch_fold(W, b, N, K, w_bits, z, s, Wq, sW, bprime, status.word(), st);
  return fold_result(e, status, sW, bprime, N, st);
}

ot_status ot_quantize_act(const uint16_t *x, int64_t M, int64_t K, int a_bits, const float *z,
                          const float *inv_s, int8_t *Xq, void *stream) {
  if (!bits_ok(a_bits) || M < 0 || K < 0) return OT_EINVAL;
  if (K < 16 || K % 16 != 0 || K > kMaxK || M > kMaxRows) return OT_ESHAPE;
  if (M == 0) return OT_OK;
  if (!x || !z || !inv_s || !Xq) return OT_EINVAL;
  if (!aligned16(x) || !aligned16(z) || !aligned16(inv_s) || !aligned16(Xq)) return OT_EINVAL;
  return hip_status(ot::launch_quantize_act(x, M, K, qmax(a_bits), z, inv_s, Xq,
                                            static_cast<hipStream_t>(stream)));
}

ot_status ot_ln_quantize_act(const uint16_t *h, int64_t M, int64_t K, const uint16_t *gamma,
                             const uint16_t *beta, float eps, int a_bits, const float *z,
                             const float *inv_s, int8_t *Xq, void *stream) {
  if (!bits_ok(a_bits) || M < 0 || K < 0 || !(eps >= 0.f) || eps > 3.4e38f) return OT_EINVAL;
  if (K < 16 || K % 16 != 0 || K > kMaxLnK || M > kMaxRows) return OT_ESHAPE;
  if (M == 0) return OT_OK;
  if (!h || !gamma || !beta || !z || !inv_s || !Xq) return OT_EINVAL;
  if (!aligned16(h) || !aligned16(gamma) || !aligned16(beta) || !aligned16(z) ||
      !aligned16(inv_s) || !aligned16(Xq))
    return OT_EINVAL;
  return hip_status(ot::launch_ln_quantize_act(h, M, K, gamma, beta, eps, qmax(a_bits), z, inv_s,
                                               Xq, static_cast<hipStream_t>(stream)));
}

ot_status ot_qlinear(const int8_t *Xq, const int8_t *Wq, const float *sW, const float *bprime,
                     int64_t M, int64_t N, int64_t K, int a_bits, int w_bits, uint16_t *Y,
                     int32_t *acc_out, void *workspace, void *stream) {
  if (!bits_ok(a_bits) || !bits_ok(w_bits) || M < 0 || N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || K < 16 || K % 16 != 0 || K > kMaxK || M > kMaxRows || N > kMaxRows)
    return OT_ESHAPE;
  if (!grid_ok(M, N)) return OT_ESHAPE;
  if (K * qmax(a_bits) * qmax(w_bits) >= (int64_t(1) << 31)) return OT_ERANGE;
  if (M == 0) return OT_OK;
  if (!Xq || !Wq || !sW || !bprime || !Y) return OT_EINVAL;
  if (!aligned16(Xq) || !aligned16(Wq) || !aligned16(sW) || !aligned16(bprime) || !aligned16(Y) ||
      (acc_out && !aligned16(acc_out)) ||
      (workspace && !aligned16(workspace)))
    return OT_EINVAL;
  return hip_status(ot::launch_qgemm(Xq, Wq, nullptr, nullptr, sW, bprime, M, N, K, Y, acc_out,
                                     workspace, static_cast<hipStream_t>(stream)));
}

ot_status ot_quantize_act_per_token(const uint16_t *x, int64_t M, int64_t K, int a_bits,
                                    int8_t *Xq, float *sX, void *stream) {
  if (!bits_ok(a_bits) || M < 0 || K < 0) return OT_EINVAL;
  if (K < 16 || K % 16 != 0 || K > kMaxLnK || M > kMaxRows) return OT_ESHAPE;
  if (M == 0) return OT_OK;
  if (!x || !Xq || !sX) return OT_EINVAL;
  if (!aligned16(x) || !aligned16(Xq) || !aligned16(sX)) return OT_EINVAL;
  return hip_status(ot::launch_quantize_act_per_token(x, M, K, qmax(a_bits), Xq, sX,
                                                      static_cast<hipStream_t>(stream)));
}

ot_status ot_fold_weights_per_token(const uint16_t *W, const uint16_t *b, const float *zres,
                                    int64_t N, int64_t K, int w_bits, int8_t *Wq, float *sW,
                                    float *bprime, void *stream) {
  if (!bits_ok(w_bits) || N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || K == 0 || N > kMaxRows || K > kMaxRows) return OT_ESHAPE;
  if (!W || !Wq || !sW || !bprime) return OT_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  StatusWord status(st);
  const hipError_t e =
      ot::launch_fold_per_token(W, b, zres, N, K, w_bits, Wq, sW, bprime, status.word(), st);
  return fold_result(e, status, sW, bprime, N, st);
}

ot_status ot_qlinear_per_token(const int8_t *Xq, const int8_t *Wq, const float *sX,
                               const float *sW, const float *bprime, int64_t M, int64_t N,
                               int64_t K, int a_bits, int w_bits, uint16_t *Y, int32_t *acc_out,
                               void *workspace, void *stream) {
  if (!bits_ok(a_bits) || !bits_ok(w_bits) || M < 0 || N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || K < 16 || K % 16 != 0 || K > kMaxK || M > kMaxRows || N > kMaxRows)
    return OT_ESHAPE;
  if (!grid_ok(M, N)) return OT_ESHAPE;
  if (K * qmax(a_bits) * qmax(w_bits) >= (int64_t(1) << 31)) return OT_ERANGE;
  if (M == 0) return OT_OK;
  if (!Xq || !Wq || !sX || !sW || !bprime || !Y) return OT_EINVAL;
  if (!aligned16(Xq) || !aligned16(Wq) || !aligned16(sW) || !aligned16(bprime) || !aligned16(Y) ||
      (acc_out && !aligned16(acc_out)) ||
      (workspace && !aligned16(workspace)))
    return OT_EINVAL;
  return hip_status(ot::launch_qgemm(Xq, Wq, sX, nullptr, sW, bprime, M, N, K, Y, acc_out,
                                     workspace, static_cast<hipStream_t>(stream)));
}

ot_status ot_fold_weights_asym(const uint16_t *W, const uint16_t *b, int64_t N, int64_t K,
                               int w_bits, const float *z, const float *s, int8_t *Wq, float *sW,
                               int32_t *zW, float *bprime, void *stream) {
  if (!W || !z || !s || !Wq || !sW || !zW || !bprime) return OT_EINVAL;
  if (!bits_ok(w_bits) || N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || K == 0 || N > kMaxRows || K > kMaxRows) return OT_ESHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  StatusWord status(st);
  const hipError_t e =
      ot::launch_fold_asym(W, b, N, K, w_bits, z, s, Wq, sW, zW, bprime, status.word(), st);
  return fold_result(e, status, sW, bprime, N, st);
}

ot_status ot_qlinear_asym(const int8_t *Xq, const int8_t *Wq, const float *sW, const int32_t *zW,
                          const float *bprime, int64_t M, int64_t N, int64_t K, int a_bits,
                          int w_bits, uint16_t *Y, int32_t *acc_out, void *workspace,
                          void *stream) {
  if (!bits_ok(a_bits) || !bits_ok(w_bits) || M < 0 || N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || K < 16 || K % 16 != 0 || K > kMaxK || M > kMaxRows || N > kMaxRows)
    return OT_ESHAPE;
  if (!grid_ok(M, N)) return OT_ESHAPE;
  // |Xq| <= qa against stored codes and zero points of magnitude <= 2^(w_bits-1):
  // every partial sum stays below K qa 2^w_bits
  if (K * qmax(a_bits) * (int64_t(1) << w_bits) >= (int64_t(1) << 31)) return OT_ERANGE;
  if (M == 0) return OT_OK;
  if (!Xq || !Wq || !sW || !zW || !bprime || !Y) return OT_EINVAL;
  if (!aligned16(Xq) || !aligned16(Wq) || !aligned16(sW) || !aligned16(zW) ||
      !aligned16(bprime) || !aligned16(Y) || (acc_out && !aligned16(acc_out)) ||
      (workspace && !aligned16(workspace)))
    return OT_EINVAL;
  return hip_status(ot::launch_qgemm(Xq, Wq, nullptr, zW, sW, bprime, M, N, K, Y, acc_out,
                                     workspace, static_cast<hipStream_t>(stream)));
}

size_t ot_packed_weights_size(int64_t N, int64_t K) {
  if (N <= 0 || K < 16 || K % 16 != 0 || N > kMaxRows || K > kMaxK) return 0;
  return ot::packed_weights_bytes(N, K);
}

ot_status ot_pack_weights(const int8_t *Wq, int64_t N, int64_t K, int8_t *Wp, void *stream) {
  if (N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || K < 16 || K % 16 != 0 || K > kMaxK || N > kMaxRows) return OT_ESHAPE;
  if (!Wq || !Wp || !aligned16(Wq) || !aligned16(Wp)) return OT_EINVAL;
  return hip_status(ot::launch_pack_weights(Wq, N, K, Wp, static_cast<hipStream_t>(stream)));
}

ot_status ot_qlinear_packed(const int8_t *Xq, const int8_t *Wp, const float *sW,
                            const float *bprime, int64_t M, int64_t N, int64_t K, int a_bits,
                            int w_bits, uint16_t *Y, int32_t *acc_out, void *workspace,
                            void *stream) {
  if (!bits_ok(a_bits) || !bits_ok(w_bits) || M < 0 || N < 0 || K < 0) return OT_EINVAL;
  if (M > 64 || N == 0 || K < 16 || K % 16 != 0 || K > kMaxK || N > kMaxRows) return OT_ESHAPE;
  if (K * qmax(a_bits) * qmax(w_bits) >= (int64_t(1) << 31)) return OT_ERANGE;
  if (M == 0) return OT_OK;
  if (!Xq || !Wp || !sW || !bprime || !Y) return OT_EINVAL;
  if (!aligned16(Xq) || !aligned16(Wp) || !aligned16(sW) || !aligned16(bprime) || !aligned16(Y) ||
      (acc_out && !aligned16(acc_out)) || (workspace && !aligned16(workspace)))
    return OT_EINVAL;
  return hip_status(ot::launch_qgemm_decode(Xq, Wp, nullptr, nullptr, sW, bprime, M, N, K, Y,
                                            acc_out, workspace, true,
                                            static_cast<hipStream_t>(stream)));
}

ot_status ot_qlinear_plan(int64_t M, int64_t N, int64_t K, int packed, int with_workspace,
                          char *buf, size_t len) {
  if (!buf || len == 0 || M < 0 || N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || K < 16 || K % 16 != 0 || K > kMaxK || M > kMaxRows || N > kMaxRows ||
      !grid_ok(M, N) || (packed && M > 64))
    return OT_ESHAPE;
  if (M == 0)
    snprintf(buf, len, "none");
  else if (M <= 64)
    ot::describe_decode(M, N, K, packed != 0, with_workspace != 0, buf, len);
  else
    snprintf(buf, len, "%s", ot::prefill_tile_name(M, N, K));
  return OT_OK;
}

size_t ot_qlinear_workspace_size(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0 || K <= 0 || M > kMaxRows || N > kMaxRows || K > kMaxK) return 0;
  return ot::qgemm_workspace_bytes(M, N, K);
}

ot_status ot_quantize_act_mx4(const uint16_t *x, int64_t M, int64_t K, const float *z,
                              const float *inv_s, uint8_t *Xc, uint8_t *Xe, void *stream) {
  if (M < 0 || K < 0) return OT_EINVAL;
  if (!mx4_k_ok(K) || M > kMaxRows) return OT_ESHAPE;
  if (M == 0) return OT_OK;
  if (!x || !Xc || !Xe || (z == nullptr) != (inv_s == nullptr)) return OT_EINVAL;
  if (!aligned16(x) || !aligned16(z) || !aligned16(inv_s) || !aligned16(Xc) || !aligned16(Xe))
    return OT_EINVAL;
  return hip_status(
      ot::launch_quantize_act_mx4(x, M, K, z, inv_s, Xc, Xe, static_cast<hipStream_t>(stream)));
}

ot_status ot_ln_quantize_act_mx4(const uint16_t *h, int64_t M, int64_t K, const uint16_t *gamma,
                                 const uint16_t *beta, float eps, const float *z,
                                 const float *inv_s, uint8_t *Xc, uint8_t *Xe, void *stream) {
  if (M < 0 || K < 0 || !(eps >= 0.f) || eps > 3.4e38f) return OT_EINVAL;
  if (!mx4_k_ok(K) || K > kMaxLnK || M > kMaxLnMx4Rows) return OT_ESHAPE;
  if (M == 0) return OT_OK;
  if (!h || !gamma || !beta || !z || !inv_s || !Xc || !Xe) return OT_EINVAL;
  if (!aligned16(h) || !aligned16(gamma) || !aligned16(beta) || !aligned16(z) ||
      !aligned16(inv_s) || !aligned16(Xc) || !aligned16(Xe))
    return OT_EINVAL;
  return hip_status(ot::launch_ln_quantize_act_mx4(h, M, K, gamma, beta, eps, z, inv_s, Xc, Xe,
                                                   static_cast<hipStream_t>(stream)));
}

ot_status ot_fold_weights_mx4(const uint16_t *W, const uint16_t *b, int64_t N, int64_t K,
                              const float *z, const float *s, uint8_t *Wc, uint8_t *We,
                              float *bprime, void *stream) {
  if (N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || !mx4_k_ok(K) || N > kMaxRows) return OT_ESHAPE;
  if (!W || !Wc || !We || !bprime) return OT_EINVAL;
  if (!aligned16(W) || !aligned16(z) || !aligned16(s) || !aligned16(Wc) || !aligned16(We))
    return OT_EINVAL;
  // b and b' go by single elements
  if (reinterpret_cast<uintptr_t>(b) % sizeof(*b) || reinterpret_cast<uintptr_t>(bprime) % sizeof(*bprime))
    return OT_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  StatusWord status(st);
  const hipError_t e = ot::launch_fold_mx4(W, b, N, K, z, s, Wc, We, bprime, status.word(), st);
  return fold_result(e, status, bprime, bprime, N, st);  // a row's NaN b' marks it
}

ot_status ot_dequantize_mx4(const uint8_t *c, const uint8_t *e, int64_t rows, int64_t K, float *y,
                            void *stream) {
  if (rows < 0 || K < 0) return OT_EINVAL;
  if (!mx4_k_ok(K) || rows > kMaxRows) return OT_ESHAPE;
  if (rows == 0) return OT_OK;
  if (!c || !e || !y || !aligned16(c) || !aligned16(e) || !aligned16(y)) return OT_EINVAL;
  return hip_status(ot::launch_dequantize_mx4(c, e, rows, K, y, static_cast<hipStream_t>(stream)));
}

size_t ot_packed_weights_mx4_size(int64_t N, int64_t K) {
  if (N <= 0 || !mx4_k_ok(K) || N > kMaxRows) return 0;
  return ot::mx4_packed_bytes(N, K);
}

ot_status ot_pack_weights_mx4(const uint8_t *Wc, const uint8_t *We, int64_t N, int64_t K,
                              uint8_t *Wp, void *stream) {
  if (N < 0 || K < 0) return OT_EINVAL;
  if (N == 0 || !mx4_k_ok(K) || N > kMaxRows) return OT_ESHAPE;
  if (!Wc || !We || !Wp || !aligned16(Wc) || !aligned16(We) || !aligned16(Wp)) return OT_EINVAL;
  return hip_status(
      ot::launch_pack_weights_mx4(Wc, We, N, K, Wp, static_cast<hipStream_t>(stream)));
}

static bool mx4_linear_ok(int64_t M, int64_t N, int64_t K) {
  return N > 0 && mx4_k_ok(K) && M <= kMaxRows && N <= kMaxMx4N && ot::mx4_gemm_fits(M, N);
}

ot_status ot_qlinear_mx4(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                         const float *bprime, int64_t M, int64_t N, int64_t K, uint16_t *Y,
                         void *workspace, void *stream) {
  if (M < 0 || N < 0 || K < 0) return OT_EINVAL;
  if (!mx4_linear_ok(M, N, K)) return OT_ESHAPE;
  if (M == 0) return OT_OK;
  if (!Xc || !Xe || !Wp || !bprime || !Y) return OT_EINVAL;
  if (!aligned16(Xc) || !aligned16(Xe) || !aligned16(Wp) || !aligned16(bprime) || !aligned16(Y) ||
      !aligned16(workspace))
    return OT_EINVAL;
  return hip_status(ot::launch_mx4_linear(Xc, Xe, Wp, bprime, M, N, K, Y, workspace,
                                          static_cast<hipStream_t>(stream)));
}

size_t ot_qlinear_mx4_workspace_size(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || !mx4_linear_ok(M, N, K)) return 0;
  return ot::mx4_linear_workspace_bytes(M, N, K);
}

size_t ot_qlinear_mx4_workspace_max(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || !mx4_linear_ok(M, N, K)) return 0;
  return ot::mx4_linear_workspace_max(M, N, K);
}

ot_status ot_qlinear_mx4_plan(int64_t M, int64_t N, int64_t K, int with_workspace, char *buf,
                              size_t len) {
  if (!buf || len == 0 || M < 0 || N < 0 || K < 0) return OT_EINVAL;
  if (!mx4_linear_ok(M, N, K)) return OT_ESHAPE;
  if (M == 0)
    snprintf(buf, len, "none");
  else
    ot::describe_mx4_linear(M, N, K, with_workspace != 0, buf, len);
  return OT_OK;
}

// Sizes of a mixture-of-experts layer: M == 0 is fine.
static bool moe_shape_ok(int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k) {
  return M <= OT_MOE_MAX_TOKENS && H > 0 && H % 32 == 0 && H <= kMaxLnK && F > 0 && F % 32 == 0 &&
         F <= kMaxLnK && E > 0 && E <= OT_MOE_MAX_EXPERTS && top_k > 0 && top_k <= E &&
         top_k <= OT_MOE_MAX_TOP_K;
}

size_t ot_moe_mx4_workspace_size(int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k) {
  if (M <= 0 || !moe_shape_ok(M, H, F, E, top_k)) return 0;
  return ot::moe_mx4_workspace_bytes(M, H, F, E, top_k);
}

ot_status ot_moe_mx4(const uint8_t *Xc, const uint8_t *Xe, const uint16_t *logits,
                     const uint8_t *W1p, const float *b1, const uint8_t *W2p, const float *b2,
                     int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k, int act,
                     uint16_t *Y, void *workspace, void *stream) {
  if (M < 0 || H < 0 || F < 0 || E < 0 || top_k < 0) return OT_EINVAL;
  if (act != OT_MOE_RELU && act != OT_MOE_SWIGLU) return OT_EINVAL;
  if (!moe_shape_ok(M, H, F, E, top_k)) return OT_ESHAPE;
  if (M == 0) return OT_OK;
  if (!Xc || !Xe || !logits || !W1p || !W2p || !Y || !workspace) return OT_EINVAL;
  if (!aligned16(Xc) || !aligned16(Xe) || !aligned16(logits) || !aligned16(W1p) ||
      !aligned16(b1) || !aligned16(W2p) || !aligned16(b2) || !aligned16(Y) ||
      !aligned16(workspace))
    return OT_EINVAL;
  return hip_status(ot::launch_moe_mx4(Xc, Xe, logits, W1p, b1, W2p, b2, M, H, F, E, top_k,
                                       act == OT_MOE_SWIGLU, Y, workspace,
                                       static_cast<hipStream_t>(stream)));
}

// Sizes of an 8-bit cache and a batch over it.
static bool kv8_ok(int64_t T, int64_t B, int64_t H, int64_t D, int64_t max_pages,
                   int64_t num_pages) {
  return D >= 16 && D <= 256 && D % 16 == 0 && H >= 1 && H <= kMaxKv8Heads && B <= kMaxKv8Batch &&
         T <= kMaxKv8Tokens && max_pages >= 1 && max_pages <= kMaxKv8Pages && num_pages >= 1 &&
         num_pages <= kMaxRows;
}
// A wave to a page, a head and keys or values fits a launch (fewer than 2^32 work-items).
static bool kv8_pages_fit(int64_t T, int64_t B, int64_t H) {
  return ot::kv8_page_slots(T, B) * ((2 * H + 3) / 4) * 256 < (int64_t(1) << 32);
}
static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int64_t ot_kv8_row_size(int64_t D) {
  return D >= 16 && D <= 256 && D % 16 == 0 ? ot::kv8_width(D) : 0;
}

ot_status ot_kv8_append(const uint16_t *k, int64_t ldk, const uint16_t *v, int64_t ldv, int64_t T,
                        int64_t B, int64_t H, int64_t D, const int32_t *cu, const int32_t *kv_len,
                        const int32_t *table, int64_t max_pages, int64_t num_pages, uint8_t *Kc,
                        uint8_t *Vc, float *Ks, float *Vs, void *stream) {
  if (T < 0 || B < 0 || H < 0 || D < 0 || max_pages < 0 || num_pages < 0) return OT_EINVAL;
  if (!kv8_ok(T, B, H, D, max_pages, num_pages) || !kv8_pages_fit(T, B, H)) return OT_ESHAPE;
  if (T == 0 || B == 0) return OT_OK;
  if (!kv8_ld_ok(ldk, H * D) || !kv8_ld_ok(ldv, H * D)) return OT_EINVAL;
  if (!k || !v || !cu || !kv_len || !table || !Kc || !Vc || !Ks || !Vs) return OT_EINVAL;
  if (!aligned16(k) || !aligned16(v) || !aligned16(Kc) || !aligned16(Vc) || !aligned4(cu) ||
      !aligned4(kv_len) || !aligned4(table) || !aligned4(Ks) || !aligned4(Vs))
    return OT_EINVAL;
  const ot::Kv8Cache cache{Kc, Vc, Ks, Vs, table, max_pages, num_pages};
  return hip_status(ot::launch_kv8_append(k, ldk, v, ldv, T, B, H, D, cu, kv_len, cache,
                                          static_cast<hipStream_t>(stream)));
}

ot_status ot_kv8_read(const uint8_t *Kc, const uint8_t *Vc, const float *Ks, const float *Vs,
                      int64_t num_pages, const int32_t *cu, const int32_t *start,
                      const int32_t *table, int64_t max_pages, int64_t T, int64_t B, int64_t H,
                      int64_t D, uint16_t *k, uint16_t *v, void *stream) {
  if (T < 0 || B < 0 || H < 0 || D < 0 || max_pages < 0 || num_pages < 0) return OT_EINVAL;
  if (!kv8_ok(T, B, H, D, max_pages, num_pages) || !kv8_pages_fit(T, B, H)) return OT_ESHAPE;
  if (T == 0 || B == 0) return OT_OK;
  if (!k || !v || !cu || !start || !table || !Kc || !Vc || !Ks || !Vs) return OT_EINVAL;
  if (!aligned16(k) || !aligned16(v) || !aligned16(Kc) || !aligned16(Vc) || !aligned4(cu) ||
      !aligned4(start) || !aligned4(table) || !aligned4(Ks) || !aligned4(Vs))
    return OT_EINVAL;
  const ot::Kv8Cache cache{const_cast<uint8_t *>(Kc), const_cast<uint8_t *>(Vc),
                           const_cast<float *>(Ks), const_cast<float *>(Vs), table, max_pages,
                           num_pages};
  return hip_status(ot::launch_kv8_read(cache, H, D, cu, start, T, B, k, v,
                                        static_cast<hipStream_t>(stream)));
}

static bool attn_kv8_ok(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D, int64_t max_pages,
                        int64_t num_pages) {
  return kv8_ok(T, B, Hkv, D, max_pages, num_pages) && Hq >= Hkv && Hq <= kMaxKv8Queries &&
         Hq % Hkv == 0 && ot::attn_kv8_fits(T, B, Hq, Hkv);
}

ot_status ot_attn_kv8(const uint16_t *q, int64_t ldq, int64_t T, int64_t B, int64_t Hq, int64_t Hkv,
                      int64_t D, const int32_t *cu, const int32_t *kv_len, const int32_t *table,
                      int64_t max_pages, int64_t num_pages, const uint8_t *Kc, const uint8_t *Vc,
                      const float *Ks, const float *Vs, float scale, int causal, int64_t window,
                      int64_t max_q, uint16_t *Y, float *lse, void *workspace, void *stream) {
  if (T < 0 || B < 0 || Hq < 0 || Hkv < 0 || D < 0 || max_pages < 0 || num_pages < 0)
    return OT_EINVAL;
  if (!isfinite(scale) || window < 0 || (window > 0 && !causal)) return OT_EINVAL;
  if (!attn_kv8_ok(T, B, Hq, Hkv, D, max_pages, num_pages)) return OT_ESHAPE;
  if (T == 0 || B == 0) return OT_OK;
  if (max_q < 1 || max_q > T || !kv8_ld_ok(ldq, Hq * D)) return OT_EINVAL;
  if (!q || !cu || !kv_len || !table || !Kc || !Vc || !Ks || !Vs || !Y) return OT_EINVAL;
  if (!aligned16(q) || !aligned16(Kc) || !aligned16(Vc) || !aligned16(Y) || !aligned16(workspace) ||
      !aligned4(cu) || !aligned4(kv_len) || !aligned4(table) || !aligned4(Ks) || !aligned4(Vs) ||
      !aligned4(lse))
    return OT_EINVAL;
  ot::Kv8Attn a{};
  a.q = q;
  a.ldq = ldq;
  a.T = (int)T;
  a.B = (int)B;
  a.Hq = (int)Hq;
  a.Hkv = (int)Hkv;
  a.D = (int)D;
  a.max_q = (int)max_q;
  a.cu = cu;
  a.kv_len = kv_len;
  a.cache = ot::Kv8Cache{const_cast<uint8_t *>(Kc), const_cast<uint8_t *>(Vc),
                         const_cast<float *>(Ks), const_cast<float *>(Vs), table, max_pages,
                         num_pages};
  a.scale = scale;
  a.causal = causal != 0;
  a.window = window < kMaxRows ? window : kMaxRows;  // past every position
  a.Y = Y;
  a.lse = lse;
  return hip_status(ot::launch_attn_kv8(a, workspace, static_cast<hipStream_t>(stream)));
}

size_t ot_attn_kv8_workspace_size(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D,
                                  int64_t max_q) {
  if (T <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || max_q < 1 || max_q > T ||
      !attn_kv8_ok(T, B, Hq, Hkv, D, 1, 1))
    return 0;
  return ot::attn_kv8_workspace_bytes(T, B, Hq, Hkv, D, max_q);
}

ot_status ot_attn_kv8_plan(int64_t T, int64_t B, int64_t Hq, int64_t Hkv, int64_t D, int64_t max_q,
                           int with_workspace, char *buf, size_t len) {
  if (!buf || len == 0 || T < 0 || B < 0 || Hq < 0 || Hkv < 0 || D < 0) return OT_EINVAL;
  if (!attn_kv8_ok(T, B, Hq, Hkv, D, 1, 1)) return OT_ESHAPE;
  if (T == 0 || B == 0) {
    snprintf(buf, len, "none");
    return OT_OK;
  }
  if (max_q < 1 || max_q > T) return OT_EINVAL;
  ot::describe_attn_kv8(T, B, Hq, Hkv, D, max_q, with_workspace != 0, buf, len);
  return OT_OK;
}

}  // extern "C"
