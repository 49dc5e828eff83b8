// The dense layer of include/dl.h: arguments and entry points (dl_calls.h: kernels and launches).
#include <initializer_list>
#include <string>

#include "dl_plan.h"

namespace dl {
namespace {

using sc::DeviceGuard;
using sc::misaligned;
using sc::set_error;

sc_status check_config(const char* fn, const dl_config* cfg, int64_t n) {
  auto bad = [&](sc_status st, const char* what) { return set_error(st, std::string(fn) + ": " + what); };
  if (!cfg) return bad(SC_ERR_INVALID_ARG, "cfg is NULL");
  if (cfg->struct_size != static_cast<int32_t>(sizeof(dl_config)))
    return bad(SC_ERR_INVALID_ARG, "struct_size does not match this library's dl_config");
  if (cfg->k_in < 1 || cfg->k_out < 1) return bad(SC_ERR_INVALID_ARG, "k_in or k_out < 1");
  if (cfg->k_in > DL_MAX_WIDTH || cfg->k_out > DL_MAX_WIDTH) return bad(SC_ERR_UNSUPPORTED, "k_in or k_out above DL_MAX_WIDTH");
  if (cfg->activation < DL_NONE || cfg->activation > DL_GELU) return bad(SC_ERR_INVALID_ARG, "bad activation");
  if (cfg->dtype != SC_F32 && cfg->dtype != SC_F64 && cfg->dtype != SC_BF16) return bad(SC_ERR_INVALID_ARG, "bad dtype");
  if (cfg->ld_in != 0 && cfg->ld_in < cfg->k_in) return bad(SC_ERR_INVALID_ARG, "ld_in below k_in");
  if (cfg->ld_out != 0 && cfg->ld_out < cfg->k_out) return bad(SC_ERR_INVALID_ARG, "ld_out below k_out");
  if (cfg->ld_in > DL_MAX_STRIDE || cfg->ld_out > DL_MAX_STRIDE) return bad(SC_ERR_UNSUPPORTED, "ld_in or ld_out above DL_MAX_STRIDE");
  if (n < 0 || n > (int64_t(1) << 30)) return bad(SC_ERR_INVALID_ARG, "n_rows outside 0..2^30");
  return SC_OK;
}

Entries entries_of(const dl_config* c) { return c->dtype == SC_F64 ? entries_f64() : c->dtype == SC_BF16 ? entries_bf16() : entries_f32(); }

sc_status check_tensors(const char* fn, std::initializer_list<const void*> needed, std::initializer_list<const void*> optional) {
  for (const void* p : needed)
    if (!p) return set_error(SC_ERR_INVALID_ARG, std::string(fn) + ": NULL tensor argument");
  for (auto list : {needed, optional})
    for (const void* p : list)
      if (misaligned(p, 16)) return set_error(SC_ERR_INVALID_ARG, std::string(fn) + ": tensor pointer not 16-byte aligned");
  return SC_OK;
}

sc_status check_workspace(const char* fn, const dl_config* cfg, int64_t n, const void* workspace, size_t given) {
  if (!workspace || given < workspace_bytes(cfg, n))
    return set_error(SC_ERR_WORKSPACE, std::string(fn) + ": workspace missing or smaller than dl_workspace_bytes()");
  if (misaligned(workspace, 256)) return set_error(SC_ERR_WORKSPACE, std::string(fn) + ": workspace not 256-byte aligned");
  return SC_OK;
}

sc_status launched(const char* fn, hipError_t e) {
  return e == hipSuccess ? SC_OK : set_error(SC_ERR_HIP, std::string(fn) + ": kernel launch: " + hipGetErrorString(e));
}

}  // namespace
}  // namespace dl

extern "C" {

sc_status dl_forward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* b, const void* residual, void* Y,
                     void* Z, void* hip_stream) {
  using namespace dl;
  sc_status st = check_config("dl_forward", cfg, n_rows);
  if (st != SC_OK || n_rows == 0) return st;
  st = check_tensors("dl_forward", {X, W, Y}, {b, residual, Z});
  if (st != SC_OK) return st;
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "dl_forward: cannot make cfg->device current");
  return launched("dl_forward", entries_of(cfg).forward(cfg, n_rows, static_cast<hipStream_t>(hip_stream), X, W, b, residual, Y, Z));
}

sc_status dl_workspace_bytes(const dl_config* cfg, int64_t n_rows, size_t* bytes) {
  using namespace dl;
  const sc_status st = check_config("dl_workspace_bytes", cfg, n_rows);
  if (st != SC_OK) return st;
  if (!bytes) return set_error(SC_ERR_INVALID_ARG, "dl_workspace_bytes: bytes is NULL");
  *bytes = workspace_bytes(cfg, n_rows);
  return SC_OK;
}

sc_status dl_backward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* Z, const void* dY, void* dX, void* dW,
                      void* db, void* workspace, size_t workspace_bytes_given, void* hip_stream) {
  using namespace dl;
  sc_status st = check_config("dl_backward", cfg, n_rows);
  if (st != SC_OK) return st;
  if (!dX && !dW && !db) return set_error(SC_ERR_INVALID_ARG, "dl_backward: dX, dW and db are all NULL");
  st = check_tensors("dl_backward", {}, {X, W, Z, dY, dX, dW, db});
  if (st != SC_OK) return st;
  if (n_rows > 0) {
    st = check_tensors("dl_backward", {X, W, dY}, {});
    if (st == SC_OK && cfg->activation != DL_NONE) st = check_tensors("dl_backward", {Z}, {});
    if (st == SC_OK) st = check_workspace("dl_backward", cfg, n_rows, workspace, workspace_bytes_given);
    if (st != SC_OK) return st;
  }
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "dl_backward: cannot make cfg->device current");
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const Entries calls = entries_of(cfg);
  return launched("dl_backward", n_rows == 0 ? calls.zero(cfg, stream, dW, db) : calls.backward(cfg, n_rows, stream, X, W, Z, dY, dX, dW, db, workspace));
}

sc_status dl_double_backward(const dl_config* cfg, int64_t n_rows, const void* X, const void* W, const void* Z, const void* dY,
                             const void* HX, void* ddY, void* X2, void* W2, void* b2, void* workspace, size_t workspace_bytes_given,
                             void* hip_stream) {
  using namespace dl;
  sc_status st = check_config("dl_double_backward", cfg, n_rows);
  if (st != SC_OK) return st;
  st = check_tensors("dl_double_backward", {}, {X, W, Z, dY, HX, ddY, X2, W2, b2});
  if (st != SC_OK) return st;
  if (n_rows > 0) {
    st = check_tensors("dl_double_backward", {X, W, dY, HX, ddY}, {});
    if (st == SC_OK && cfg->activation != DL_NONE) st = check_tensors("dl_double_backward", {Z}, {});
    if (st == SC_OK) st = check_workspace("dl_double_backward", cfg, n_rows, workspace, workspace_bytes_given);
    if (st != SC_OK) return st;
  }
  DeviceGuard guard(cfg->device);
  if (!guard.ok) return set_error(SC_ERR_HIP, "dl_double_backward: cannot make cfg->device current");
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const Entries calls = entries_of(cfg);
  return launched("dl_double_backward", n_rows == 0 ? calls.zero(cfg, stream, W2, b2)
                                                     : calls.double_backward(cfg, n_rows, stream, X, W, Z, dY, HX, ddY, X2, W2, b2, workspace));
}

}  // extern "C"
