// Entry points of the dense layers: checks of arguments, workspace, and which kernels a call takes.
#include "dense.h"

using namespace spcfg;

namespace {

constexpr int64_t kMaxDim = 1 << 24, kMaxElems = (int64_t)1 << 36;

int check(const spcfg_dense_config* c) {
  if (!c || c->struct_size != sizeof(spcfg_dense_config)) return SPCFG_ERR_ARG;
  if (c->rows < 0 || c->in < 1 || c->out < 1 || c->rows > kMaxDim || c->in > kMaxDim || c->out > kMaxDim) return SPCFG_ERR_SHAPE;
  const int64_t R = c->rows, I = c->in, O = c->out;
  if (R * I > kMaxElems || R * O > kMaxElems || I * O > kMaxElems) return SPCFG_ERR_SHAPE;
  const bool f32 = c->in_type == SPCFG_TYPE_F32 && c->out_type == SPCFG_TYPE_F32;
  const bool b16 = c->in_type == SPCFG_TYPE_BF16 && (c->out_type == SPCFG_TYPE_F32 || c->out_type == SPCFG_TYPE_BF16);
  if (!f32 && !b16) return SPCFG_ERR_UNSUPPORTED;
  if (c->activation < SPCFG_ACT_NONE || c->activation > SPCFG_ACT_SILU) return SPCFG_ERR_UNSUPPORTED;
  if (c->flags & ~(uint32_t)SPCFG_FLAG_ACCUMULATE_GRADS) return SPCFG_ERR_UNSUPPORTED;
  return SPCFG_OK;
}

size_t need(const spcfg_dense_config* c) {
  return c->rows == 0 ? 0 : dense::tiled_workspace(c->rows, c->in, c->out, c->in_type, c->out_type, c->activation);
}

int check_workspace(size_t n, const void* ws, size_t bytes) {
  if (n == 0) return SPCFG_OK;
  if (!ws) return SPCFG_ERR_ARG;
  return ((uintptr_t)ws & 255) != 0 || bytes < n ? SPCFG_ERR_WORKSPACE : SPCFG_OK;
}

bool on_type(const void* p, int type) { return ((uintptr_t)p & (type == SPCFG_TYPE_F32 ? 3 : 1)) == 0; }

int64_t size_of(int type) { return type == SPCFG_TYPE_F32 ? 4 : 2; }

dense::Args args_of(const spcfg_dense_config* c) {
  dense::Args a{};
  a.R = c->rows;
  a.I = c->in;
  a.O = c->out;
  a.act = c->activation;
  a.accumulate = (c->flags & SPCFG_FLAG_ACCUMULATE_GRADS) != 0;
  return a;
}

}  // namespace

extern "C" {

int spcfg_dense_workspace_bytes(const spcfg_dense_config* cfg, size_t* out_bytes) {
  const int rc = check(cfg);
  if (rc) return rc;
  if (!out_bytes) return SPCFG_ERR_ARG;
  *out_bytes = need(cfg);
  return SPCFG_OK;
}

int spcfg_dense_forward(const spcfg_dense_config* cfg, const void* x, const void* W, const void* bias, const void* residual,
                        void* y, void* preact, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check(cfg);
  if (rc) return rc;
  if (cfg->rows == 0) return SPCFG_OK;
  if (!x || !W || !y) return SPCFG_ERR_ARG;
  const int ti = cfg->in_type, to = cfg->out_type;
  if (!on_type(x, ti) || !on_type(W, ti) || !on_type(bias, ti) || !on_type(residual, to) || !on_type(y, to) || !on_type(preact, to))
    return SPCFG_ERR_ARG;
  dense::Args a = args_of(cfg);
  const int64_t si = size_of(ti), nx = a.R * a.I * si, nw = a.O * a.I * si, ny = a.R * a.O * size_of(to);
  const size_t n = need(cfg);
  const Memory all[] = {{y, ny}, {preact, ny}, {workspace, (int64_t)n}, {x, nx}, {W, nw}, {bias, a.O * si}, {residual, ny}};
  if (clash(all, 3, 7, 0, 6)) return SPCFG_ERR_ARG;
  if ((rc = check_workspace(n, workspace, workspace_bytes))) return rc;
  a.x = x; a.W = W; a.bias = bias; a.residual = residual; a.y = y; a.preact = preact;
  if (!dense::tiled_forward(a, ti, to, workspace, (hipStream_t)hip_stream))
    dense::launch_direct_forward(a, ti, to, (hipStream_t)hip_stream);
  return launch_status();
}

int spcfg_dense_backward(const spcfg_dense_config* cfg, const void* x, const void* W, const void* preact, const void* grad_y,
                         const void* grad_x_add, void* grad_x, void* grad_W, void* grad_bias, void* workspace,
                         size_t workspace_bytes, void* hip_stream) {
  int rc = check(cfg);
  if (rc) return rc;
  const bool act = cfg->activation != SPCFG_ACT_NONE;
  if (cfg->rows > 0 && !grad_x && !grad_W && !grad_bias) return SPCFG_ERR_ARG;  // (an empty grad_x has no address)
  if (grad_bias && !grad_W) return SPCFG_ERR_ARG;
  if (cfg->rows > 0 && (!x || !W || !grad_y || (act && !preact) || (grad_x_add && !grad_x))) return SPCFG_ERR_ARG;
  const int ti = cfg->in_type, to = cfg->out_type;
  if (!on_type(x, ti) || !on_type(W, ti) || !on_type(preact, to) || !on_type(grad_y, to) || !on_type(grad_x_add, ti) ||
      !on_type(grad_x, ti) || !on_type(grad_W, ti) || !on_type(grad_bias, ti))
    return SPCFG_ERR_ARG;
  dense::Args a = args_of(cfg);
  const int64_t si = size_of(ti), nx = a.R * a.I * si, nw = a.O * a.I * si, ny = a.R * a.O * size_of(to);
  const size_t n = need(cfg);
  const Memory all[] = {{grad_x, nx}, {grad_W, nw}, {grad_bias, a.O * si}, {workspace, (int64_t)n}, {x, nx}, {W, nw}, {preact, ny},
                        {grad_y, ny}, {grad_x_add, nx}};
  if (clash(all, 4, 9, 0, 8)) return SPCFG_ERR_ARG;
  if ((rc = check_workspace(n, workspace, workspace_bytes))) return rc;
  if (cfg->rows == 0 && !grad_W) return SPCFG_OK;
  a.x = x; a.W = W; a.preact_in = act ? preact : nullptr; a.grad_y = grad_y; a.grad_x_add = grad_x_add;
  a.grad_x = cfg->rows > 0 ? grad_x : nullptr; a.grad_W = grad_W; a.grad_bias = grad_bias;
  if (cfg->rows == 0 || !dense::tiled_backward(a, ti, to, workspace, (hipStream_t)hip_stream))
    dense::launch_direct_backward(a, ti, to, (hipStream_t)hip_stream);
  return launch_status();
}

}  // extern "C"
