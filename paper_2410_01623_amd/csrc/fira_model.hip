// Host side of the operators that complete a training step (include/fira.h): checks of the arguments and launches.  gfx950 only; no
// state, no allocation, nothing that throws.
#include "fira_host.h"
#include "fira_adamw.h"

namespace {

fira_status check_adamw(const fira_adamw_desc* d, int i) {
  if (d->rows < 0 || d->cols < 0 || d->rows > kMost) return refuse(FIRA_ERR_SHAPE, "tensor %d of %lld x %lld", i, (long long)d->rows, (long long)d->cols);
  if (!known(d->dtype) || !known(d->grad_dtype)) return refuse(FIRA_ERR_DTYPE, "types of tensor %d", i);
  if (d->state_type != FIRA_STATE_F32 && d->state_type != FIRA_STATE_E4M3) return refuse(FIRA_ERR_DTYPE, "state type of tensor %d", i);
  if (!(d->weight_decay >= 0.0) || !std::isfinite((float)d->weight_decay)) return refuse(FIRA_ERR_INVALID_ARG, "weight decay of tensor %d", i);
  FIRA_LEADING(d->ld_w, d->cols, d->rows);
  FIRA_LEADING(d->ld_g, d->cols, d->rows);
  if (d->rows > 1 && (d->ld_w != d->cols || d->ld_g != d->cols) && d->cols > kMost) return refuse(FIRA_ERR_SHAPE, "tensor %d has rows apart of %lld", i, (long long)d->cols);
  return FIRA_OK;
}

fira_status check_adamw_hparams(const fira_adamw_hparams* hp, bool norm) {
  if (!hp) return refuse(FIRA_ERR_INVALID_ARG, "null hyper-parameters");
  if (!std::isfinite((float)hp->lr)) return refuse(FIRA_ERR_INVALID_ARG, "lr is not finite");
  // (1 - beta has to be there in fp32, as beta itself)
  if (!(hp->beta1 >= 0.0 && hp->beta2 >= 0.0) || !((float)hp->beta1 < 1.0f && (float)hp->beta2 < 1.0f)) return refuse(FIRA_ERR_INVALID_ARG, "a beta is not in [0, 1)");
  if (!((float)hp->eps > 0.0f) || !std::isfinite((float)hp->eps)) return refuse(FIRA_ERR_INVALID_ARG, "eps is not positive and finite");
  if (norm && !(hp->max_norm >= 0.0)) return refuse(FIRA_ERR_INVALID_ARG, "max_norm is negative or not a number");
  return FIRA_OK;
}

}  // namespace

extern "C" {

int64_t fira_adamw_scales(const fira_adamw_desc* d) {
  if (!d || check_adamw(d, 0) || d->state_type != FIRA_STATE_E4M3) return 0;
  return (d->rows * d->cols + kAdamBlock - 1) / kAdamBlock;
}

fira_status fira_adamw_step(const fira_adamw_desc* d, int count, const fira_adamw_hparams* hp, void* const* dev_W, const void* const* dev_G,
                            const fira_adamw_state* dev_state, int64_t* dev_t, const float* dev_lr, const float* dev_norm, void* hip_stream) {
  if (count < 0 || (count && (!d || !dev_W || !dev_G || !dev_state))) return refuse(FIRA_ERR_INVALID_ARG, "%d tensors, or a null list", count);
  if (const fira_status st = check_adamw_hparams(hp, dev_norm != nullptr)) return st;
  FIRA_POINTER(dev_t, 8);
  if (!aligned(dev_lr, 4) || !aligned(dev_norm, 4)) return refuse(FIRA_ERR_INVALID_ARG, "dev_lr or dev_norm is not aligned to its elements");
  for (int i = 0; i < count; ++i) {
    if (const fira_status st = check_adamw(d + i, i)) return st;
    if (!d[i].rows || !d[i].cols) continue;
    const fira_adamw_state& s = dev_state[i];
    const bool eight = d[i].state_type == FIRA_STATE_E4M3;
    if (!dev_W[i] || !dev_G[i] || !s.m || !s.v || (eight && (!s.m_scale || !s.v_scale))) return refuse(FIRA_ERR_INVALID_ARG, "tensor %d has a null pointer", i);
    if (!aligned(dev_W[i], size_of(d[i].dtype)) || !aligned(dev_G[i], size_of(d[i].grad_dtype)) ||
        (eight ? !aligned(s.m_scale, 4) || !aligned(s.v_scale, 4) : !aligned(s.m, 4) || !aligned(s.v, 4)))
      return refuse(FIRA_ERR_INVALID_ARG, "tensor %d is not aligned to its elements", i);
    if (dev_W[i] == dev_G[i] || s.m == s.v) return refuse(FIRA_ERR_INVALID_ARG, "tensor %d overlaps its gradient or its states each other", i);
  }
  const hipStream_t q = (hipStream_t)hip_stream;
  const FiraAdamHp h{hp->lr, std::log(hp->beta1), std::log(hp->beta2), hp->max_norm, (float)hp->beta1, (float)hp->beta2, (float)(1.0 - hp->beta1), (float)(1.0 - hp->beta2),
                     (float)hp->eps};
  for (int i = 0; i < count; ++i) {
    const int64_t n = d[i].rows * d[i].cols;
    if (!n) continue;
    const fira_adamw_state& s = dev_state[i];
    const FiraAdamTensor a{dev_W[i], dev_G[i], s.m, s.v, s.m_scale, s.v_scale, n, d[i].cols, d[i].ld_w, d[i].ld_g, d[i].weight_decay, d[i].seed};
    with_types(d[i].dtype, d[i].grad_dtype, [&](auto t, auto r) {
      with_flag(d[i].state_type == FIRA_STATE_E4M3, [&](auto eight) {
        hipLaunchKernelGGL((fira_adamw_kernel<decltype(t), decltype(r), decltype(eight)::value>), dim3(std::min<int64_t>((n + kAdamBlock - 1) / kAdamBlock, 1 << 20)),
                           dim3(kAdamBlock), 0, q, a, h, dev_lr, dev_norm, (const long long*)dev_t);
      });
    });
  }
  hipLaunchKernelGGL(fira_adamw_count_kernel<>, dim3(1), dim3(1), 0, q, (long long*)dev_t);
  return launched("AdamW step");
}

}  // extern "C"
