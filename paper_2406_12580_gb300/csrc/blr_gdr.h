// Problem checks shared by the entry points of the gated delta rule.
#pragma once

#include <math.h>

#include "blr_host.h"

namespace blr {

struct GdrSizes {
  int64_t B, L, Hk, Hv, Dk, Dv;
  int64_t ldq, ldk, ldv;  // elements between steps, filled in
  bool empty;             // nothing to do but states
};

inline blr_status gdr_check(const blr_gdr_desc* d, GdrSizes* s) {
  if (d == nullptr) return fail(BLR_ERR_INVALID_ARG, "desc is NULL");
  if (d->B < 0 || d->L < 0 || d->Hk < 0 || d->Hv < 0)
    return fail(BLR_ERR_INVALID_ARG, "negative size B=%lld L=%lld Hk=%lld Hv=%lld", (long long)d->B,
                (long long)d->L, (long long)d->Hk, (long long)d->Hv);
  if (d->io != BLR_F32 && d->io != BLR_BF16)
    return fail(BLR_ERR_INVALID_ARG, "unknown io dtype %d", (int)d->io);
  if (!isfinite(d->scale)) return fail(BLR_ERR_INVALID_ARG, "scale must be finite");
  if (d->Dk != 64 && d->Dk != 128)
    return fail(BLR_ERR_UNSUPPORTED, "Dk=%lld is neither 64 nor 128", (long long)d->Dk);
  if (d->Dv < 64 || d->Dv > 256 || d->Dv % 64 != 0)
    return fail(BLR_ERR_UNSUPPORTED, "Dv=%lld is not 64, 128, 192 or 256", (long long)d->Dv);
  s->empty = d->B == 0 || d->Hv == 0;
  if (!s->empty && (d->Hk == 0 || d->Hv % d->Hk != 0))
    return fail(BLR_ERR_INVALID_ARG, "Hv=%lld is not a multiple of Hk=%lld", (long long)d->Hv,
                (long long)d->Hk);
  if (d->B >= ((int64_t)1 << 31) || d->L >= ((int64_t)1 << 30) || d->Hv >= ((int64_t)1 << 16) ||
      (double)d->B * (double)d->L * (double)d->Hv * 256.0 > 1e17)
    return fail(BLR_ERR_UNSUPPORTED, "problem too large");
  s->B = d->B;
  s->L = d->L;
  s->Hk = d->Hk;
  s->Hv = d->Hv;
  s->Dk = d->Dk;
  s->Dv = d->Dv;
  const int64_t given[3] = {d->ldq, d->ldk, d->ldv};
  const int64_t least[3] = {d->Hk * d->Dk, d->Hk * d->Dk, d->Hv * d->Dv};
  int64_t* out[3] = {&s->ldq, &s->ldk, &s->ldv};
  for (int i = 0; i < 3; ++i) {
    if (given[i] != 0 && (given[i] < least[i] || given[i] % 8 != 0 || given[i] > ((int64_t)1 << 31)))
      return fail(BLR_ERR_INVALID_ARG, "ld%c=%lld: at least %lld and a multiple of 8 is wanted", "qkv"[i],
                  (long long)given[i], (long long)least[i]);
    *out[i] = given[i] != 0 ? given[i] : least[i];
  }
  return BLR_OK;
}

}  // namespace blr
