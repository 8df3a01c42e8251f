// C entry points of rotary positions: frequencies, argument checks and dispatch.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "rope.h"

namespace rs {

static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

rs_status check_rope(const rs_rope *r, int d) {
  if (!r) return fail(RS_ERR_INVALID_ARG, "rope is NULL");
  if (r->dim < 2 || r->dim % 2 != 0 || r->dim > d) return fail(RS_ERR_INVALID_ARG, "rope: dim must be even, from 2 to the head dim");
  if (r->layout != RS_ROPE_HALF && r->layout != RS_ROPE_INTERLEAVED) return fail(RS_ERR_INVALID_ARG, "rope: unknown layout");
  if (!std::isfinite(r->mscale)) return fail(RS_ERR_INVALID_ARG, "rope: mscale must be finite");
  for (int i = 0; i < r->dim / 2; ++i)
    if (!std::isfinite(r->turns[i])) return fail(RS_ERR_INVALID_ARG, "rope: turns must be finite");
  return RS_OK;
}

rs_status check_rope_part(const rs_rope_part *p, int dtype, int d, int n, const char *what) {
  const std::string name(what);
  if (!p->x || !p->y || !aligned16(p->x) || !aligned16(p->y))
    return fail(RS_ERR_INVALID_ARG, name + ": x and y must be 16-byte aligned device pointers");
  if (p->heads < 1 || p->heads > 65535) return fail(RS_ERR_INVALID_ARG, name + ": need 1 <= heads <= 65535");
  const int vec = dtype == RS_BF16 ? 8 : 4;
  const int64_t s[4] = {p->sx_t, p->sx_h, p->sy_t, p->sy_h};
  for (int i = 0; i < 4; ++i)
    if (s[i] < 0 || s[i] % vec != 0) return fail(RS_ERR_INVALID_ARG, name + ": strides must be non-negative multiples of 16 bytes");
  // heads within tokens, or tokens within heads
  const int64_t token = (p->heads - 1) * p->sy_h + d, head = (int64_t)(n - 1) * p->sy_t + d;
  if ((n > 1 && p->sy_t < d) || (p->heads > 1 && p->sy_h < d) || (n > 1 && p->heads > 1 && p->sy_t < token && p->sy_h < head))
    return fail(RS_ERR_INVALID_ARG, name + ": rows of y overlap");
  if (p->x == p->y && (p->sx_t != p->sy_t || p->sx_h != p->sy_h))
    return fail(RS_ERR_INVALID_ARG, name + ": in place x and y have the same strides");
  return RS_OK;
}

}  // namespace rs

using namespace rs;

extern "C" {

rs_status rs_rope_init(const rs_rope_cfg *cfg, rs_rope *rope) {
  set_error("");
  if (!cfg || !rope) return fail(RS_ERR_INVALID_ARG, "rope: cfg or rope is NULL");
  const rs_rope_cfg &c = *cfg;
  const bool ramp = c.scaling == RS_ROPE_TURNS || c.scaling == RS_ROPE_PAIRS;
  if (c.dim < 2 || c.dim > 128 || c.dim % 2 != 0) return fail(RS_ERR_INVALID_ARG, "rope: dim must be even, from 2 to 128");
  if (c.layout != RS_ROPE_HALF && c.layout != RS_ROPE_INTERLEAVED) return fail(RS_ERR_INVALID_ARG, "rope: unknown layout");
  if (c.scaling < RS_ROPE_PLAIN || c.scaling > RS_ROPE_PAIRS) return fail(RS_ERR_INVALID_ARG, "rope: unknown scaling");
  if (!(c.base > 1.0) || !std::isfinite(c.base)) return fail(RS_ERR_INVALID_ARG, "rope: base must be finite and above 1");
  if (c.scaling != RS_ROPE_PLAIN && (!(c.factor >= 1.0) || !std::isfinite(c.factor)))
    return fail(RS_ERR_INVALID_ARG, "rope: factor must be finite and at least 1");
  if (ramp && (!(c.context > 0.0) || !std::isfinite(c.context) || !(c.low > 0.0) || !(c.high > c.low) || !std::isfinite(c.high)))
    return fail(RS_ERR_INVALID_ARG, "rope: ramps need context > 0 and 0 < low < high");
  if (!std::isfinite((float)c.mscale)) return fail(RS_ERR_INVALID_ARG, "rope: mscale must be finite");
  const double two_pi = 6.283185307179586476925;
  const int half = c.dim / 2;
  const auto pair_of = [&](double turns) { return half * std::log(c.context / (two_pi * turns)) / std::log(c.base); };
  double first = 0.0, width = 1.0;
  if (c.scaling == RS_ROPE_PAIRS) {
    first = std::fmax(std::floor(pair_of(c.high)), 0.0);
    width = std::fmax(std::fmin(std::ceil(pair_of(c.low)), c.dim - 1.0) - first, 0.001);
  }
  *rope = rs_rope{};
  rope->dim = c.dim;
  rope->layout = c.layout;
  rope->mscale = c.mscale == 0.0 ? 1.f : (float)c.mscale;
  for (int i = 0; i < half; ++i) {
    const double g = std::pow(c.base, -2.0 * i / c.dim);
    double keep = 1.0;
    if (c.scaling == RS_ROPE_LINEAR) keep = 0.0;
    if (c.scaling == RS_ROPE_TURNS) keep = std::fmin(std::fmax((c.context * g / two_pi - c.low) / (c.high - c.low), 0.0), 1.0);
    if (c.scaling == RS_ROPE_PAIRS) keep = 1.0 - std::fmin(std::fmax((i - first) / width, 0.0), 1.0);
    rope->turns[i] = (keep == 1.0 ? g : g * (keep + (1.0 - keep) / c.factor)) / two_pi;
  }
  return RS_OK;
}

rs_status rs_rope_apply(const rs_rope *rope, const rs_rope_rows *rows, int32_t transpose, rs_stream stream) {
  set_error("");
  if (!rows) return fail(RS_ERR_INVALID_ARG, "rope: rows is NULL");
  if (rows->dtype != RS_BF16 && rows->dtype != RS_F32) return fail(RS_ERR_INVALID_ARG, "rope: unknown dtype");
  if (rows->d != 64 && rows->d != 128) return fail(RS_ERR_UNSUPPORTED, "rope: head dim must be 64 or 128");
  if (rows->n < 0) return fail(RS_ERR_INVALID_ARG, "rope: n < 0");
  if (rows->n > 1 << 24) return fail(RS_ERR_UNSUPPORTED, "rope: at most 16777216 rows");
  if (rows->nparts < 1 || rows->nparts > 4) return fail(RS_ERR_INVALID_ARG, "rope: need 1 to 4 parts");
  if (rows->pos0 < -(1ll << 31) || rows->pos0 > 1ll << 31) return fail(RS_ERR_INVALID_ARG, "rope: pos0 beyond 2^31");
  rs_status st;
  if ((st = check_rope(rope, rows->d)) != RS_OK) return st;
  if (rows->n == 0) return RS_OK;
  for (int k = 0; k < rows->nparts; ++k)
    if ((st = check_rope_part(&rows->part[k], rows->dtype, rows->d, rows->n, "rope")) != RS_OK) return st;
  return rope_launch(*rope, *rows, transpose != 0, (hipStream_t)stream);
}

}  // extern "C"
