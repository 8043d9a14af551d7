// Host layer of the operators on packed rows: argument validation and launches behind crisp_rope_init, crisp_rope and
// crisp_packed_attn of include/crisp.h.
#include "host_checks.h"
#include "packed_internal.h"

namespace crisp {

namespace {

constexpr int64_t kMaxKeyStride = (int64_t)1 << 23;  // elements: a tile of 64 keys stays within 32-bit byte offsets
constexpr int64_t kMaxBlocks = (int64_t)1 << 23;     // workgroups of 256 threads: a launch has fewer than 2^32

crisp_status check_packed(const crisp_packed_shape* s, PackedDims* d) {
  if (!s) return fail(CRISP_EINVAL, "packed shape is null");
  if (s->n_seqs < 0 || s->n_rows < 0 || s->n_q_heads < 0 || s->n_kv_heads < 0)
    return fail(CRISP_EINVAL, "bad packed shape: n_seqs=%d n_rows=%d n_q_heads=%d n_kv_heads=%d", s->n_seqs, s->n_rows,
                s->n_q_heads, s->n_kv_heads);
  if (s->head_dim != kHeadDim) return fail(CRISP_EUNSUPPORTED, "head_dim %d unsupported (only 128)", s->head_dim);
  if (s->n_rows > kMaxRows) return fail(CRISP_EUNSUPPORTED, "n_rows %d above the supported %d", s->n_rows, kMaxRows);
  if (s->n_seqs > kMaxSeqs) return fail(CRISP_EUNSUPPORTED, "n_seqs %d above the supported %d", s->n_seqs, kMaxSeqs);
  if (s->n_q_heads > 65535 || s->n_kv_heads > 65535)
    return fail(CRISP_EUNSUPPORTED, "n_q_heads %d or n_kv_heads %d above the supported 65535", s->n_q_heads, s->n_kv_heads);
  *d = PackedDims{s->n_seqs, s->n_rows, s->n_q_heads, s->n_kv_heads};
  return CRISP_OK;
}

crisp_status check_rotation(int rotary_dim, int layout) {
  if (rotary_dim < 16 || rotary_dim > kHeadDim || rotary_dim % 16)
    return fail(CRISP_EUNSUPPORTED, "rotary_dim %d unsupported (a multiple of 16 in [16, 128])", rotary_dim);
  if (layout != CRISP_ROPE_HALF && layout != CRISP_ROPE_INTERLEAVED) return fail(CRISP_EINVAL, "rotary layout %d unknown", layout);
  return CRISP_OK;
}

crisp_status check_rotated(const RopeTensor& x, int rows, const char* name) {
  if (x.heads == 0) return CRISP_OK;
  CHECK(check_ptr(x.in, 16, name));
  CHECK(check_ptr(x.out, 16, name));
  if (x.in == x.out && ((x.heads > 1 && x.is.head != x.os.head) || (rows > 1 && x.is.row != x.os.row)))
    return fail(CRISP_EINVAL, "%s: in place its strides (%lld, %lld) and (%lld, %lld) must agree", name, (long long)x.is.head,
                (long long)x.is.row, (long long)x.os.head, (long long)x.os.row);
  return CRISP_OK;
}

}  // namespace

}  // namespace crisp

using namespace crisp;

extern "C" {

crisp_status crisp_rope_init(const crisp_rope_params* params, crisp_rope_table* table) {
  if (!params || !table) return fail(CRISP_EINVAL, "params or table is null");
  const crisp_rope_params& p = *params;
  CHECK(check_rotation(p.rotary_dim, p.layout));
  if (p.scaling < CRISP_ROPE_PLAIN || p.scaling > CRISP_ROPE_RAMP) return fail(CRISP_EINVAL, "rotary scaling %d unknown", p.scaling);
  if (!(p.base > 1.0) || !isfinite(p.base)) return fail(CRISP_EINVAL, "base %g must be finite and > 1", p.base);
  if (p.scaling != CRISP_ROPE_PLAIN && (!(p.factor >= 1.0) || !isfinite(p.factor)))
    return fail(CRISP_EINVAL, "factor %g must be finite and >= 1", p.factor);
  if (p.scaling == CRISP_ROPE_BANDS || p.scaling == CRISP_ROPE_RAMP) {
    if (!(p.original_len > 0.0) || !isfinite(p.original_len))
      return fail(CRISP_EINVAL, "original_len %g must be finite and > 0", p.original_len);
    if (!(p.low > 0.0) || !(p.high > p.low) || !isfinite(p.high))
      return fail(CRISP_EINVAL, "low %g and high %g must be finite and 0 < low < high", p.low, p.high);
  }
  const double two_pi = 6.283185307179586476925286766559, dim = p.rotary_dim;
  const double base = p.scaling == CRISP_ROPE_BASE ? p.base * pow(p.factor, dim / (dim - 2.0)) : p.base;
  if (!isfinite(base)) return fail(CRISP_EINVAL, "base %g and factor %g are too large together", p.base, p.factor);
  const auto at = [&](double turns) { return dim * log(p.original_len / (two_pi * turns)) / (2.0 * log(p.base)); };
  double from = 0.0, to = 0.0;
  if (p.scaling == CRISP_ROPE_RAMP) {
    from = fmax(floor(at(p.high)), 0.0);
    to = fmin(ceil(at(p.low)), dim - 1.0);
  }
  const auto unit = [](double x) { return fmin(fmax(x, 0.0), 1.0); };
  *table = crisp_rope_table{};
  table->rotary_dim = p.rotary_dim;
  table->layout = p.layout;
  table->gain = p.scaling == CRISP_ROPE_RAMP ? (float)(0.1 * log(p.factor) + 1.0) : 1.0f;
  for (int i = 0; i < p.rotary_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / dim);
    if (p.scaling == CRISP_ROPE_LINEAR) f /= p.factor;
    if (p.scaling == CRISP_ROPE_BANDS || p.scaling == CRISP_ROPE_RAMP) {
      const double x = p.scaling == CRISP_ROPE_BANDS ? unit((p.original_len * f / two_pi - p.low) / (p.high - p.low))
                                                     : 1.0 - unit((i - from) / fmax(to - from, 0.001));
      f *= x + (1.0 - x) / p.factor;
    }
    table->turns[i] = f / two_pi;
  }
  return CRISP_OK;
}

crisp_status crisp_rope(const crisp_packed_shape* shape, const crisp_rope_table* table, const int32_t* start,
                        const int32_t* row_ptr, const crisp_bf16* q, int64_t q_head_stride, int64_t q_row_stride,
                        const crisp_bf16* k, int64_t k_head_stride, int64_t k_row_stride, crisp_bf16* q_out,
                        int64_t q_out_head_stride, int64_t q_out_row_stride, crisp_bf16* k_out,
                        int64_t k_out_head_stride, int64_t k_out_row_stride, crisp_stream stream) {
  PackedDims d;
  CHECK(check_packed(shape, &d));
  if (!table) return fail(CRISP_EINVAL, "rope table is null");
  CHECK(check_rotation(table->rotary_dim, table->layout));
  CHECK(check_strides(q_head_stride, q_row_stride, false, d.hq, d.n_rows, "q"));
  CHECK(check_strides(k_head_stride, k_row_stride, false, d.hkv, d.n_rows, "k"));
  CHECK(check_strides(q_out_head_stride, q_out_row_stride, d.hq > 0, d.hq, d.n_rows, "q_out"));
  CHECK(check_strides(k_out_head_stride, k_out_row_stride, d.hkv > 0, d.hkv, d.n_rows, "k_out"));
  if (d.n_seqs == 0 || d.n_rows == 0 || d.hq + d.hkv == 0) return CRISP_OK;
  CHECK(check_ptr(start, 4, "start"));
  CHECK(check_ptr(row_ptr, 4, "row_ptr"));
  const RopeTensor qt{q, q_out, {q_head_stride, q_row_stride}, {q_out_head_stride, q_out_row_stride}, d.hq};
  const RopeTensor kt{k, k_out, {k_head_stride, k_row_stride}, {k_out_head_stride, k_out_row_stride}, d.hkv};
  CHECK(check_rotated(qt, d.n_rows, "q"));
  CHECK(check_rotated(kt, d.n_rows, "k"));
  RopeTable t{table->rotary_dim, table->layout == CRISP_ROPE_INTERLEAVED, table->gain, {}};
  for (int i = 0; i < t.dim / 2; ++i) t.turns[i] = table->turns[i];
  return hip_status(launch_rope(d, t, start, row_ptr, qt, kt, (hipStream_t)stream), "crisp_rope launch");
}

crisp_status crisp_packed_attn(const crisp_packed_shape* shape, float softmax_scale, const int32_t* row_ptr,
                               const crisp_bf16* q, int64_t q_head_stride, int64_t q_row_stride, const crisp_bf16* k,
                               int64_t k_head_stride, int64_t k_row_stride, const crisp_bf16* v, int64_t v_head_stride,
                               int64_t v_row_stride, crisp_bf16* o, int64_t o_head_stride, int64_t o_row_stride,
                               crisp_stream stream) {
  PackedDims d;
  CHECK(check_packed(shape, &d));
  if (d.hkv < 1 || d.hq % d.hkv) return fail(CRISP_EINVAL, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", d.hq, d.hkv);
  if (!(softmax_scale >= 0.f) || !isfinite(softmax_scale))
    return fail(CRISP_EINVAL, "softmax_scale must be finite and >= 0");
  CHECK(check_strides(q_head_stride, q_row_stride, false, d.hq, d.n_rows, "q"));
  CHECK(check_strides(k_head_stride, k_row_stride, false, d.hkv, d.n_rows, "k"));
  CHECK(check_strides(v_head_stride, v_row_stride, false, d.hkv, d.n_rows, "v"));
  CHECK(check_strides(o_head_stride, o_row_stride, true, d.hq, d.n_rows, "o"));
  if (k_row_stride >= kMaxKeyStride || v_row_stride >= kMaxKeyStride)
    return fail(CRISP_EUNSUPPORTED, "row strides of k (%lld) and v (%lld) must be below 2^23", (long long)k_row_stride,
                (long long)v_row_stride);
  if ((int64_t)((d.n_rows + 127) / 128) * d.hq > kMaxBlocks)
    return fail(CRISP_EUNSUPPORTED, "n_rows %d of %d query heads above the supported 2^23 blocks of 128 rows", d.n_rows, d.hq);
  if (d.n_seqs == 0 || d.n_rows == 0 || d.hq == 0) return CRISP_OK;
  CHECK(check_ptr(row_ptr, 4, "row_ptr"));
  CHECK(check_ptr(q, 16, "q"));
  CHECK(check_ptr(k, 16, "k"));
  CHECK(check_ptr(v, 16, "v"));
  CHECK(check_ptr(o, 16, "o"));
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)kHeadDim);
  return hip_status(launch_packed_attn(d, scale, row_ptr, q, Strides{q_head_stride, q_row_stride}, k,
                                       Strides{k_head_stride, k_row_stride}, v, Strides{v_head_stride, v_row_stride}, o,
                                       Strides{o_head_stride, o_row_stride}, (hipStream_t)stream),
                    "crisp_packed_attn launch");
}

}  // extern "C"
