// C ABI of the calls that need no cache: rotary tables, turning a tensor, cross attention, encoder states in 4 bits.  Checks and the conversion of
// strides to bytes; everything else is in the kernels' files.
#include <algorithm>
#include <cmath>
#include <limits>

#include "amskv_internal.hpp"

namespace {

using amskv::RowMap;

inline bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Strides of a tensor of `n` = {batch, heads, tokens} rows of head_dim elements, in bytes.  False: a row would not start at a
// multiple of 16 bytes, a stride is negative or out of range, or (written) the dimensions do not nest, so that rows might
// share an address.
bool map_of(const amskv_strides* s, const int64_t (&n)[3], int head_dim, int elem, bool written, RowMap* out) {
  if (!s) return false;
  const int64_t st[3] = {s->batch, s->head, s->token};
  int64_t bytes[3];
  for (int i = 0; i < 3; ++i) {
    bytes[i] = 0;
    if (n[i] <= 1) continue;
    if (st[i] < 0 || st[i] > ((int64_t)1 << 40) || st[i] * elem % 16 != 0) return false;
    bytes[i] = st[i] * elem;
  }
  if (written) {
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return st[a] < st[b]; });
    __int128 span = head_dim;  // (strides up to 2^40, sizes up to 2^26)
    for (int i : order) {
      if (n[i] <= 1) continue;
      if (st[i] < span) return false;
      span += (__int128)st[i] * (n[i] - 1);
    }
  }
  *out = RowMap{bytes[0], bytes[1], bytes[2]};
  return true;
}

bool positive(double x) { return std::isfinite(x) && x > 0; }

int check_cross(const amskv_cross* x) {
  if (!x || x->batch < 0 || x->heads < 0 || x->kv_heads < 0 || x->q_tokens < 0 || x->kv_tokens < 0) return AMSKV_ERR_INVALID_ARG;
  if (x->head_dim != 64 && x->head_dim != 128) return AMSKV_ERR_INVALID_ARG;
  if ((x->dtype != AMSKV_DTYPE_BF16 && x->dtype != AMSKV_DTYPE_BF16_KV4) || !(x->softmax_scale >= 0.f) || !std::isfinite(x->softmax_scale)) return AMSKV_ERR_INVALID_ARG;
  if (x->heads > 0 && (x->kv_heads == 0 || x->heads % x->kv_heads != 0)) return AMSKV_ERR_INVALID_ARG;
  // grids count (b, head, block of rows) in 32 bits, rows of a unit too
  if ((int64_t)x->batch * x->heads > (1 << 24) || x->q_tokens > (1 << 22) || x->kv_tokens > (1 << 26)) return AMSKV_ERR_INVALID_ARG;
  if ((int64_t)x->batch * x->heads * x->q_tokens > ((int64_t)1 << 32)) return AMSKV_ERR_INVALID_ARG;
  if (x->heads > 0) {
    const int64_t rows = (int64_t)(x->heads / x->kv_heads) * x->q_tokens;
    if (rows > (1 << 26)) return AMSKV_ERR_INVALID_ARG;
    // a launch has fewer than 2^32 threads, 64 of them to 32 rows; a grid is rounded up by 7 at most
    if ((int64_t)x->batch * x->kv_heads * ((rows + 31) / 32) > (1 << 26) - 8) return AMSKV_ERR_INVALID_ARG;
  }
  return AMSKV_OK;
}

uint64_t workspace_of(const amskv_cross* x) {
  if (x->heads == 0) return 0;
  auto bytes = x->dtype == AMSKV_DTYPE_BF16_KV4 ? amskv::cross_workspace_bytes4 : amskv::cross_workspace_bytes;
  return bytes(x->batch, x->heads, x->kv_heads, x->head_dim, x->q_tokens, x->kv_tokens);
}

// Bytes of a held tensor of this shape in 4 bits.
int64_t held_bytes(const amskv_cross* x, bool packed) {
  const int64_t units = packed ? x->kv_heads : (int64_t)x->batch * x->kv_heads;
  return units * (packed ? x->kv_rows : x->kv_tokens) * (x->head_dim / 2 + x->head_dim / AMSKV_KV4_GROUP);
}

// The shape of a call about held tensors, and where the batch elements' states are.
int check_held(const amskv_cross* x, const int32_t* lengths_dev, const int32_t* offsets_dev) {
  if (int rc = check_cross(x)) return rc;
  if (x->dtype != AMSKV_DTYPE_BF16_KV4) return AMSKV_ERR_INVALID_ARG;
  if ((lengths_dev && offsets_dev) || ((uintptr_t)lengths_dev & 3) != 0 || ((uintptr_t)offsets_dev & 3) != 0) return AMSKV_ERR_INVALID_ARG;
  if (offsets_dev && (x->kv_rows < 0 || x->kv_rows > INT32_MAX)) return AMSKV_ERR_INVALID_ARG;
  if (x->kv_heads > (1 << 24) || (int64_t)x->batch * x->kv_heads > (1 << 24)) return AMSKV_ERR_INVALID_ARG;  // (heads or batch may be 0)
  return AMSKV_OK;
}

// Both directions between bf16 states and held tensors.
int hold(const amskv_cross* x, const void* k, const void* v, const void* k_held, const void* v_held, const int32_t* lengths_dev,
         const int32_t* offsets_dev, bool back, void* stream) {
  if (int rc = check_held(x, lengths_dev, offsets_dev)) return rc;
  const int64_t n[3] = {offsets_dev ? 1 : x->batch, x->kv_heads, offsets_dev ? x->kv_rows : x->kv_tokens};
  amskv::HoldCall c{};
  // (the strides of a tensor that is left out are not looked at)
  if ((k && !map_of(&x->k, n, x->head_dim, 2, back, &c.k_map)) || (v && !map_of(&x->v, n, x->head_dim, 2, back, &c.v_map)))
    return AMSKV_ERR_INVALID_ARG;
  if (misaligned(k) || misaligned(v) || misaligned(k_held) || misaligned(v_held)) return AMSKV_ERR_INVALID_ARG;
  if (n[0] * n[1] * n[2] > ((int64_t)1 << 36)) return AMSKV_ERR_INVALID_ARG;  // the launch counts blocks of 64 rows in 31 bits
  if (held_bytes(x, offsets_dev != nullptr) == 0 || (offsets_dev && x->batch == 0)) return AMSKV_OK;
  if ((!k && !v) || (k && !k_held) || (v && !v_held)) return AMSKV_ERR_INVALID_ARG;
  // what is written is no other tensor of the call
  if (k && v && (back ? k == v : k_held == v_held)) return AMSKV_ERR_INVALID_ARG;
  for (const void* a : {k, v})
    for (const void* b : {k_held, v_held})
      if (a && a == b) return AMSKV_ERR_INVALID_ARG;
  c.k = const_cast<void*>(k);
  c.v = const_cast<void*>(v);
  c.k_held = (unsigned char*)const_cast<void*>(k_held);
  c.v_held = (unsigned char*)const_cast<void*>(v_held);
  c.lengths = lengths_dev;
  c.offsets = offsets_dev;
  c.batch = x->batch;
  c.kv_heads = x->kv_heads;
  c.head_dim = x->head_dim;
  c.kv_tokens = x->kv_tokens;
  c.kv_rows = x->kv_rows;
  return (back ? amskv::launch_unhold(c, (hipStream_t)stream) : amskv::launch_hold(c, (hipStream_t)stream)) == hipSuccess ? AMSKV_OK
                                                                                                                        : AMSKV_ERR_HIP;
}

}  // namespace

extern "C" {

int32_t amskv_rope_table(const amskv_rope* r, const double* positions_dev, int64_t n, float* table_dev, void* stream) {
  if (int rc = amskv::check_turn(r, 128)) return rc;
  if ((r->axes != 1 && r->axes != 2) || !positive(r->base) || !std::isfinite(r->factor) || r->factor < 1 || !positive(r->amplitude))
    return AMSKV_ERR_INVALID_ARG;
  const bool ramp = r->low != 0 || r->high != 0;
  if (ramp && (!(r->low >= 0) || !(r->low < r->high) || !std::isfinite(r->high) || !positive(r->original))) return AMSKV_ERR_INVALID_ARG;
  if (n < 0 || n > (1 << 25) || misaligned(table_dev) || ((uintptr_t)positions_dev & 7) != 0) return AMSKV_ERR_INVALID_ARG;
  if (n == 0) return AMSKV_OK;
  if (!positions_dev || !table_dev) return AMSKV_ERR_INVALID_ARG;
  const int pairs = r->rot_dim / 2, per_axis = pairs / r->axes;
  double f[64];
  for (int i = 0; i < per_axis; ++i) {
    const double own = std::pow(r->base, -(double)i / per_axis);
    double g = 0;
    if (ramp) {
      g = (r->original * own / (2 * 3.14159265358979323846) - r->low) / (r->high - r->low);
      g = g < 0 ? 0 : g > 1 ? 1 : g;
    }
    f[i] = own * (g + (1 - g) / r->factor);
  }
  return amskv::launch_rope_table(f, pairs, r->axes, r->amplitude, positions_dev, n, table_dev, (hipStream_t)stream) == hipSuccess
             ? AMSKV_OK : AMSKV_ERR_HIP;
}

int32_t amskv_rotate(const amskv_rope* rope, int32_t dtype, int32_t head_dim, int32_t batch, int32_t heads, int32_t tokens,
                     const float* table_dev, int64_t table_batch, int32_t inverse, const void* x_dev, const amskv_strides* x,
                     void* out_dev, const amskv_strides* out, void* stream) {
  if ((head_dim != 64 && head_dim != 128) || (dtype != AMSKV_DTYPE_F32 && dtype != AMSKV_DTYPE_BF16)) return AMSKV_ERR_INVALID_ARG;
  if (int rc = amskv::check_turn(rope, head_dim)) return rc;
  if (batch < 0 || heads < 0 || tokens < 0 || tokens > (1 << 22) || (int64_t)batch * heads > (1 << 24)) return AMSKV_ERR_INVALID_ARG;
  if ((int64_t)batch * heads * tokens > (1 << 29)) return AMSKV_ERR_INVALID_ARG;  // 4 lanes to a row, rows in blocks of 16: 2^32 lanes
  if (table_batch < 0 || table_batch % 4 != 0 || table_batch > ((int64_t)1 << 40)) return AMSKV_ERR_INVALID_ARG;
  const int elem = dtype == AMSKV_DTYPE_F32 ? 4 : 2;
  const int64_t n[3] = {batch, heads, tokens};
  amskv::Take t{};
  if (!map_of(x, n, head_dim, elem, false, &t.q_map) || !map_of(out, n, head_dim, elem, true, &t.q_out_map)) return AMSKV_ERR_INVALID_ARG;
  if (misaligned(table_dev) || misaligned(x_dev) || misaligned(out_dev)) return AMSKV_ERR_INVALID_ARG;
  if (batch == 0 || heads == 0 || tokens == 0) return AMSKV_OK;
  if (!table_dev || !x_dev || !out_dev) return AMSKV_ERR_INVALID_ARG;
  if (x_dev == out_dev &&
      (t.q_map.batch != t.q_out_map.batch || t.q_map.head != t.q_out_map.head || t.q_map.tok != t.q_out_map.tok))
    return AMSKV_ERR_INVALID_ARG;
  t.q = x_dev;
  t.q_out = out_dev;
  t.table = table_dev;
  t.table_batch = table_batch;
  t.rot_dim = rope->rot_dim;
  t.pairing = rope->pairing;
  t.inverse = inverse != 0;
  t.batch = batch;
  t.heads = heads;
  t.tokens = tokens;
  t.head_dim = head_dim;
  t.dtype = dtype;
  return amskv::launch_take(t, (hipStream_t)stream) == hipSuccess ? AMSKV_OK : AMSKV_ERR_HIP;
}

int32_t amskv_cross_workspace_bytes(const amskv_cross* x, uint64_t* bytes_out) {
  if (!bytes_out) return AMSKV_ERR_INVALID_ARG;
  if (int rc = check_cross(x)) return rc;
  *bytes_out = workspace_of(x);
  return AMSKV_OK;
}

int32_t amskv_cross_held_bytes(const amskv_cross* x, int32_t packed, uint64_t* bytes_out) {
  if (!bytes_out || (packed != 0 && packed != 1)) return AMSKV_ERR_INVALID_ARG;
  if (int rc = check_held(x, nullptr, nullptr)) return rc;
  if (packed && (x->kv_rows < 0 || x->kv_rows > INT32_MAX)) return AMSKV_ERR_INVALID_ARG;
  *bytes_out = (uint64_t)held_bytes(x, packed != 0);
  return AMSKV_OK;
}

int32_t amskv_cross_hold(const amskv_cross* x, const void* K_dev, const void* V_dev, void* K_held_dev, void* V_held_dev,
                         const int32_t* lengths_dev, const int32_t* offsets_dev, void* stream) {
  return hold(x, K_dev, V_dev, K_held_dev, V_held_dev, lengths_dev, offsets_dev, false, stream);
}

int32_t amskv_cross_export(const amskv_cross* x, const void* K_held_dev, const void* V_held_dev, void* K_out_dev, void* V_out_dev,
                           const int32_t* lengths_dev, const int32_t* offsets_dev, void* stream) {
  return hold(x, K_out_dev, V_out_dev, K_held_dev, V_held_dev, lengths_dev, offsets_dev, true, stream);
}

int32_t amskv_cross_attend(const amskv_cross* x, const void* Q_dev, const void* K_dev, const void* V_dev, void* O_dev,
                           const int32_t* lengths_dev, const int32_t* offsets_dev, void* workspace_dev, uint64_t workspace_bytes,
                           void* stream) {
  if (int rc = check_cross(x)) return rc;
  if ((lengths_dev && offsets_dev) || ((uintptr_t)lengths_dev & 3) != 0 || ((uintptr_t)offsets_dev & 3) != 0) return AMSKV_ERR_INVALID_ARG;
  if (offsets_dev && (x->kv_rows < 0 || x->kv_rows > INT32_MAX)) return AMSKV_ERR_INVALID_ARG;
  const int64_t nq[3] = {x->batch, x->heads, x->q_tokens};
  // packed: one axis of rows, whatever the batch strides say
  const int64_t nk[3] = {offsets_dev ? 1 : x->batch, x->kv_heads, offsets_dev ? x->kv_rows : x->kv_tokens};
  amskv::CrossCall c{};
  c.four_bits = x->dtype == AMSKV_DTYPE_BF16_KV4;  // held tensors have no strides
  if (!map_of(&x->q, nq, x->head_dim, 2, false, &c.q_map) || !map_of(&x->o, nq, x->head_dim, 2, true, &c.o_map) ||
      (!c.four_bits && (!map_of(&x->k, nk, x->head_dim, 2, false, &c.k_map) || !map_of(&x->v, nk, x->head_dim, 2, false, &c.v_map))))
    return AMSKV_ERR_INVALID_ARG;
  if (c.k_map.tok >= (1 << 24) || c.v_map.tok >= (1 << 24)) return AMSKV_ERR_INVALID_ARG;  // 64 rows of a tile by 32-bit offsets
  if (misaligned(Q_dev) || misaligned(K_dev) || misaligned(V_dev) || misaligned(O_dev) || misaligned(workspace_dev)) return AMSKV_ERR_INVALID_ARG;
  if (x->batch == 0 || x->heads == 0 || x->q_tokens == 0) return AMSKV_OK;
  // (K and V may be absent where there can be no states)
  if (!Q_dev || !O_dev || ((!K_dev || !V_dev) && x->kv_tokens > 0 && (!offsets_dev || x->kv_rows > 0))) return AMSKV_ERR_INVALID_ARG;
  if (workspace_dev && workspace_bytes < workspace_of(x))
    return AMSKV_ERR_ARENA_TOO_SMALL;
  c.q = Q_dev;
  c.k = K_dev;
  c.v = V_dev;
  c.o = O_dev;
  c.lengths = lengths_dev;
  c.offsets = offsets_dev;
  c.batch = x->batch;
  c.heads = x->heads;
  c.kv_heads = x->kv_heads;
  c.head_dim = x->head_dim;
  c.q_tokens = x->q_tokens;
  c.kv_tokens = x->kv_tokens;
  c.kv_rows = x->kv_rows;
  c.softmax_scale = x->softmax_scale > 0.f ? x->softmax_scale : 1.0f / std::sqrt((float)x->head_dim);
  c.workspace = (float*)workspace_dev;
  return amskv::launch_cross(c, (hipStream_t)stream) == hipSuccess ? AMSKV_OK : AMSKV_ERR_HIP;
}

}  // extern "C"
