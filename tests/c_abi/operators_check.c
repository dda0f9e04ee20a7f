/* The rotary, 8-bit and cross-attention calls used the way a C program would: this file includes include/amskv.h and the HIP runtime API
 * and nothing else.  Keys and queries of two scales are turned on their way into an 8-bit cache, attended and read back, a tensor
 * is turned there and back, and the queries attend to states of two lengths through a workspace; every result is compared with its
 * definition written out below in double precision.  With an argument it prints the structures' layout instead and needs no GPU.
 *
 * Test program: built and run by tests/test_gpu_operators_c_abi.py.  Tolerances: 2e-2 (bf16), 2^-4 of a value and 2^-10 (codes), max-abs. */
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "amskv.h"

#define B 2
#define H 3
#define D 64
#define P (D / 2)
#define T0 4
#define T1 9
#define HK 1
#define LK 2000

#define HIP(x)                                                                        \
  do {                                                                                \
    hipError_t e_ = (x);                                                              \
    if (e_ != hipSuccess) {                                                           \
      fprintf(stderr, "%s:%d: %s -> %s\n", __FILE__, __LINE__, #x, hipGetErrorString(e_)); \
      exit(1);                                                                        \
    }                                                                                 \
  } while (0)
#define AMS(x)                                                                        \
  do {                                                                                \
    int32_t s_ = (x);                                                                 \
    if (s_ != AMSKV_OK) {                                                             \
      fprintf(stderr, "%s:%d: %s -> %s\n", __FILE__, __LINE__, #x, amskv_status_string(s_)); \
      exit(1);                                                                        \
    }                                                                                 \
  } while (0)
#define EXPECT(cond)                                                  \
  do {                                                                \
    if (!(cond)) {                                                    \
      fprintf(stderr, "%s:%d: not so: %s\n", __FILE__, __LINE__, #cond); \
      exit(1);                                                        \
    }                                                                 \
  } while (0)

static uint32_t g_state = 4711u;
static float draw(void) { /* uniform in [-1.5, 1.5), a plain linear congruential generator */
  g_state = g_state * 1664525u + 1013904223u;
  return ((float)(g_state >> 8) / 16777216.0f - 0.5f) * 3.0f;
}
static uint16_t to_bf16(float x) { /* round to nearest even */
  uint32_t u;
  memcpy(&u, &x, 4);
  u += 0x7fffu + ((u >> 16) & 1u);
  return (uint16_t)(u >> 16);
}
static float from_bf16(uint16_t h) {
  uint32_t u = (uint32_t)h << 16;
  float x;
  memcpy(&x, &u, 4);
  return x;
}

/* a bf16 tensor on the device, and its values */
typedef struct {
  uint16_t* dev;
  double* val;
  size_t n;
} Tensor;
static Tensor made(size_t n) {
  Tensor t = {NULL, malloc(n * sizeof(double)), n};
  uint16_t* host = malloc(n * 2);
  for (size_t i = 0; i < n; ++i) {
    host[i] = to_bf16(draw());
    t.val[i] = from_bf16(host[i]);
  }
  HIP(hipMalloc((void**)&t.dev, n * 2));
  HIP(hipMemcpy(t.dev, host, n * 2, hipMemcpyHostToDevice));
  free(host);
  return t;
}
static void fetch(Tensor* t) {
  uint16_t* host = malloc(t->n * 2);
  HIP(hipDeviceSynchronize());
  HIP(hipMemcpy(host, t->dev, t->n * 2, hipMemcpyDeviceToHost));
  for (size_t i = 0; i < t->n; ++i) t->val[i] = from_bf16(host[i]);
  free(host);
}

/* rows [units][T][D] turned by positions first, first + 1, .. (halves) */
static void turned(const double* x, double* y, int units, int T, double first, double sign) {
  for (int u = 0; u < units; ++u)
    for (int t = 0; t < T; ++t)
      for (int i = 0; i < P; ++i) {
        const double angle = (first + t) * pow(10000.0, -(double)i / P), c = cos(angle), s = sign * sin(angle);
        const double *a = x + ((size_t)u * T + t) * D;
        double* b = y + ((size_t)u * T + t) * D;
        b[i] = a[i] * c - a[i + P] * s;
        b[i + P] = a[i + P] * c + a[i] * s;
      }
}
static void attended(const double* q, const double* k, const double* v, size_t k_row, int n, double* o) {
  double top = -1e300, sum = 0, *w = malloc((size_t)n * sizeof(double));
  for (int j = 0; j < n; ++j) {
    double s = 0;
    for (int d = 0; d < D; ++d) s += q[d] * k[j * k_row + d];
    w[j] = s / sqrt((double)D);
    if (w[j] > top) top = w[j];
  }
  for (int j = 0; j < n; ++j) sum += w[j] = exp(w[j] - top);
  for (int d = 0; d < D; ++d) {
    o[d] = 0;
    for (int j = 0; j < n; ++j) o[d] += w[j] / sum * v[j * k_row + d];
  }
  free(w);
}
static void same(const char* what, const double* a, const double* b, size_t n, double rel, double abs_) {
  for (size_t i = 0; i < n; ++i) {
    const double off = fabs(a[i] - b[i]) - rel * fabs(b[i]);
    if (!(off <= abs_)) {
      fprintf(stderr, "%s: element %zu is %g, not %g\n", what, i, a[i], b[i]);
      exit(1);
    }
  }
  printf("%s: ok\n", what);
}

static int layout(void) {
#define SIZE(t) printf(#t " %zu\n", sizeof(t))
#define AT(t, m) printf(#t "." #m " %zu\n", offsetof(t, m))
  SIZE(amskv_rope);
  AT(amskv_rope, rot_dim), AT(amskv_rope, pairing), AT(amskv_rope, axes), AT(amskv_rope, base), AT(amskv_rope, factor);
  AT(amskv_rope, original), AT(amskv_rope, low), AT(amskv_rope, high), AT(amskv_rope, amplitude);
  SIZE(amskv_strides);
  AT(amskv_strides, batch), AT(amskv_strides, head), AT(amskv_strides, token);
  SIZE(amskv_cross);
  AT(amskv_cross, batch), AT(amskv_cross, heads), AT(amskv_cross, kv_heads), AT(amskv_cross, head_dim), AT(amskv_cross, dtype);
  AT(amskv_cross, q_tokens), AT(amskv_cross, kv_tokens), AT(amskv_cross, kv_rows), AT(amskv_cross, softmax_scale);
  AT(amskv_cross, q), AT(amskv_cross, k), AT(amskv_cross, v), AT(amskv_cross, o);
  return 0;
}

int main(int argc, char** argv) {
  (void)argv;
  if (argc > 1) return layout();
  const amskv_rope rope = {D, AMSKV_ROPE_HALF, 1, 10000.0, 1.0, 0.0, 0.0, 0.0, 1.0};
  const int T[2] = {T0, T1}, units = B * H;
  const int32_t side_h[2] = {1, 1}, side_w[2] = {T0, T1};
  float* table[2];
  for (int s = 0, first = 0; s < 2; first += T[s], ++s) {
    double where[T1], *dev;
    for (int t = 0; t < T[s]; ++t) where[t] = first + t;
    HIP(hipMalloc((void**)&dev, sizeof(where)));
    HIP(hipMemcpy(dev, where, (size_t)T[s] * sizeof(double), hipMemcpyHostToDevice));
    HIP(hipMalloc((void**)&table[s], (size_t)T[s] * P * 2 * sizeof(float)));
    AMS(amskv_rope_table(&rope, dev, T[s], table[s], NULL));
  }

  /* an 8-bit cache of one layer that keeps both scales; keys and queries turned on the way */
  const amskv_layer_policy pol = {0, 0, 1};
  const amskv_schedule sc = {2, side_h, side_w, B, AMSKV_DTYPE_BF16_KV8};
  const amskv_policy po = {1, &pol, 0.f, AMSKV_LAYOUT_COMPACT, 0, 0, AMSKV_MODE_SCALE_WINDOW, NULL};
  uint64_t need = 0;
  void* arena;
  amskv_cache* h = NULL;
  AMS(amskv_cache_required_bytes(1, H, D, &sc, &po, &need));
  HIP(hipMalloc(&arena, need));
  AMS(amskv_cache_create(1, H, D, &sc, &po, arena, need, &h));
  Tensor q[2], k[2], v[2], qt[2], o[2];
  double* want_k[2];
  for (int s = 0; s < 2; ++s) {
    const size_t n = (size_t)units * T[s] * D;
    q[s] = made(n), k[s] = made(n), v[s] = made(n), qt[s] = made(n), o[s] = made(n);
    AMS(amskv_append_scale_rotary(h, 0, s, &rope, table[s], q[s].dev, 0, qt[s].dev, k[s].dev, v[s].dev, NULL));
    AMS(amskv_attend(h, 0, s, qt[s].dev, o[s].dev, NULL));
    double* want = malloc(n * sizeof(double));
    turned(q[s].val, want, units, T[s], s ? T0 : 0, 1);
    fetch(&qt[s]);
    same("turned queries", qt[s].val, want, n, 1.0 / 256, 2e-6);
    want_k[s] = malloc(n * sizeof(double));
    turned(k[s].val, want_k[s], units, T[s], s ? T0 : 0, 1);
  }
  Tensor ko = made((size_t)units * (T0 + T1) * D), vo = made((size_t)units * (T0 + T1) * D);
  AMS(amskv_cache_export(h, 0, ko.dev, vo.dev, NULL));
  fetch(&ko), fetch(&vo);
  for (int u = 0; u < units; ++u)
    for (int s = 0; s < 2; ++s) {
      const size_t at = ((size_t)u * (T0 + T1) + (s ? T0 : 0)) * D, from = (size_t)u * T[s] * D, n = (size_t)T[s] * D;
      same("cached keys", ko.val + at, want_k[s] + from, n, 1.0 / 16, 1.0 / 1024);
      same("cached values", vo.val + at, v[s].val + from, n, 1.0 / 16, 1.0 / 1024);
    }
  for (int s = 0; s < 2; ++s) { /* attention over what the cache says it holds */
    double* want = malloc(o[s].n * sizeof(double));
    fetch(&o[s]);
    for (int u = 0; u < units; ++u)
      for (int t = 0; t < T[s]; ++t)
        attended(qt[s].val + ((size_t)u * T[s] + t) * D, ko.val + (size_t)u * (T0 + T1) * D, vo.val + (size_t)u * (T0 + T1) * D, D, s ? T0 + T1 : T0,
                 want + ((size_t)u * T[s] + t) * D);
    same("attention over codes", o[s].val, want, o[s].n, 0, 2e-2);
  }
  amskv_cache_destroy(h);

  /* there and back */
  const amskv_strides rows = {(int64_t)H * T1 * D, (int64_t)T1 * D, D};
  Tensor there = made(q[1].n), back = made(q[1].n);
  AMS(amskv_rotate(&rope, AMSKV_DTYPE_BF16, D, B, H, T1, table[1], 0, 0, q[1].dev, &rows, there.dev, &rows, NULL));
  AMS(amskv_rotate(&rope, AMSKV_DTYPE_BF16, D, B, H, T1, table[1], 0, 1, there.dev, &rows, back.dev, &rows, NULL));
  fetch(&there), fetch(&back);
  same("the turn of the append", there.val, qt[1].val, there.n, 0, 0);
  same("back again", back.val, q[1].val, back.n, 0, 2e-2);

  /* the queries over padded states of 2000 and 700, one kv head for all */
  const int32_t lengths[B] = {LK, 700};
  int32_t* lengths_dev;
  HIP(hipMalloc((void**)&lengths_dev, sizeof(lengths)));
  HIP(hipMemcpy(lengths_dev, lengths, sizeof(lengths), hipMemcpyHostToDevice));
  Tensor ck = made((size_t)B * LK * HK * D), cv = made((size_t)B * LK * HK * D), co = made(q[1].n);
  amskv_cross x;
  memset(&x, 0, sizeof(x));
  x.batch = B, x.heads = H, x.kv_heads = HK, x.head_dim = D, x.dtype = AMSKV_DTYPE_BF16, x.q_tokens = T1, x.kv_tokens = LK;
  x.q = x.o = rows;
  x.k.batch = (int64_t)LK * HK * D, x.k.head = D, x.k.token = HK * D;
  x.v = x.k;
  AMS(amskv_cross_workspace_bytes(&x, &need));
  EXPECT(need > 0);
  void* space;
  HIP(hipMalloc(&space, need));
  EXPECT(amskv_cross_attend(&x, q[1].dev, ck.dev, cv.dev, co.dev, lengths_dev, NULL, space, need - 1, NULL) == AMSKV_ERR_ARENA_TOO_SMALL);
  AMS(amskv_cross_attend(&x, q[1].dev, ck.dev, cv.dev, co.dev, lengths_dev, NULL, space, need, NULL));
  fetch(&co);
  double* want = malloc(co.n * sizeof(double));
  for (int u = 0; u < units; ++u)
    for (int t = 0; t < T1; ++t)
      attended(q[1].val + ((size_t)u * T1 + t) * D, ck.val + (size_t)(u / H) * LK * D, cv.val + (size_t)(u / H) * LK * D, D, lengths[u / H],
               want + ((size_t)u * T1 + t) * D);
  same("cross attention", co.val, want, co.n, 0, 2e-2);
  printf("operators_check: ok\n");
  return 0;
}
