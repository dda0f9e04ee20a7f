// Sanitizer driver for the host side of K and V in 4 bits (csrc/amskv_api.cpp, csrc/operators_api.cpp): built by
// tests/test_host_sanitize_four_bits.py with -fsanitize=address,undefined.  The launchers are stubs that do to ordinary host memory what
// the kernels do to the device's, row by row, with a number for every row in place of its channels and its low byte in place of its
// groups' powers.  Arenas and held tensors are exactly as large as the library asks for.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "amskv_internal.hpp"
#include "attend_rows_choice.hpp"

static int failures = 0;
#define CHECK(cond)                                                                   \
  do {                                                                                \
    if (!(cond)) {                                                                    \
      if (++failures < 20) std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
    }                                                                                 \
  } while (0)

[[noreturn]] static void unexpected(const char* what) {
  std::fprintf(stderr, "%s is no part of these walks\n", what);
  std::exit(2);
}

using amskv::Codes4;
using amskv::RowMap;

static const int32_t kTurned = 1 << 30, kValue = 1 << 29;
static int32_t id_of(int scale, int token) { return (scale + 1) << 16 | token; }
static int32_t get(const void* row) {
  int32_t x;
  std::memcpy(&x, row, 4);
  return x;
}
static void put(void* row, int32_t id, int bytes) {
  std::memset(row, 0x5a, bytes);
  std::memcpy(row, &id, 4);
}
static char* at(const void* base, const RowMap& m, int bh, int heads, int64_t t) {
  return (char*)base + (bh / heads) * m.batch + (bh % heads) * m.head + t * m.tok;
}
static int32_t coded(const unsigned char* codes, const unsigned char* groups, int64_t row, int D) {
  const int32_t id = get(codes + row * (D / 2));
  for (int g = 0; g < D / 32; ++g) CHECK(groups[row * (D / 32) + g] == (unsigned char)id);
  return id;
}

static std::vector<int32_t> g_expect;
static int g_takes = 0, g_moves = 0, g_attends = 0, g_holds = 0, g_crosses = 0;
static bool g_turns = false;

namespace amskv {
hipError_t launch_move_codes4(const Codes4& c, int bh, int D, int64_t cap, const MoveList& mv, hipStream_t) {
  ++g_moves;
  for (int m = 0; m < mv.n; ++m) {
    CHECK(mv.dst[m] >= 0 && mv.dst[m] < mv.src[m] && mv.src[m] + mv.len[m] <= cap);
    for (int u = 0; u < bh; ++u)
      for (unsigned char* p : {c.k, c.v, c.k_group, c.v_group}) {
        const int row = p == c.k || p == c.v ? D / 2 : D / 32;
        std::memmove(p + (u * cap + mv.dst[m]) * row, p + (u * cap + mv.src[m]) * row, (size_t)mv.len[m] * row);
      }
  }
  return hipSuccess;
}
hipError_t launch_take(const Take& t, hipStream_t st) {
  ++g_takes;
  const int D = t.head_dim;
  CHECK(!t.eight_bits && t.dtype == AMSKV_DTYPE_BF16);
  if (t.four_bits) {
    CHECK(t.dst_new >= 0 && t.dst_new + t.tokens <= t.cap_tokens);
    if (t.moves && t.moves->n > 0) (void)launch_move_codes4(t.codes4, t.batch * t.heads, D, t.cap_tokens, *t.moves, st);
  }
  const void* src[3] = {t.k, t.v, t.q};
  void* dst[3] = {t.k_out, t.v_out, t.q_out};
  for (int i = 0; i < 3; ++i)
    for (int u = 0; src[i] && u < t.batch * t.heads; ++u)
      for (int j = 0; j < t.tokens; ++j) {
        int32_t id = get(at(src[i], i == 2 ? t.q_map : t.kv_map, u, t.heads, j));
        CHECK((id & kTurned) == 0);
        if (t.table && i != 1) id |= kTurned;
        if (t.four_bits && i < 2) {
          const int64_t row = u * t.cap_tokens + t.dst_new + j;
          put((i ? t.codes4.v : t.codes4.k) + row * (D / 2), id, D / 2);
          std::memset((i ? t.codes4.v_group : t.codes4.k_group) + row * (D / 32), id & 0xff, D / 32);
        } else {
          put(at(dst[i], i == 2 ? t.q_out_map : t.out_map, u, t.heads, j), id, 2 * D);
        }
      }
  return hipSuccess;
}
hipError_t launch_attend_codes4(const void* q, void* o, const Codes4& c, int bh, int t_q, int D, int64_t cap, const SegTable& seg, const ExtKV& ext,
                                const CallerIo& io, float, hipStream_t) {
  ++g_attends;
  CHECK(seg.total == (int)g_expect.size() && ext.alt_if == nullptr && ext.wb_from >= seg.total);
  for (int u = 0; u < bh; ++u) {
    for (int t = 0; t < t_q; ++t) {
      CHECK(((get(at(q, io.q, u, io.heads, t)) & kTurned) != 0) == g_turns);
      put(at(o, io.o, u, io.heads, t), 0, 2 * D);
    }
    for (int g = 0; g < seg.n; ++g)
      for (int i = 0; i < seg.len[g]; ++i) {
        const int j = seg.virt_start[g] + i;
        const bool outside = j >= seg.ext_start;
        if (!outside) CHECK(seg.phys_off[g] >= 0 && seg.phys_off[g] + i < cap);
        const int64_t row = u * cap + seg.phys_off[g] + i;
        const int32_t k = outside ? get(at(ext.k, io.kv, u, io.heads, j - seg.ext_start)) : coded(c.k, c.k_group, row, D);
        const int32_t v = outside ? get(at(ext.v, io.kv, u, io.heads, j - seg.ext_start)) : coded(c.v, c.v_group, row, D);
        CHECK(k == (g_expect[j] | (g_turns ? kTurned : 0)) && v == (g_expect[j] | kValue));
      }
  }
  return hipSuccess;
}
hipError_t launch_export_codes4(const Codes4& c, void* k_out, void* v_out, int bh, int D, int64_t cap, const SegTable& seg, const ExtKV& ext,
                                const RowMap& map, int heads, hipStream_t) {
  for (int u = 0; u < bh; ++u)
    for (int g = 0; g < seg.n; ++g)
      for (int i = 0; i < seg.len[g]; ++i) {
        const int j = seg.virt_start[g] + i;
        const bool outside = j >= seg.ext_start;
        const int64_t row = u * cap + seg.phys_off[g] + i, to = ((int64_t)u * seg.total + j) * 2 * D;
        put((char*)k_out + to, outside ? get(at(ext.k, map, u, heads, j - seg.ext_start)) : coded(c.k, c.k_group, row, D), 2 * D);
        put((char*)v_out + to, outside ? get(at(ext.v, map, u, heads, j - seg.ext_start)) : coded(c.v, c.v_group, row, D), 2 * D);
      }
  return hipSuccess;
}

// every state of a held tensor, codes and groups, and the rows it comes from or goes to
static hipError_t hold(const HoldCall& c, bool back) {
  ++g_holds;
  const int D = c.head_dim;
  const int64_t rows = c.offsets ? c.kv_rows : c.kv_tokens, units = c.offsets ? c.kv_heads : (int64_t)c.batch * c.kv_heads;
  for (int i = 0; i < 2; ++i) {
    char* x = (char*)(i ? c.v : c.k);
    unsigned char* held = i ? c.v_held : c.k_held;
    if (!x) continue;
    CHECK(held != nullptr && units * rows > 0);
    for (int64_t u = 0; u < units; ++u)
      for (int64_t r = 0; r < rows; ++r) {
        if (!c.offsets && c.lengths && r >= c.lengths[u / c.kv_heads]) continue;
        if (c.offsets && (r < c.offsets[0] || r >= c.offsets[c.batch])) continue;
        char* row = at(x, i ? c.v_map : c.k_map, (int)u, c.kv_heads, r);
        unsigned char *codes = held + (u * rows + r) * (D / 2), *groups = held + units * rows * (D / 2);
        if (back) {
          put(row, coded(held, groups, u * rows + r, D), 2 * D);
        } else {
          const int32_t id = get(row);
          put(codes, id, D / 2);
          std::memset(groups + (u * rows + r) * (D / 32), id & 0xff, D / 32);
        }
      }
  }
  return hipSuccess;
}
hipError_t launch_hold(const HoldCall& c, hipStream_t) { return hold(c, false); }
hipError_t launch_unhold(const HoldCall& c, hipStream_t) { return hold(c, true); }
uint64_t cross_workspace_bytes4(int batch, int heads, int kv_heads, int D, int q_tokens, int kv_tokens) {
  const long long units = (long long)batch * kv_heads, n = (long long)(heads / kv_heads) * q_tokens;
  if (units == 0 || n == 0 || kv_tokens == 0) return 0;
  const rows::Division d = rows::divide4(D, units, n, kv_tokens, 48);
  return d.splits == 1 ? 0 : (uint64_t)units * ((n + 32 * d.team_waves - 1) / (32 * d.team_waves)) * d.splits * rows::partial_floats(32 * d.team_waves, D) * 4;
}
hipError_t launch_cross(const CrossCall& c, hipStream_t) {
  ++g_crosses;
  CHECK(c.four_bits && c.batch >= 1 && c.heads >= 1 && c.q_tokens >= 1 && c.softmax_scale > 0 && !(c.lengths && c.offsets));
  return hipSuccess;
}

// of other caches
hipError_t launch_append(void*, void*, const void*, const void*, int, int, int64_t, const MoveList&, int, int, int, const RowMap&, int, hipStream_t) { unexpected(__func__); }
hipError_t launch_roll(void*, void*, const void*, const void*, int, int, int64_t, const MoveList&, const NewRanges&, const RowMap&, int, hipStream_t) { unexpected(__func__); }
hipError_t launch_export(const void*, const void*, void*, void*, int, int, int64_t, const SegTable&, const ExtKV&, const RowMap&, int, hipStream_t) { unexpected(__func__); }
hipError_t launch_attend_bf16(const void*, void*, void*, void*, int, int, int, int64_t, const SegTable&, const ExtKV&, const CallerIo&, float, hipStream_t) { unexpected(__func__); }
hipError_t launch_attend_f32(const void*, void*, void*, void*, int, int, int, int64_t, const SegTable&, const ExtKV&, const CallerIo&, float, hipStream_t) { unexpected(__func__); }
hipError_t launch_similarity(const ScaleRef&, const ScaleRef&, int, int, int, int, int, int, int, int, float*, float*, hipStream_t) { unexpected(__func__); }
hipError_t launch_similarity_static(const ScaleRef&, const ScaleRef&, int, int, int, int, int, int, int, int, float*, hipStream_t) { unexpected(__func__); }
hipError_t launch_density(const void*, const void*, int, int, int, int, int, int64_t, const SegTable&, const ExtKV&, const CallerIo&, float, float*,
                          float*, hipStream_t) { unexpected(__func__); }
hipError_t launch_theta_flag(const float*, int, double, float, int32_t*, int32_t*, hipStream_t) { unexpected(__func__); }
bool attend_density_fused(int) { unexpected(__func__); }
bool attend_owns_unit(int, int) { unexpected(__func__); }
hipError_t launch_attend_density_bf16(const void*, void*, void*, void*, int, int, int, int, int64_t, const SegTable&, const ExtKV&, const CallerIo&,
                                      float, const GroupEnds&, float*, float*, hipStream_t) { unexpected(__func__); }
}  // namespace amskv
extern "C" hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t) { unexpected(__func__); }
extern "C" hipError_t hipStreamSynchronize(hipStream_t) { unexpected(__func__); }
extern "C" hipError_t hipHostMalloc(void**, size_t, unsigned int) { unexpected(__func__); }
extern "C" hipError_t hipHostFree(void*) { unexpected(__func__); }
extern "C" hipError_t hipEventCreateWithFlags(hipEvent_t*, unsigned) { unexpected(__func__); }
extern "C" hipError_t hipEventDestroy(hipEvent_t) { unexpected(__func__); }
extern "C" hipError_t hipEventRecord(hipEvent_t, hipStream_t) { unexpected(__func__); }
extern "C" hipError_t hipEventSynchronize(hipEvent_t) { unexpected(__func__); }

struct Buffer {  // nothing behind it
  char* p;
  explicit Buffer(size_t n) : p((char*)std::aligned_alloc(16, (n + 15) / 16 * 16)) {}
  ~Buffer() { std::free(p); }
  Buffer(const Buffer&) = delete;
};

static void walk(const std::vector<int32_t>& hs, const std::vector<int32_t>& ws, int D, int32_t layout, int32_t borrow, bool packed, bool turns) {
  const int n = (int)hs.size(), B = 2, H = 3, row = 2 * D;
  std::vector<amskv_layer_policy> pols;
  for (int c = 0; c < 4; ++c)
    for (int w = 0; w < 4; ++w) pols.push_back({c, w, 0});
  pols.push_back({0, 0, 1});
  const int L = (int)pols.size();
  amskv_schedule sc{n, hs.data(), ws.data(), B, AMSKV_DTYPE_BF16_KV4};
  amskv_policy po{L, pols.data(), 0.f, layout, borrow, 0, AMSKV_MODE_SCALE_WINDOW, nullptr};
  uint64_t need = 0;
  CHECK(amskv_cache_required_bytes(L, H, D, &sc, &po, &need) == AMSKV_OK && need > 0);
  char* arena = (char*)std::aligned_alloc(256, need);
  std::memset(arena, 0xff, need);
  amskv_cache* h = nullptr;
  CHECK(amskv_cache_create(L, H, D, &sc, &po, arena, need, &h) == AMSKV_OK && h);
  if (!h) std::exit(2);
  if (packed) CHECK(amskv_cache_set_io_layout(h, AMSKV_IO_TOKEN_MAJOR, turns ? H * D : 3 * H * D, 3 * H * D, H * D) == AMSKV_OK);
  const amskv_rope rope{D / 2, AMSKV_ROPE_HALF, 1, 1e4, 1, 0, 0, 0, 1};
  Buffer table(64);
  g_turns = turns;
  for (int image = 0; image < 2; ++image) {
    CHECK(amskv_cache_reset(h) == AMSKV_OK);
    std::vector<Buffer*> alive(L, nullptr);
    for (int s = 0; s < n; ++s)
      for (int l = 0; l < L; ++l) {
        const int T = hs[s] * ws[s];
        const size_t whole = (size_t)B * H * T * row;
        auto* data = new Buffer(3 * whole);
        const RowMap in = packed ? RowMap{(int64_t)T * 3 * H * row, row, (int64_t)3 * H * row} : RowMap{(int64_t)H * T * row, (int64_t)T * row, row};
        char* part[3];
        for (int i = 0; i < 3; ++i) {
          part[i] = data->p + (packed ? (size_t)i * H * row : i * whole);
          for (int u = 0; u < B * H; ++u)
            for (int t = 0; t < T; ++t) put(at(part[i], in, u, H, t), id_of(s, t) | (i == 2 ? kValue : 0), row);
        }
        Buffer o(whole), turned(whole);
        g_expect.clear();
        int64_t held = 0;
        for (int k = 0; k <= s; ++k)
          if (k == s || pols[l].keep_all || k < pols[l].n_condensed || s - k <= pols[l].window) {
            for (int t = 0; t < hs[k] * ws[k]; ++t) g_expect.push_back(id_of(k, t));
            held += k < s ? hs[k] * ws[k] : 0;
          }
        char* q = part[0];
        if (turns) {
          CHECK(amskv_append_scale_rotary(h, l, s, &rope, (float*)table.p, q, packed ? 3 * H * D : 0, turned.p, part[1], part[2], nullptr) == AMSKV_OK);
          q = turned.p;
        } else {
          CHECK(amskv_append_scale(h, l, s, part[1], part[2], nullptr) == AMSKV_OK);
        }
        CHECK(amskv_attend(h, l, s, q, o.p, nullptr) == AMSKV_OK);
        CHECK(amskv_cache_bytes_held(h, l, 0) == 2ll * B * H * held * (D / 2 + D / 32));
        Buffer ko(B * H * g_expect.size() * row), vo(B * H * g_expect.size() * row);
        CHECK(amskv_cache_export(h, l, ko.p, vo.p, nullptr) == AMSKV_OK);
        for (int u = 0; u < B * H; ++u)
          for (size_t j = 0; j < g_expect.size(); ++j) {
            CHECK(get(ko.p + (u * g_expect.size() + j) * row) == (g_expect[j] | (turns ? kTurned : 0)));
            CHECK(get(vo.p + (u * g_expect.size() + j) * row) == (g_expect[j] | kValue));
          }
        delete alive[l];  // the caller's tensors live until the next append on the layer
        alive[l] = data;
      }
    for (Buffer* b : alive) delete b;
    CHECK(amskv_cache_reset(h) == AMSKV_OK);
  }
  amskv_cache_destroy(h);
  std::free(arena);
}

static void held_tensors() {
  for (int D : {64, 128})
    for (int packed : {0, 1})
      for (int lengths_given : {0, 1}) {
        const int B = 3, H = 2, T = 7, rows = 17;
        int32_t lengths[B] = {7, 0, 4}, offsets[B + 1] = {2, 9, 9, 15};
        const amskv_strides st = packed ? amskv_strides{0, D, H * D} : amskv_strides{T * H * D, D, H * D};
        amskv_cross x{B, 4, H, D, AMSKV_DTYPE_BF16_KV4, 5, T, packed ? rows : 0, 0.f, {20 * D, 5 * D, D}, st, st, {20 * D, 5 * D, D}};
        uint64_t need = 0;
        CHECK(amskv_cross_held_bytes(&x, packed, &need) == AMSKV_OK);
        const int total = (packed ? rows : B * T) * H, bytes = total * 2 * D;
        CHECK(need == (uint64_t)total * (D / 2 + D / 32));
        char *kh = (char*)std::malloc(need), *vh = (char*)std::malloc(need);
        Buffer k(bytes), v(bytes), ko(bytes), vo(bytes);
        for (int i = 0; i < total; ++i) put(k.p + (size_t)i * 2 * D, i, 2 * D), put(v.p + (size_t)i * 2 * D, i | kValue, 2 * D);
        std::memset(ko.p, 0, bytes), std::memset(vo.p, 0, bytes);
        const int32_t *l = lengths_given && !packed ? lengths : nullptr, *o = packed ? offsets : nullptr;
        CHECK(amskv_cross_hold(&x, k.p, v.p, kh, vh, l, o, nullptr) == AMSKV_OK);
        CHECK(amskv_cross_export(&x, kh, vh, ko.p, vo.p, l, o, nullptr) == AMSKV_OK);
        for (int i = 0; i < total; ++i) {
          const int r = i / H, in = packed ? r >= 2 && r < 15 : !l || r % T < lengths[r / T];
          CHECK(get(ko.p + (size_t)i * 2 * D) == (in ? i : 0) && get(vo.p + (size_t)i * 2 * D) == (in ? (i | kValue) : 0));
        }
        std::free(kh), std::free(vh);
      }
}

static void refusals() {
  const int64_t far[] = {0, 1, -1, 64, 100, 1ll << 40, 1ll << 62, INT64_MAX, INT64_MIN};
  const int32_t sizes[] = {0, 1, 2, 33, 1 << 22, 1 << 26, INT32_MAX, -1, INT32_MIN};
  Buffer some(4096);
  void *p = some.p, *p2 = some.p + 64, *p3 = some.p + 128, *p4 = some.p + 192;
  for (int32_t b : sizes)
    for (int32_t h : sizes)
      for (int32_t kv : sizes)
        for (int64_t s : far)
          for (int64_t rows : {(int64_t)0, (int64_t)7, (int64_t)INT32_MAX, (int64_t)1 << 31, (int64_t)-1}) {
            const amskv_strides st{s, 64, 64};
            amskv_cross x{b, h, h, 64, AMSKV_DTYPE_BF16_KV4, 1, kv, rows, 0.f, st, st, st, st};
            uint64_t need = 0;
            const int32_t a = amskv_cross_held_bytes(&x, 0, &need), c = amskv_cross_held_bytes(&x, 1, &need);
            // (calls that would do something are left to held_tensors())
            const int32_t d = amskv_cross_hold(&x, nullptr, nullptr, p3, p4, nullptr, nullptr, nullptr);
            CHECK(d == AMSKV_ERR_INVALID_ARG || (a == AMSKV_OK && (b == 0 || h == 0 || kv == 0)));
            const int32_t e = amskv_cross_export(&x, p3, p4, nullptr, nullptr, nullptr, (const int32_t*)p, nullptr);
            CHECK(e == AMSKV_ERR_INVALID_ARG || (c == AMSKV_OK && (b == 0 || h == 0 || rows == 0)));
            const int32_t f = amskv_cross_workspace_bytes(&x, &need);
            const int32_t g = amskv_cross_attend(&x, p, p2, p3, p4, nullptr, rows > 0 ? (const int32_t*)p : nullptr, nullptr, 0, nullptr);
            CHECK(f == AMSKV_OK || g == AMSKV_ERR_INVALID_ARG);
          }
}

int main() {
  const std::vector<std::vector<int32_t>> hs = {{1, 2, 3, 4, 5, 6, 8, 10}, {4, 1, 5, 2, 3, 1, 1}, {1, 16, 17, 1, 4}},
                                          ws = {{1, 2, 3, 4, 5, 6, 8, 10}, {5, 1, 7, 3, 3, 2, 1}, {1, 1, 1, 31, 4}};
  for (size_t i = 0; i < hs.size(); ++i)
    for (int32_t layout : {AMSKV_LAYOUT_COMPACT, AMSKV_LAYOUT_PLANNED})
      for (int32_t borrow : {0, 1})
        for (bool packed : {false, true})
          for (bool turns : {false, true}) walk(hs[i], ws[i], i == 1 ? 128 : 64, layout, borrow, packed, turns);
  held_tensors();
  refusals();
  CHECK(g_takes > 0 && g_moves > 0 && g_attends > 0 && g_holds == 16 && g_crosses > 0);
  std::printf("%d launches that take, %d that move, %d attentions, %d of held tensors, %d check(s) failed\n", g_takes, g_moves, g_attends, g_holds,
              failures);
  return failures != 0;
}
