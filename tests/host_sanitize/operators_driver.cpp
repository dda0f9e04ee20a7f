// Sanitizer driver for the host side of the rotary, 8-bit and cross-attention calls (csrc/amskv_api.cpp, csrc/operators_api.cpp): built by
// tests/test_host_sanitize_operators.py with -fsanitize=address,undefined.  The launchers are stubs that do to ordinary host memory what
// the kernels do to the device's, row by row, with a number for every row in place of its channels: scale and token, and whether it
// has been turned.  Arenas and tensors are exactly as large as the library asks for, so a region, slot or stride that is wrong
// ends in the sanitizer, and a row that is lost, in another's place, turned twice or not at all in a check.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
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

using amskv::Codes;
using amskv::RowMap;

[[noreturn]] static void unexpected(const char* what) {
  std::fprintf(stderr, "%s is no part of these walks\n", what);
  std::exit(2);
}

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

// what the next attention launch has to see, in order, and how many launches there were
static std::vector<int32_t> g_expect;
static int g_attends = 0, g_takes = 0, g_moves = 0;
static bool g_q_turned = false;

static void move_rows(char* base, int64_t cap, int row, int bh, const amskv::MoveList& mv) {
  for (int m = 0; m < mv.n; ++m) {
    CHECK(mv.dst[m] >= 0 && mv.dst[m] < mv.src[m] && mv.src[m] + mv.len[m] <= cap);
    CHECK(m == 0 || mv.src[m] >= mv.src[m - 1] + mv.len[m - 1]);
    for (int u = 0; u < bh; ++u)
      std::memmove(base + (u * cap + mv.dst[m]) * row, base + (u * cap + mv.src[m]) * row, (size_t)mv.len[m] * row);
  }
}

namespace amskv {
hipError_t launch_move_codes(const Codes& c, int bh, int head_dim, int64_t cap, const MoveList& mv, hipStream_t) {
  ++g_moves;
  MoveList blocks = mv;
  for (int m = 0; m < mv.n; ++m) {
    CHECK(mv.src[m] % 16 == 0 && mv.dst[m] % 16 == 0 && mv.len[m] % 16 == 0);
    blocks.src[m] /= 16, blocks.dst[m] /= 16, blocks.len[m] /= 16;
  }
  move_rows((char*)c.k, cap, head_dim, bh, mv);
  move_rows((char*)c.v, cap, head_dim, bh, mv);
  move_rows((char*)c.k_scale, cap / 16, 4, bh, blocks);
  move_rows((char*)c.v_scale, cap / 16, 4, bh, blocks);
  return hipSuccess;
}

hipError_t launch_take(const Take& t, hipStream_t st) {
  ++g_takes;
  const int bh = t.batch * t.heads, row = t.head_dim * (t.dtype == AMSKV_DTYPE_F32 ? 4 : 2);
  CHECK(t.tokens >= 1 && (t.table == nullptr || (t.rot_dim >= 16 && t.rot_dim <= t.head_dim && t.rot_dim % 16 == 0)));
  if (t.eight_bits) {
    CHECK(t.dtype == AMSKV_DTYPE_BF16 && t.cap_tokens % 16 == 0 && t.dst_new % 16 == 0 && t.dst_new + (t.tokens + 15) / 16 * 16 <= t.cap_tokens);
    if (t.moves && t.moves->n > 0) (void)launch_move_codes(t.codes, bh, t.head_dim, t.cap_tokens, *t.moves, st);
  }
  const void* src[3] = {t.k, t.v, t.q};
  void* dst[3] = {t.k_out, t.v_out, t.q_out};
  for (int i = 0; i < 3; ++i) {
    if (!src[i]) continue;
    for (int u = 0; u < bh; ++u)
      for (int j = 0; j < t.tokens; ++j) {
        const char* from = at(src[i], i == 2 ? t.q_map : t.kv_map, u, t.heads, j);
        int32_t id = get(from);
        CHECK((id & kTurned) == 0);
        if (t.table && i != 1) id |= kTurned;
        if (t.eight_bits && i < 2) {
          const int64_t to = u * t.cap_tokens + t.dst_new + j;
          put((i ? t.codes.v : t.codes.k) + to * t.head_dim, id, t.head_dim);
          (i ? t.codes.v_scale : t.codes.k_scale)[to / 16] = 1.f;
        } else {
          put(at(dst[i], i == 2 ? t.q_out_map : t.out_map, u, t.heads, j), id, row);
        }
      }
  }
  return hipSuccess;
}

// `row`: bytes of a cached row, `ext_row` of one of the caller's
static hipError_t attend(const void* q, void* o, char* kc, char* vc, int row, int ext_row, int bh, int t_q, int64_t cap, const SegTable& seg,
                         const ExtKV& ext, const CallerIo& io) {
  ++g_attends;
  CHECK(ext.alt_if == nullptr && seg.total == (int)g_expect.size());
  for (int u = 0; u < bh; ++u) {
    for (int t = 0; t < t_q; ++t) {
      CHECK(((get(at(q, io.q, u, io.heads, t)) & kTurned) != 0) == g_q_turned);
      put(at(o, io.o, u, io.heads, t), 0, ext_row);
    }
    for (int g = 0; g < seg.n; ++g)
      for (int i = 0; i < seg.len[g]; ++i) {
        const int j = seg.virt_start[g] + i;
        const bool outside = j >= seg.ext_start;
        if (!outside) CHECK(seg.phys_off[g] + i < cap);
        const int64_t in_cache = u * cap + seg.phys_off[g] + i;
        const int32_t k = get(outside ? at(ext.k, io.kv, u, io.heads, j - seg.ext_start) : kc + in_cache * row);
        const int32_t v = get(outside ? at(ext.v, io.kv, u, io.heads, j - seg.ext_start) : vc + in_cache * row);
        CHECK(j < (int)g_expect.size() && k == (g_expect[j] | (g_q_turned ? kTurned : 0)) && v == (g_expect[j] | kValue));
        const int to = write_back_row(ext, j, seg.total, seg.ext_start);
        if (to >= 0) {
          CHECK(to < cap && row == ext_row);
          put(kc + (u * cap + to) * row, k, row);
          put(vc + (u * cap + to) * row, v, row);
        }
      }
  }
  return hipSuccess;
}
hipError_t launch_attend_codes(const void* q, void* o, const Codes& c, int bh, int t_q, int head_dim, int64_t cap, const SegTable& seg,
                               const ExtKV& ext, const CallerIo& io, float, hipStream_t) {
  CHECK(ext.wb_from >= seg.total && ext.wb_head_end <= seg.ext_start);     // codes are written by the append alone
  for (int g = 0; g < seg.n; ++g) CHECK(seg.virt_start[g] >= seg.ext_start || seg.phys_off[g] % 16 == 0);
  for (int u = 0; u < bh; ++u)
    for (int g = 0; g < seg.n; ++g)
      for (int i = 0; i < seg.len[g] && seg.virt_start[g] < seg.ext_start; ++i) {
        const int64_t block = (u * cap + seg.phys_off[g] + i) / 16;
        CHECK(c.k_scale[block] == 1.f && c.v_scale[block] == 1.f);
      }
  return attend(q, o, (char*)c.k, (char*)c.v, head_dim, 2 * head_dim, bh, t_q, cap, seg, ext, io);
}
hipError_t launch_attend_bf16(const void* q, void* o, void* kc, void* vc, int bh, int t_q, int head_dim, int64_t cap, const SegTable& seg,
                              const ExtKV& ext, const CallerIo& io, float, hipStream_t) {
  return attend(q, o, (char*)kc, (char*)vc, 2 * head_dim, 2 * head_dim, bh, t_q, cap, seg, ext, io);
}
hipError_t launch_attend_f32(const void* q, void* o, void* kc, void* vc, int bh, int t_q, int head_dim, int64_t cap, const SegTable& seg,
                             const ExtKV& ext, const CallerIo& io, float, hipStream_t) {
  return attend(q, o, (char*)kc, (char*)vc, 4 * head_dim, 4 * head_dim, bh, t_q, cap, seg, ext, io);
}
hipError_t launch_roll(void* kc, void* vc, const void* k_new, const void* v_new, int bh, int row, int64_t cap, const MoveList& mv,
                       const NewRanges& nr, const RowMap& src, int heads, hipStream_t) {
  move_rows((char*)kc, cap, row, bh, mv);
  move_rows((char*)vc, cap, row, bh, mv);
  for (int r = 0; r < nr.n; ++r) {
    CHECK(nr.dst[r] >= 0 && nr.dst[r] + nr.len[r] <= cap);
    for (int u = 0; u < bh; ++u)
      for (int j = 0; j < nr.len[r]; ++j) {
        put((char*)kc + (u * cap + nr.dst[r] + j) * row, get(at(k_new, src, u, heads, nr.src_first[r] + j)), row);
        put((char*)vc + (u * cap + nr.dst[r] + j) * row, get(at(v_new, src, u, heads, nr.src_first[r] + j)), row);
      }
  }
  return hipSuccess;
}
hipError_t launch_append(void* kc, void* vc, const void* k_new, const void* v_new, int bh, int row, int64_t cap, const MoveList& mv, int t_new,
                         int dst_new, int src_first, const RowMap& src, int heads, hipStream_t st) {
  NewRanges nr{};
  if (k_new && t_new > 0) nr.n = 1, nr.src_first[0] = src_first, nr.dst[0] = dst_new, nr.len[0] = t_new;
  return launch_roll(kc, vc, k_new, v_new, bh, row, cap, mv, nr, src, heads, st);
}
static hipError_t export_rows(const char* kc, const char* vc, void* k_out, void* v_out, int bh, int row, int ext_row, int64_t cap,
                              const SegTable& seg, const ExtKV& ext, const RowMap& map, int heads) {
  for (int u = 0; u < bh; ++u)
    for (int g = 0; g < seg.n; ++g)
      for (int i = 0; i < seg.len[g]; ++i) {
        const int j = seg.virt_start[g] + i;
        const bool outside = j >= seg.ext_start;
        const int64_t from = u * cap + seg.phys_off[g] + i, to = ((int64_t)u * seg.total + j) * ext_row;
        put((char*)k_out + to, get(outside ? at(ext.k, map, u, heads, j - seg.ext_start) : kc + from * row), ext_row);
        put((char*)v_out + to, get(outside ? at(ext.v, map, u, heads, j - seg.ext_start) : vc + from * row), ext_row);
      }
  return hipSuccess;
}
hipError_t launch_export(const void* kc, const void* vc, void* k_out, void* v_out, int bh, int row, int64_t cap, const SegTable& seg,
                         const ExtKV& ext, const RowMap& map, int heads, hipStream_t) {
  return export_rows((const char*)kc, (const char*)vc, k_out, v_out, bh, row, row, cap, seg, ext, map, heads);
}
hipError_t launch_export_codes(const Codes& c, void* k_out, void* v_out, int bh, int head_dim, int64_t cap, const SegTable& seg,
                               const ExtKV& ext, const RowMap& map, int heads, hipStream_t) {
  return export_rows((const char*)c.k, (const char*)c.v, k_out, v_out, bh, head_dim, 2 * head_dim, cap, seg, ext, map, heads);
}

static int g_tables = 0, g_crosses = 0;
hipError_t launch_rope_table(const double* f, int pairs, int axes, double amplitude, const double*, int64_t n, float*, hipStream_t) {
  ++g_tables;
  CHECK(pairs >= 8 && pairs <= 64 && pairs % axes == 0 && n >= 1 && amplitude > 0);
  for (int i = 0; i < pairs / axes; ++i) CHECK(f[i] > 0 && std::isfinite(f[i]) && (i == 0 || f[i] <= f[i - 1] || f[0] < 1));
  return hipSuccess;
}
uint64_t cross_workspace_bytes(int batch, int heads, int kv_heads, int head_dim, int q_tokens, int kv_tokens) {
  if (batch == 0 || q_tokens == 0 || kv_tokens == 0) return 0;
  const rows::Division d = rows::divide(head_dim, (long long)batch * kv_heads, (long long)(heads / kv_heads) * q_tokens, kv_tokens);
  return d.splits == 1 ? 0 : 4096;
}
hipError_t launch_cross(const CrossCall& c, hipStream_t) {
  ++g_crosses;
  CHECK(c.batch >= 1 && c.heads >= 1 && c.q_tokens >= 1 && c.softmax_scale > 0 && !(c.lengths && c.offsets));
  CHECK(c.k_map.tok < (1 << 24) && c.v_map.tok < (1 << 24) && c.o_map.batch % 16 == 0 && c.q_map.head % 16 == 0);
  return hipSuccess;
}

hipError_t launch_similarity(const ScaleRef&, const ScaleRef&, int, int, int, int, int, int, int, int, float*, float*, hipStream_t) { unexpected(__func__); }
hipError_t launch_similarity_static(const ScaleRef&, const ScaleRef&, int, int, int, int, int, int, int, int, float*, hipStream_t) { unexpected(__func__); }
hipError_t launch_density(const void*, const void*, int, int, int, int, int, int64_t, const SegTable&, const ExtKV&, const CallerIo&, float, float*,
                          float*, hipStream_t) { unexpected(__func__); }
hipError_t launch_theta_flag(const float*, int, double, float, int32_t*, int32_t*, hipStream_t) { unexpected(__func__); }
bool attend_density_fused(int) { unexpected(__func__); }
bool attend_owns_unit(int head_dim, int t_q) { return t_q <= (head_dim == 64 ? 256 : 128); }
hipError_t launch_attend_density_bf16(const void*, void*, void*, void*, int, int, int, int, int64_t, const SegTable&, const ExtKV&, const CallerIo&,
                                      float, const GroupEnds&, float*, float*, hipStream_t) { unexpected(__func__); }
}  // namespace amskv
extern "C" hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t) { unexpected(__func__); }
extern "C" hipError_t hipStreamSynchronize(hipStream_t) { unexpected(__func__); }
extern "C" hipError_t hipHostMalloc(void** p, size_t n, unsigned int) { return (*p = std::calloc(1, n)) ? hipSuccess : hipErrorOutOfMemory; }
extern "C" hipError_t hipHostFree(void* p) { std::free(p); return hipSuccess; }
extern "C" hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { *e = reinterpret_cast<hipEvent_t>(std::malloc(1)); return hipSuccess; }
extern "C" hipError_t hipEventDestroy(hipEvent_t e) { std::free(e); return hipSuccess; }
extern "C" hipError_t hipEventRecord(hipEvent_t, hipStream_t) { unexpected(__func__); }
extern "C" hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }  // (destroy and reset of a token-mode cache)

struct Buffer {  // 16-byte aligned, nothing behind it
  char* p;
  explicit Buffer(size_t n, size_t align = 256) : p((char*)std::aligned_alloc(align, (n + align - 1) / align * align)) {}
  ~Buffer() { std::free(p); }
  Buffer(const Buffer&) = delete;
};

struct Kind {
  int32_t dtype, layout, borrow, fuse, mode;
  bool packed, turns, apart;
};

static void walk(const std::vector<int32_t>& hs, const std::vector<int32_t>& ws, int D, const Kind& kind) {
  const int n = (int)hs.size(), B = 2, H = 3, bytes = kind.dtype == AMSKV_DTYPE_F32 ? 4 : 2, row = D * bytes;
  const bool window = kind.mode == AMSKV_MODE_TOKEN_WINDOW;
  std::vector<amskv_layer_policy> pols;
  for (int c = 0; c < 4; ++c)
    for (int w = 0; w < 4; ++w) pols.push_back({c, w, 0});
  pols.push_back({0, 0, 1});
  std::vector<amskv_layer_budget> budgets = {{30, 30, 5, 0.f}, {7, 7, 0, 0.f}, {500, 500, 3, 0.f}};
  const int L = window ? (int)budgets.size() : (int)pols.size();
  amskv_schedule sc{n, hs.data(), ws.data(), B, kind.dtype};
  amskv_policy po{L, window ? nullptr : pols.data(), 0.f, kind.layout, kind.borrow, kind.fuse, kind.mode, window ? budgets.data() : nullptr};
  uint64_t need = 0;
  CHECK(amskv_cache_required_bytes(L, H, D, &sc, &po, &need) == AMSKV_OK && need > 0);
  Buffer arena(need);
  std::memset(arena.p, 0xff, need);
  amskv_cache* h = nullptr;
  CHECK(amskv_cache_create(L, H, D, &sc, &po, arena.p, need, &h) == AMSKV_OK && h);
  if (!h) return;
  if (kind.packed) {
    const int64_t width = H * D;
    CHECK(amskv_cache_set_io_layout(h, AMSKV_IO_TOKEN_MAJOR, kind.turns && kind.apart ? width : 3 * width, 3 * width, width) == AMSKV_OK);
  }
  const amskv_rope rope{D / 2, AMSKV_ROPE_HALF, 1, 1e4, 1, 0, 0, 0, 1};
  Buffer table(64);
  for (int image = 0; image < (kind.borrow ? 1 : 2); ++image) {
    CHECK(amskv_cache_reset(h) == AMSKV_OK);
    std::vector<std::vector<Buffer*>> alive(L);
    for (int s = 0; s < n; ++s)
      for (int l = 0; l < L; ++l) {
        const int T = hs[s] * ws[s];
        const size_t whole = (size_t)B * H * T * row;
        // [B][T][3][H][D], or three tensors [B][H][T][D]
        auto* data = new Buffer(3 * whole, 16);
        const RowMap in = kind.packed ? RowMap{(int64_t)T * 3 * H * row, row, (int64_t)3 * H * row} : RowMap{(int64_t)H * T * row, (int64_t)T * row, row};
        char* part[3];
        for (int i = 0; i < 3; ++i) {
          part[i] = data->p + (kind.packed ? (size_t)i * H * row : i * whole);
          for (int u = 0; u < B * H; ++u)
            for (int t = 0; t < T; ++t) put(at(part[i], in, u, H, t), id_of(s, t) | (i == 2 ? kValue : 0), row);
        }
        Buffer o(whole, 16), turned(whole, 16);
        g_expect.clear();
        if (window) {
          int32_t m = 0, scale[AMSKV_MAX_SCALES], first[AMSKV_MAX_SCALES], len[AMSKV_MAX_SCALES];
          int64_t off[AMSKV_MAX_SCALES];
          CHECK(amskv_cache_segments(h, l, &m, scale, first, off, len) == AMSKV_OK);
          for (int i = 0; i < m; ++i)
            for (int t = 0; t < len[i]; ++t) g_expect.push_back(id_of(scale[i], first[i] + t));
        } else {
          for (int k = 0; k < s; ++k)
            if (pols[l].keep_all || k < pols[l].n_condensed || s - k <= pols[l].window)
              for (int t = 0; t < hs[k] * ws[k]; ++t) g_expect.push_back(id_of(k, t));
        }
        for (int t = 0; t < T; ++t) g_expect.push_back(id_of(s, t));
        char* q = part[0];
        g_q_turned = kind.turns;
        if (kind.turns) {
          const bool apart = !kind.packed || kind.apart;
          CHECK(amskv_append_scale_rotary(h, l, s + 1, &rope, (float*)table.p, q, 0, apart ? turned.p : q, part[1], part[2], nullptr) != AMSKV_OK);
          CHECK(amskv_append_scale_rotary(h, l, s, &rope, (float*)table.p, q, kind.packed && kind.apart ? 3 * H * D : 0, apart ? turned.p : q, part[1],
                                          part[2], nullptr) == AMSKV_OK);
          if (apart) q = turned.p;
        } else {
          CHECK(amskv_append_scale(h, l, s, part[1], part[2], nullptr) == AMSKV_OK);
        }
        const int before = g_attends;
        if (kind.fuse == 0 || s % 3 != 1) {     // an attend that never comes leaves its copy to the next append
          CHECK(amskv_attend(h, l, s, q, o.p, nullptr) == AMSKV_OK);
          CHECK(g_attends == before + 1);
        }
        if (kind.dtype == AMSKV_DTYPE_BF16_KV8) CHECK(amskv_cache_capacity_tokens(h, l) % 16 == 0);
        if (!window) {
          Buffer ko(B * H * g_expect.size() * row, 16), vo(B * H * g_expect.size() * row, 16);
          CHECK(amskv_cache_export(h, l, ko.p, vo.p, nullptr) == AMSKV_OK);
          for (int u = 0; u < B * H; ++u)
            for (size_t j = 0; j < g_expect.size(); ++j) {
              CHECK(get(ko.p + (u * g_expect.size() + j) * row) == (g_expect[j] | (kind.turns ? kTurned : 0)));
              CHECK(get(vo.p + (u * g_expect.size() + j) * row) == (g_expect[j] | kValue));
            }
        }
        // the caller's tensors live until the next append on the layer
        alive[l].push_back(data);
        if (alive[l].size() > 1) delete alive[l].front(), alive[l].erase(alive[l].begin());
      }
    CHECK(amskv_cache_reset(h) == AMSKV_OK);
    for (auto& a : alive)
      for (Buffer* b : a) delete b;
  }
  amskv_cache_destroy(h);
}

static void refusals() {
  const double inf = std::numeric_limits<double>::infinity(), nan = std::nan("");
  const int64_t far[] = {0, 1, -1, 8, 64, 100, 1ll << 23, 1ll << 40, (1ll << 40) + 8, 1ll << 62, INT64_MAX, INT64_MIN};
  const int32_t sizes[] = {0, 1, 2, 33, 1 << 22, 1 << 24, INT32_MAX, -1, INT32_MIN};
  Buffer some(4096);
  void* p = some.p;
  int calls = 0, ok = 0;
  for (int32_t rot : {0, 16, 24, 64, 112, 128, 144, INT32_MIN, INT32_MAX})
    for (int32_t axes : {0, 1, 2, 3})
      for (double base : {1e4, 0.0, -1.0, inf, nan, 1.5})
        for (double factor : {1.0, 32.0, 0.5, inf, nan})
          for (double low : {0.0, 1.0, -1.0, nan})
            for (double high : {0.0, 32.0, inf, nan}) {
              const amskv_rope r{rot, AMSKV_ROPE_HALF, axes, base, factor, 4096.0, low, high, 1.1};
              ok += amskv_rope_table(&r, (const double*)p, 3, (float*)p, nullptr) == AMSKV_OK;
              ++calls;
            }
  CHECK(ok == amskv::g_tables && ok > 0 && ok < calls);
  for (int64_t n : {(int64_t)-1, (int64_t)0, (int64_t)1 << 25, ((int64_t)1 << 25) + 1, INT64_MAX}) {
    const amskv_rope r{64, AMSKV_ROPE_INTERLEAVED, 1, 1e4, 1, 0, 0, 0, 1};
    CHECK((amskv_rope_table(&r, (const double*)p, n, (float*)p, nullptr) == AMSKV_OK) == (n >= 0 && n <= (1 << 25)));
  }
  // turning: what the checks let through reaches the launcher; sizes are large only where they are refused or nothing is to be done
  const amskv_rope r{64, AMSKV_ROPE_HALF, 1, 1e4, 1, 0, 0, 0, 1};
  for (int32_t b : sizes)
    for (int32_t t : sizes)
      for (int64_t s0 : far)
        for (int64_t s1 : far) {
          if ((int64_t)b * t > 1 && b > 0 && t > 0 && (int64_t)b * t <= (1 << 29)) continue;
          const amskv_strides x{s0, 64, s1}, out{64 * (int64_t)(t > 0 ? t : 1), 64, 64};
          const int32_t rc = amskv_rotate(&r, AMSKV_DTYPE_BF16, 64, b, 1, t, (const float*)p, 0, 0, nullptr, &x, p, &out, nullptr);
          CHECK(rc == AMSKV_ERR_INVALID_ARG || (rc == AMSKV_OK && (b == 0 || t == 0)));
        }
  const int before = amskv::g_crosses;
  for (int32_t b : sizes)
    for (int32_t h : sizes)
      for (int32_t q : sizes)
        for (int32_t kv : sizes)
          for (int64_t s : far)
            for (int64_t rows : {(int64_t)0, (int64_t)7, (int64_t)INT32_MAX, (int64_t)1 << 31, (int64_t)-1}) {
              const amskv_strides st{s, 64, 64};
              amskv_cross x{b, h, h > 2 && h % 2 == 0 ? h / 2 : h, 64, AMSKV_DTYPE_BF16, q, kv, rows, 0.f, st, st, st, st};
              uint64_t need = 0;
              const int32_t a = amskv_cross_workspace_bytes(&x, &need);
              const int32_t c = amskv_cross_attend(&x, p, p, p, p, nullptr, rows > 0 ? (const int32_t*)p : nullptr, p, 4096, nullptr);
              CHECK(a == AMSKV_OK || c == AMSKV_ERR_INVALID_ARG);
              if (a == AMSKV_OK && (b == 0 || h == 0 || q == 0)) CHECK(need == 0);
            }
  CHECK(amskv::g_crosses > before);
  CHECK(amskv_cross_workspace_bytes(nullptr, nullptr) == AMSKV_ERR_INVALID_ARG);
  CHECK(amskv_cross_attend(nullptr, p, p, p, p, nullptr, nullptr, nullptr, 0, nullptr) == AMSKV_ERR_INVALID_ARG);
  CHECK(amskv_rotate(nullptr, AMSKV_DTYPE_BF16, 64, 1, 1, 1, (const float*)p, 0, 0, p, nullptr, p, nullptr, nullptr) == AMSKV_ERR_INVALID_ARG);
}

int main() {
  const std::vector<std::vector<int32_t>> hs = {{1, 2, 3, 4, 5, 6, 8, 10}, {4, 1, 5, 2, 3, 1, 1}, {1, 16, 17, 1, 4}},
                                          ws = {{1, 2, 3, 4, 5, 6, 8, 10}, {5, 1, 7, 3, 3, 2, 1}, {1, 1, 1, 31, 4}};
  for (size_t i = 0; i < hs.size(); ++i)
    for (int D : {i == 1 ? 128 : 64})
      for (int32_t dtype : {AMSKV_DTYPE_F32, AMSKV_DTYPE_BF16, AMSKV_DTYPE_BF16_KV8})
        for (bool packed : {false, true})
          for (int turns = 0; turns < (packed ? 3 : 2); ++turns) {      // 2: out of the projection into a tensor of their own
            for (int32_t layout : {AMSKV_LAYOUT_COMPACT, AMSKV_LAYOUT_PLANNED})
              for (int32_t borrow : {0, 1})
                for (int32_t fuse : {0, 1})
                  if (!(fuse && dtype == AMSKV_DTYPE_BF16_KV8))
                    walk(hs[i], ws[i], D, {dtype, layout, borrow, fuse, AMSKV_MODE_SCALE_WINDOW, packed, turns > 0, turns == 2});
            if (dtype != AMSKV_DTYPE_BF16_KV8)
              walk(hs[i], ws[i], D, {dtype, AMSKV_LAYOUT_COMPACT, 0, 0, AMSKV_MODE_TOKEN_WINDOW, packed, turns > 0, turns == 2});
          }
  CHECK(g_takes > 0 && g_moves > 0 && g_attends > 0);
  refusals();
  std::printf("%d launches that take, %d that move codes, %d attentions, %d check(s) failed\n", g_takes, g_moves, g_attends, failures);
  return failures != 0;
}
