// Attention of up to 32 * kTeamWaves query rows over keys in 4 bits, for teams of waves: attend_rows.hpp's formulation with K's codes as
// they are.
//
// The matrix cores take e2m1 numbers with a power of two to every 32 along the sum: S^T = K Q^T is formed by
// v_mfma_scale_f32_32x32x64_f8f6f4 from K's codes and powers straight out of LDS, a quarter of bf16's bytes there and no
// conversion.  Its other operand may have 6 bits without loss of speed (4 times bf16's rate; 8 bits: twice), so Q is held as the
// sum of two e2m3 numbers (4 significant bits each), made once for a workgroup: 32 channels with largest element m, 2^a the least power
// with m <= 7.5 * 2^a, are hi * 2^a + lo * 2^(a - 4), hi the number nearest to q * 2^-a, lo nearest to what is left.  What is left of a
// bf16 number of at least 2^a is a multiple of half of hi's step times 2^-3, which lo holds exactly; smaller elements are off by at most
// 2^(a - 8), 2^-9.9 of m.  Two products at 4 times the rate: half of the time of bf16's.  (e4m3 parts would be exact over a wider range
// and take bf16's time.)  V becomes bf16 on its way to LDS, once for all waves: weights in 6 bits would have to be split in two for
// every block, which takes the vector ALUs more (a conversion of 32 numbers 38 ns, back 33) than the matrix cores save.
//
// kExt: rows of bf16 may follow the codes (a scale that is read in place); they are walked as in attend_rows.hpp, with Q as it is.
#pragma once
#include "attend_rows.hpp"

#if defined(__HIPCC__)
namespace amskv {
namespace rows {

typedef unsigned u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Q of a lane: channels 64 c + 32 h .. + 31 of its row in two parts, and the bytes of their powers (0: hi, 1: lo).
template <int D>
struct QueryParts {
  u32x6 hi[D / 64], lo[D / 64];
  unsigned power[D / 64];
};
template <int D>
__device__ __forceinline__ void split_query(QueryParts<D>& q, const char* row, int h) {
  u32x4 raw[D / 64][4];
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[c][i] = *reinterpret_cast<const u32x4*>(row + 128 * c + 64 * h + 16 * i);
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    f32x16 even, odd;
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      even[i] = __builtin_bit_cast(float, raw[c][i / 4][i % 4] << 16);
      odd[i] = __builtin_bit_cast(float, raw[c][i / 4][i % 4] & 0xffff0000u);
      m = max3(m, __builtin_fabsf(even[i]), __builtin_fabsf(odd[i]));
    }
    const int bits = __builtin_bit_cast(int, m);  // 7.5 = 1.875 * 2^2
    const int a = min(max((bits >> 23) - 127 - 2 + ((bits & 0x7fffff) > 0x700000 ? 1 : 0), -120), 126);
    q.power[c] = (unsigned)(a + 127) | (unsigned)(a + 123) << 8;
    const float by = power_of_byte(a + 127);
    q.hi[c] = __builtin_bit_cast(u32x6, __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, by));
    const f32x32 held = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(q.hi[c], by);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      even[i] -= held[2 * i];
      odd[i] -= held[2 * i + 1];
    }
    q.lo[c] = __builtin_bit_cast(u32x6, __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, power_of_byte(a + 123)));
    // (the conversion writes its first results before it has read all operands, and the compiler lets the two overlap where the
    // operands are not read again: here they are)
    asm volatile("" ::"v"(even), "v"(odd));
  }
}

template <int D, int kTeamWaves, bool kExt>
struct FourBitTeam : Unit<D, kTeamWaves, 1, 4> {
  typedef Unit<D, kTeamWaves, 1, 4> Base;
  typedef typename Base::Result Result;
  typedef typename Base::Behind Behind;
  typedef typename Base::Staged Staged;
  typedef typename Base::Aim Aim;
  static constexpr int RB = Base::RB, KS = Base::KS, kTile = Base::kTile, kThreads = Base::kThreads;
  static constexpr int kRowK = D / 2;                   // bytes of a row of codes
  static constexpr int kPowers = kTile * kRowK;         // where the powers of a tile's K begin: 32 bytes to a row
  static constexpr int kOfK = kExt ? Base::kTensor : kPowers + 32 * kTile;
  static constexpr int kStage = kOfK + Base::kTensor;
  static constexpr int kLds = 4 * kStage;
  static_assert(kPowers + 32 * kTile <= kOfK && kThreads == 8 * kTile, "eight threads bring a row of K and of V");

  __device__ static __forceinline__ int tiles(const Keys& k) { return kExt ? Base::tiles(k) : Base::tiles_of_codes(k); }
  __device__ static __forceinline__ int valid(const Keys& k, int it) {
    return kExt ? Base::valid(k, it) : min(kTile, k.n_codes - it * kTile);
  }

  // ---- from memory to LDS.  A thread has an eighth of a row of K and the same of V: D / 8 channels each, and their powers.
  // Where chunk c (16 bytes) of a row of K's codes sits: reads of 8 rows then spread over all banks
  __device__ static __forceinline__ int chunk_of_k(int row, int c) { return D == 64 ? c ^ ((row >> 3) & 1) : c ^ ((row >> 2) & 3); }
  __device__ static __forceinline__ void aim_codes(Aim& a, const Keys& k, const SegTable& seg, int it, int member) {
    const int first = it * kTile, last = k.n_codes - 1;
    member = Base::fresh(member);
    if (first >= a.end)  // a handful of times: the segment that holds `first`
      for (int g = 0; g < seg.n; ++g)
        if (first >= seg.virt_start[g]) {
          a.end = seg.virt_start[g] + seg.len[g];
          a.delta = seg.phys_off[g] - seg.virt_start[g];
        }
    const int j = min(first + member / 8, last);
    a.row[0] = j + a.delta;
    if (min(first + kTile - 1, last) >= a.end)  // rows of several segments
      for (int g = 0; g < seg.n; ++g)
        if (j >= seg.virt_start[g]) a.row[0] = j + seg.phys_off[g] - seg.virt_start[g];
  }
  // (x[0]: K's codes, V's; x[1]: the powers of K's row, of V's piece)
  __device__ static __forceinline__ void fetch_codes(Staged& s, const Aim& a, const Keys& k, int member) {
    member = Base::fresh(member);
    const unsigned piece = member % 8, at = a.row[0] * kRowK + piece * (D / 16), group = a.row[0] * (D / AMSKV_KV4_GROUP);
    if constexpr (D == 64) {
      s.x[0][0] = *reinterpret_cast<const unsigned*>(k.k_codes + at);
      s.x[0][2] = *reinterpret_cast<const unsigned*>(k.v_codes + at);
      s.x[1][0] = *reinterpret_cast<const unsigned short*>(k.k_group + group);
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(k.k_codes + at), y = *reinterpret_cast<const u32x2*>(k.v_codes + at);
      s.x[0] = u32x4{x[0], x[1], y[0], y[1]};
      s.x[1][0] = *reinterpret_cast<const unsigned*>(k.k_group + group);
    }
    s.x[1][1] = k.v_group[group + piece * (D / 8) / AMSKV_KV4_GROUP];
  }
  __device__ static __forceinline__ void store_codes(const Staged& s, char* lds_all, int lds, int member) {
    member = Base::fresh(member);
    const int row = member / 8, piece = member % 8;
    char* tile = lds_all + lds;
    *reinterpret_cast<unsigned*>(tile + kPowers + 32 * row + 4 * piece) = s.x[1][0];  // (eight times: no lane stands aside)
    const float by = power_of_byte(s.x[1][1]);
    if constexpr (D == 64) {
      *reinterpret_cast<unsigned*>(tile + row * kRowK + 16 * chunk_of_k(row, piece / 4) + 4 * (piece % 4)) = s.x[0][0];
      *reinterpret_cast<u32x4*>(tile + kOfK + row * RB + 16 * (piece ^ swizzle<D>(row))) = values4(s.x[0][2], by);
    } else {
      *reinterpret_cast<u32x2*>(tile + row * kRowK + 16 * chunk_of_k(row, piece / 2) + 8 * (piece % 2)) = u32x2{s.x[0][0], s.x[0][1]};
      char* v = tile + kOfK + row * RB;
      const int at = 16 * ((2 * piece) ^ swizzle<D>(row));
      *reinterpret_cast<u32x4*>(v + at) = values4(s.x[0][2], by);
      *reinterpret_cast<u32x4*>(v + (at ^ 16)) = values4(s.x[0][3], by);
    }
  }
  // of a tile of either kind (found out uniformly)
  __device__ static __forceinline__ void aim_any(Aim& a, const Keys& k, const SegTable& seg, int it, int member) {
    if (!kExt || it < Base::tiles_of_codes(k))
      aim_codes(a, k, seg, it, member);
    else
      Base::template aim<Base::kRowsOnly>(a, k, seg, it, member);
  }
  __device__ static __forceinline__ void fetch_any(Staged& s, const Aim& a, const Keys& k, int it, int member) {
    if (!kExt || it < Base::tiles_of_codes(k))
      fetch_codes(s, a, k, member);
    else
      Base::template fetch<Base::kRowsOnly>(s, a, k, it, member);
  }
  __device__ static __forceinline__ void store_any(const Staged& s, char* lds_all, int lds, const Keys& k, int it, int member) {
    if (!kExt || it < Base::tiles_of_codes(k))
      store_codes(s, lds_all, lds, member);
    else
      Base::template store<Base::kRowsOnly>(s, lds_all, lds, k, it, member);
  }

  // ---- scores.  K of 32 keys: lane (r, h) has channels 64 c + 32 h .. + 31 of key r.
  struct KeyCodes {
    u32x4 code[D / 64];
    unsigned powers;  // c's in byte 2 c
  };
  __device__ static __forceinline__ int k_lane4(int lane) { return (lane & 31) * kRowK + 16 * chunk_of_k(lane & 31, lane >> 5); }
  // block: of 32 keys inside the tile at `slot`
  __device__ static __forceinline__ void load_codes(KeyCodes& kc, const char* lds_all, int slot, int block, int ka, int lane) {
    const int r = lane & 31;
    const char* at = lds_all + slot + block * 32 * kRowK;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) kc.code[c] = *reinterpret_cast<const u32x4*>(at + (ka ^ (32 * c)));
    kc.powers = *reinterpret_cast<const unsigned*>(lds_all + slot + kPowers + 32 * 32 * block + 32 * r + 4 * (r >> 3)) >> (8 * (lane >> 5));
  }
  __device__ static __forceinline__ f32x16 product(const KeyCodes& kc, const QueryParts<D>& q) {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
    auto wide4 = [](const u32x4& x) { return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}; };
    auto wide6 = [](const u32x6& x) { return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0}; };
    // (4: e2m1, 2: e2m3; the bytes of the powers are picked by constants)
    s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide4(kc.code[0]), wide6(q.lo[0]), s, 4, 2, 0, kc.powers, 1, q.power[0]);
    s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide4(kc.code[0]), wide6(q.hi[0]), s, 4, 2, 0, kc.powers, 0, q.power[0]);
    if constexpr (D == 128) {
      s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide4(kc.code[1]), wide6(q.lo[1]), s, 4, 2, 2, kc.powers, 1, q.power[1]);
      s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide4(kc.code[1]), wide6(q.hi[1]), s, 4, 2, 2, kc.powers, 0, q.power[1]);
    }
    return s;
  }
  template <bool kFull, class Between>
  __device__ static __forceinline__ void step_codes(Result& x, Behind& w, KeyCodes& kc, const QueryParts<D>& q, const char* lds_all, int va, int block,
                                                    int n_valid, float c, int lane, Between between) {
    if (!Base::kOneBlock && __builtin_expect(w.rescale, 0)) Base::scale_by(x, w.alpha);
    f32x16 s = product(kc, q);
    between();
    Base::template behind_scores<kFull>(x, w, s, lds_all, va, block, n_valid, c, lane);
  }

  // Tiles [from, to) of the keys, as Unit::walk.  q_row(): the lane's row of Q, for rows of bf16 (asked for when it comes to them).
  template <class QueryRow>
  __device__ static __forceinline__ void walk(Result& x, const QueryParts<D>& q, QueryRow q_row, char* lds_all, const Keys& k, const SegTable& seg,
                                              int from, int to, float c, bool active) {
    const int lane = threadIdx.x & 63, member = threadIdx.x;
    const int t8 = min(Base::tiles_of_codes(k), to);
    int it = from;
    const int ka = k_lane4(lane), va = Base::v_lane(lane) - Base::kTensor + kOfK;
    Staged s;
    Aim to_come;
    auto load = [&](Staged& y, int i) {
      aim_any(to_come, k, seg, i, member);
      fetch_any(y, to_come, k, i, member);
    };
    if (it < to) load(s, it);
    {
      Staged s2;
      if (it + 1 < to) load(s2, it + 1);
      if (it < to) store_any(s, lds_all, 0, k, it, member);
      if (it + 1 < to) store_any(s2, lds_all, kStage, k, it + 1, member);
    }
    if (it + 2 < to) load(s, it + 2);
    __syncthreads();
    int slot = 0, next = kStage, after = 2 * kStage, spare = 3 * kStage;
    auto turn_over = [&]() {
      __syncthreads();
      if (it + 2 < to) {
        store_any(s, lds_all, after, k, it + 2, member);
        if (it + 3 < to) fetch_any(s, to_come, k, it + 3, member);
      }
    };
    auto next_tile = [&]() {
      const int freed = slot;
      slot = next;
      next = after;
      after = spare;
      spare = freed;
      ++it;
    };
    if (!active) {  // a wave without rows only brings its part of the tiles
      while (it < to) {
        if (it + 3 < to) aim_any(to_come, k, seg, it + 3, member);
        turn_over();
        next_tile();
      }
      return;
    }
    if (it >= to) return;
    Behind w;
    w.rescale = false;
    w.first = true;
    w.alpha = 1.f;
    w.block = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) w.pf[u][e] = (__bf16)0.f;
    KeyCodes kc;
    if (it < t8) load_codes(kc, lds_all, slot, 0, ka, lane);
    // tiles of which everything is known have no branch between their instructions
    while (it + 3 < t8) {
      aim_codes(to_come, k, seg, it + 3, member);
      if constexpr (kTile == 64)
        step_codes<true>(x, w, kc, q, lds_all, va, slot, 32, c, lane, [&]() { load_codes(kc, lds_all, slot, 1, ka, lane); });
      step_codes<true>(x, w, kc, q, lds_all, va, slot + (kTile - 32) * RB, 32, c, lane, [&]() {
        if constexpr (kTile == 32) __syncthreads();
        store_codes(s, lds_all, after, member);
        fetch_codes(s, to_come, k, member);
        if constexpr (kTile == 64) __syncthreads();
        load_codes(kc, lds_all, next, 0, ka, lane);
      });
      next_tile();
    }
    while (it < t8) {
      if (it + 3 < to) aim_any(to_come, k, seg, it + 3, member);
      int left = valid(k, it), done = 0;
      if (kTile == 64 && left > 32) {
        step_codes<true>(x, w, kc, q, lds_all, va, slot, 32, c, lane, [&]() { load_codes(kc, lds_all, slot, 1, ka, lane); });
        done = 32;
      }
      step_codes<false>(x, w, kc, q, lds_all, va, slot + done * RB, left - done, c, lane, [&]() {
        turn_over();
        if (it + 1 < t8) load_codes(kc, lds_all, next, 0, ka, lane);
      });
      next_tile();
    }
    if constexpr (kExt) {
      if (it < to) {
        bf16x8 qf[KS], kf[KS];
        const char* row = q_row();
#pragma unroll
        for (int t = 0; t < KS; ++t) qf[t] = *reinterpret_cast<const bf16x8*>(row + 32 * t + 16 * (lane >> 5));
        Base::settle(qf);
        const int kr = Base::k_lane(lane);
        constexpr bool kAhead = Base::kAhead;
        if constexpr (kAhead) Base::load_k(kf, lds_all, slot + kr);
        while (it < to) {
          while (it + 3 < to && (it - 1 >= t8 || it == from)) {  // (Unit::walk: behind a tile of two blocks)
            Base::template aim<Base::kRowsOnly>(to_come, k, seg, it + 3, member);
            if constexpr (kTile == 64)
              Base::template step<true>(x, w, kf, qf, lds_all, kr, va, slot, 32, c, lane, [&]() {
                if constexpr (kAhead) Base::load_k(kf, lds_all, slot + kr + 32 * RB);
              });
            Base::template step<true>(x, w, kf, qf, lds_all, kr, va, slot + (kTile - 32) * RB, 32, c, lane, [&]() {
              if constexpr (kTile == 32) __syncthreads();
              Base::template store<Base::kRowsOnly>(s, lds_all, after, k, it + 2, member);
              Base::template fetch<Base::kRowsOnly>(s, to_come, k, it + 3, member);
              if constexpr (kTile == 64) __syncthreads();
              if constexpr (kAhead) Base::load_k(kf, lds_all, next + kr);
            });
            next_tile();
          }
          if (it + 3 < to) Base::template aim<Base::kRowsOnly>(to_come, k, seg, it + 3, member);
          int left = valid(k, it), done = 0;
          if (kTile == 64 && left > 32) {
            Base::template step<false>(x, w, kf, qf, lds_all, kr, va, slot, 32, c, lane, [&]() {
              if constexpr (kAhead) Base::load_k(kf, lds_all, slot + kr + 32 * RB);
            });
            done = 32;
          }
          Base::template step<false>(x, w, kf, qf, lds_all, kr, va, slot + done * RB, left - done, c, lane, [&]() {
            __syncthreads();
            if (it + 2 < to) {
              Base::template store<Base::kRowsOnly>(s, lds_all, after, k, it + 2, member);
              if (it + 3 < to) Base::template fetch<Base::kRowsOnly>(s, to_come, k, it + 3, member);
            }
            if (kAhead && it + 1 < to) Base::load_k(kf, lds_all, next + kr);
          });
          next_tile();
        }
      }
    }
    Base::finish(x, w, lds_all, va);
  }
};

}  // namespace rows
}  // namespace amskv
#endif
