// Attention of up to 32 * kTeamWaves query rows over the keys of one (b,h) or (b, kv head), for kernels whose keys are not
// plain rows of a bf16 cache: codes in 8 bits (attend_codes.hip), rows whose number only the device knows (cross.hip).
//
// Formulation as in attend_bf16.hip: a wave owns 32 query rows and forms S^T = K Q^T and O^T += V^T P^T with
// v_mfma_f32_32x32x16_bf16, 32 keys at a time; a lane holds 16 keys of one query, so softmax sums are in-lane, and the
// probabilities already lie as the second product's B operand wants them; V is transposed by ds_read_b64_tr_b16.  One pass,
// with the reference of the exponentials lagging behind the running maximum by up to kMaxLag powers of two.
//
// A team of kTeamWaves waves shares tiles of keys (64, or 32 where a wave works alone).  A tile goes from memory to
// registers one tile ahead, is made bf16 there -- once for all waves that read it, which is why codes do not go to LDS as they
// are -- and is written to LDS when the tile before it is done: two tiles in LDS and one barrier a tile for a team, one
// tile and no barrier for a wave by itself.  kTeams teams of a workgroup hold the same rows and take every kTeams-th tile;
// their results meet in LDS at the end.
#pragma once
#include "codes.hpp"

#if defined(__HIPCC__)
namespace amskv {
namespace rows {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
#define AMSKV_ROWS_LDS __attribute__((address_space(3)))

// the reference of the exponentials may lag behind the maximum by this many powers of two: weights stay below 2^kMaxLag
constexpr float kMaxLag = 6.0f;

// Keys of a unit: n8 rows of codes, located by the segment table, then nx rows of bf16 at a fixed stride.
struct Keys {
  const unsigned char *k8, *v8, *k_exp, *v_exp;
  const char *kx, *vx;
  long long k_tok, v_tok;  // bytes
  int n8, nx;
};

// chunk c (16 bytes) of row `row` of a tile sits at chunk c ^ swizzle(row): fragment reads of 32 rows and transposing reads of
// 4 rows then spread over all banks
template <int D>
__device__ __forceinline__ constexpr int swizzle(int row) {
  return D == 64 ? (row & 7) : (((row & 3) << 1) | ((row >> 2) & 1) | (row & 8));
}

// v_max3_f32 written out (fmaxf canonicalises every operand first), and the wait states that it needs behind an 8-pass matrix
// instruction, which the compiler does not see into inline assembly for; acc is passed through so that it stays between the two
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ void settle_mfma(f32x16& acc) { asm volatile("s_nop 11" : "+v"(acc)); }

template <int D, int kTeamWaves, int kTeams, bool kEight>
struct Unit {
  static constexpr int RB = 2 * D, KS = D / 16, DB = D / 32, CPR = D / 8, CP8 = D / 16;
  static constexpr int kTile = kTeamWaves == 1 ? 32 : 64;
  static constexpr int kStages = kTeamWaves == 1 ? 1 : 2;
  static constexpr int kThreads = 64 * kTeamWaves;
  static constexpr int kItems = 2 * kTile * CPR / kThreads;  // 16-byte pieces of K and V a thread brings per tile, as bf16
  static constexpr int kItems8 = kItems / 2;                 // ... as codes
  static constexpr int kTensor = kTile * RB, kStage = 2 * kTensor, kTeamLds = kStages * kStage;
  static constexpr int kLds = kTeams * kTeamLds;
  static constexpr int kRows = 32 * kTeamWaves;
  static_assert(kTeams == 1 || kTeamLds >= kTeamWaves * 32 * D * 4, "a wave parks its O^T in its share of the tiles");

  struct Staged {
    u32x4 x[kItems];
    float scale[kEight ? kItems8 : 1];
  };

  // tiles [0, tiles8) are codes, [tiles8, tiles) bf16 rows
  __device__ static __forceinline__ int tiles8(const Keys& k) { return kEight ? (k.n8 + kTile - 1) / kTile : 0; }
  __device__ static __forceinline__ int tiles(const Keys& k) { return tiles8(k) + (k.nx + kTile - 1) / kTile; }
  __device__ static __forceinline__ int valid(const Keys& k, int it) {
    const int t8 = tiles8(k);
    return kEight && it < t8 ? min(kTile, k.n8 - it * kTile) : min(kTile, k.nx - (it - t8) * kTile);
  }

  // `member`: thread inside the team
  __device__ static __forceinline__ void load(Staged& s, const Keys& k, const SegTable& seg, int it, int member) {
    const int t8 = tiles8(k);
    if (kEight && it < t8) {
      const int first = it * kTile;
      int end = k.n8, delta = 0;  // of the segment that holds `first`
      for (int g = 0; g < seg.n; ++g)
        if (first >= seg.virt_start[g]) {
          end = seg.virt_start[g] + seg.len[g];
          delta = seg.phys_off[g] - seg.virt_start[g];
        }
      const bool whole = min(first + kTile, k.n8) <= end;  // uniform
#pragma unroll
      for (int i = 0; i < kItems8; ++i) {
        constexpr int kPer = kTile * CP8;
        const int at = i * kThreads + member;
        const bool is_v = kItems8 > 1 ? i >= kItems8 / 2 : __builtin_amdgcn_readfirstlane(at) >= kPer;
        const int idx = at & (kPer - 1), c = idx % CP8, j = min(first + idx / CP8, k.n8 - 1);
        int row = j + delta;
        if (!whole)
          for (int g = 0; g < seg.n; ++g)
            if (j >= seg.virt_start[g]) row = j + seg.phys_off[g] - seg.virt_start[g];
        s.x[i] = *reinterpret_cast<const u32x4*>((is_v ? k.v8 : k.k8) + ((long long)row * D + 16 * c));
        s.scale[i] = __int_as_float((int)(is_v ? k.v_exp : k.k_exp)[row / AMSKV_KV8_BLOCK] << 23);
      }
      return;
    }
    const int first = (it - t8) * kTile;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const bool is_v = i >= kItems / 2;
      const int idx = (i % (kItems / 2)) * kThreads + member, c = idx % CPR, j = min(first + idx / CPR, k.nx - 1);
      s.x[i] = *reinterpret_cast<const u32x4*>((is_v ? k.vx : k.kx) + ((long long)j * (is_v ? k.v_tok : k.k_tok) + 16 * c));
    }
  }

  // `lds`: byte offset of the tile.  (Offsets of a lane's pieces differ from the first one's by a constant and by the flip of
  // address bits that the swizzle of a constant number of rows makes -- swizzle() moves bits, so the swizzles of bits apart add up.)
  __device__ static __forceinline__ void store(const Staged& s, char* lds_all, int lds, const Keys& k, int it, int member) {
    if (kEight && it < tiles8(k)) {
      constexpr int kPer = kTile * CP8, kStep = kThreads / CP8 < kTile ? kThreads / CP8 : kTile;  // rows from a piece to the next
      const int first = member & (kPer - 1), row = first / CP8;
      const int at = lds + row * RB + 16 * ((2 * (first % CP8)) ^ swizzle<D>(row));
#pragma unroll
      for (int i = 0; i < kItems8; ++i) {
        const int n = kItems8 > 1 ? i % (kItems8 / 2) : 0;
        const bool is_v = kItems8 > 1 ? i >= kItems8 / 2 : __builtin_amdgcn_readfirstlane(member) >= kPer;
        u32x4 w[2];
        values16(s.x[i], s.scale[i], w);
        char* to = lds_all + ((at ^ (16 * swizzle<D>(n * kStep))) + (is_v ? kTensor : 0) + n * kStep * RB);
        char* to2 = lds_all + ((at ^ (16 * swizzle<D>(n * kStep)) ^ 16) + (is_v ? kTensor : 0) + n * kStep * RB);
        *reinterpret_cast<u32x4*>(to) = w[0];
        *reinterpret_cast<u32x4*>(to2) = w[1];
      }
      return;
    }
    constexpr int kStep = kThreads / CPR;
    const int row = member / CPR, at = lds + row * RB + 16 * ((member % CPR) ^ swizzle<D>(row));
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int n = i % (kItems / 2);
      *reinterpret_cast<u32x4*>(lds_all + ((at ^ (16 * swizzle<D>(n * kStep))) + (i >= kItems / 2 ? kTensor : 0) + n * kStep * RB)) = s.x[i];
    }
  }

  // What a wave has of its 32 rows: lane (r, h) row r; O^T rows 32d + 8(v/4) + 4h + v%4; sums over the lane's own keys.
  struct Result {
    f32x16 o[DB];
    float ref, sum;  // reference times c; sum of 2^(s c - ref)
  };

  __device__ static __forceinline__ void clear(Result& x) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int v = 0; v < 16; ++v) x.o[d][v] = 0.f;
    x.ref = -INFINITY;
    x.sum = 0.f;
  }

  // the keys of a tile in LDS
  __device__ static __forceinline__ void attend(Result& x, const bf16x8 (&qf)[KS], const char* lds_all, int lds, int n_valid, float c, int lane) {
    const int r = lane & 31, h = lane >> 5;
    const int tr_key = 4 * h + ((lane & 15) >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int ka = lds + r * RB + 16 * (h ^ swizzle<D>(r));
    const int va = lds + kTensor + tr_key * RB + 16 * ((tr_col >> 3) ^ swizzle<D>(tr_key)) + 2 * (tr_col & 7);
#pragma unroll 1
    for (int b = 0; b < kTile / 32; ++b) {
      if (b > 0 && 32 * b >= n_valid) break;  // uniform
      f32x16 s;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(lds_all + (ka ^ (32 * t)) + 32 * b * RB);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[t], s, 0, 0, 0);
      }
      if (n_valid < 32 * b + 32) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (32 * b + 8 * (v >> 2) + 4 * h + (v & 3) >= n_valid) s[v] = -INFINITY;
      }
      // the reference moves when a score of the block lies more than kMaxLag powers of two above it (from -inf on the first)
      settle_mfma(s);
      float m = max3(s[0], s[1], s[2]);
#pragma unroll
      for (int v = 3; v < 15; v += 2) m = max3(m, s[v], s[v + 1]);
      m = max3(m, s[15], s[15]);
      asm volatile("s_nop 1" : "+v"(m));  // (a lane swap reads what inline assembly wrote)
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(m), __float_as_int(m), false, false);
      const float full = fmaxf(__int_as_float(sw[0]), __int_as_float(sw[1])) * c;  // finite: a tile's first key is valid
      if (__builtin_amdgcn_ballot_w64(full - x.ref > kMaxLag) != 0) {
        const float ref = full - x.ref > kMaxLag ? full : x.ref;
        const float alpha = __builtin_amdgcn_exp2f(x.ref - ref);
        x.ref = ref;
        x.sum *= alpha;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int v = 0; v < 16; ++v) x.o[d][v] *= alpha;
      }
      bf16x8 pf[2];
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[v], c, -x.ref)), p1 = __builtin_amdgcn_exp2f(fmaf(s[v + 1], c, -x.ref));
        s0 += p0;
        s1 += p1;
        // bf16: the matrix cores' type; a weight is off by 2^-8 of itself at most, the sum stays in fp32
        pf[v >> 3][v & 7] = (__bf16)p0;
        pf[v >> 3][(v & 7) + 1] = (__bf16)p1;
      }
      x.sum += s0 + s1;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const bf16x4 lo = tr16(lds_all + (va ^ (64 * d)) + (32 * b + 16 * u) * RB);
          const bf16x4 hi = tr16(lds_all + (va ^ (64 * d) ^ (16 * swizzle<D>(8))) + (32 * b + 16 * u + 8) * RB);
          const bf16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          x.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pf[u], x.o[d], 0, 0, 0);
        }
    }
  }
  // within 16 lanes, lane i gives the address of 4 channels of key i/4 and receives 4 keys of channel i
  __device__ static __forceinline__ bf16x4 tr16(const char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((AMSKV_ROWS_LDS bf16x4*)(p));
  }

  // Tiles [from, to) of the keys.  Every wave of the workgroup calls this; one without rows only brings its part of the tiles.
  __device__ static __forceinline__ void walk(Result& x, const bf16x8 (&qf)[KS], char* lds_all, const Keys& k, const SegTable& seg, int from,
                                              int to, float c, bool active) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int team = wave / kTeamWaves, member = threadIdx.x - team * kThreads;
    const int lds = team * kTeamLds;
    Staged s;
    int it = from + team;
    if constexpr (kTeamWaves == 1) {
      if (it < to) load(s, k, seg, it, member);
      for (; it < to; it += kTeams) {
        store(s, lds_all, lds, k, it, member);
        if (it + kTeams < to) load(s, k, seg, it + kTeams, member);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();  // the rows written above by all lanes are read below
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        attend(x, qf, lds_all, lds, valid(k, it), c, lane);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();  // ... and overwritten by the next trip
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
    } else {
      const int trips = (to - from + kTeams - 1) / kTeams;  // of every team: the barriers are the workgroup's
      int stage = 0;
      if (it < to) {
        load(s, k, seg, it, member);
        store(s, lds_all, lds, k, it, member);
        if (it + kTeams < to) load(s, k, seg, it + kTeams, member);
      }
      __syncthreads();
      for (int n = 0; n < trips; ++n, it += kTeams) {
        if (active && it < to) attend(x, qf, lds_all, lds + stage, valid(k, it), c, lane);
        stage ^= kStage;
        if (it + kTeams < to) {
          store(s, lds_all, lds + stage, k, it + kTeams, member);
          if (it + 2 * kTeams < to) load(s, k, seg, it + 2 * kTeams, member);
        }
        __syncthreads();
      }
    }
  }

  // The results of all teams.  Afterwards a wave holds, of its 32 rows, chunks i (i % kTeams == team) of 8 channels: o[i/4][4 (i%4)
  // + ..]; ref, sum are the rows' (over all keys).  Every wave of the workgroup calls this.
  __device__ static __forceinline__ void meet(Result& x, char* lds_all) {
    x.sum += __shfl_xor(x.sum, 32, 64);
    if constexpr (kTeams > 1) {
      __shared__ float2 stat[kTeams * kTeamWaves][32];
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31;
      const int team = wave / kTeamWaves, rows_of = wave - team * kTeamWaves;
      constexpr int kPark = 32 * D * 4;
      if constexpr (kTeamWaves == 1) __builtin_amdgcn_wave_barrier();  // its own tile; a team's last barrier was behind its last tile
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = x.o[i >> 2][4 * (i & 3) + e];
        *reinterpret_cast<f32x4*>(lds_all + wave * kPark + i * 1024 + lane * 16) = y;
      }
      if (lane < 32) stat[wave][r] = make_float2(x.ref, x.sum);
      __syncthreads();
      float top = -INFINITY, total = 0.f, w[kTeams];
#pragma unroll
      for (int p = 0; p < kTeams; ++p) top = fmaxf(top, stat[p * kTeamWaves + rows_of][r].x);
#pragma unroll
      for (int p = 0; p < kTeams; ++p) {
        const float2 y = stat[p * kTeamWaves + rows_of][r];
        w[p] = y.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y.x - top);  // (a team without keys)
        total = fmaf(w[p], y.y, total);
      }
#pragma unroll
      for (int i0 = 0; i0 < 4 * DB; i0 += kTeams) {
        const char* from = lds_all + rows_of * kPark + (i0 + team) * 1024 + lane * 16;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < kTeams; ++p) {
          const f32x4 z = *reinterpret_cast<const f32x4*>(from + p * kTeamWaves * kPark);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = fmaf(w[p], z[e], y[e]);
        }
        // (kept at chunk i0, which every team has: register arrays are not indexed by the team)
#pragma unroll
        for (int e = 0; e < 4; ++e) x.o[i0 >> 2][4 * (i0 & 3) + e] = y[e];
      }
      x.ref = top;
      x.sum = total;
    }
  }

  // O of row r as bf16 at `dst` (the lanes of a row that is stored)
  __device__ static __forceinline__ void put(const Result& x, __bf16* dst, bool stored) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
    const float inv = x.sum > 0.f ? 1.0f / x.sum : 0.f;  // no keys: O = 0
    if constexpr (kTeams == 1) {
      // the lane halves hold alternate 8-byte pieces of a row; a lane swap per register pairs them up to 16-byte stores
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          bf16x4 wa, wb;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            wa[e] = (__bf16)(x.o[d][8 * k + e] * inv);
            wb[e] = (__bf16)(x.o[d][8 * k + 4 + e] * inv);
          }
          const u32x2 a = __builtin_bit_cast(u32x2, wa), b = __builtin_bit_cast(u32x2, wb);
          const auto s0 = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
          const auto s1 = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
          const u32x4 w = {s0[0], s1[0], s0[1], s1[1]};
          if (stored) *reinterpret_cast<u32x4*>(dst + 32 * d + 16 * k + 8 * h) = w;
        }
    } else {
      const int team = wave / kTeamWaves;
#pragma unroll
      for (int i0 = 0; i0 < 4 * DB; i0 += kTeams) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (__bf16)(x.o[i0 >> 2][4 * (i0 & 3) + e] * inv);
        if (stored) *reinterpret_cast<bf16x4*>(dst + 8 * (i0 + team) + 4 * h) = w;
      }
    }
  }

  // ... as fp32, not divided, at `dst`
  __device__ static __forceinline__ void put_partial(const Result& x, float* dst) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
    const int team = kTeams == 1 ? 0 : wave / kTeamWaves;
#pragma unroll
    for (int i0 = 0; i0 < 4 * DB; i0 += kTeams) {
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = x.o[i0 >> 2][4 * (i0 & 3) + e];
      *reinterpret_cast<f32x4*>(dst + 8 * (i0 + team) + 4 * h) = y;
    }
  }
};

}  // namespace rows
}  // namespace amskv
#endif
