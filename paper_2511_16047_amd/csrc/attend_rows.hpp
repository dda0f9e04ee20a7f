// Attention of up to 32 * kTeamWaves query rows over the keys of one (b,h) or (b, kv head), for kernels whose keys are not
// plain rows of a bf16 cache: codes in 8 or 4 bits (attend_codes.hip), rows whose number only the device knows (cross.hip).
//
// Formulation as in attend_bf16.hip: a wave owns 32 query rows and forms S^T = K Q^T and O^T += V^T P^T with
// v_mfma_f32_32x32x16_bf16, 32 keys at a time; a lane holds 16 keys of one query, so softmax sums are in-lane, and the
// probabilities already lie as the second product's B operand wants them; V is transposed by ds_read_b64_tr_b16.  One pass,
// with the reference of the exponentials lagging behind the running maximum by up to kMaxLag powers of two.
//
// A team of kTeamWaves waves shares tiles of keys (64, or 32 for teams of fewer than eight).  A tile goes from memory to
// registers one tile ahead, is made bf16 there -- once for all waves that read it, which is why codes do not go to LDS as they
// are -- and is written to LDS: a ring of four tiles and one barrier a tile for a team, which has the workgroup to itself.  A wave by
// itself (kTeamWaves 1) takes K straight to registers and has one tile of V in LDS, no barriers; kTeams such waves of a
// workgroup hold the same rows, take every kTeams-th tile, and their results meet in LDS at the end.
//
// Bound: where keys are many the matrix and vector pipes and what power leaves of them (head dim 128, 64 units 4096 x 6421, codes: 772
// to 800 us from card to card, 1.12 to 1.08 PFLOP/s; a large library product reaches 1.22;
// head dim 64, 3840 units 256 x 530: 190 to 195 us, 0.70 to 0.68 PFLOP/s, the exponentials' share is twice as large); where they are few, the
// latency of arguments, Q, the first tiles and O in turn: 3.5 to 7 us.
#pragma once
#include "codes.hpp"

#if defined(__HIPCC__)
namespace amskv {
namespace rows {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
#define AMSKV_ROWS_LDS __attribute__((address_space(3)))

// the reference of the exponentials may lag behind the maximum by this many powers of two; a lane's 16 new weights then sum to
// at most kTripSum = 16 * 2^kMaxLag, and a larger sum says that the reference has to move
constexpr float kMaxLag = 6.0f, kTripSum = 1024.0f;
// the reference before any key: finite, so that a block whose scores are all -inf (products beyond fp32) weighs nothing
constexpr float kNoKeys = -0x1.fffffep127f;

// Keys of a unit: n_codes rows of codes in 8 or 4 bits, located by the segment table, then n_rows rows of bf16 at a fixed stride.
struct Keys {
  const unsigned char *k_codes, *v_codes;
  const float *k_scale, *v_scale;  // 8 bits: of every 16 rows of codes
  const char *kx, *vx;
  long long k_tok, v_tok;  // bytes, below 2^24
  int n_codes, n_rows;
  const unsigned char *k_group, *v_group;  // 4 bits: of every 32 channels of a row
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

// kBits: of an element of the codes that keys may be (8 or 4), or 16: there are none
template <int D, int kTeamWaves, int kTeams, int kBits>
struct Unit {
  static constexpr bool kCoded = kBits != 16;
  static constexpr int RB = 2 * D, KS = D / 16, DB = D / 32, CPR = D / 8;
  static_assert(kTeamWaves == 1 || kTeams == 1, "a team of several waves has the workgroup to itself");
  static constexpr int kTile = kTeamWaves == 8 ? 64 : 32;
  static constexpr int kStages = 4;
  static constexpr bool kAlone = kTeamWaves == 8 && D == 128;  // 128 KB of LDS
  static constexpr int kThreads = 64 * kTeamWaves;
  // a piece of codes: 16 of 8 bits, or a quarter of a row of 4 bits (a wave by itself: 32)
  static constexpr int kPiece = kBits == 8 ? 16 : kTeamWaves == 1 ? 32 : D / 4, kPieces = D / kPiece;
  static constexpr int kItems = 2 * kTile * CPR / kThreads, kItemsC = kTeamWaves == 1 ? 2 * kTile * kPieces / 64 : kBits == 8 ? kItems / 2 : 1;
  // rows from a thread's piece to its next one of the same tensor; with one piece of codes, half of the waves bring K and half V
  static constexpr int kStep = kThreads / CPR, kStepC = kItemsC == 1 ? kTile : 2 * kStep;
  static constexpr int kRowsC = kItemsC == 1 ? 1 : kItemsC / 2;
  static constexpr int kTensor = kTile * RB, kStage = 2 * kTensor;
  // a wave by itself has a block of V there; afterwards teams park their O^T
  static constexpr int kTeamLds = kTeamWaves > 1 ? kStages * kStage : kTeams > 1 ? 32 * D * 4 : kTensor;
  static constexpr int kLds = kTeams * kTeamLds;
  static constexpr int kRows = 32 * kTeamWaves;
  // K fragments of the next block are asked for while the softmax of this one runs, where there are registers for them
  static constexpr bool kAhead = D == 128 || !kCoded;
  static_assert(kTeams == 1 || kTeamLds >= kTeamWaves * 32 * D * 4, "a wave parks its O^T in its share of the tiles");

  // A thread's part of a tile: 16 bytes each of 8 bf16 channels (kItems of them, the first half K) or pieces of codes (kItemsC) with
  // their powers of two (8 bits: as fp32; 4 bits: as bytes).
  typedef typename std::conditional<kBits == 4, unsigned, float>::type Scale;
  struct Staged {
    u32x4 x[kItems];
    Scale scale[kCoded ? kItemsC : 1];
  };
  // Where the pieces of the next tile lie: uniform bases of bf16 rows, and a row per piece.  Found at the top of a tile, so that the table walk at
  // a segment's end does not stand between matrix instructions.
  struct Aim {
    const char *kb, *vb;
    unsigned k_step, v_step;     // bytes from row to row
    unsigned row[kItems / 2];    // (of codes: the first kRowsC)
    int end = 0, delta = 0;      // codes: segment of the tile's first row, its end, from virtual row to row
  };
  // Kinds of tile a loop meets: kAny is found out (uniformly), kCodes and kRows are known.
  enum Kind { kAny, kCodes, kRowsOnly };
  template <Kind kKind>
  struct Of {
    static constexpr Kind value = kKind;
  };
  template <Kind kKind>
  __device__ static __forceinline__ bool is_codes(const Keys& k, int it) {
    return kCoded && (kKind == kCodes || (kKind == kAny && it < tiles_of_codes(k)));
  }

  // tiles [0, tiles_of_codes) are codes, [tiles_of_codes, tiles) bf16 rows
  __device__ static __forceinline__ int tiles_of_codes(const Keys& k) { return kCoded ? (k.n_codes + kTile - 1) / kTile : 0; }
  __device__ static __forceinline__ int tiles(const Keys& k) { return tiles_of_codes(k) + (k.n_rows + kTile - 1) / kTile; }
  __device__ static __forceinline__ int valid(const Keys& k, int it) {
    const int t8 = tiles_of_codes(k);
    return kCoded && it < t8 ? min(kTile, k.n_codes - it * kTile) : min(kTile, k.n_rows - (it - t8) * kTile);
  }

  // `member`: thread inside the team.  (Through an empty asm, so that what is derived from it is not kept in registers from
  // before the loop: this is where the widest forms would spill.)
  __device__ static __forceinline__ int fresh(int x) {
    if (D == 64 || kTeamWaves == 1) asm volatile("" : "+v"(x));
    return x;
  }
  // row inside a tile of a thread's first piece of codes, its channel group, and whether it is V's (one piece: by the wave)
  __device__ static __forceinline__ bool is_vC(int i, int member) {
    return kItemsC == 1 ? __builtin_amdgcn_readfirstlane(member) >= kThreads / 2 : i >= kItemsC / 2;
  }
  __device__ static __forceinline__ int memberC(int member) { return kItemsC == 1 ? member & (kThreads / 2 - 1) : member; }
  template <Kind kKind>
  __device__ static __forceinline__ void aim(Aim& a, const Keys& k, const SegTable& seg, int it, int member) {
    const bool codes = is_codes<kKind>(k, it);  // uniform
    const int first = (codes ? it : it - tiles_of_codes(k)) * kTile, last = (codes ? k.n_codes : k.n_rows) - 1;
    member = fresh(member);
    if (codes) {
      if (first >= a.end)  // a handful of times: the segment that holds `first`
        for (int g = 0; g < seg.n; ++g)
          if (first >= seg.virt_start[g]) {
            a.end = seg.virt_start[g] + seg.len[g];
            a.delta = seg.phys_off[g] - seg.virt_start[g];
          }
      const int row0 = first + memberC(member) / kPieces;
#pragma unroll
      for (int i = 0; i < kRowsC; ++i) a.row[i] = min(row0 + i * kStepC, last) + a.delta;
      if (min(first + kTile - 1, last) >= a.end) {  // rows of several segments
#pragma unroll
        for (int i = 0; i < kRowsC; ++i) {
          const int j = min(row0 + i * kStepC, last);
          for (int g = 0; g < seg.n; ++g)
            if (j >= seg.virt_start[g]) a.row[i] = j + seg.phys_off[g] - seg.virt_start[g];
        }
      }
    } else {
      a.kb = k.kx + first * k.k_tok;
      a.vb = k.vx + first * k.v_tok;
      a.k_step = (unsigned)k.k_tok;
      a.v_step = (unsigned)k.v_tok;
#pragma unroll
      for (int i = 0; i < kItems / 2; ++i) a.row[i] = min(member / CPR + i * kStep, last - first);
    }
  }
  // (offsets from the bases stay below 2^31: 64 rows at strides below 2^24 bytes, or a unit's codes)
  template <Kind kKind>
  __device__ static __forceinline__ void fetch(Staged& s, const Aim& a, const Keys& k, int it, int member) {
    member = fresh(member);
    if (is_codes<kKind>(k, it)) {
      const unsigned piece = memberC(member) % kPieces;
#pragma unroll
      for (int i = 0; i < kItemsC; ++i) {
        const bool v = is_vC(i, member);
        const unsigned row = a.row[kItemsC == 1 ? 0 : i % kRowsC];
        const unsigned char* from = (v ? k.v_codes : k.k_codes) + (row * (D * kBits / 8) + kPiece * kBits / 8 * piece);
        if constexpr (kBits == 4) {
          if constexpr (D == 64) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(from);
            s.x[i][0] = x[0];
            s.x[i][1] = x[1];
          } else {
            s.x[i] = *reinterpret_cast<const u32x4*>(from);
          }
          s.scale[i] = (v ? k.v_group : k.k_group)[row * (D / AMSKV_KV4_GROUP) + piece * kPiece / AMSKV_KV4_GROUP];
        } else {
          s.x[i] = *reinterpret_cast<const u32x4*>(from);
          s.scale[i] = (v ? k.v_scale : k.k_scale)[row / AMSKV_KV8_BLOCK];
        }
      }
      return;
    }
    const unsigned in_row = 16 * (member % CPR);
#pragma unroll
    for (int i = 0; i < kItems / 2; ++i) {
      s.x[i] = *reinterpret_cast<const u32x4*>(a.kb + (a.row[i] * a.k_step + in_row));
      s.x[kItems / 2 + i] = *reinterpret_cast<const u32x4*>(a.vb + (a.row[i] * a.v_step + in_row));
    }
  }
  template <Kind kKind>
  __device__ static __forceinline__ void load(Staged& s, Aim& a, const Keys& k, const SegTable& seg, int it, int member) {
    aim<kKind>(a, k, seg, it, member);
    fetch<kKind>(s, a, k, it, member);
  }

  // a piece of codes as bf16, 8 channels to a chunk; chunk j of it at `to` ^ 16 j
  __device__ static __forceinline__ void put_piece(char* lds, int to, const u32x4& x, Scale scale) {
    if constexpr (kBits == 4) {
      const float by = power_of_byte(scale);
#pragma unroll
      for (int j = 0; j < kPiece / 8; ++j) *reinterpret_cast<u32x4*>(lds + (to ^ (16 * j))) = values4(x[j], by);
    } else {
      *reinterpret_cast<u32x4*>(lds + to) = values8(u32x2{x[0], x[1]}, scale);
      *reinterpret_cast<u32x4*>(lds + (to ^ 16)) = values8(u32x2{x[2], x[3]}, scale);
    }
  }
  // `lds`: byte offset of the tile.  (Offsets of a lane's pieces differ from the first one's by a constant and by the flip of
  // address bits that the swizzle of a constant number of rows makes -- swizzle() moves bits, so the swizzles of bits apart add up.)
  template <Kind kKind>
  __device__ static __forceinline__ void store(const Staged& s, char* lds_all, int lds, const Keys& k, int it, int member) {
    member = fresh(member);
    if (is_codes<kKind>(k, it)) {
      const int m = memberC(member), row = m / kPieces, c = kPiece / 8 * (m % kPieces), at = lds + row * RB + 16 * (c ^ swizzle<D>(row));
#pragma unroll
      for (int i = 0; i < kItemsC; ++i) {
        const int n = kItemsC == 1 ? 0 : i % kRowsC;
        const int to = (at ^ (16 * swizzle<D>(n * kStepC))) + n * kStepC * RB;
        const int tensor = is_vC(i, member) ? kTensor : 0;
        put_piece(lds_all + tensor, to, s.x[i], s.scale[i]);
      }
      return;
    }
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
    x.ref = kNoKeys;
    x.sum = 0.f;
  }

  // byte offsets, inside a tile, of a lane's K fragment (t = 0) and V fragment (d, u = 0) of the tile's first 32 keys
  __device__ static __forceinline__ int k_lane(int lane) {
    const int r = lane & 31, h = lane >> 5;
    return r * RB + 16 * (h ^ swizzle<D>(r));
  }
  __device__ static __forceinline__ int v_lane(int lane) {
    const int key = 4 * (lane >> 5) + ((lane & 15) >> 2), col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    return kTensor + key * RB + 16 * ((col >> 3) ^ swizzle<D>(key)) + 2 * (col & 7);
  }

  // K fragments of 32 keys; `at`: k_lane + the block's offset
  __device__ static __forceinline__ void load_k(bf16x8 (&kf)[KS], const char* lds_all, int at) {
#pragma unroll
    for (int t = 0; t < KS; ++t) kf[t] = *reinterpret_cast<const bf16x8*>(lds_all + (at ^ (32 * t)));
  }
  // S^T of these keys
  __device__ static __forceinline__ f32x16 scores(const bf16x8 (&kf)[KS], const bf16x8 (&qf)[KS]) {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
    for (int t = 0; t < KS; ++t) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t], qf[t], s, 0, 0, 0);
    return s;
  }
  // only the first n_valid keys weigh anything
  __device__ static __forceinline__ void mask(f32x16& s, int n_valid, int lane) {
    if (n_valid < 32) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v >> 2) + 4 * (lane >> 5) + (v & 3) >= n_valid) s[v] = -INFINITY;
    }
  }
  // O^T += V^T P^T, keys 16u .. 16u + 15 of a block; `at`: v_lane + the block's offset
  __device__ static __forceinline__ void add_values(Result& x, const bf16x8& pf, const char* lds_all, int at, int u) {
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      const bf16x4 lo = tr16(lds_all + (at ^ (64 * d)) + 16 * u * RB);
      const bf16x4 hi = tr16(lds_all + (at ^ (64 * d) ^ (16 * swizzle<D>(8))) + (16 * u + 8) * RB);
      const bf16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      x.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pf, x.o[d], 0, 0, 0);
    }
  }
  // weights of keys 16u .. 16u + 15; returns the lane's sum.  bf16 is the matrix cores' type: a weight is off by 2^-8 of itself at
  // most.  The sum, in fp32, is over the weights as the second product multiplies them: two to an instruction, and the roundings
  // of numerator and denominator cancel in part.
  __device__ static __forceinline__ float weights(const f32x16& s, bf16x8& pf, float c, float ref, int u) {
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < 8; v += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[8 * u + v], c, -ref)), p1 = __builtin_amdgcn_exp2f(fmaf(s[8 * u + v + 1], c, -ref));
      const bf16x2 pk = {(__bf16)p0, (__bf16)p1};
      sum = __builtin_amdgcn_fdot2_f32_bf16(pk, ones, sum, false);
      pf[v] = pk[0];
      pf[v + 1] = pk[1];
    }
    return sum;
  }
  // the largest score of each query, over both lane halves, times c
  __device__ static __forceinline__ float largest(f32x16& s, float c) {
    settle_mfma(s);
    float m = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int v = 3; v < 15; v += 2) m = max3(m, s[v], s[v + 1]);
    m = max3(m, s[15], s[15]);
    asm volatile("s_nop 1" : "+v"(m));  // (a lane swap reads what inline assembly wrote)
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_int(m), __float_as_int(m), false, false);
    return fmaxf(__int_as_float(sw[0]), __int_as_float(sw[1])) * c;
  }
  __device__ static __forceinline__ void scale_by(Result& x, float alpha) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int v = 0; v < 16; ++v) x.o[d][v] *= alpha;
  }

  // A block from its scores on, start to end (a wave by itself: other waves of the SIMD fill its gaps).
  __device__ static __forceinline__ void whole_step(Result& x, f32x16& s, const char* lds_all, int v_at, int n_valid, float c, int lane) {
    mask(s, n_valid, lane);
    const float full = largest(s, c);
    if (__builtin_amdgcn_ballot_w64(full - x.ref > kMaxLag) != 0) {
      const float ref = full - x.ref > kMaxLag ? full : x.ref, alpha = __builtin_amdgcn_exp2f(x.ref - ref);
      x.ref = ref;
      x.sum *= alpha;
      scale_by(x, alpha);
    }
    bf16x8 pf[2];
    x.sum += weights(s, pf[0], c, x.ref, 0) + weights(s, pf[1], c, x.ref, 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) add_values(x, pf[u], lds_all, v_at, u);
  }

  // A block, one behind: its softmax on the vector ALUs runs beside the second product of the block before it, whose weights
  // wait in pf; the two share no data and stand in one basic block.  Weights are formed against the reference as it is; only
  // when a lane's sum shows that some score lay far above it is the maximum taken and the block's weights formed again, and O^T
  // follows the new reference at the top of the next step.
  //
  // Codes at head dim 128: the first block, which has none before it, is no question but weights of 0 for what lies in its
  // slot, and O^T follows at once: one basic block from K to the weights (both sides on one card: 64 units 2304 x 3925 363 -> 349 us, 32
  // units 209 -> 196, 4096 x 6421 808 -> 784).  Elsewhere walks are short for four products more, and their registers (head dim 64, 256 x 530 188 -> 193).
  static constexpr bool kOneBlock = D == 128 && kCoded;
  struct Behind {
    bf16x8 pf[2];
    float alpha;
    int block;  // byte offset of the block before (uniform)
    bool rescale, first;
  };
  // Where a team of eight has the CU to itself (head dim 128), the softmax goes before the score products of the wave it shares a SIMD
  // with, so that the two come to differ in what they do: 64 units 4096 x 6421 834 -> 802 us, before the one basic block above.  Waves of two teams on a SIMD hold each
  // other up instead: teams of four, 80 units 1024 x 2000, 121 -> 134, of eight at head dim 64, 150 units 1100 x 2000, 112 -> 125.
  // `between`, behind the score products, replaces kf by the next block's fragments: they arrive beside the softmax.
  template <bool kFull, class Between>
  __device__ static __forceinline__ void step(Result& x, Behind& w, bf16x8 (&kf)[KS], const bf16x8 (&qf)[KS], const char* lds_all, int ka, int va,
                                              int block, int n_valid, float c, int lane, Between between) {
    if (!kOneBlock && __builtin_expect(w.rescale, 0)) scale_by(x, w.alpha);
    if constexpr (!kAhead) load_k(kf, lds_all, block + ka);
    f32x16 s = scores(kf, qf);
    between();
    if constexpr (!kFull) mask(s, n_valid, lane);
    if constexpr (kAlone) __builtin_amdgcn_s_setprio(1);
    float sum = 0.f;
    bool trip = true;
    const bool first = !kOneBlock && w.first;
    if (!first) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        add_values(x, w.pf[u], lds_all, w.block + va, u);
        sum += weights(s, w.pf[u], c, x.ref, u);
      }
      trip = __builtin_amdgcn_ballot_w64(!(sum <= kTripSum)) != 0;
    }
    w.rescale = trip && !first;  // (nothing has been added up before the first block)
    if (__builtin_expect(trip, 0)) {
      const float full = largest(s, c), ref = full - x.ref > kMaxLag ? full : x.ref;
      w.alpha = __builtin_amdgcn_exp2f(x.ref - ref);
      x.ref = ref;
      x.sum *= w.alpha;
      if constexpr (kOneBlock) scale_by(x, w.alpha);
      sum = weights(s, w.pf[0], c, ref, 0);
      sum += weights(s, w.pf[1], c, ref, 1);
    }
    if constexpr (kAlone) __builtin_amdgcn_s_setprio(0);
    x.sum += sum;
    w.first = false;
    w.block = block;
  }
  __device__ static __forceinline__ void finish(Result& x, const Behind& w, const char* lds_all, int va) {
    if (!kOneBlock && w.rescale) scale_by(x, w.alpha);
#pragma unroll
    for (int u = 0; u < 2; ++u) add_values(x, w.pf[u], lds_all, w.block + va, u);
  }
  // within 16 lanes, lane i gives the address of 4 channels of key i/4 and receives 4 keys of channel i
  __device__ static __forceinline__ bf16x4 tr16(const char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((AMSKV_ROWS_LDS bf16x4*)(p));
  }

  // The wait for Q's loads, here: left to the compiler it stands in the loop, where it waits for the tile just asked for as well.
  __device__ static __forceinline__ void settle(const bf16x8 (&qf)[KS]) {
#pragma unroll
    for (int t = 0; t < KS; ++t) asm volatile("" ::"v"(qf[t]));
  }

  // A wave by itself: 32 keys at a time.  K goes from memory to the registers that the first product wants, lane (r, h) from key r.
  // Where keys may be codes its channels are h D/2 .. in order, so that 16 codes of a load are two fragments, and Q's fragments
  // are taken in the same order (q_at), which the sum over channels does not mind.  V goes through LDS, where it is transposed.
  struct Brought {
    u32x4 k[KS], v[kItems / 2];
    Scale k_scale[D / 64], v_scale[kCoded ? kItemsC / 2 : 1];  // (8 bits: K's row has one)
  };
  // byte offset in a row of Q (and of bf16 K, for a wave by itself) of fragment t
  static constexpr bool kHalves = kTeamWaves == 1 && kCoded;
  __device__ static __forceinline__ int q_at(int t, int h) { return kHalves ? h * D + 16 * t : 32 * t + 16 * h; }
  template <bool kCodesNow>
  __device__ static __forceinline__ void bring(Brought& n, const Keys& k, const SegTable& seg, int it, int lane) {
    const int r = lane & 31, h = lane >> 5;
    if constexpr (kCodesNow) {
      const int first = it * kTile, last = k.n_codes - 1;
      constexpr int kV = kItemsC / 2, kVStep = 64 / kPieces;
      // rows of the lane's pieces, K's and V's, in one walk of the table
      int row[kV + 1], at[kV + 1];
#pragma unroll
      for (int i = 0; i <= kV; ++i) row[i] = at[i] = min(first + (i < kV ? i * kVStep + lane / kPieces : r), last);
      for (int g = 0; g < seg.n; ++g) {
        const int from = seg.virt_start[g], by = seg.phys_off[g] - seg.virt_start[g];
#pragma unroll
        for (int i = 0; i <= kV; ++i) row[i] = at[i] >= from ? at[i] + by : row[i];
      }
      constexpr int kRowBytes = D * kBits / 8, kGroups = D / AMSKV_KV4_GROUP;
      const unsigned k_from = (unsigned)row[kV] * kRowBytes + h * (kRowBytes / 2);
#pragma unroll
      for (int i = 0; i < kRowBytes / 32; ++i) n.k[i] = *reinterpret_cast<const u32x4*>(k.k_codes + (k_from + 16 * i));
      if constexpr (kBits == 4) {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) n.k_scale[i] = k.k_group[(unsigned)row[kV] * kGroups + h * (kGroups / 2) + i];
      } else {
        n.k_scale[0] = k.k_scale[(unsigned)row[kV] / AMSKV_KV8_BLOCK];
      }
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        n.v[i] = *reinterpret_cast<const u32x4*>(k.v_codes + ((unsigned)row[i] * kRowBytes + 16 * (lane % kPieces)));
        if constexpr (kBits == 4)
          n.v_scale[i] = k.v_group[(unsigned)row[i] * kGroups + lane % kPieces];
        else
          n.v_scale[i] = k.v_scale[(unsigned)row[i] / AMSKV_KV8_BLOCK];
      }
    } else {
      const int first = (it - tiles_of_codes(k)) * kTile, last = k.n_rows - 1;
      const char *kb = k.kx + first * k.k_tok, *vb = k.vx + first * k.v_tok;
      const unsigned k_from = (unsigned)min(r, last - first) * (unsigned)k.k_tok;
#pragma unroll
      for (int i = 0; i < KS; ++i) n.k[i] = *reinterpret_cast<const u32x4*>(kb + (k_from + q_at(i, h)));
#pragma unroll
      for (int i = 0; i < kItems / 2; ++i)
        n.v[i] = *reinterpret_cast<const u32x4*>(vb + ((unsigned)min(i * (64 / CPR) + lane / CPR, last - first) * (unsigned)k.v_tok + 16 * (lane % CPR)));
    }
  }
  template <bool kCodesNow>
  __device__ static __forceinline__ void put_down(const Brought& n, bf16x8 (&kf)[KS], char* lds, int lane) {
    if constexpr (kCodesNow) {
      constexpr int kVStep = 64 / kPieces;
      const int row = lane / kPieces, c = kPiece / 8 * (lane % kPieces), at = row * RB + 16 * (c ^ swizzle<D>(row));
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        if constexpr (kBits == 4)
          kf[i] = __builtin_bit_cast(bf16x8, values4(n.k[i / 4][i % 4], power_of_byte(n.k_scale[i / 4])));
        else
          kf[i] = __builtin_bit_cast(bf16x8, values8(u32x2{n.k[i / 2][2 * (i & 1)], n.k[i / 2][2 * (i & 1) + 1]}, n.k_scale[0]));
      }
#pragma unroll
      for (int i = 0; i < kItemsC / 2; ++i) {
        const int to = (at ^ (16 * swizzle<D>(i * kVStep))) + i * kVStep * RB;
        put_piece(lds, to, n.v[i], n.v_scale[i]);
      }
    } else {
      constexpr int kVStep = 64 / CPR;
      const int row = lane / CPR, at = row * RB + 16 * ((lane % CPR) ^ swizzle<D>(row));
#pragma unroll
      for (int i = 0; i < KS; ++i) kf[i] = __builtin_bit_cast(bf16x8, n.k[i]);
#pragma unroll
      for (int i = 0; i < kItems / 2; ++i) *reinterpret_cast<u32x4*>(lds + ((at ^ (16 * swizzle<D>(i * kVStep))) + i * kVStep * RB)) = n.v[i];
    }
  }
  __device__ static __forceinline__ void alone(Result& x, const bf16x8 (&qf)[KS], char* lds, const Keys& k, const SegTable& seg, int it, int to,
                                               float c, int lane) {
    Brought n;
    const int t8 = min(tiles_of_codes(k), to), va = v_lane(lane) - kTensor;
    if (kCoded && it < t8) bring<kCoded>(n, k, seg, it, lane);
    else if (it < to) bring<false>(n, k, seg, it, lane);
    settle(qf);
    auto block = [&](auto now, auto next, bool more) {
      bf16x8 kf[KS];
      // to the score products before other waves' softmax: their next block is asked for behind them (us, head dim 128, 960 units 64 x
      // 130 18.2 -> 17.0, 64 units 256 x 530 14.6 -> 13.9; head dim 64, 3840 units 1 x 1 5.69 -> 5.55; shared by eight 9.3 -> 9.6)
      if constexpr (kTeams < 8) __builtin_amdgcn_s_setprio(1);
      put_down<decltype(now)::value == kCodes>(n, kf, lds, lane);
      f32x16 s = scores(kf, qf);
      if constexpr (kTeams < 8) __builtin_amdgcn_s_setprio(0);
      if (more) bring<decltype(next)::value == kCodes>(n, k, seg, it + kTeams, lane);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();  // the rows written above by all lanes are read below
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      whole_step(x, s, lds, va, valid(k, it), c, lane);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();  // ... and overwritten by the next block
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      it += kTeams;
    };
    if constexpr (kCoded) {
      while (it + kTeams < t8) block(Of<kCodes>{}, Of<kCodes>{}, true);
      if (it < t8) block(Of<kCodes>{}, Of<kRowsOnly>{}, it + kTeams < to);
    }
    while (it < to) block(Of<kRowsOnly>{}, Of<kRowsOnly>{}, it + kTeams < to);
  }

  // Tiles [from, to) of the keys.  Every wave of the workgroup calls this; one without rows only brings its part of the tiles.
  __device__ static __forceinline__ void walk(Result& x, const bf16x8 (&qf)[KS], char* lds_all, const Keys& k, const SegTable& seg, int from,
                                              int to, float c, bool active) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if constexpr (kTeamWaves == 1) {
      alone(x, qf, lds_all + wave * kTeamLds, k, seg, from + wave, to, c, lane);
    } else {
      const int member = threadIdx.x;
      int it = from;
      // A ring of four tiles: the one before, whose last V rows may still be to be multiplied (a tile of one block), the one in
      // use, the next one, whose first keys are asked for in the last step of this one, and the one that is being written.  One
      // barrier a tile, behind the score products of its last block.
      const int ka = k_lane(lane), va = v_lane(lane);
      Staged s;
      Aim to_come;
      if (it < to) load<kAny>(s, to_come, k, seg, it, member);
      {
        Staged s2;
        if (it + 1 < to) load<kAny>(s2, to_come, k, seg, it + 1, member);
        if (it < to) store<kAny>(s, lds_all, 0, k, it, member);
        if (it + 1 < to) store<kAny>(s2, lds_all, kStage, k, it + 1, member);
      }
      if (it + 2 < to) load<kAny>(s, to_come, k, seg, it + 2, member);
      settle(qf);
      __syncthreads();
      int slot = 0, next = kStage, after = 2 * kStage, spare = 3 * kStage;
      bf16x8 kf[KS];
      auto turn_over = [&](auto kind) {
        constexpr Kind kKind = decltype(kind)::value;  // of the tile to bring
        __syncthreads();
        if (it + 2 < to) {
          store<kAny>(s, lds_all, after, k, it + 2, member);
          if (it + 3 < to) fetch<kKind>(s, to_come, k, it + 3, member);
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
          if (it + 3 < to) aim<kAny>(to_come, k, seg, it + 3, member);
          turn_over(Of<kAny>{});
          next_tile();
        }
      } else if (it < to) {
        Behind w;
        w.rescale = false;
        w.first = true;
        w.alpha = 1.f;
        w.block = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) w.pf[u][e] = (__bf16)0.f;
        if constexpr (kAhead) load_k(kf, lds_all, slot + ka);
        // Tiles of which everything is known -- they are full, so are the next two, the one to bring exists and all are of one
        // kind -- have no branch between their instructions; the others are walked with every question asked.  Tiles of two blocks
        // are written in front of the barrier, beside the score products: the V rows that lay in the slot were multiplied in the
        // first step of the tile before this one, if that had two blocks.
        auto known = [&](auto kind, int end) {
          constexpr Kind kKind = decltype(kind)::value;
          while (it + 3 < end) {
            aim<kKind>(to_come, k, seg, it + 3, member);
            if constexpr (kTile == 64)
              step<true>(x, w, kf, qf, lds_all, ka, va, slot, 32, c, lane, [&]() {
                if constexpr (kAhead) load_k(kf, lds_all, slot + ka + 32 * RB);
              });
            step<true>(x, w, kf, qf, lds_all, ka, va, slot + (kTile - 32) * RB, 32, c, lane, [&]() {
              if constexpr (kTile == 32) __syncthreads();
              store<kKind>(s, lds_all, after, k, it + 2, member);
              fetch<kKind>(s, to_come, k, it + 3, member);
              if constexpr (kTile == 64) __syncthreads();
              if constexpr (kAhead) load_k(kf, lds_all, next + ka);
            });
            next_tile();
          }
        };
        const int t8 = min(tiles_of_codes(k), to);
        if constexpr (kCoded) known(Of<kCodes>{}, t8);
        while (it < to) {
          if (it - 1 >= t8 || (it >= t8 && it == from)) known(Of<kRowsOnly>{}, to);
          if (it + 3 < to) aim<kRowsOnly>(to_come, k, seg, it + 3, member);  // (codes: all brought above)
          int left = valid(k, it), done = 0;
          if (kTile == 64 && left > 32) {
            step<false>(x, w, kf, qf, lds_all, ka, va, slot, 32, c, lane, [&]() {
                if constexpr (kAhead) load_k(kf, lds_all, slot + ka + 32 * RB);
              });
            done = 32;
          }
          step<false>(x, w, kf, qf, lds_all, ka, va, slot + done * RB, left - done, c, lane, [&]() {
            turn_over(Of<kRowsOnly>{});
            if (kAhead && it + 1 < to) load_k(kf, lds_all, next + ka);
          });
          next_tile();
        }
        finish(x, w, lds_all, va);
      }
    }
  }

  // The results of all teams.  Afterwards a wave holds, of its 32 rows, chunks i (i % kTeams == wave) of 8 channels: o[i/4][4 (i%4)
  // + ..]; ref, sum are the rows' (over all keys).  Every wave of the workgroup calls this.
  __device__ static __forceinline__ void meet(Result& x, char* lds_all) {
    x.sum += __shfl_xor(x.sum, 32, 64);
    if constexpr (kTeams > 1) {
      __shared__ float2 stat[kTeams][32];
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31;
      constexpr int kPark = 32 * D * 4;  // where the wave's own tile was
      __builtin_amdgcn_wave_barrier();
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
      for (int p = 0; p < kTeams; ++p) top = fmaxf(top, stat[p][r].x);
#pragma unroll
      for (int p = 0; p < kTeams; ++p) {
        const float2 y = stat[p][r];
        w[p] = __builtin_amdgcn_exp2f(y.x - top);  // (a team without keys: of sums that are 0)
        total = fmaf(w[p], y.y, total);
      }
#pragma unroll
      for (int i0 = 0; i0 < 4 * DB; i0 += kTeams) {
        const char* from = lds_all + (i0 + wave) * 1024 + lane * 16;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < kTeams; ++p) {
          const f32x4 z = *reinterpret_cast<const f32x4*>(from + p * kPark);
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
#pragma unroll
      for (int i0 = 0; i0 < 4 * DB; i0 += kTeams) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (__bf16)(x.o[i0 >> 2][4 * (i0 & 3) + e] * inv);
        if (stored) *reinterpret_cast<bf16x4*>(dst + 8 * (i0 + wave) + 4 * h) = w;
      }
    }
  }

  // ... as fp32, not divided, at `dst`
  __device__ static __forceinline__ void put_partial(const Result& x, float* dst) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
    const int part = kTeams == 1 ? 0 : wave;
#pragma unroll
    for (int i0 = 0; i0 < 4 * DB; i0 += kTeams) {
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = x.o[i0 >> 2][4 * (i0 & 3) + e];
      *reinterpret_cast<f32x4*>(dst + 8 * (i0 + part) + 4 * h) = y;
    }
  }
};

}  // namespace rows
}  // namespace amskv
#endif
