// How the launches of take_kernels.hip that move an 8-bit cache's codes are divided: plain host code.  A launch has fewer than 2^32
// threads along an axis.
#pragma once

namespace amskv {

constexpr long long kMostThreads = 0xffffffffll;

// Threads of a workgroup, one to a (b,h) and tensor, that slides `blocks` blocks of 16 tokens: the smallest that takes them in one pass
// where there are many (b,h), else a large one; smaller ones again where the (b,h) are so many that large ones are no launch.
inline int move_threads(long long blocks, int head_dim, int bh) {
  int threads = blocks * head_dim <= 1024 && bh >= 128 ? 256 : 1024;
  while ((long long)bh * threads > kMostThreads) threads /= 2;   // (bh up to 2^24: 128 and more)
  return threads;
}

// Whether the workgroup that owns a (b,h) of a tensor slides its survivors and takes the new scale in one launch, or two launches share
// the work.  us an append, at once / in two, units x tokens, survivors as short.  D 64: 16 x 16 3.6 / 4.6, 16 x 256 4.9 / 5.1, 16 x 512 7.1 /
// 5.8, 256 x 64 4.8 / 6.4, 256 x 256 9.4 / 13.1, 256 x 512 16.3 / 20.4 (turned: 29.8 / 28.3), 960 x 16 9.1 / 6.8, 960 x 256 30.7 / 32.8.  D 128: 16 x
// 128 4.6 / 5.4, 16 x 256 6.2 / 6.1, 256 x 128 10.8 / 11.6, 256 x 256 20.3 / 20.2, 960 x 64 21.2 / 17.3.  So: where a workgroup to a
// (b,h) and tensor has few blocks to a wave, and there are no more of them than the chip holds at once.  And where few tokens slide:
// they are passes of 512 threads, of 1024 in a launch of their own.  16 units, 16 tokens behind survivors of 256 / 512 / 1024 / 4096, D 64: 4.6 / 5.6,
// 5.9 / 6.7, 8.6 / 8.2, 25.0 / 18.9; D 128: 6.2 / 7.1, 8.8 / 8.5, 14.3 / 12.0, 42.4 / 29.5; 256 units, D 128, 128 / 256 / 4096: 10.6 / 10.7, 12.5 /
// 12.1, 156 / 110.  (256 units, D 64, 1024 13.5 / 14.4.)
inline bool slides_at_once(int bh, long long tokens, long long blocks, int head_dim) {
  return bh <= 256 && tokens * head_dim <= 16384 && 16 * blocks * head_dim <= 32768;
}

// Workgroups of 256 threads, `parts` to a (b,h), for a read-back of `rows` rows: units of them along one axis of the grid, as many as it
// may have threads for, and `layers` of these along another.
struct ExportGrid {
  long long parts, units, layers;
};
inline ExportGrid export_grid(int bh, long long rows, int head_dim) {
  const long long parts = (rows * (head_dim / 16) + 255) / 256, most = kMostThreads / 256 / parts, units = bh < most ? bh : most;
  return {parts, units, (bh + units - 1) / units};
}

}  // namespace amskv
