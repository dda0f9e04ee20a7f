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
