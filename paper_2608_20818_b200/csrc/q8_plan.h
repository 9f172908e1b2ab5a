// Grids of the persistent and cooperative launches: arithmetic on sizes alone, so that a host without a device
// can check it.  `sms`: SMs of the device, a part of a B200's where it is divided up.
#pragma once

#include <algorithm>
#include <cstdint>

#ifdef __CUDACC__
#define PRM_HOST_DEVICE __host__ __device__
#else
#define PRM_HOST_DEVICE
#endif

namespace prm {

// SMs of a B200, one persistent CTA to each.  Launches use no more, for the scratch is sized by it.
constexpr int kRingBlocks = 148;

// Blocks of `threads` threads that an SM holds in the gradient's kernels without a ring: 768 threads at 80
// registers with one oct per thread, 512 at 128 with more.
PRM_HOST_DEVICE constexpr int grad_blocks(int threads, int nv = 1) {
  return threads <= 32 ? 8 : threads <= 128 ? 6 : threads <= 256 ? (nv == 1 ? 3 : 2) : 1;
}

// Lines of partial sums of grad_w: what the launches come to at most.
inline int grad_parts(int64_t rows, int64_t cols) {
  return (int)std::min<int64_t>(rows, kRingBlocks * (cols <= 256 ? 8 : cols <= 1024 ? 6 : cols <= 6144 ? 3 : 1));
}

// Threads per row and octs per thread for rows that start anywhere (no threads: too wide).
struct GradForm {
  int threads, nv;
};
inline GradForm grad_shifted_form(int64_t cols) {
  const int64_t c = cols + 7;             // a row may need one more oct
  return c <= 256 ? GradForm{32, 1} : c <= 1024 ? GradForm{128, 1} : c <= 2048 ? GradForm{256, 1}
       : c <= 4096 ? GradForm{256, 2} : c <= 6144 ? GradForm{256, 3} : c <= 8192 ? GradForm{512, 2}
       : c <= 16384 ? GradForm{1024, 2} : GradForm{0, 0};
}

// At least as many blocks as share the columns of grad_w at the end (1 x 4096, one block: 56 us).
inline int64_t grad_grid_for_columns(int64_t blocks, int64_t cols, int sms) {
  return std::max<int64_t>(blocks, std::min<int64_t>(sms, (cols + 31) / 32));
}
// A block per row and turn: two blocks per SM until they have six rows each, for a block more is a line more
// of partial sums (512 x 2041: 10.5 us, three per SM 12.9; 5000 x 1001: 24.5 us, two per SM 32).
inline int64_t grad_grid(int64_t rows, int64_t cols, int per_sm, int sms) {
  const int64_t want = std::min<int64_t>(rows, std::max<int64_t>(2 * sms, (rows + 47) / 48 * 8));
  return grad_grid_for_columns(std::min<int64_t>(want, (int64_t)per_sm * sms), cols, sms);
}
// The same for rows that start anywhere: a block that has several rows keeps the offset of its first one's
// start from an oct's boundary, so its rows lie a multiple of eight apart.  Rounded after all else.
inline int64_t grad_shifted_grid(int64_t rows, int64_t cols, GradForm form, int sms = kRingBlocks) {
  const int64_t grid = grad_grid(rows, cols, grad_blocks(form.threads, form.nv), sms);
  return grid >= rows ? grid : grid / 8 * 8;
}

// The streamed quantiser without codes by row: panels of up to 8192 columns, one block for each at least.
inline int stream_panels(int64_t cols) { return (int)((cols + 8191) / 8192); }
inline int stream_panel(int64_t cols, int panels) { return (int)((cols + 8 * panels - 1) / (8 * panels) * 8); }
inline bool stream_takes(int64_t cols, int sms) { return cols >= 256 && cols <= 32 * 8192 && stream_panels(cols) <= sms; }

// Blocks of a kernel on rings: as many as there are groups' worth of rows, a whole number for each panel.
inline int64_t ring_grid(int64_t rows, int rows_per_set, int groups, int panels, int sms) {
  const int64_t sets = (rows + rows_per_set - 1) / rows_per_set;
  return std::min<int64_t>(sms / panels, (sets + groups - 1) / groups) * panels;
}

}  // namespace prm
