// Rotary positions: query and key rows turned by their positions.
//
// A thread has a piece of a row, W pairs of channels, in some of the row's heads: its cosines and sines are taken once
// and serve all of them from registers.  Every row is read once and written once: bound by memory where rows are many,
// 16384 rows of 40 + 8 heads of 128 in bf16 83.6 us, 403 MB at 4.8 TB/s of the 5.1 that a large copy reaches; 5001 rows of 32
// heads of 80 in fp32 26.9 us, 102 MB at 3.8, as long as a launch's start and end are in it.  80 rows take the 3.6 us of a
// launch behind another.
#include "rotary_dev.h"

namespace lvspec {

namespace {

constexpr int kRotaryThreads = 256;

template <class T, int W>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryCallArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kRotaryThreads + threadIdx.x;
  const int64_t t = i / a.pieces;
  if (t >= a.n_rows) return;
  const Piece e = piece_of((int)(i - t * a.pieces), W, a.rot.half, a.D, a.rot.interleaved != 0);
  if (!e.turned && a.in_place) return;
  const int h0 = blockIdx.y * a.heads, h1 = h0 + a.heads;
  Turn<W> turn;
  bool ready = false;
  rotate_heads<T, W>(a.q, a.rot, turn, ready, e, t, min(h0, a.q.H), min(h1, a.q.H));
  if (a.k.H > 0)
    rotate_heads<T, W>(a.k, a.rot, turn, ready, e, t, max(h0 - a.q.H, 0), min(max(h1 - a.q.H, 0), a.k.H));
}

template <class T, int W>
hipError_t launch(RotaryCallArgs a, hipStream_t stream) {
  a.pieces = pieces(W, a.rot.half, a.D);
  const int64_t threads = a.n_rows * a.pieces, all = a.q.H + a.k.H;
  // enough threads for the chip, then as many heads as there are for each
  int64_t groups = ((int64_t)kRotaryEnough + threads - 1) / threads;
  groups = groups < 1 ? 1 : groups > all ? all : groups;
  a.heads = (int)((all + groups - 1) / groups);
  groups = (all + a.heads - 1) / a.heads;
  rotary_kernel<T, W><<<dim3((unsigned)((threads + kRotaryThreads - 1) / kRotaryThreads), (unsigned)groups),
                        dim3(kRotaryThreads), 0, stream>>>(a);
  return hipGetLastError();
}

template <class T>
hipError_t launch_type(const RotaryCallArgs& a, hipStream_t stream) {
  // Four pairs of channels where halves and heads are whole numbers of four, or one by one (odd heads, and what is in
  // between).  One row, 40 + 8 heads of 128 in bf16: eight pairs 3.9 us, four 3.5, one 3.4; 1500 rows 10.6, 10.2 and 12.0;
  // 16384 rows 85.5, 83.6 and 83.3; 5001 rows of 32 heads of 80 in fp32: four 29.4, one 32.9.  Eight read 16 bytes at a
  // time and take twice the angles one behind the other, and twice the instructions to fetch.
  if (a.rot.half % 4 == 0 && a.D % 4 == 0) return launch<T, 4>(a, stream);
  return launch<T, 1>(a, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryCallArgs& a, int dtype, hipStream_t stream) {
  if (dtype == LVSPEC_F32) return launch_type<float>(a, stream);
  if (dtype == LVSPEC_F16) return launch_type<_Float16>(a, stream);
  return launch_type<__bf16>(a, stream);
}

}  // namespace lvspec
