// Rotary positions: query and key rows turned by their positions.
//
// A thread has a piece of a row, W pairs of channels, in some of the row's heads: its cosines and sines are taken once
// and serve all of them from registers.
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

template <class T, int MOST>
hipError_t launch_type(const RotaryCallArgs& a, hipStream_t stream) {
  // 16 bytes at a time where halves and heads are whole numbers of them, 8, or channel by channel
  if (a.rot.half % MOST == 0 && a.D % MOST == 0) return launch<T, MOST>(a, stream);
  if constexpr (MOST == 8)
    if (a.rot.half % 4 == 0 && a.D % 4 == 0) return launch<T, 4>(a, stream);
  return launch<T, 1>(a, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryCallArgs& a, int dtype, hipStream_t stream) {
  if (dtype == LVSPEC_F32) return launch_type<float, 4>(a, stream);
  if (dtype == LVSPEC_F16) return launch_type<_Float16, 8>(a, stream);
  return launch_type<__bf16, 8>(a, stream);
}

}  // namespace lvspec
