// The table of rotary angles (ptc_rope_table).
#include <cmath>

#include "ptc_rope.cuh"

namespace ptc {
namespace {

// Angles are kept as fractions of a turn in 64-bit integers: a frequency f is
// floor(f / 2 pi * 2^64) of them a position (its error, 2^-52 of it and 2^-64 of a
// turn, grows with the position: at angles of 2^24 it is below 2^-30 of a turn), a
// position's angle the product modulo 2^64, exact.  The two upper bits after rounding to the nearest quarter are the
// quarter; the rest, within an eighth of a turn, becomes 32-bit radians with a
// relative error of 2^-23, and the Taylor series about 0 give both functions (next
// terms: 1.7e-9 and 2.4e-9).  A thread has a frequency and goes down the positions, a
// warp writes 128 bytes in a row.  131,072 positions of 64 frequencies, 67 MB, take
// 13.4 us, 5.0 TB/s: some 45 instructions an angle.
constexpr int kTableThreads = 256;

struct TableArgs {
  const double* freq;
  float* table;
  uint32_t n_freq, n_pos;
  float factor;
};

__global__ void __launch_bounds__(kTableThreads) k_rope_table(TableArgs a) {
  grid_dep_sync();
  __shared__ uint64_t s_step[PTC_MAX_HEAD_DIM / 2];
  __shared__ bool s_fine[PTC_MAX_HEAD_DIM / 2];
  const uint32_t F = a.n_freq, across = kTableThreads / F, i = threadIdx.x % F, row = threadIdx.x / F;
  // The fraction of a turn, once a frequency: 64-bit numbers are slow here (a
  // division by 2 pi in every thread took as long as all the rest).
  if (threadIdx.x < F) {
    double t = a.freq[threadIdx.x] * 0.15915494309189533577;
    t -= floor(t);
    const bool fine = t >= 0.0 && t <= 1.0;  // not of an infinity or NaN
    s_fine[threadIdx.x] = fine;
    s_step[threadIdx.x] = fine && t < 1.0 ? (uint64_t)(t * 18446744073709551616.0) : 0;
  }
  __syncthreads();
  if (row >= across) return;
  const uint64_t step = s_step[i];
  const bool fine = s_fine[i];
  const uint64_t first = (uint64_t)blockIdx.x * across + row, apart = (uint64_t)gridDim.x * across;
  uint64_t at = first * step + (uint64_t(1) << 61);
  float* to = a.table + first * 2 * F + i;
  for (uint64_t p = first; p < a.n_pos; p += apart, at += apart * step, to += apart * 2 * F) {
    const uint32_t quarter = (uint32_t)(at >> 62);
    // 2 pi / 2^32 times the rest's upper half, and 2^-32 of that times the lower
    const float hi = (float)((int32_t)((uint32_t)(at >> 32) & 0x3FFFFFFFu) - (1 << 29)), lo = (float)(uint32_t)at;
    const float x = fmaf(lo, 0x1p-32f, hi) * 1.4629180792671596e-9f, z = x * x;
    float s = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 0.f);
    s = fmaf(x, s, x);
    float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f);
    c = fmaf(z, c, 1.f);
    if (quarter & 1) {
      const float y = s;
      s = c;
      c = -y;
    }
    if (quarter & 2) {
      s = -s;
      c = -c;
    }
    if (!fine) s = c = __int_as_float(0x7FC00000);
    to[0] = a.factor * c;
    to[F] = a.factor * s;
  }
}

}  // namespace
}  // namespace ptc

using namespace ptc;

extern "C" ptc_status ptc_rope_table(const double* freq, uint32_t n_freq, uint32_t n_pos, float factor, float* table,
                                     void* stream) {
  if (n_freq < 1 || n_freq > PTC_MAX_HEAD_DIM / 2 || !std::isfinite(factor)) return PTC_ERR_INVALID_ARG;
  if (n_pos == 0) return PTC_OK;
  if (!freq || ((uintptr_t)freq & 7) || !aligned16(table)) return PTC_ERR_INVALID_ARG;
  const TableArgs a{freq, table, n_freq, n_pos, factor};
  const uint32_t across = kTableThreads / n_freq, rows = (n_pos - 1) / across + 1, most = 2 * num_sms();
  PTC_KERNEL("k_rope_table", static_cast<cudaStream_t>(stream), k_rope_table, rows < most ? rows : most, kTableThreads, 0, a);
  return cudaGetLastError() == cudaSuccess ? PTC_OK : PTC_ERR_CUDA;
}
