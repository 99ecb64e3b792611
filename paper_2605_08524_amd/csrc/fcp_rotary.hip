// Rotary positions with several axes: kernel and launcher.
//
// Memory-bound: every element is read once and written once, 6 FLOP a pair.  A workgroup takes kRows rows of one tensor; it first works
// out cos and sin of their angles, one per (row, pair), into LDS, where all heads of the row share them, and then streams the rows,
// 16 dimensions (8 pairs) of a head a thread and step: two 16-byte accesses each way in bf16, 128-byte lines in whole.
// Angles.  A position times a frequency of 1 in fp32 is off by 0.03 at position 10^6 (half a unit of 2^-4), so the frequency comes as a 64-bit fraction
// of a turn and the product wraps modulo 2^64, that is modulo one turn, exactly.  What is left is the fraction's own error times the position,
// |pos| (1 + |freq| / 4) 2^-64 turns, and 2^-33 where the product is rounded to 32 bits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "fcp_internal.h"
#include "fcp_rotary.h"

namespace fcp {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kMaxPairs = FCP_ROTARY_MAX_DIM / 2;
constexpr int kThreads = 256;
constexpr int64_t kMaxGroups = ((int64_t)1 << 32) / kThreads - 1;     // a launch has fewer than 2^32 threads

struct RotaryArgs {
  fcp_rotary_part part[FCP_ROTARY_MAX_PARTS];
  int64_t first_group[FCP_ROTARY_MAX_PARTS + 1];    // workgroups of part i: first_group[i] .. first_group[i + 1]
  int32_t rows, head_dim, n_pairs, n_axes;          // rows: of a workgroup
  float sign;                                       // of the sine
  uint64_t turn[kMaxPairs];                         // frequency, 2^-64 turns per position
  uint8_t axis[kMaxPairs];
};

// 16 dimensions of a head
struct Chunk { float x[16]; };

template <bool F32>
__device__ __forceinline__ void load8(float* x, const void* p, int64_t at) {
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(p) + at + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; j++) x[4 * i + j] = v[j];
    }
  } else {
    const u32x4 v = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(p) + at);
#pragma unroll
    for (int i = 0; i < 4; i++) { x[2 * i] = __uint_as_float(v[i] << 16); x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
  }
}
template <bool F32>
__device__ __forceinline__ void store8(void* p, int64_t at, const float* x) {
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 2; i++) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(p) + at + 4 * i) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
  } else {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const f32x2 f = {x[2 * i], x[2 * i + 1]};
      v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));     // round to nearest even
    }
    *reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(p) + at) = v;
  }
}

template <bool INTERLEAVED, bool SRC32, bool DST32>
__device__ __forceinline__ void rotate_rows(const RotaryArgs& a, const fcp_rotary_part& p, int64_t row0, int n_rows, const f32x2* cs) {
  const int per_head = a.head_dim / 16, per_row = p.n_heads * per_head, n = n_rows * per_row, turned = a.n_pairs / 8;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int row = i / per_row, rest = i - row * per_row, head = rest / per_head, c = rest - head * per_head;
    const int64_t src = (row0 + row) * p.src_row_stride + head * a.head_dim, dst = (row0 + row) * p.dst_row_stride + head * a.head_dim;
    // dimensions of the chunk: two runs of eight
    const bool halves = !INTERLEAVED && c < turned;
    const int d0 = halves ? 8 * c : 16 * c, d1 = halves ? a.n_pairs + 8 * c : 16 * c + 8;
    float x[16];
    load8<SRC32>(x, p.src, src + d0);
    load8<SRC32>(x + 8, p.src, src + d1);
    if (c < turned) {
      const f32x2* t = cs + row * a.n_pairs + 8 * c;
#pragma unroll
      for (int k = 0; k < 8; k++) {
        const f32x2 w = t[k];
        float &u = x[INTERLEAVED ? 2 * k : k], &v = x[INTERLEAVED ? 2 * k + 1 : k + 8];
        const float u1 = u * w[0] - v * w[1], v1 = u * w[1] + v * w[0];
        u = u1; v = v1;
      }
    }
    store8<DST32>(p.dst, dst + d0, x);
    store8<DST32>(p.dst, dst + d1, x + 8);
  }
}

template <bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a) {
  extern __shared__ __attribute__((aligned(16))) f32x2 cs[];      // [rows][n_pairs]: cos, sin
  int part = 0;
  while (part < FCP_ROTARY_MAX_PARTS - 1 && (int64_t)blockIdx.x >= a.first_group[part + 1]) part++;
  const fcp_rotary_part p = a.part[part];
  const int64_t row0 = ((int64_t)blockIdx.x - a.first_group[part]) * a.rows;
  const int n_rows = (int)min((int64_t)a.rows, p.n_rows - row0);
  for (int i = threadIdx.x; i < n_rows * a.n_pairs; i += kThreads) {
    const int row = i / a.n_pairs, pair = i - row * a.n_pairs;
    const int pos = p.pos[(row0 + row) * a.n_axes + a.axis[pair]];
    // the top 32 bits of the turn as a signed fraction: half turns in [-1, 1)
    const int32_t top = (int32_t)(((uint64_t)(int64_t)pos * a.turn[pair] + 0x80000000u) >> 32);
    float s, c;
    sincospif((float)top * 0x1p-31f, &s, &c);
    cs[i] = f32x2{c, s * a.sign};
  }
  __syncthreads();
  if (p.src_f32) {
    if (p.dst_f32) rotate_rows<INTERLEAVED, true, true>(a, p, row0, n_rows, cs); else rotate_rows<INTERLEAVED, true, false>(a, p, row0, n_rows, cs);
  } else {
    if (p.dst_f32) rotate_rows<INTERLEAVED, false, true>(a, p, row0, n_rows, cs); else rotate_rows<INTERLEAVED, false, false>(a, p, row0, n_rows, cs);
  }
}

}  // namespace fcp

using namespace fcp;

extern "C" int fcp_rotary_turns(const double* freq, int32_t n, uint64_t* turn) {
  if (n < 0 || (n > 0 && (!freq || !turn))) { set_error("fcp_rotary_turns: invalid argument"); return FCP_ERR_INVALID_ARG; }
  for (int p = 0; p < n; p++) {
    if (!(std::fabs(freq[p]) <= 1e6)) { set_error("fcp_rotary_turns: |freq[%d]| must be at most 1e6", p); return FCP_ERR_INVALID_ARG; }
    // 64 bits of mantissa: the divisor and the quotient are off by half a unit each, 1.5 2^-64 freq / 2 pi at most; cutting the rest off is one more 2^-64
    const long double turns = (long double)freq[p] / 6.28318530717958647692528676655900577L;
    const long double fraction = turns - floorl(turns);
    turn[p] = fraction >= 1.0L ? 0 : (uint64_t)(fraction * 18446744073709551616.0L);
  }
  return FCP_OK;
}

extern "C" int fcp_rotary_apply(const fcp_rotary* r, const fcp_rotary_part* parts, int32_t n_parts, int32_t inverse, void* stream) {
  if (!r || !parts || n_parts < 1 || n_parts > FCP_ROTARY_MAX_PARTS || !r->axis || !r->turn) { set_error("fcp_rotary_apply: NULL pointer, or not 1 to %d parts", FCP_ROTARY_MAX_PARTS); return FCP_ERR_INVALID_ARG; }
  if (r->head_dim < 16 || r->head_dim > FCP_ROTARY_MAX_DIM || r->head_dim % 16 != 0) {
    set_error("fcp_rotary_apply: head_dim %d unsupported (a multiple of 16 up to %d)", r->head_dim, FCP_ROTARY_MAX_DIM); return FCP_ERR_UNSUPPORTED;
  }
  if (r->n_pairs < 8 || r->n_pairs > r->head_dim / 2 || r->n_pairs % 8 != 0) {
    set_error("fcp_rotary_apply: n_pairs %d unsupported (a multiple of 8 up to head_dim / 2)", r->n_pairs); return FCP_ERR_UNSUPPORTED;
  }
  if (r->n_axes < 1 || r->n_axes > FCP_ROTARY_MAX_AXES) { set_error("fcp_rotary_apply: n_axes must be 1 to %d", FCP_ROTARY_MAX_AXES); return FCP_ERR_INVALID_ARG; }
  RotaryArgs a{};
  a.head_dim = r->head_dim; a.n_pairs = r->n_pairs; a.n_axes = r->n_axes; a.sign = inverse ? -1.0f : 1.0f;
  for (int p = 0; p < r->n_pairs; p++) {
    if (r->axis[p] < 0 || r->axis[p] >= r->n_axes) { set_error("fcp_rotary_apply: axis[%d] = %d out of range", p, r->axis[p]); return FCP_ERR_INVALID_ARG; }
    a.axis[p] = (uint8_t)r->axis[p];
    a.turn[p] = r->turn[p];
  }
  int64_t rows = 0;
  for (int i = 0; i < n_parts; i++) {
    const fcp_rotary_part& p = parts[i];
    if (p.n_rows < 0 || p.n_heads <= 0) { set_error("fcp_rotary_apply: part %d: n_rows must be >= 0 and n_heads positive", i); return FCP_ERR_INVALID_ARG; }
    if (p.n_rows == 0) continue;
    if (!p.src || !p.dst || !p.pos) { set_error("fcp_rotary_apply: part %d: NULL pointer", i); return FCP_ERR_INVALID_ARG; }
    const int64_t width = (int64_t)p.n_heads * r->head_dim;
    if (width > INT32_MAX / 64) { set_error("fcp_rotary_apply: part %d: a row of more than 2^25 elements", i); return FCP_ERR_UNSUPPORTED; }
    if (p.n_rows > 1 && (p.src_row_stride < width || p.dst_row_stride < width)) { set_error("fcp_rotary_apply: part %d: a row stride is less than a row", i); return FCP_ERR_INVALID_ARG; }
    if (p.src == p.dst && (p.src_row_stride != p.dst_row_stride || !p.src_f32 != !p.dst_f32)) {
      set_error("fcp_rotary_apply: part %d: in place needs one stride and one type", i); return FCP_ERR_INVALID_ARG;
    }
    if (((uintptr_t)p.src | (uintptr_t)p.dst) & 15 || (p.n_rows > 1 && (p.src_row_stride % (p.src_f32 ? 4 : 8) != 0 || p.dst_row_stride % (p.dst_f32 ? 4 : 8) != 0))) {
      set_error("fcp_rotary_apply: part %d: rows must be aligned to 16 bytes", i); return FCP_ERR_UNSUPPORTED;
    }
    rows += p.n_rows;
  }
  if (rows == 0) return FCP_OK;
  // enough workgroups for two to a compute unit, as long as there are rows
  a.rows = (int32_t)std::max<int64_t>(1, std::min<int64_t>(4, rows / 512));
  int64_t n = 0;
  for (int i = 0; i < FCP_ROTARY_MAX_PARTS; i++) {
    a.first_group[i + 1] = a.first_group[i];
    if (i >= n_parts) continue;
    a.part[i] = parts[i];
    n += ((int64_t)parts[i].n_rows + a.rows - 1) / a.rows;
    a.first_group[i + 1] = n;
  }
  if (n > kMaxGroups) { set_error("fcp_rotary_apply: too many rows for one launch (%lld groups of %d, at most %lld)", (long long)n, a.rows, (long long)kMaxGroups); return FCP_ERR_UNSUPPORTED; }
  void (*kern)(RotaryArgs) = r->interleaved ? rotary_kernel<true> : rotary_kernel<false>;
  hipLaunchKernelGGL(kern, dim3((unsigned)n), dim3(kThreads), a.rows * a.n_pairs * sizeof(f32x2), (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("fcp_rotary_apply: %s", hipGetErrorString(e)); return FCP_ERR_HIP; }
  return FCP_OK;
}
