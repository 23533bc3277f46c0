// Block-scaled values (mx.h): quantisation, its inverse, and the norm that adds
// a residual and writes its output in 8 (or 4) bits with scales.
#include "kernels.h"
#include "mx.h"

namespace dlmc {
namespace {

// Columns col .. col + 7 of a row as fp32, zeros from column cols on.  VEC: cols
// and the row are whole 16-byte chunks; otherwise the chunks are loaded all the same,
// at their elements' alignment, and a row's last columns one by one.
template <bool BF16, bool VEC>
__device__ __forceinline__ void load8(const void* row, int col, int cols, float (&v)[8]) {
  const uint8_t* p = (const uint8_t*)row + (size_t)col * (BF16 ? 2 : 4);
  u32x4 a{}, b{};
  if constexpr (VEC) {
    if (col < cols) {
      a = *reinterpret_cast<const u32x4*>(p);
      if constexpr (!BF16) b = *reinterpret_cast<const u32x4*>(p + 16);
    }
  } else if (col + 8 <= cols) {
    __builtin_memcpy(&a, p, 16);
    if constexpr (!BF16) __builtin_memcpy(&b, p + 16, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.0f;
      if (col + i < cols) {
        if constexpr (BF16)
          v[i] = bf16_to_f32(((const bf16_t*)row)[col + i]);
        else
          v[i] = ((const float*)row)[col + i];
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (BF16)
      v[i] = __builtin_bit_cast(float, i % 2 ? a[i / 2] & 0xFFFF0000u : a[i / 2] << 16);
    else
      v[i] = __builtin_bit_cast(float, i < 4 ? a[i % 4] : b[i % 4]);
  }
}

template <bool BF16, bool VEC>
__device__ __forceinline__ void store8(void* row, int col, int cols, const float (&v)[8]) {
  if (VEC ? col >= cols : col + 8 > cols) {
    if constexpr (!VEC) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < cols) {
          if constexpr (BF16)
            ((bf16_t*)row)[col + i] = f32_to_bf16(v[i]);
          else
            ((float*)row)[col + i] = v[i];
        }
    }
    return;
  }
  uint8_t* p = (uint8_t*)row + (size_t)col * (BF16 ? 2 : 4);
  auto put = [](uint8_t* d, auto x) {
    if constexpr (VEC)
      *reinterpret_cast<decltype(x)*>(d) = x;
    else
      __builtin_memcpy(d, &x, 16);
  };
  if constexpr (BF16) {
    put(p, u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])});
  } else {
    put(p, f32x4{v[0], v[1], v[2], v[3]});
    put(p + 16, f32x4{v[4], v[5], v[6], v[7]});
  }
}

// A lane's eight codes, and its block's scale by the first of the block's four
// lanes; col is a multiple of 8 below the pitch in columns.
template <int FMT>
__device__ __forceinline__ void put8(uint8_t* codes, size_t pitch, uint8_t* scales, size_t slots, int row,
                                     int col, const float (&v)[8]) {
  uint32_t lo, hi;
  const uint32_t s = mx_encode8<FMT>(v, lo, hi);
  if constexpr (FMT == DLMC_MX_FP4)
    *reinterpret_cast<uint32_t*>(codes + (size_t)row * pitch + col / 2) = lo;
  else
    *reinterpret_cast<u32x2*>(codes + (size_t)row * pitch + col) = u32x2{lo, hi};
  if (col % MX_BLOCK == 0)
    scales[((size_t)(col / MX_GROUP) * slots + row) * 8 + col / MX_BLOCK % 8] = (uint8_t)s;
}

// Groups of columns that a block of mx_quantize / mx_dequantize takes of each of
// its eight rows (32 lanes to a group, eight columns a lane).  HBM bound: 32768 x 4096
// from bf16 to E2M1 62 us, 5.6 TB/s, and back to bf16 58 us, each alone (in turn 77 and
// 49, as the caches hold the other's data).  The blocks of a row follow each other, so
// that what is in flight lies together in memory (rows first: 73 and 73, each alone);
// four groups a block take 64 and 59.
constexpr int Q_GROUPS = 2;

template <int FMT, bool BF16, bool VEC>
__global__ void __launch_bounds__(256)
mx_quantize_kernel(const void* __restrict__ x, size_t ldx, int rows, int cols, uint8_t* __restrict__ codes,
                   size_t pitch, uint8_t* __restrict__ scales, size_t slots, int groups) {
  const int parts = (groups + Q_GROUPS - 1) / Q_GROUPS;
  const int row = blockIdx.x / parts * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (row >= rows) return;  // whole halves of a wave
  const void* xr = (const uint8_t*)x + (size_t)row * ldx * (BF16 ? 2 : 4);
  float v[Q_GROUPS][8];
  const int g0 = blockIdx.x % parts * Q_GROUPS;
#pragma unroll
  for (int e = 0; e < Q_GROUPS; ++e) load8<BF16, VEC>(xr, (g0 + e) * MX_GROUP + lane * 8, cols, v[e]);
#pragma unroll
  for (int e = 0; e < Q_GROUPS; ++e)
    if (g0 + e < groups) put8<FMT>(codes, pitch, scales, slots, row, (g0 + e) * MX_GROUP + lane * 8, v[e]);
}

template <int FMT, bool BF16, bool VEC>
__global__ void __launch_bounds__(256)
mx_dequantize_kernel(const uint8_t* __restrict__ codes, size_t pitch, const uint8_t* __restrict__ scales,
                     size_t slots, int rows, int cols, int groups, void* __restrict__ out, size_t ldo) {
  const int parts = (groups + Q_GROUPS - 1) / Q_GROUPS;
  const int row = blockIdx.x / parts * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (row >= rows) return;
  void* orow = (uint8_t*)out + (size_t)row * ldo * (BF16 ? 2 : 4);
  const int g0 = blockIdx.x % parts * Q_GROUPS;
  uint32_t lo[Q_GROUPS], hi[Q_GROUPS], s[Q_GROUPS];
#pragma unroll
  for (int e = 0; e < Q_GROUPS; ++e) {
    lo[e] = hi[e] = s[e] = 0;
    if (g0 + e >= groups) continue;
    const int col = (g0 + e) * MX_GROUP + lane * 8;
    if constexpr (FMT == DLMC_MX_FP4) {
      lo[e] = *reinterpret_cast<const uint32_t*>(codes + (size_t)row * pitch + col / 2);
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2*>(codes + (size_t)row * pitch + col);
      lo[e] = w[0];
      hi[e] = w[1];
    }
    s[e] = scales[((size_t)(g0 + e) * slots + row) * 8 + lane / 4];
  }
#pragma unroll
  for (int e = 0; e < Q_GROUPS; ++e) {
    if (g0 + e >= groups) continue;
    float v[8];
    mx_decode8<FMT>(lo[e], hi[e], s[e], v);
    store8<BF16, VEC>(orow, (g0 + e) * MX_GROUP + lane * 8, cols, v);
  }
}

__device__ __forceinline__ float wave_total(float t) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o);
  return t;
}

// r = x + delta, y = norm(r) * gain, y in codes with scales.  A row is held in
// registers by WAVES waves, eight columns a lane and step, PER steps; with one
// wave a row a block takes four rows.  Which form a row takes goes by its
// columns alone, so its sums, and with them its codes, do not depend on the
// number of rows.  HBM bound: x and delta are read once, and everything is in
// flight before the first value is used (2048 x 4096 in fp32 with a bf16 delta, to E4M3:
// 17.6 us, 5.3 TB/s).
template <int FMT, bool XB, bool VEC, int WAVES, int PER>
__global__ void __launch_bounds__(256)
add_norm_mx_kernel(AddNormMx a) {
  constexpr int STEP = 512 * WAVES;
  __shared__ float part[2][4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int row = WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= a.rows || (a.n_dev && row >= *a.n_dev)) return;  // whole waves, or the whole block
  const int src = a.gather ? a.gather[row] : row;
  const int c0 = (WAVES == 1 ? lane : (int)threadIdx.x) * 8;
  const void* xr = (const uint8_t*)a.x + (size_t)src * a.ldx * (XB ? 2 : 4);
  float v[PER][8];
#pragma unroll
  for (int e = 0; e < PER; ++e) load8<XB, VEC>(xr, c0 + e * STEP, a.cols, v[e]);
  if (a.delta) {
    float d[PER][8];
    if (a.delta_bf16) {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        load8<true, VEC>((const bf16_t*)a.delta + (size_t)src * a.ldd, c0 + e * STEP, a.cols, d[e]);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        load8<false, VEC>((const float*)a.delta + (size_t)src * a.ldd, c0 + e * STEP, a.cols, d[e]);
    }
#pragma unroll
    for (int e = 0; e < PER; ++e)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[e][i] += d[e][i];
        // a bf16 stream: the norm is of the values that are stored, so that it
        // can be taken again from the stream
        if constexpr (XB) v[e][i] = bf16_to_f32(f32_to_bf16(v[e][i]));
      }
  }
  if (a.sum) {
    void* sr = (uint8_t*)a.sum + (size_t)src * a.lds * (XB ? 2 : 4);
#pragma unroll
    for (int e = 0; e < PER; ++e) store8<XB, VEC>(sr, c0 + e * STEP, a.cols, v[e]);
  }
  auto total = [&](float t, int k) {
    t = wave_total(t);
    if constexpr (WAVES == 1) return t;
    if (lane == 0) part[k][wave] = t;
    __syncthreads();
    return (part[k][0] + part[k][1]) + (part[k][2] + part[k][3]);
  };
  float shift = 0.0f;
  if (a.norm_kind == DLMC_NORM_LAYER) {
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < PER; ++e)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[e][i];
    shift = total(s, 0) / (float)a.cols;
  }
  float q = 0.0f;
#pragma unroll
  for (int e = 0; e < PER; ++e)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // columns past cols hold zero and add nothing
      const float t = c0 + e * STEP + i < a.cols ? v[e][i] - shift : 0.0f;
      v[e][i] = t;
      q = fmaf(t, t, q);
    }
  const float scale = 1.0f / sqrtf(total(q, 1) / (float)a.cols + a.eps);
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int col = c0 + e * STEP;
    if (col >= a.pitch_cols) continue;  // four lanes of a block together
#pragma unroll
    for (int i = 0; i < 8; ++i) v[e][i] *= scale;
    if (a.gain) {
      float g[8];
      load8<false, VEC>(a.gain, col, a.cols, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[e][i] *= g[i];
    }
    put8<FMT>(a.q.codes, a.pitch, a.q.scales, a.slots, row, col, v[e]);
  }
}

template <int FMT, bool XB, bool VEC>
void launch_add_norm(hipStream_t st, const AddNormMx& a) {
  const unsigned by4 = (unsigned)ceil_div(a.rows, 4);
  if (a.cols <= 512)
    add_norm_mx_kernel<FMT, XB, VEC, 1, 1><<<by4, 256, 0, st>>>(a);
  else if (a.cols <= 1024)
    add_norm_mx_kernel<FMT, XB, VEC, 1, 2><<<by4, 256, 0, st>>>(a);
  else if (a.cols <= 2048)
    add_norm_mx_kernel<FMT, XB, VEC, 4, 1><<<a.rows, 256, 0, st>>>(a);
  else if (a.cols <= 4096)
    add_norm_mx_kernel<FMT, XB, VEC, 4, 2><<<a.rows, 256, 0, st>>>(a);
  else
    add_norm_mx_kernel<FMT, XB, VEC, 4, 4><<<a.rows, 256, 0, st>>>(a);
}

// Blocks of a launch: a grid's threads are counted in 32 bits.
constexpr int LAUNCH_BLOCKS = 1 << 23;

inline bool whole16(const void* p, size_t ld, size_t esz) {
  return ((uintptr_t)p & 15) == 0 && ld * esz % 16 == 0;
}

}  // namespace

void mx_quantize(hipStream_t st, const void* x, bool bf16, size_t ldx, int rows, int cols, int fmt, MxView q) {
  if (rows <= 0) return;
  const int groups = mx_groups(cols);
  const size_t esz = bf16 ? 2 : 4, pitch = mx_pitch(fmt, cols);
  const bool vec = cols % 8 == 0 && whole16(x, ldx, esz);
  auto go = [&](auto kernel) {
    const size_t parts = ceil_div(groups, Q_GROUPS), most = LAUNCH_BLOCKS / parts * 8;
    for (size_t r = 0; r < (size_t)rows; r += most) {
      const int n = (int)std::min<size_t>(rows - r, most);
      const unsigned grid = (unsigned)(ceil_div(n, 8) * parts);
      kernel<<<grid, 256, 0, st>>>((const uint8_t*)x + r * ldx * esz, ldx, n, cols, q.codes + r * pitch, pitch,
                                   q.scales + r * 8, mx_slots(rows), groups);
    }
  };
  if (fmt == DLMC_MX_FP4) {
    if (bf16) vec ? go(mx_quantize_kernel<DLMC_MX_FP4, true, true>) : go(mx_quantize_kernel<DLMC_MX_FP4, true, false>);
    else vec ? go(mx_quantize_kernel<DLMC_MX_FP4, false, true>) : go(mx_quantize_kernel<DLMC_MX_FP4, false, false>);
  } else {
    if (bf16) vec ? go(mx_quantize_kernel<DLMC_MX_FP8, true, true>) : go(mx_quantize_kernel<DLMC_MX_FP8, true, false>);
    else vec ? go(mx_quantize_kernel<DLMC_MX_FP8, false, true>) : go(mx_quantize_kernel<DLMC_MX_FP8, false, false>);
  }
  DLMC_HIP(hipGetLastError());
}

void mx_dequantize(hipStream_t st, MxView q, int fmt, int rows, int cols, void* out, bool bf16, size_t ldo) {
  if (rows <= 0) return;
  const int groups = mx_groups(cols);
  const size_t esz = bf16 ? 2 : 4, pitch = mx_pitch(fmt, cols);
  const bool vec = cols % 8 == 0 && whole16(out, ldo, esz);
  auto go = [&](auto kernel) {
    const size_t parts = ceil_div(groups, Q_GROUPS), most = LAUNCH_BLOCKS / parts * 8;
    for (size_t r = 0; r < (size_t)rows; r += most) {
      const int n = (int)std::min<size_t>(rows - r, most);
      const unsigned grid = (unsigned)(ceil_div(n, 8) * parts);
      kernel<<<grid, 256, 0, st>>>(q.codes + r * pitch, pitch, q.scales + r * 8, mx_slots(rows), n, cols, groups,
                                   (uint8_t*)out + r * ldo * esz, ldo);
    }
  };
  if (fmt == DLMC_MX_FP4) {
    if (bf16) vec ? go(mx_dequantize_kernel<DLMC_MX_FP4, true, true>) : go(mx_dequantize_kernel<DLMC_MX_FP4, true, false>);
    else vec ? go(mx_dequantize_kernel<DLMC_MX_FP4, false, true>) : go(mx_dequantize_kernel<DLMC_MX_FP4, false, false>);
  } else {
    if (bf16) vec ? go(mx_dequantize_kernel<DLMC_MX_FP8, true, true>) : go(mx_dequantize_kernel<DLMC_MX_FP8, true, false>);
    else vec ? go(mx_dequantize_kernel<DLMC_MX_FP8, false, true>) : go(mx_dequantize_kernel<DLMC_MX_FP8, false, false>);
  }
  DLMC_HIP(hipGetLastError());
}

void add_norm_mx(hipStream_t st, AddNormMx a) {
  if (a.rows <= 0) return;
  DLMC_CHECK(a.cols >= 1 && a.cols <= ADD_NORM_MAX_COLS, DLMC_E_INVAL, "norm of more columns than a block holds");
  a.pitch_cols = mx_groups(a.cols) * MX_GROUP;
  a.pitch = mx_pitch(a.fmt, a.cols);
  if (a.rows > LAUNCH_BLOCKS) {
    DLMC_CHECK(!a.gather && !a.n_dev, DLMC_E_INVAL, "too many gathered rows");
    const AddNormMx all = a;
    const size_t xs = a.x_bf16 ? 2 : 4, ds = a.delta_bf16 ? 2 : 4;
    for (size_t r = 0; r < (size_t)all.rows; r += LAUNCH_BLOCKS) {
      AddNormMx part = all;
      part.rows = (int)std::min<size_t>(all.rows - r, LAUNCH_BLOCKS);
      part.x = (const uint8_t*)all.x + r * all.ldx * xs;
      if (all.delta) part.delta = (const uint8_t*)all.delta + r * all.ldd * ds;
      if (all.sum) part.sum = (uint8_t*)all.sum + r * all.lds * xs;
      part.q = MxView{all.q.codes + r * all.pitch, all.q.scales + r * 8};
      add_norm_mx(st, part);
    }
    return;
  }
  const bool vec = a.cols % 8 == 0 && whole16(a.x, a.ldx, a.x_bf16 ? 2 : 4) &&
                   (!a.delta || whole16(a.delta, a.ldd, a.delta_bf16 ? 2 : 4)) &&
                   (!a.sum || whole16(a.sum, a.lds, a.x_bf16 ? 2 : 4)) && (!a.gain || ((uintptr_t)a.gain & 15) == 0);
  if (a.fmt == DLMC_MX_FP4) {
    if (a.x_bf16) vec ? launch_add_norm<DLMC_MX_FP4, true, true>(st, a) : launch_add_norm<DLMC_MX_FP4, true, false>(st, a);
    else vec ? launch_add_norm<DLMC_MX_FP4, false, true>(st, a) : launch_add_norm<DLMC_MX_FP4, false, false>(st, a);
  } else {
    if (a.x_bf16) vec ? launch_add_norm<DLMC_MX_FP8, true, true>(st, a) : launch_add_norm<DLMC_MX_FP8, true, false>(st, a);
    else vec ? launch_add_norm<DLMC_MX_FP8, false, true>(st, a) : launch_add_norm<DLMC_MX_FP8, false, false>(st, a);
  }
  DLMC_HIP(hipGetLastError());
}

}  // namespace dlmc
