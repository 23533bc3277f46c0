// Product of block-scaled matrices (mx.h): C = A B^T on
// v_mfma_scale_f32_32x32x64_f8f6f4, A in E4M3 or E2M1, B in E2M1, fp32
// accumulation.
//
// C[m][n] = sum over blocks b of 32 columns of 2^(sa[m][b] + sb[n][b] - 254) sum_k
// a[m][k] b[n][k].  One instruction multiplies 64 columns and applies both blocks'
// scales, at four times the bf16 rate with E2M1 on both sides, at twice with E4M3.
//
// Operand registers (found by measurement): lane l holds row l % 32 of its operand.
// E2M1: the 32 columns of block l / 32.  E4M3: columns 16 (l / 32) .. + 15 of block
// 0 in the first four registers, of block 1 in the last four.  The scale of block
// b is taken from the lanes l / 32 = b.
//
// Precision: products of E2M1 values are summed exactly.  With E4M3 the unit aligns
// the products it adds together to the largest and drops what lies 2^13 below it:
// about 4e-6 of a result's root mean square for normal values, far below the
// 2^-4 half step of the values themselves.
//
// Numerics: each output is a sequential sum over groups of 256 columns, each four
// instructions in order, whatever the tile, so a row's result does not depend on
// the launch's other rows.
#include "kernels.h"

namespace dlmc {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Direct 16-byte load to LDS; `lds` is wave-uniform, lane l writes lds + 16 l.
__device__ __forceinline__ void dma16(const uint8_t* g, uint8_t* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(g, lds, 16, 0, 0);
#endif
}
__device__ __forceinline__ void bare_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// s_waitcnt immediate: vmcnt(n) alone
constexpr int wait_vm(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }

// 16-byte chunks of a tile row are stored XOR-swizzled, so that the 16 rows that a
// ds_read_b128 serves at a time fall on the 16 slots of the 64 banks: rows of 128
// bytes by (row / 2) % 8, rows of 256 bytes by row % 16.
template <int ROW>
__device__ __forceinline__ int swizzle(int row) {
  return ROW == 128 ? (row >> 1) & 7 : row & 15;
}

// This block's tile among those with live rows; hardware block ids go round robin
// over the 8 XCDs, and each XCD takes a contiguous range of tiles in groups of
// eight row tiles, which share their operand panels in its L2.
__device__ __forceinline__ bool tile_of(int bid, int n_tm, int n_tn, int bm, int Mv, int& tm, int& tn) {
  const int live_m = min(n_tm, (Mv + bm - 1) / bm), live = live_m * n_tn, nb = (live + 7) & ~7;
  if (bid >= nb) return false;
  const int l = (bid & 7) * (nb >> 3) + (bid >> 3);
  if (l >= live) return false;
  const int per = 8 * n_tn, g = l / per, first = g * 8, size = min(live_m - first, 8), r = l - g * per;
  tm = first + r % size;
  tn = r / size;
  return true;
}

struct MxArgs {
  const uint8_t *a, *as, *b, *bs;
  size_t a_slots, b_slots;
  int M, N, groups;
  const int* M_dev;
  void* out;
  size_t ldo;
  int n_tm, n_tn;
};

// BM x BN tiles by WR x WC waves, a ring of NS stages of one group (256 columns)
// of both operands and their scales.
template <int FA, int BM, int BN, int WR, int WC, int NS, bool OUT_BF16>
__global__ void __launch_bounds__(64 * WR * WC)
mx_ring_kernel(MxArgs p) {
  constexpr int NW = WR * WC, WM = BM / WR, WN = BN / WC, TM = WM / 32, TN = WN / 32;
  constexpr int AROW = FA == DLMC_MX_FP4 ? 128 : 256, BROW = 128;
  constexpr int A_B = BM * AROW, B_B = BN * BROW, S_N = ((BM + BN) * 8 + 1023) / 1024;
  constexpr int S_IN = (S_N + NW - 1) / NW, S_B = S_IN * NW * 1024;
  constexpr int A_IN = A_B / 1024 / NW, B_IN = B_B / 1024 / NW, NL = A_IN + B_IN + S_IN;
  constexpr int STAGE = A_B + B_B + S_B;
  static_assert(A_IN * NW * 1024 == A_B && B_IN * NW * 1024 == B_B, "whole windows per wave");
  static_assert(NS * STAGE <= 160 * 1024 && (NS - 2) * NL < 64, "LDS / vmcnt field");
  __shared__ __attribute__((aligned(16))) uint8_t smem[NS * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WC, wn = wave % WC, lr = lane & 31, lg = lane >> 5;
  const int Mv = p.M_dev ? min(*p.M_dev, p.M) : p.M;
  int tm, tn;
  if (!tile_of(blockIdx.x, p.n_tm, p.n_tn, BM, Mv, tm, tn)) return;
  const int m0 = tm * BM, n0 = tn * BN, ng = p.groups;

  // windows of 1 KB: a lane's row and chunk; rows past the live ones are clamped
  const size_t a_pitch = (size_t)ng * AROW, b_pitch = (size_t)ng * BROW;
  const uint8_t* a_src[A_IN];
  const uint8_t* b_src[B_IN];
  const uint8_t* s_src[S_IN];
  size_t s_step[S_IN];
#pragma unroll
  for (int j = 0; j < A_IN; ++j) {
    const int slot = (wave * A_IN + j) * 64 + lane, row = slot / (AROW / 16), c = slot % (AROW / 16);
    a_src[j] = p.a + (size_t)min(m0 + row, Mv - 1) * a_pitch + ((c ^ swizzle<AROW>(row)) << 4);
  }
#pragma unroll
  for (int j = 0; j < B_IN; ++j) {
    const int slot = (wave * B_IN + j) * 64 + lane, row = slot / 8, c = slot % 8;
    b_src[j] = p.b + (size_t)min(n0 + row, p.N - 1) * b_pitch + ((c ^ swizzle<BROW>(row)) << 4);
  }
#pragma unroll
  for (int j = 0; j < S_IN; ++j) {  // two rows' scales a lane, A's rows first
    const int row = ((wave * S_IN + j) * 64 + lane) * 2;
    if (row < BM) {
      s_src[j] = p.as + (size_t)min((size_t)(m0 + row), p.a_slots - 2) * 8;
      s_step[j] = p.a_slots * 8;
    } else {
      s_src[j] = p.bs + (size_t)min((size_t)(n0 + row - BM), p.b_slots - 2) * 8;
      s_step[j] = p.b_slots * 8;
    }
  }
  auto load = [&](int kt) {
    uint8_t* st = smem + (kt % NS) * STAGE;
#pragma unroll
    for (int j = 0; j < A_IN; ++j) dma16(a_src[j] + (size_t)kt * AROW, st + (wave * A_IN + j) * 1024);
#pragma unroll
    for (int j = 0; j < B_IN; ++j) dma16(b_src[j] + (size_t)kt * BROW, st + A_B + (wave * B_IN + j) * 1024);
#pragma unroll
    for (int j = 0; j < S_IN; ++j)
      dma16(s_src[j] + (size_t)kt * s_step[j], st + A_B + B_B + (wave * S_IN + j) * 1024);
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  for (int k = 0; k < NS - 1 && k < ng; ++k) load(k);
  for (int kt = 0; kt < ng; ++kt) {
    // this wave's loads of group kt have landed: NS - 2 younger groups may be in
    // flight, fewer (all waited for) towards the end
    if (kt + NS - 2 < ng)
      __builtin_amdgcn_s_waitcnt(wait_vm((NS - 2) * NL));
    else
      __builtin_amdgcn_s_waitcnt(wait_vm(0));
    bare_barrier();  // every wave's have, and group kt - 1 is read
    if (kt + NS - 1 < ng) load(kt + NS - 1);
    const uint8_t* as = smem + (kt % NS) * STAGE;
    const uint8_t* bs = as + A_B;
    const uint8_t* sc = bs + B_B;
    // lane's scales of its row: even and odd blocks by its half, so that bytes 0
    // and 2 are those of the steps' block
    u32x2 sa[TM], sb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      sa[i] = *reinterpret_cast<const u32x2*>(sc + (wm * WM + i * 32 + lr) * 8);
      sa[i] = u32x2{sa[i][0] >> (8 * lg), sa[i][1] >> (8 * lg)};
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      sb[j] = *reinterpret_cast<const u32x2*>(sc + (BM + wn * WN + j * 32 + lr) * 8);
      sb[j] = u32x2{sb[j][0] >> (8 * lg), sb[j][1] >> (8 * lg)};
    }
    auto step = [&](auto s_) {
      constexpr int S = decltype(s_)::value;
      i32x8 fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int row = wm * WM + i * 32 + lr;
        const uint8_t* r = as + row * AROW;
        const int x = swizzle<AROW>(row);
        if constexpr (FA == DLMC_MX_FP4) {
          const i32x4 q = *reinterpret_cast<const i32x4*>(r + (((2 * S + lg) ^ x) << 4));
          fa[i] = i32x8{q[0], q[1], q[2], q[3], 0, 0, 0, 0};
        } else {
          const i32x4 q = *reinterpret_cast<const i32x4*>(r + (((4 * S + lg) ^ x) << 4));
          const i32x4 t = *reinterpret_cast<const i32x4*>(r + (((4 * S + 2 + lg) ^ x) << 4));
          fa[i] = i32x8{q[0], q[1], q[2], q[3], t[0], t[1], t[2], t[3]};
        }
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int row = wn * WN + j * 32 + lr;
        const i32x4 q = *reinterpret_cast<const i32x4*>(bs + row * BROW + (((2 * S + lg) ^ swizzle<BROW>(row)) << 4));
        fb[j] = i32x8{q[0], q[1], q[2], q[3], 0, 0, 0, 0};
      }
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
              fa[i], fb[j], acc[i][j], FA == DLMC_MX_FP4 ? 4 : 0, 4, 2 * (S & 1), (int)sa[i][S >> 1], 2 * (S & 1),
              (int)sb[j][S >> 1]);
#endif
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
  }
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = m0 + wm * WM + i * 32 + (r >> 2) * 8 + lg * 4 + (r & 3);
      if (row >= Mv) continue;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int col = n0 + wn * WN + j * 32 + lr;
        if (col >= p.N) continue;
        if constexpr (OUT_BF16)
          ((bf16_t*)p.out)[(size_t)row * p.ldo + col] = f32_to_bf16(acc[i][j][r]);
        else
          ((float*)p.out)[(size_t)row * p.ldo + col] = acc[i][j][r];
      }
    }
}

template <int FA, int BM, int BN, int WR, int WC, int NS>
void launch_ring(hipStream_t st, MxArgs p, bool out_bf16) {
  p.n_tm = ceil_div(p.M, BM);
  p.n_tn = ceil_div(p.N, BN);
  const int64_t tiles = (int64_t)p.n_tm * p.n_tn;
  DLMC_CHECK(tiles < (1ll << 30), DLMC_E_INVAL, "product with too many tiles");
  const unsigned grid = (unsigned)((tiles + 7) & ~7ll);
  if (out_bf16)
    mx_ring_kernel<FA, BM, BN, WR, WC, NS, true><<<grid, 64 * WR * WC, 0, st>>>(p);
  else
    mx_ring_kernel<FA, BM, BN, WR, WC, NS, false><<<grid, 64 * WR * WC, 0, st>>>(p);
  DLMC_HIP(hipGetLastError());
}

}  // namespace

void mx_matmul(hipStream_t st, MxView A, int fmt_a, size_t a_slots, MxView B, int M, int N, int K, const int* M_dev,
               void* out, bool out_bf16, size_t ldo, int rows_hint) {
  if (M <= 0 || N <= 0) return;
  MxArgs p{};
  p.a = A.codes;
  p.as = A.scales;
  p.b = B.codes;
  p.bs = B.scales;
  p.a_slots = a_slots;
  p.b_slots = mx_slots(N);
  p.M = M;
  p.N = N;
  p.groups = mx_groups(K);
  p.M_dev = M_dev;
  p.out = out;
  p.ldo = ldo;
  const int rows = rows_hint >= 0 && rows_hint < M ? rows_hint : M;
  const bool fp4 = fmt_a == DLMC_MX_FP4;
  const int64_t big = (int64_t)ceil_div(rows, fp4 ? 256 : 128) * ceil_div(N, 256);
  if (rows <= 32) {
    if (fp4)
      launch_ring<DLMC_MX_FP4, 32, 128, 1, 4, 3>(st, p, out_bf16);
    else
      launch_ring<DLMC_MX_FP8, 32, 128, 1, 4, 3>(st, p, out_bf16);
  } else if (big >= 256) {
    if (fp4)
      launch_ring<DLMC_MX_FP4, 256, 256, 2, 2, 2>(st, p, out_bf16);
    else
      launch_ring<DLMC_MX_FP8, 128, 256, 2, 2, 2>(st, p, out_bf16);
  } else {
    if (fp4)
      launch_ring<DLMC_MX_FP4, 128, 128, 2, 2, 4>(st, p, out_bf16);
    else
      launch_ring<DLMC_MX_FP8, 128, 128, 2, 2, 3>(st, p, out_bf16);
  }
}

}  // namespace dlmc
