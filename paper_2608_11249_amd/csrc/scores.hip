// Scores of logit rows: log2 probabilities of given tokens (their code lengths in
// bits, negated), entropies, and the most probable alternatives, in one pass over
// the logits.
//
// With t_i = (l_i - M) log2 e, M the row's largest logit: Z = sum 2^t_i, A = sum 2^t_i
// t_i, log2 p_i = t_i - log2 Z, H = log2 Z - A / Z.  Every lane keeps its own running
// M, Z, A and rescales them when its M rises.  (The difference comes first: l_i
// log2 e would overflow in a row masked with the type's lowest value throughout.)
//
// Alternatives: each wave keeps a threshold that at least k of its logits so far
// reach, and collects the logits above it in LDS.  The threshold bounds the k-th largest
// of the 64 lanes' running maxima (for many alternatives, of the maxima of the lanes'
// two halves), taken anew with tiles 0, 1, 2, 4, 8, ...: about k logits pass it in the
// first tile, and fewer and fewer later.  A list that fills up all the same is cut
// to its k best.  A wave's tiles come in the order of
// their columns, so among equal logits the ones collected first have the lowest ids,
// and later ones equal to the threshold need not be looked at.
#include "kernels.h"

#include <type_traits>

namespace dlmc {
namespace {

constexpr int TILE = 512;            // columns a wave takes at a time, eight a lane
// Entries of a wave's list before it is cut: with 96, and room for a tile on top, a CU
// holds eight blocks, so that 2048 rows are on the chip at once.  With more
// alternatives than 16 it would be cut too often: 192, and room for half a tile (2048 x
// 126464 with 20 alternatives 208 us; with 256 and a whole tile, six blocks a CU, 255).
constexpr int FEW_TOP = 16, FEW_LIST = 96, LONG_LIST = 192;
constexpr int MAX_SPLIT = 32, MAX_TOP = 64;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float NEG_INF = -__builtin_inff();

struct Stat {
  float M, Z, A;  // M = -inf: nothing above -inf (Z then 0, or NaN where a logit is NaN)
};

__device__ __forceinline__ Stat merge(Stat x, Stat y) {
  if (y.M == NEG_INF) {
    if (y.Z != y.Z) x.Z = x.A = y.Z;
    return x;
  }
  if (x.M == NEG_INF) {
    if (x.Z != x.Z) y.Z = y.A = x.Z;
    return y;
  }
  // bounded, so that a sum scaled to nothing stays zero where the difference overflows
  const float M = fmaxf(x.M, y.M);
  const float dx = fmaxf((x.M - M) * LOG2E, -1.0e30f), dy = fmaxf((y.M - M) * LOG2E, -1.0e30f);
  const float cx = __builtin_amdgcn_exp2f(dx), cy = __builtin_amdgcn_exp2f(dy);
  return {M, fmaf(cx, x.Z, cy * y.Z), fmaf(cx, fmaf(dx, x.Z, x.A), cy * fmaf(dy, y.Z, y.A))};
}

// Order of logits as unsigned numbers, -0 as +0; and back.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t LEAST_KEY = 0x007FFFFFu;  // of -inf: numbers below it are no logit's
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// The number before x, a logit above -inf (there is none between -0 and +0).
__device__ __forceinline__ float before(float x) {
  const uint32_t k = order_of(x);
  return value_of(k - (k == 0x80000000u ? 2 : 1));
}

__device__ __forceinline__ int count(bool p) { return __popcll(__ballot(p)); }
__device__ __forceinline__ int rank_in(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Keeps the k best of the entries key[e], id[e] (key 0: none) of a wave: sets keep[e]
// and returns the k-th best's key, or 0 where there are no more than k.  Equal
// keys: the lowest ids.
template <int E>
__device__ __forceinline__ uint32_t cut(const uint32_t (&key)[E], const uint32_t (&id)[E], int k, bool (&keep)[E]) {
  uint32_t T = 0;
  for (int bit = 31; bit >= 0; --bit) {  // the largest T that k keys reach
    const uint32_t c = T | 1u << bit;
    int n = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) n += count(key[e] >= c);
    if (n >= k) T = c;
  }
  if (T == 0) {
#pragma unroll
    for (int e = 0; e < E; ++e) keep[e] = key[e] != 0;
    return 0;
  }
  int above = 0, ties = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    above += count(key[e] > T);
    ties += count(key[e] == T);
  }
  const int need = k - above;  // of the ties
  uint32_t last = 0xFFFFFFFFu;
  if (ties > need) {  // the largest id that fewer than `need` ties lie below
    last = 0;
    for (int bit = 30; bit >= 0; --bit) {
      const uint32_t c = last | 1u << bit;
      int n = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) n += count(key[e] == T && id[e] < c);
      if (n < need) last = c;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) keep[e] = key[e] > T || (key[e] == T && id[e] <= last);
  return T;
}

// The kept entries side by side in keys / ids; returns their number.
template <int E>
__device__ __forceinline__ int pack(const uint32_t (&key)[E], const uint32_t (&id)[E], const bool (&keep)[E],
                                    uint32_t* keys, uint32_t* ids) {
  int n = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint64_t mask = __ballot(keep[e]);
    if (keep[e]) {
      const int at = n + rank_in(mask);
      keys[at] = key[e];
      ids[at] = id[e];
    }
    n += __popcll(mask);
  }
  return n;
}

// Entries as one number, in descending order of key, then ascending order of id.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, uint32_t id) { return (uint64_t)key << 32 | (uint32_t)~id; }

// The place of a lane's entry among those of the first n lanes, all different (64
// comparisons with a scalar each: a third of the time of sorting over the lanes,
// whose every step waits for a shuffle).
__device__ __forceinline__ int place_of(uint64_t x, int n) {
  int at = 0;
#pragma unroll 8
  for (int j = 0; j < n; ++j) {
    const uint64_t y = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), j) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, j);
    at += y > x;
  }
  return at;
}

// A bound that at least k of the lanes' numbers reach, E in each (0 if so many are not
// above 0): their k-th largest in its upper 20 bits, two bits a step.  (The logit's
// sign, exponent and eleven bits: what little passes in excess costs less than the
// 22 steps that the whole number would take bit by bit, each of which waits for a
// comparison to reach the scalar side: 1.1 us against 0.35.)
template <int E>
__device__ __forceinline__ uint32_t bound_of_lanes(const uint32_t (&x)[E], int k) {
  uint32_t T = 0;
#pragma unroll 1
  for (int bit = 30; bit >= 12; bit -= 2) {
    const uint32_t one = 1u << bit;
    int n1 = 0, n2 = 0, n3 = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      n1 += count(x[e] >= T + one);
      n2 += count(x[e] >= T + 2 * one);
      n3 += count(x[e] >= T + 3 * one);
    }
    T += n3 >= k ? 3 * one : n2 >= k ? 2 * one : n1 >= k ? one : 0u;
  }
  return T;
}

// A bound that at least k of the entries reach, or 0: of the lanes' best, those of
// even and of odd entries.
template <int E>
__device__ __forceinline__ uint32_t bound_of(const uint32_t (&key)[E], int k) {
  uint32_t best[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < E; ++e) best[e % 2] = max(best[e % 2], key[e]);
  return bound_of_lanes(best, k);
}

// The entries that may be among the k best, side by side in keys / ids: at most
// `most` of them, k where the bound leaves more.  Sets a bound that k of them reach.
// MOVE: keys and ids have room for NARROW_ROOM entries; what the bound leaves is moved
// there and cut as four entries a lane instead of E (the cut counts every entry 32
// times: one row with 64 alternatives 31 -> 25 us).  With few alternatives, whose bound
// leaves few, the added code costs up to 8%.
constexpr int NARROW_ROOM = 256;
template <int E, bool MOVE>
__device__ __forceinline__ int narrow(const uint32_t (&key)[E], const uint32_t (&id)[E], int k, int most,
                                      uint32_t* keys, uint32_t* ids, uint32_t& bound) {
  bool keep[E];
  bound = bound_of(key, k);
  int n = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    keep[e] = key[e] != 0 && key[e] >= bound;
    n += count(keep[e]);
  }
  if constexpr (MOVE) {
    if (n > most && n <= NARROW_ROOM) {
      pack<E>(key, id, keep, keys, ids);
      constexpr int F = NARROW_ROOM / 64;
      uint32_t ke[F], ie[F];
      bool kept[F];
      const int lane = __lane_id();
#pragma unroll
      for (int e = 0; e < F; ++e) {
        const int at = e * 64 + lane;
        ke[e] = at < n ? keys[at] : 0u;
        ie[e] = at < n ? ids[at] : 0xFFFFFFFFu;
      }
      bound = cut<F>(ke, ie, k, kept);
      return pack<F>(ke, ie, kept, keys, ids);
    }
  }
  if (n > most) bound = cut<E>(key, id, k, keep);
  return pack<E>(key, id, keep, keys, ids);
}

struct ScoreArgs {
  const void* logits;
  size_t ld;
  int n_rows, V, splits, k;
  const int32_t* tokens;
  float *logp, *entropy;
  int32_t* top_ids;
  float* top_logp;
  // per (row, split), record_bytes(k) apart: (M, Z, A, 0), then k (key, id) pairs
  uint8_t* ws;
};

__host__ __device__ inline size_t record_bytes(int k) { return 16 + 16 * (size_t)((k + 1) / 2); }

// The logit of the row's token; 0 without one within the vocabulary.  (Read ahead of
// the work that leads up to write_row: two loads one after the other.)
template <bool BF16>
__device__ __forceinline__ float token_logit(const ScoreArgs& p, int row, int& t) {
  t = p.tokens ? p.tokens[row] : -1;
  if (t < 0 || t >= p.V) return 0.0f;
  const size_t at = (size_t)row * p.ld + t;
  return BF16 ? bf16_to_f32(((const bf16_t*)p.logits)[at]) : ((const float*)p.logits)[at];
}

// A row's results by one wave: its statistics, its token t with logit l, and n >= k
// entries (one a lane) with the k best among them (n may be less in a row without a
// distribution).
__device__ __forceinline__ void write_row(const ScoreArgs& p, int row, Stat s, uint32_t key, uint32_t id, int n, int lane,
                                          int t, float l) {
  // no distribution: nothing above -inf, a NaN, or an infinity
  const bool ok = s.M > NEG_INF && s.M < -NEG_INF && s.Z == s.Z;
  const float nan = __builtin_nanf(""), lz = ok ? log2f(s.Z) : nan;
  if (p.k) {
    const int at = ok ? place_of(entry_of(key, id), n) : lane;
    if (at < p.k && (lane < n || !ok)) {
      const size_t o = (size_t)row * p.k + at;
      p.top_ids[o] = ok ? (int32_t)id : -1;
      p.top_logp[o] = ok ? (value_of(key) - s.M) * LOG2E - lz : nan;
    }
  }
  if (lane != 0) return;
  // a sum of nonnegative terms, up to rounding
  const float h = lz - s.A / s.Z;
  p.entropy[row] = ok ? (h < 0.0f ? 0.0f : h) : nan;
  if (p.tokens) p.logp[row] = t == -1 ? 0.0f : ok && t >= 0 && t < p.V ? (l - s.M) * LOG2E - lz : nan;
}

// A number reduced over the wave's lanes, the same in all of them: within 16 lanes by
// DPP moves, then the four results (a shuffle would go through LDS, six times in turn).
template <typename F>
__device__ __forceinline__ float reduce_lanes(float x, F f) {
#if defined(__HIP_DEVICE_COMPILE__)
  auto at = [&](auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x = f(x, at(std::integral_constant<int, 0xB1>{}));   // lane ^ 1
  x = f(x, at(std::integral_constant<int, 0x4E>{}));   // lane ^ 2
  x = f(x, at(std::integral_constant<int, 0x141>{}));  // 7 - lane, of each eight
  x = f(x, at(std::integral_constant<int, 0x140>{}));  // 15 - lane, of each sixteen
  auto lane = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); };
  x = f(f(lane(0), lane(16)), f(lane(32), lane(48)));
#endif
  return x;
}

// The lanes' statistics joined.  Without a logit above -inf a lane's Z is zero or NaN,
// and stays so whatever it is scaled with.
__device__ __forceinline__ Stat merge_lanes(Stat s) {
  const float M = reduce_lanes(s.M, [](float a, float b) { return fmaxf(a, b); });
  if (M > NEG_INF) {
    const float d = fmaxf((s.M - M) * LOG2E, -1.0e30f), c = __builtin_amdgcn_exp2f(d);
    s.A = c * fmaf(d, s.Z, s.A);
    s.Z *= c;
  }
  auto add = [](float a, float b) { return a + b; };
  return {M, reduce_lanes(s.Z, add), reduce_lanes(s.A, add)};
}

// ROWS 1: a row, or one of its `splits` parts, by a block's four waves; ROWS 4: a row
// by each of them.  CUT: entries before a list is cut, 0 without alternatives.
template <bool BF16, int CUT, int ROWS>
__global__ void __launch_bounds__(256, 8)
scores_kernel(ScoreArgs p) {
  constexpr bool TOP = CUT > 0;
  constexpr int ROOM = CUT == LONG_LIST ? TILE / 2 : TILE, LIST = CUT + ROOM;
  static_assert(LIST >= NARROW_ROOM, "room of a wave's list");
  __shared__ uint32_t keys[TOP ? 4 : 1][TOP ? LIST : 1], ids[TOP ? 4 : 1][TOP ? LIST : 1];
  __shared__ Stat stats[4];
  __shared__ int counts[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = ROWS == 4 ? blockIdx.x * 4 + wave : blockIdx.x / p.splits;
  const int split = ROWS == 4 ? 0 : blockIdx.x % p.splits;
  if (ROWS == 4 && row >= p.n_rows) return;  // a whole wave; they do not wait for each other
  constexpr int CH = BF16 ? 8 : 4;  // columns of a 16-byte load
  const uint8_t* base = (const uint8_t*)p.logits + (size_t)row * p.ld * (BF16 ? 2 : 4);
  // columns are counted from the 16-byte border at or below the row's start
  const int shift = (int)((uintptr_t)base / (BF16 ? 2 : 4) % CH);
  const int nt = (p.V + shift + TILE - 1) / TILE;
  const int per = ROWS == 4 ? nt : (nt + 4 * p.splits - 1) / (4 * p.splits);
  const int t0 = ROWS == 4 ? 0 : (split * 4 + wave) * per, t1 = min(t0 + per, nt);

  // read by the wave that writes the row, ahead of its logits
  int tok = -1;
  float tok_logit = 0.0f;
  if (ROWS == 4 || (p.splits == 1 && wave == 0)) tok_logit = token_logit<BF16>(p, row, tok);

  auto column = [&](int t, int q) {  // first column of the lane's chunk q of tile t
    return t * TILE - shift + (BF16 ? lane * 8 : q * 256 + lane * 4);
  };
  auto load = [&](int t, float (&v)[8]) {
#pragma unroll
    for (int q = 0; q < 8 / CH; ++q) {
      const int c = column(t, q);
      if (c >= 0 && c + CH <= p.V) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(base + (size_t)c * (BF16 ? 2 : 4));
#pragma unroll
        for (int i = 0; i < CH; ++i)
          v[q * CH + i] = BF16 ? __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16) : __uint_as_float(w[i % 4]);
      } else {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          v[q * CH + i] = NEG_INF;
          if (c + i >= 0 && c + i < p.V)
            v[q * CH + i] = BF16 ? bf16_to_f32(((const bf16_t*)base)[c + i]) : ((const float*)base)[c + i];
        }
      }
    }
  };

  Stat s{NEG_INF, 0.0f, 0.0f};
  float thr = NEG_INF, half[2] = {NEG_INF, NEG_INF};
  int n = 0;
  uint32_t* wk = keys[TOP ? wave : 0];
  uint32_t* wi = ids[TOP ? wave : 0];
  // a list's entries e * 64 + lane of n
  auto entry = [&](int w, int e, int n, uint32_t& key, uint32_t& id) {
    const int at = e * 64 + lane;
    key = at < n ? keys[w][at] : 0u;
    id = at < n ? ids[w][at] : 0xFFFFFFFFu;
  };
  auto shrink = [&] {
    constexpr int E = (LIST + 63) / 64;
    uint32_t key[E], id[E], bound;
#pragma unroll
    for (int e = 0; e < E; ++e) entry(wave, e, n, key[e], id[e]);
    n = narrow<E, CUT == LONG_LIST>(key, id, p.k, CUT, wk, wi, bound);
    thr = value_of(max(bound, LEAST_KEY));
  };

  auto take = [&](int t, const float (&v)[8]) {
    const float lo = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), hi = fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7]));
    const float top = fmaxf(lo, hi);
    if constexpr (CUT == LONG_LIST) {
      half[0] = fmaxf(half[0], lo);
      half[1] = fmaxf(half[1], hi);
    }
    if (top > s.M) {
      if (s.M > NEG_INF) {
        const float d = fmaxf((s.M - top) * LOG2E, -1.0e30f), c = __builtin_amdgcn_exp2f(d);
        s.A = c * fmaf(d, s.Z, s.A);
        s.Z *= c;
      }
      s.M = top;
    }
    if (s.M > NEG_INF) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = (v[i] - s.M) * LOG2E, e = __builtin_amdgcn_exp2f(x);
        s.Z += e;
        s.A = fmaf(e, fmaxf(x, -1.0e30f), s.A);  // -inf: adds 0
      }
    } else {  // the max passes over NaN
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (v[i] != v[i]) s.Z = s.A = v[i];
    }
    if constexpr (TOP) {
      const int seen = t - t0;
      bool ties = n < p.k;  // logits equal to the threshold count
      if (seen == 0 || ((seen & (seen - 1)) == 0 && t1 - t > 2)) {
        uint32_t best[2] = {order_of(s.M), 0u};
        if constexpr (CUT == LONG_LIST) {
          best[0] = order_of(half[0]);
          best[1] = order_of(half[1]);
        }
        const float up = value_of(max(bound_of_lanes(best, p.k), LEAST_KEY));
        if (seen == 0 || up > thr) {
          thr = up;
          ties = true;
        }
      }
      auto push = [&](bool in, float x, int c) {
        const uint64_t mask = __ballot(in);
        if (mask == 0) return;
        if (in) {
          const int at = n + rank_in(mask);
          wk[at] = order_of(x);
          wi[at] = (uint32_t)c;
        }
        n += __popcll(mask);
      };
      const bool all = ties && thr == NEG_INF;  // -inf too, but nothing beside the row
      // where ties count, what lies above the number before the threshold
      float above = ties ? before(thr) : thr;
      if (all || __any(top > above)) {
        constexpr int PARTS = TILE / ROOM, EACH = 8 / PARTS;
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            const float x = PARTS == 1 || h == 0 ? v[j] : v[8 - EACH + j];
            const int c = PARTS == 1 ? column(t, j / CH) + j % CH : CH == 8 ? column(t, 0) + h * EACH + j : column(t, h) + j;
            bool in = x > above;
            if (all) in = x >= thr && c >= 0 && c < p.V;
            push(in, x, c);
          }
          if (n > CUT) {
            shrink();
            // the tile's other part may have lower ids
            if (PARTS > 1 && thr > NEG_INF) above = before(thr);
          }
        }
      }
    }
  };

  int t = t0;
  for (; t + 1 < t1; t += 2) {
    float a[8], b[8];
    load(t, a);
    load(t + 1, b);
    take(t, a);
    take(t + 1, b);
  }
  if (t < t1) {
    float a[8];
    load(t, a);
    take(t, a);
  }

  if constexpr (ROWS == 4) {
    s = merge_lanes(s);
    uint32_t key = 0, id = 0xFFFFFFFFu;
    if constexpr (TOP) {
      constexpr int E = (CUT + 63) / 64;
      uint32_t ke[E], ie[E], bound;
#pragma unroll
      for (int e = 0; e < E; ++e) entry(wave, e, n, ke[e], ie[e]);
      if (n > 64) n = narrow<E, (E > 4 && CUT == LONG_LIST)>(ke, ie, p.k, 64, wk, wi, bound);
      if (lane < n) {
        key = wk[lane];
        id = wi[lane];
      }
    }
    write_row(p, row, s, key, id, n, lane, tok, tok_logit);
    return;
  }
  if (TOP && lane == 0) counts[wave] = n;
  s = merge_lanes(s);
  if (lane == 0) stats[wave] = s;
  __syncthreads();
  if (wave != 0) return;
  s = merge(merge(stats[0], stats[1]), merge(stats[2], stats[3]));
  uint32_t key = 0, id = 0xFFFFFFFFu;
  if constexpr (TOP) {
    auto join = [&](auto each_) {
      constexpr int EACH = decltype(each_)::value, E = 4 * EACH;
      uint32_t ke[E], ie[E], bound;
#pragma unroll
      for (int e = 0; e < E; ++e) entry(e & 3, e >> 2, counts[e & 3], ke[e], ie[e]);
      n = narrow<E, (E > 4 && CUT == LONG_LIST)>(ke, ie, p.k, 64, wk, wi, bound);
    };
    // mostly the lists have an entry a lane at most
    if (max(max(counts[0], counts[1]), max(counts[2], counts[3])) <= 64)
      join(std::integral_constant<int, 1>{});
    else
      join(std::integral_constant<int, (CUT + 63) / 64>{});
    if (lane < n) {
      key = wk[lane];
      id = wi[lane];
    }
  }
  if (p.splits == 1) {
    write_row(p, row, s, key, id, n, lane, tok, tok_logit);
    return;
  }
  uint8_t* w = p.ws + (size_t)blockIdx.x * record_bytes(p.k);
  if (lane == 0) *reinterpret_cast<f32x4*>(w) = f32x4{s.M, s.Z, s.A, 0.0f};
  if constexpr (TOP) {
    // the k best in order; fewer in a row's short last split
    const int at = lane < n ? place_of(entry_of(key, id), n) : lane;
    if (at < p.k) *reinterpret_cast<u32x2*>(w + 16 + 8 * at) = u32x2{key, id};
  }
}

// The splits of a row joined, by one block a row.  The first wave takes all their
// entries where a lane has no more than eight; otherwise each wave narrows those of
// eight splits, and the first wave what they leave (one wave for 32 splits took
// 30 us with 64 alternatives).
template <bool BF16>
__global__ void __launch_bounds__(256)
scores_join_kernel(ScoreArgs p) {
  constexpr int EACH = MAX_SPLIT / 4;
  __shared__ uint32_t keys[4][NARROW_ROOM], ids[4][NARROW_ROOM];
  __shared__ int counts[4];
  const int row = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const size_t rec = record_bytes(p.k);
  const uint8_t* w = p.ws + (size_t)row * p.splits * rec;
  const bool alone = p.splits * p.k <= EACH * 64;
  if (alone && wave != 0) return;
  int tok = -1;
  const float tok_logit = wave == 0 ? token_logit<BF16>(p, row, tok) : 0.0f;
  Stat s{NEG_INF, 0.0f, 0.0f};
  if (wave == 0 && lane < p.splits) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(w + lane * rec);
    s = Stat{v[0], v[1], v[2]};
  }
  uint32_t key = 0, id = 0xFFFFFFFFu;
  int n = 0;
  if (p.k) {
    uint32_t ke[EACH], ie[EACH], bound;
    const int first = alone ? 0 : wave * EACH;
    const int total = min(alone ? p.splits : EACH, p.splits - first) * p.k;  // none of a wave past the splits
    // entry e * 64 + lane of the splits' lists one after another
    int from = lane / p.k, at = lane % p.k;
    const int step = 64 / p.k, rest = 64 % p.k;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      u32x2 x{0u, 0xFFFFFFFFu};
      if (e * 64 + lane < total) x = *reinterpret_cast<const u32x2*>(w + (first + from) * rec + 16 + 8 * at);
      ke[e] = x[0];
      ie[e] = x[1];
      from += step;
      at += rest;
      if (at >= p.k) {
        at -= p.k;
        ++from;
      }
    }
    n = total > 0 ? narrow<EACH, true>(ke, ie, p.k, MAX_TOP, keys[wave], ids[wave], bound) : 0;
    if (!alone) {
      if (lane == 0) counts[wave] = n;
      __syncthreads();
      if (wave != 0) return;
      uint32_t k4[4], i4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = lane < counts[e];
        k4[e] = in ? keys[e][lane] : 0u;
        i4[e] = in ? ids[e][lane] : 0xFFFFFFFFu;
      }
      n = narrow<4, false>(k4, i4, p.k, MAX_TOP, keys[0], ids[0], bound);
    }
    if (lane < n) {
      key = keys[0][lane];
      id = ids[0][lane];
    }
  }
  write_row(p, row, merge_lanes(s), key, id, n, lane, tok, tok_logit);
}

// Whether each wave takes a row: where a row is a tile or two, or the blocks would not
// all be on the chip at once (256 CUs hold eight each).  Then the joining of a block's
// waves costs most, unless rows are so long that a CU's 32 rows at a time keep less of
// memory busy than eight: without alternatives, whose joining is short, from ten tiles
// on, and with alternatives up to 4096 rows from twenty on.  us with 0 / 8 / 20
// alternatives, a row a block and a row a wave, fp32 (bf16 where marked):
//    3000 x  1000   6.7 /  16 /  17    5.8 /  10 /  12
//    1272 x  2000   5.4 /  11 /  12    6.1 /  13 /  15
//    1272 x  4099   7.9 /  15 /  16    9.2 /  21 /  23
//    2500 x  4099    12 /  23 /  25     11 /  23 /  26
//    3000 x  9000    24 /  42 /  46     24 /  40 /  43
//    5000 x 20000    78 / 105 / 112     77 /  92 /  98
//    5000 x 20000    47 /  89 /  97     52 /  80 /  87  bf16
//   42115 x   265    52 / 140 / 129     18 /  38 /  46
//   44113 x  4099   141 / 262 / 265    125 / 170 / 192
//    2100 x126464   241 / 272 / 285    250 / 306 / 323
bool rows_by_waves(int n_rows, int V, int n_top) {
  if (V <= 2 * TILE) return true;
  if (n_rows <= 2048) return false;
  return n_top ? n_rows >= 4096 || V <= 20 * TILE : V <= 10 * TILE;
}

// Blocks a row's columns are split over: enough blocks for the chip's 256 CUs eight
// times over, but at least two tiles to a wave, and three blocks, as joining costs a
// launch (1000 x 32768 with 5 alternatives in two 49 us, unsplit 45; 600 x 126464 in
// three 86, unsplit 113).
int splits_of(int n_rows, int V, int n_top) {
  if (rows_by_waves(n_rows, V, n_top)) return 1;
  const int s = std::min({2048 / n_rows, ceil_div(V + 7, 8 * TILE), MAX_SPLIT});
  return s < 3 ? 1 : s;
}

void launch_scores(hipStream_t st, bool bf16, bool wave_rows, const ScoreArgs& p) {
  const int n_rows = p.n_rows, n_top = p.k;
  const unsigned grid = wave_rows ? (unsigned)ceil_div(n_rows, 4) : (unsigned)n_rows * p.splits;
  auto go = [&](auto four, auto one) { (wave_rows ? four : one)<<<grid, 256, 0, st>>>(p); };
  if (n_top == 0)
    bf16 ? go(scores_kernel<true, 0, 4>, scores_kernel<true, 0, 1>) : go(scores_kernel<false, 0, 4>, scores_kernel<false, 0, 1>);
  else if (n_top <= FEW_TOP)
    bf16 ? go(scores_kernel<true, FEW_LIST, 4>, scores_kernel<true, FEW_LIST, 1>)
         : go(scores_kernel<false, FEW_LIST, 4>, scores_kernel<false, FEW_LIST, 1>);
  else
    bf16 ? go(scores_kernel<true, LONG_LIST, 4>, scores_kernel<true, LONG_LIST, 1>)
         : go(scores_kernel<false, LONG_LIST, 4>, scores_kernel<false, LONG_LIST, 1>);
  DLMC_HIP(hipGetLastError());
  if (p.splits > 1) {
    if (bf16) scores_join_kernel<true><<<n_rows, 256, 0, st>>>(p);
    else scores_join_kernel<false><<<n_rows, 256, 0, st>>>(p);
    DLMC_HIP(hipGetLastError());
  }
}

}  // namespace

// A launch's rows from n_rows in parts of as many as a grid's threads, counted in 32 bits,
// allow with a block a row.  How a row is taken goes by all rows: a short last part
// decides nothing for itself, so that no part needs a workspace that the whole does not.
ScoreLaunch score_launch(int n_rows, int V, int n_top, int i) {
  constexpr int64_t LAUNCH_ROWS = 1 << 23;
  const int64_t first = i * LAUNCH_ROWS;
  ScoreLaunch l{};
  l.first = (size_t)first;
  l.rows = (int)std::max<int64_t>(0, std::min(n_rows - first, LAUNCH_ROWS));
  if (l.rows == 0) return l;
  l.by_waves = rows_by_waves(n_rows, V, n_top);
  l.splits = splits_of(n_rows, V, n_top);
  l.ws = l.splits == 1 ? 0 : (size_t)l.rows * l.splits * record_bytes(n_top);
  return l;
}

size_t token_scores_ws(int n_rows, int V, int n_top) { return score_launch(n_rows, V, n_top, 0).ws; }

void token_scores(hipStream_t st, const void* logits, bool bf16, size_t ld, int n_rows, int V, const int32_t* tokens,
                  int n_top, float* logp, float* entropy, int32_t* top_ids, float* top_logp, void* ws) {
  DLMC_CHECK(n_top >= 0 && n_top <= MAX_TOP && n_top <= V, DLMC_E_INVAL, "alternatives a row");
  for (int i = 0;; ++i) {
    const ScoreLaunch l = score_launch(n_rows, V, n_top, i);
    if (l.rows == 0) return;
    const size_t r = l.first;
    launch_scores(st, bf16, l.by_waves,
                  ScoreArgs{(const uint8_t*)logits + r * ld * (bf16 ? 2 : 4), ld, l.rows, V, l.splits, n_top,
                            tokens ? tokens + r : nullptr, tokens ? logp + r : nullptr, entropy + r,
                            n_top ? top_ids + r * n_top : nullptr, n_top ? top_logp + r * n_top : nullptr, (uint8_t*)ws});
  }
}

}  // namespace dlmc
