// Proposals from a denoiser's logits: epic_sample and epic_propose.
#include "rows.inc"

namespace epic_rows {

// ---------------------------------------------------------------- sampling
//
// One workgroup per row.  The row is read once into registers, J vectors a
// lane (J = 0, rows too long for that: every pass reads it again).  Two passes
// over the registers give the largest logit and the weights' sum W.
//
// Without a filter, one wavefront then finds the token.  With top-k or top-p
// the tokens that can matter are few in most rows: those above a bound that
// follows from the largest logits of the lanes (top-k), or from the mass that
// top-p leaves out (a token below (1 - p) W / V cannot be needed).  If there
// are at most kList of them they go into LDS in the order of their ids, are
// sorted by logit, and everything else happens there.  If there are more (flat
// rows), the threshold is found by rounds of a histogram over the row, which
// is read again from L2 by every round.
//
// Weights are whole numbers (2^31 for the likeliest token), so the order of
// the sums, the atomics' order among them, changes no result.
constexpr float kOne = 2147483648.0f;
constexpr int kBins = 1024;

struct SampleArgs {
  const char* data;
  int64_t seq_stride, row_stride;  // bytes
  int rows, V;
  Window win;
  const float *uniform, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tok;
  float* conf;
};

// floor(mass * part / 2^24) for part <= 2^24
EPIC_DEV uint64_t share(uint64_t mass, uint32_t part) {
  return (mass >> 24) * part + (((mass & 0xFFFFFFu) * part) >> 24);
}

// v_cvt_u32_f32 truncates and makes NaN 0
EPIC_DEV uint32_t to_u32(float f) {
  uint32_t r;
  asm("v_cvt_u32_f32 %0, %1" : "=v"(r) : "v"(f));
  return r;
}

// The weight of a logit: the two roundings of (l - M) * c are part of its
// definition, so they may not be contracted into one.
EPIC_DEV float power(float l, float M, float c) {
  return __builtin_amdgcn_exp2f(__fmul_rn(__fsub_rn(l, M), c));
}
EPIC_DEV uint32_t weight(float l, float M, float c) {
  return to_u32(__builtin_fmaf(power(l, M, c), kOne, 0.5f));  // 2^31 e is exact: one rounding either way
}

// Ordered keys: the logits' own bits as whole numbers in the order of the
// values, 0.0 and -0.0 the same.
template <int DT>
EPIC_DEV uint32_t key_of(float l) {
  if constexpr (DT == EPIC_F16) {
    const uint32_t h = __half_as_ushort(__float2half(l + 0.0f));
    return (h & 0x8000u) ? 0xFFFFu - h : h + 0x8000u;
  }
  const uint32_t u = __float_as_uint(l + 0.0f);
  const uint32_t k = (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return DT == EPIC_BF16 ? k >> 16 : k;
}
template <int DT>
EPIC_DEV float of_key(uint32_t k) {
  if constexpr (DT == EPIC_F16) return __half2float(__ushort_as_half((unsigned short)((k & 0x8000u) ? k - 0x8000u : 0xFFFFu - k)));
  if constexpr (DT == EPIC_BF16) return __uint_as_float((k & 0x8000u) ? (k - 0x8000u) << 16 : (0xFFFFu - k) << 16);
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

template <int DT>
constexpr float kLowest = DT == EPIC_F16 ? -65504.f : -3.38e38f;

// A row read from memory by every pass; wavefronts have the same ids as the
// lanes that hold it in registers.
template <int DT>
struct Row {
  const char* base;
  int V, first, steps, lane;  // first vector of the wavefront; vectors a lane

  // id of element 0 of the lane's vector j
  EPIC_DEV int id(int j) const { return (first + j * 64 + lane) * kPer<DT>; }
  EPIC_DEV Vec load(int j) const { return load_vec<DT>(base, first + j * 64 + lane, V); }
  template <class F>
  EPIC_DEV void elements(F&& f) const {
#pragma unroll 1
    for (int j = 0; j < steps; ++j) {
      const Vec x = load(j);
#pragma unroll
      for (int e = 0; e < kPer<DT>; ++e) f(elem<DT>(x, e), id(j) + e);
    }
  }
};

constexpr int kList = 1024;

struct SampleLds {
  union {
    uint64_t hist[kBins];
    uint64_t sorted[kList];
  };
  uint64_t list[kList];  // key of the logit, complement of the id; ascending ids
  uint64_t mass[kMaxWaves];
  float top[kMaxWaves];
  int count[kMaxWaves];
  uint64_t before;  // mass (or tokens) above the chosen bin
  uint64_t inside;  // in it
  uint32_t lo, hi;  // keys of the bin
  int32_t id;
};

// The wavefront in which the running sum of `mass` exceeds target, and what is
// left of the target there.
EPIC_DEV int owner_of(const uint64_t* mass, int waves, uint64_t target, uint64_t& left) {
  uint64_t before = 0;
  for (int w = 0; w < waves; ++w) {
    const uint64_t x = mass[w];
    if (before + x > target) {
      left = target - before;
      return w;
    }
    before += x;
  }
  left = 0;
  return -1;
}

// The element of the vectors x of a wavefront (first id of a lane's: `id`) at
// which the running sum of part(l, id) exceeds `left`; own = the lane's sum.
// One lane calls found.
template <int DT, class P, class F>
EPIC_DEV void find_element(const Vec& x, int id, uint64_t own, uint64_t left, int lane, P&& part, F&& found) {
  const uint64_t upto = scan64(own);
  const uint64_t here = __ballot(upto > left);
  if (here == 0 || lane != __ffsll((unsigned long long)here) - 1) return;
  uint64_t rest = left - (upto - own);
  int at = -1;
#pragma unroll
  for (int e = 0; e < kPer<DT>; ++e) {
    if (at >= 0) continue;
    const uint64_t p = part(elem<DT>(x, e), id + e);
    if (p > rest)
      at = e;
    else
      rest -= p;
  }
  if (at >= 0) found(id + at, elem_at<DT>(x, at));
}

// First id at which the sum of part(l, id) over the row's ids up to it exceeds
// `target`; the wavefronts' sums are in `mass`.  Called by the whole workgroup;
// the wavefront that holds the id reads its part of the row again.
template <int DT, class P, class F>
EPIC_DEV void locate(const Row<DT>& row, const uint64_t* mass, int wave, int waves, uint64_t target, P&& part,
                     F&& found) {
  uint64_t left;
  if (owner_of(mass, waves, target, left) != wave) return;
#pragma unroll 1
  for (int j = 0; j < row.steps; ++j) {
    const Vec x = row.load(j);
    uint64_t own = 0;
#pragma unroll
    for (int e = 0; e < kPer<DT>; ++e) own += part(elem<DT>(x, e), row.id(j) + e);
    const uint64_t all = wave_sum64(own);
    if (all > left) {
      find_element<DT>(x, row.id(j), own, left, row.lane, part, found);
      return;
    }
    left -= all;
  }
}

// The largest key in [lo, hi] for which `holds`, true at lo and, once false,
// false from there on.  64 probes a step; called by one wavefront.
template <class P>
EPIC_DEV uint32_t last_key(uint32_t lo, uint32_t hi, int lane, P&& holds) {
  while (lo < hi) {
    const uint32_t step = (hi - lo) / 64 + 1;
    const uint64_t at = (uint64_t)lo + (uint64_t)step * lane;
    const uint64_t yes = __ballot(at <= hi && holds((uint32_t)at));
    const int last = 63 - __clzll((long long)(yes | 1));
    lo += step * last;
    const uint64_t top = (uint64_t)lo + step - 1;
    hi = (uint32_t)(top < hi ? top : hi);
  }
  return lo;
}

// Where the ordered tokens' running sum reaches `target`: of their number
// (MASS false) or their weight (MASS true), counting tokens of the order up to
// (cut, cut_id) only.  Logits below `least` are not looked at.  Sets (cut,
// cut_id) to the token that reaches it; leaves it alone when none does.
//
// Rounds: the bins of [lo, hi] get their tokens' number or weight by LDS
// atomics, a wavefront finds the bin in which the target is reached, and the
// next round is that bin.  Bins are even steps of the logit; of the key where
// there are no more keys than bins, and the last round's bin is one key, whose
// tokens are equal and go by their ids.
template <int DT, bool MASS>
EPIC_DEV void find_cut(const Row<DT>& row, SampleLds& s, int wave, int waves, float M, float c, uint64_t target,
                       float least, float& cut, int& cut_id) {
  const int tid = (int)threadIdx.x, threads = waves * 64;
  uint32_t lo = key_of<DT>(least), hi = key_of<DT>(M);
  if (lo > hi) lo = hi;
  const float old_cut = cut;
  const int old_id = cut_id;
  while (true) {
    const float flo = of_key<DT>(lo), fhi = of_key<DT>(hi);
    const bool by_key = hi - lo < (uint32_t)kBins;
    const float scale = (float)kBins * 0.999f / (fhi - flo);
    // even steps of the logit need a finite, normal scale
    const bool even = !by_key && scale > 1e-30f && scale < 1e30f;
    int shift = 0;
    while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
    auto bin_of = [&](float l, uint32_t k) {
      const int i = even ? (int)((fhi - l) * scale) : (int)((hi - k) >> shift);
      return i < 0 ? 0 : i < kBins ? i : kBins - 1;
    };
    for (int i = tid; i < kBins; i += threads) s.hist[i] = 0;
    __syncthreads();
    row.elements([&](float l, int id) {
      if (!(l >= flo && l <= fhi)) return;
      if (!(l > old_cut || (l == old_cut && id <= old_id))) return;
      const uint64_t add = MASS ? (uint64_t)weight(l, M, c) : 1ull;
      atomicAdd((unsigned long long*)&s.hist[bin_of(l, key_of<DT>(l))], (unsigned long long)add);
    });
    __syncthreads();
    if (wave == 0) {
      uint64_t own = 0;
      const int lane = row.lane;
      for (int i = 0; i < kBins / 64; ++i) own += s.hist[lane * (kBins / 64) + i];
      const uint64_t upto = scan64(own);
      const uint64_t reach = __ballot(upto >= target);
      if (reach == 0) {
        if (lane == 0) s.id = -1;
      } else {
        const int at = __ffsll((unsigned long long)reach) - 1;
        const uint64_t base = lane64(upto - own, at);
        uint64_t before = base;
        int bin = at * (kBins / 64);
        uint64_t inside = s.hist[bin];
        while (before + inside < target) {
          before += inside;
          inside = s.hist[++bin];
        }
        // the keys of the bin
        const uint32_t top = last_key(lo, hi, lane, [&](uint32_t k) { return bin_of(of_key<DT>(k), k) >= bin; });
        const bool all = bin_of(flo, lo) <= bin;
        const uint32_t under = all ? lo : last_key(lo, hi, lane, [&](uint32_t k) { return bin_of(of_key<DT>(k), k) > bin; }) + 1;
        if (lane == 0) {
          s.id = bin;
          s.before = before;
          s.inside = inside;
          s.lo = under;
          s.hi = top;
        }
      }
    }
    __syncthreads();
    if (s.id < 0) {
      __syncthreads();
      return;
    }
    target -= s.before;
    lo = s.lo;
    hi = s.hi;
    const uint64_t inside = s.inside;
    __syncthreads();
    if (of_key<DT>(lo) != of_key<DT>(hi)) continue;
    // equal tokens: as many as are needed, the lowest ids
    cut = of_key<DT>(hi);
    uint64_t each = 1;
    if constexpr (MASS) each = weight(cut, M, c);
    const uint64_t need = (target + each - 1) / each;  // target >= 1 and is reached: each >= 1
    if (need * each >= inside) {
      cut_id = old_cut == cut ? old_id : INT32_MAX;
      return;
    }
    const float equal = cut;
    auto part = [&](float l, int id) { return (uint64_t)(l == equal ? 1 : 0); };
    uint64_t own = 0;
    row.elements([&](float l, int id) { own += part(l, id); });
    own = wave_sum64(own);
    if (row.lane == 0) s.mass[wave] = own;
    __syncthreads();
    locate(row, s.mass, wave, waves, need - 1, part, [&](int id, float) { s.id = id; });
    __syncthreads();
    cut_id = s.id;
    __syncthreads();
    return;
  }
}

EPIC_DEV uint64_t swap64(uint64_t v, int x) {
  return ((uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), x, 64) << 32) | (uint32_t)__shfl_xor((int)v, x, 64);
}
// lanes x apart in order: the larger key in the lane with `up`
EPIC_DEV uint64_t order64(uint64_t v, int x, bool up) {
  const uint64_t o = swap64(v, x);
  return (v > o) == up ? v : o;
}
// 64 keys, descending by lane
EPIC_DEV uint64_t sort64(uint64_t v, int lane) {
#pragma unroll
  for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
    for (int x = k >> 1; x > 0; x >>= 1) v = order64(v, x, ((lane & k) == 0) == ((lane & x) == 0));
  return v;
}
// The token drawn from a list of N tokens in the order of their ids, in which
// all that the filters can keep are found.  k: top-k or INT32_MAX; P: top-p in
// 2^24ths; S: the mass that P is a share of, or 0 for the mass of the first k.
// Called by the whole workgroup, `found` by one lane of it.
template <int DT, class F>
EPIC_DEV void draw_from_list(SampleLds& s, int N, int wave, int waves, float M, float c, int k, uint32_t P, uint64_t S,
                             uint32_t least, uint32_t U, F&& found) {
  const int tid = (int)threadIdx.x, lane = tid & 63;
  auto weigh = [&](uint64_t key) { return key ? (uint64_t)weight(of_key<DT>((uint32_t)(key >> 32)), M, c) : 0ull; };
  if (N <= 64) {  // one wavefront, a token a lane
    if (wave != 0) return;
    const uint64_t mine = lane < N ? s.list[lane] : 0;
    const uint64_t ranked = sort64(mine, lane);
    const uint64_t w = lane < k ? weigh(ranked) : 0;
    const uint64_t upto = scan64(w);
    if (S == 0) S = lane64(upto, 63);
    const uint64_t want = share(S, P), need = want > 0 ? want : 1;
    // the tokens whose mass before is short of the need: a prefix of the order
    const uint64_t prefix = __ballot(lane < N && lane < k && upto - w < need);
    const uint64_t last = lane64(ranked, 63 - __clzll((long long)(prefix | 1)));
    uint64_t kept = weigh(mine);
    if (mine < last || kept < least) kept = 0;
    const uint64_t sum = scan64(kept);
    const uint64_t target = share(lane64(sum, 63), U);
    const uint64_t here = __ballot(sum > target);
    if (lane == __ffsll((unsigned long long)here) - 1)
      found((int)~(uint32_t)mine, of_key<DT>((uint32_t)(mine >> 32)));
    return;
  }
  int size = 128;
  while (size < N) size *= 2;
  const int threads = waves * 64;
  for (int i = tid; i < size; i += threads) s.sorted[i] = i < N ? s.list[i] : 0;
  for (int run = 2; run <= size; run *= 2)
    for (int x = run / 2; x > 0; x /= 2) {
      __syncthreads();
      for (int p = tid; p < size / 2; p += threads) {
        const int i = 2 * p - (p & (x - 1)), j = i + x;
        const uint64_t a = s.sorted[i], b = s.sorted[j];
        if ((a < b) == ((i & run) == 0)) {
          s.sorted[i] = b;
          s.sorted[j] = a;
        }
      }
    }
  __syncthreads();
  if (wave != 0) return;
  const int per = size / 64;  // a lane's tokens, adjacent
  uint64_t own = 0;
  for (int i = lane * per; i < lane * per + per; ++i)
    if (i < k) own += weigh(s.sorted[i]);
  uint64_t upto = scan64(own);
  if (S == 0) S = lane64(upto, 63);
  const uint64_t want = share(S, P), need = want > 0 ? want : 1;
  uint64_t before = upto - own, mine = ~0ull;  // the lane's last token of the prefix
  for (int i = lane * per; i < lane * per + per; ++i) {
    if (i >= N || i >= k || before >= need) break;
    mine = s.sorted[i];
    before += weigh(mine);
  }
  const uint64_t some = __ballot(mine != ~0ull);
  const uint64_t last = lane64(mine, 63 - __clzll((long long)(some | 1)));
  auto kept = [&](int i) -> uint64_t {
    const uint64_t key = i < N ? s.list[i] : 0, w = weigh(key);
    return key < last || w < least ? 0 : w;
  };
  own = 0;
  for (int i = lane * per; i < lane * per + per; ++i) own += kept(i);
  upto = scan64(own);
  const uint64_t target = share(lane64(upto, 63), U);
  const uint64_t here = __ballot(upto > target);
  if (lane != __ffsll((unsigned long long)here) - 1) return;
  uint64_t rest = target - (upto - own);
  for (int i = lane * per; i < lane * per + per; ++i) {
    const uint64_t w = kept(i);
    if (w > rest) {
      found((int)~(uint32_t)s.list[i], of_key<DT>((uint32_t)(s.list[i] >> 32)));
      return;
    }
    rest -= w;
  }
}

// A logit that at least k of the workgroup's lanes' largest reach, hence at
// least k logits: a lower bound of the k-th largest.  `none` when fewer than k
// lanes have one of any weight.
template <int DT>
EPIC_DEV float bound_of_top(SampleLds& s, float mine, int wave, int waves, float M, float c, int k, float none) {
  const int tid = (int)threadIdx.x, lane = tid & 63;
  constexpr int bins = 512;
  const float scale = c * (bins / 33.0f);
  for (int i = tid; i < bins; i += waves * 64) s.hist[i] = 0;
  __syncthreads();
  const float at = (M - mine) * scale;  // M is finite; a lane of nothing but -inf is out
  if (at < (float)bins) atomicAdd((unsigned long long*)&s.hist[(int)at], 1ull);
  __syncthreads();
  uint64_t own = 0;
  for (int i = 0; i < bins / 64; ++i) own += s.hist[lane * (bins / 64) + i];
  const uint64_t upto = scan64(own);
  const uint64_t reach = __ballot(upto >= (uint64_t)k);
  float bound = none;
  if (reach) {
    const int l = __ffsll((unsigned long long)reach) - 1;
    uint64_t before = lane64(upto - own, l);
    int bin = l * (bins / 64);
    while ((before += s.hist[bin]) < (uint64_t)k) ++bin;
    // the lanes counted have (M - l) * scale < bin + 1; a little below that is below them all
    const float low = M - (float)(bin + 1) / scale;
    bound = low - fabsf(low) * 1e-6f - fabsf(M) * 1e-6f;
  }
  __syncthreads();
  return fmaxf(bound, none);
}

template <int DT, int J>
__global__ void __launch_bounds__(1024) sample_kernel(SampleArgs a) {
  __shared__ SampleLds s;
  constexpr int E = kPer<DT>;
  const int r = (int)blockIdx.x, b = r / a.rows, i = r - b * a.rows;
  const int threads = (int)blockDim.x, waves = threads >> 6;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const bool counts = row_counts(a.win, b, i);
  const float T = a.temperature ? a.temperature[b] : 1.0f;
  if (!counts || T != T) {
    if (threadIdx.x == 0) {
      a.tok[r] = -1;
      a.conf[r] = 0.f;
    }
    return;
  }
  Row<DT> row;
  row.base = a.data + b * a.seq_stride + i * a.row_stride;
  row.V = a.V;
  row.lane = (int)threadIdx.x & 63;
  row.steps = J ? J : ((a.V + E - 1) / E + threads - 1) / threads;
  row.first = wave * row.steps * 64;
  const int lane = row.lane;
  Vec v[J ? J : 1];
  if constexpr (J > 0) {
#pragma unroll
    for (int j = 0; j < J; ++j) v[j] = row.load(j);
  }
  // Without this the compiler keeps what one pass computed of every element
  // for the next, which takes more registers than there are.
  auto forget = [&] {
    if constexpr (J > 0) {
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(v[j].d[k]));
    }
  };
  auto each = [&](auto&& f) {  // f(vector, j)
    if constexpr (J > 0) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        f(v[j], j);
        __builtin_amdgcn_sched_barrier(0);  // a vector's temporaries at a time
      }
    } else {
#pragma unroll 1
      for (int j = 0; j < row.steps; ++j) f(row.load(j), j);
    }
  };

  float mine = -kInf;
  each([&](const Vec& x, int) {
#pragma unroll
    for (int e = 0; e < E; ++e) mine = fmaxf(mine, elem<DT>(x, e));
  });
  float M = wave_max(mine);
  if (lane == 0) s.top[wave] = M;
  __syncthreads();
  for (int w = 0; w < waves; ++w) M = fmaxf(M, s.top[w]);
  M = lane32(M, 0);
  if (!(M > -kInf && M < kInf)) {  // no finite logit, or one of +inf
    if (threadIdx.x == 0) {
      a.tok[r] = -1;
      a.conf[r] = 0.f;
    }
    return;
  }
  const bool greedy = T <= 0.f;
  const float c = greedy ? kLog2e : fminf((float)(1.4426950408889634 / (double)T), 1e30f);

  // greedy is the first of the order
  int k = greedy ? 1 : a.top_k ? a.top_k[b] : 0;
  const float p = a.top_p && !greedy ? a.top_p[b] : 1.f, q = a.min_p && !greedy ? a.min_p[b] : 0.f;
  const float u = fminf(fmaxf(a.uniform[r], 0.f), 1.f);
  k = k > 0 && k < a.V ? k : INT32_MAX;
  const uint32_t P = p < 1.f ? (uint32_t)(fmaxf(p, 0.f) * 16777216.f) : 16777216u;
  const uint32_t least = q > 0.f ? to_u32(__builtin_fmaf(fminf(q, 1.f), kOne, 0.5f)) : 0u;
  const uint32_t U = min((uint32_t)(u * 16777216.f), 16777215u);
  const bool by_k = k != INT32_MAX, by_p = P < 16777216u;

  forget();
  uint64_t sums[J ? J : 1] = {};  // the lane's, by vector
  each([&](const Vec& x, int j) {
    uint64_t w = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) w += weight(elem<DT>(x, e), M, c);
    sums[J ? j : 0] += w;
  });
  uint64_t own = 0;
#pragma unroll
  for (int j = 0; j < (J ? J : 1); ++j) own += sums[j];
  own = wave_sum64(own);
  if (lane == 0) s.mass[wave] = own;
  __syncthreads();
  uint64_t W = 0;
  for (int w = 0; w < waves; ++w) W += s.mass[w];
  W = lane64(W, 0);
  auto found = [&](int id, float l) {
    a.tok[r] = id;
    a.conf[r] = power(l, M, c) * (kOne / (float)W);
  };

  if (!by_k && !by_p && !least) {
    auto part = [&](float l, int) { return (uint64_t)weight(l, M, c); };
    const uint64_t target = share(W, U);
    if constexpr (J > 0) {
      uint64_t left;
      if (owner_of(s.mass, waves, target, left) != wave) return;
      uint64_t at = 0, mass = 0;
      Vec x = v[0];
      int j = -1;
#pragma unroll
      for (int t = 0; t < J; ++t) {
        const uint64_t all = wave_sum64(sums[t]);
        if (j < 0 && all > left) {
          j = t;
          x = v[t];
          mass = sums[t];
          at = left;
        }
        left -= all;  // not read again once found
      }
      find_element<DT>(x, row.id(j), mass, at, lane, part, found);
    } else {
      locate(row, s.mass, wave, waves, target, part, found);
    }
    return;
  }

  float cut = -kInf;  // kept: logits above it, and equal ones up to cut_id
  int cut_id = INT32_MAX;
  {
    // tokens further than 33 doublings below the largest weigh nothing; -inf is no token
    const float far = M - 33.0f / c;
    const float light = fmaxf(far - fabsf(far) * 1e-5f, kLowest<DT>);
    float low = light;
    if (k == 1) {
      low = M;
    } else if (by_k) {
      if (k <= threads) low = bound_of_top<DT>(s, mine, wave, waves, M, c, k, light);
    } else {
      // what top-p leaves out, or what min-p does
      const float part = !by_p ? (float)least : (float)(16777216u - P) * (1.f / 16777216.f) * (float)W / (float)a.V;
      const float deep = M + (log2f(part * (1.f / kOne)) - 0.01f) / c;
      low = fmaxf(light, deep - fabsf(deep) * 1e-5f - fabsf(M) * 1e-5f);
    }
    low = fminf(low, M);  // rows of the type's lowest values
    forget();
    int n = 0;
    each([&](const Vec& x, int) {
#pragma unroll
      for (int e = 0; e < E; ++e) n += elem<DT>(x, e) >= low ? 1 : 0;
    });
    n = (int)wave_sum64((uint64_t)n);
    if (lane == 0) s.count[wave] = n;
    __syncthreads();
    int N = 0, at = 0;
    for (int w = 0; w < waves; ++w) {
      if (w == wave) at = N;
      N += s.count[w];
    }
    N = __builtin_amdgcn_readfirstlane(N);
    if (N <= kList) {
      forget();
      each([&](const Vec& x, int j) {
        uint32_t in = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) in |= elem<DT>(x, e) >= low ? 1u << e : 0u;
        if (__ballot(in != 0) == 0) return;
        const int upto = (int)scan64((uint64_t)__popc(in));
        int to = at + upto - __popc(in);
        at += __builtin_amdgcn_readlane(upto, 63);
        for (; in; in &= in - 1) {
          const int e = __ffs((int)in) - 1;
          s.list[to++] = ((uint64_t)key_of<DT>(elem_at<DT>(x, e)) << 32) | (uint32_t)~(row.id(j) + e);
        }
      });
      __syncthreads();
      draw_from_list<DT>(s, N, wave, waves, M, c, k, P, by_k ? 0 : W, least, U, found);
      return;
    }
    // many: by rounds over the row
    uint64_t S = W;
    if (by_k) {
      find_cut<DT, false>(row, s, wave, waves, M, c, (uint64_t)k, low, cut, cut_id);
      uint64_t some = 0;
      row.elements([&](float l, int id) {
        const uint32_t w = weight(l, M, c);
        some += (l > cut || (l == cut && id <= cut_id)) ? w : 0u;
      });
      some = wave_sum64(some);
      __syncthreads();
      if (lane == 0) s.mass[wave] = some;
      __syncthreads();
      S = 0;
      for (int w = 0; w < waves; ++w) S += s.mass[w];
    }
    if (by_p) {
      const uint64_t want = share(S, P);
      __syncthreads();
      find_cut<DT, true>(row, s, wave, waves, M, c, want > 0 ? want : 1, low, cut, cut_id);
    }
  }
  auto kept = [&](float l, int id) -> uint64_t {
    const uint32_t w = weight(l, M, c);
    return (l > cut || (l == cut && id <= cut_id)) && w >= least ? w : 0u;
  };
  uint64_t some = 0;
  row.elements([&](float l, int id) { some += kept(l, id); });
  some = wave_sum64(some);
  __syncthreads();
  if (lane == 0) s.mass[wave] = some;
  __syncthreads();
  uint64_t D = 0;
  for (int w = 0; w < waves; ++w) D += s.mass[w];
  locate(row, s.mass, wave, waves, share(D, U), kept, found);
}

// --------------------------------------------------------------- proposals
//
// One workgroup per sequence: every wavefront sorts 64 rows at a time by
// (confidence, lower row first) and keeps its best 64; the wavefronts' lists
// are merged in pairs through LDS.  Where the sequence's candidates go follows
// from how many the earlier sequences have, min(per_seq, rows with a token):
// every workgroup counts them itself, which is one load of 64 tokens for most
// sequences; a batch too large for that has them counted by a launch before.
struct ProposeArgs {
  const int32_t* tok;
  const float* conf;
  const int32_t* start;
  int32_t *seq, *pos, *out_tok;
  float* out_conf;
  int32_t* offsets;
  int B, m, P;
};

EPIC_DEV bool proposes(int32_t t, float f) { return t >= 0 && f == f; }

// descending by the high word (the ordered confidence), then by the low one
// (the complement of the row); 0: nothing
EPIC_DEV uint64_t propose_key(int32_t t, float f, int row) {
  if (!proposes(t, f)) return 0;
  const uint32_t u = __float_as_uint(f + 0.0f);
  const uint32_t k = (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return ((uint64_t)k << 32) | (uint32_t)~row;
}

// the best 64 of two descending lists, descending
EPIC_DEV uint64_t merge64(uint64_t a, uint64_t b, int lane) {
  const uint64_t r = swap64(b, 63);
  uint64_t v = a > r ? a : r;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) v = order64(v, x, (lane & x) == 0);
  return v;
}

// min(P, rows of sequence b with a token), by one wavefront
EPIC_DEV int count_rows(const ProposeArgs& a, int b, int lane) {
  int n = 0;
  for (int at = 0; at < a.m && n < a.P; at += 64) {
    const int i = at + lane;
    bool yes = false;
    if (i < a.m) yes = proposes(a.tok[(int64_t)b * a.m + i], a.conf[(int64_t)b * a.m + i]);
    n += __popcll((unsigned long long)__ballot(yes));
  }
  return min(n, a.P);
}

// the offsets of a large batch: one workgroup, sequences dealt to wavefronts
__global__ void __launch_bounds__(1024) propose_count_kernel(ProposeArgs a) {
  __shared__ int n[1024];
  __shared__ int base;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) base = a.offsets[0] = 0;
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    for (int k = wave; k < 1024; k += 16) {
      const int c = b0 + k < a.B ? count_rows(a, b0 + k, lane) : 0;
      if (lane == 0) n[k] = c;
    }
    __syncthreads();
    if (wave == 0) {
      int own = 0;
      for (int k = 0; k < 16; ++k) own += n[lane * 16 + k];
      const int upto = (int)scan64((uint64_t)own);
      int at = base + upto - own;
      for (int k = 0; k < 16; ++k) {
        at += n[lane * 16 + k];
        if (b0 + lane * 16 + k < a.B) a.offsets[b0 + lane * 16 + k + 1] = at;
      }
      if (lane == 63) base += upto;
    }
    __syncthreads();
  }
}

template <bool COUNTED>
__global__ void __launch_bounds__(1024) propose_kernel(ProposeArgs a) {
  __shared__ uint64_t list[kMaxWaves][64];
  __shared__ int part[kMaxWaves];
  const int b = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = (int)blockDim.x >> 6;
  const int32_t* tok = a.tok + (int64_t)b * a.m;
  const float* conf = a.conf + (int64_t)b * a.m;
  uint64_t best = 0;
  for (int at = wave * 64; at < a.m; at += waves * 64) {
    const int i = at + lane;
    const uint64_t k = sort64(i < a.m ? propose_key(tok[i], conf[i], i) : 0, lane);
    best = at == wave * 64 ? k : merge64(best, k, lane);
  }
  int off = 0, total = 0;
  if constexpr (!COUNTED) {
    int before = 0, all = 0;
    for (int o = wave; o < a.B; o += waves) {
      const int c = count_rows(a, o, lane);
      before += o < b ? c : 0;
      all += c;
    }
    if (lane == 0) part[wave] = before;
    __syncthreads();
    for (int w = 0; w < waves; ++w) off += part[w];
    __syncthreads();
    if (lane == 0) part[wave] = all;
    __syncthreads();
    for (int w = 0; w < waves; ++w) total += part[w];
  } else {
    off = a.offsets[b];
    total = a.offsets[a.B];
  }
  for (int half = 1; half < waves; half <<= 1) {
    list[wave][lane] = best;
    __syncthreads();
    if ((wave & (2 * half - 1)) == 0 && wave + half < waves) best = merge64(best, list[wave + half][lane], lane);
    __syncthreads();
  }
  if (wave != 0) return;
  const int mine = __popcll((unsigned long long)__ballot(best != 0 && lane < a.P));
  if (lane < mine) {
    const int row = (int)~(uint32_t)best;
    a.seq[off + lane] = b;
    a.pos[off + lane] = (a.start ? a.start[b] : 0) + row;
    a.out_tok[off + lane] = tok[row];
    a.out_conf[off + lane] = conf[row];
  }
  // the entries past the last candidate, each by the sequence that lacks it
  const int pad = total + (b * a.P - off);
  if (lane < a.P - mine) {
    a.seq[pad + lane] = -1;
    a.pos[pad + lane] = -1;
    a.out_tok[pad + lane] = -1;
    a.out_conf[pad + lane] = 0.f;
  }
  if constexpr (!COUNTED) {
    if (lane == 0) {
      if (b == 0) a.offsets[0] = 0;
      a.offsets[b + 1] = off + mine;
    }
  }
}

template <int DT>
epic_status launch_sample(const SampleArgs& a, int blocks, hipStream_t stream) {
  const int nvec = (a.V + kPer<DT> - 1) / kPer<DT>;
  auto threads = [&](int J) { return std::max(64, ((nvec + J - 1) / J + 63) / 64 * 64); };
#define EPIC_SAMPLE(J, NT) hipLaunchKernelGGL((sample_kernel<DT, J>), dim3(blocks), dim3(NT), 0, stream, a)
  if (nvec <= 2 * 64)
    EPIC_SAMPLE(2, threads(2));
  else if (nvec <= 4 * 256)
    EPIC_SAMPLE(4, threads(4));
  else if (nvec <= 8 * 512)
    EPIC_SAMPLE(8, threads(8));
  else if (nvec <= 16 * 1024)
    EPIC_SAMPLE(16, threads(16));
  else
    EPIC_SAMPLE(0, 1024);
#undef EPIC_SAMPLE
  return hipGetLastError() == hipSuccess ? EPIC_OK : EPIC_ERR_HIP;
}

}  // namespace epic_rows

extern "C" {

epic_status epic_sample(const epic_rows_desc* logits, const int32_t* d_seqs, int32_t n, const int32_t* d_start,
                        const float* d_uniform, const float* d_temperature, const int32_t* d_top_k,
                        const float* d_top_p, const float* d_min_p, int32_t* d_tok, float* d_conf,
                        hipStream_t stream) {
  using namespace epic_rows;
  epic_status st = check_rows(logits, d_seqs, n);
  if (st != EPIC_OK || logits->batch == 0 || logits->rows == 0) return st;
  if (!d_uniform || !d_tok || !d_conf) return EPIC_ERR_NULL;
  const int es = elem_size(logits->dtype);
  SampleArgs a{(const char*)logits->data, logits->seq_stride * es, logits->row_stride * es, logits->rows, logits->vocab,
               {d_seqs, d_start, n}, d_uniform, d_temperature, d_top_p, d_min_p, d_top_k, d_tok, d_conf};
  const int blocks = logits->batch * logits->rows;
  switch (logits->dtype) {
    case EPIC_F32: return launch_sample<EPIC_F32>(a, blocks, stream);
    case EPIC_F16: return launch_sample<EPIC_F16>(a, blocks, stream);
    default: return launch_sample<EPIC_BF16>(a, blocks, stream);
  }
}

epic_status epic_propose(const int32_t* d_tok, const float* d_conf, int32_t batch, int32_t rows,
                         const int32_t* d_start, int32_t per_seq, int32_t* d_cand_seq, int32_t* d_cand_pos,
                         int32_t* d_cand_tok, float* d_cand_conf, int32_t* d_offsets, hipStream_t stream) {
  using namespace epic_rows;
  if (batch < 0 || rows < 0 || per_seq < 1 || per_seq > 64) return EPIC_ERR_ARG;
  if ((int64_t)batch * rows > INT32_MAX / 2 || (int64_t)batch * per_seq > INT32_MAX / 2) return EPIC_ERR_ARG;
  if (!d_offsets) return EPIC_ERR_NULL;
  if (batch > 0 && (!d_cand_seq || !d_cand_pos || !d_cand_tok || !d_cand_conf)) return EPIC_ERR_NULL;
  if (batch > 0 && rows > 0 && (!d_tok || !d_conf)) return EPIC_ERR_NULL;
  ProposeArgs a{d_tok, d_conf, d_start, d_cand_seq, d_cand_pos, d_cand_tok, d_cand_conf, d_offsets, batch, rows, per_seq};
  const int threads = std::min(1024, std::max(64, (rows + 63) / 64 * 64));
  if (batch > 0 && batch <= 256) {
    hipLaunchKernelGGL(propose_kernel<false>, dim3(batch), dim3(threads), 0, stream, a);
  } else {
    hipLaunchKernelGGL(propose_count_kernel, dim3(1), dim3(1024), 0, stream, a);
    if (batch > 0) hipLaunchKernelGGL(propose_kernel<true>, dim3(batch), dim3(threads), 0, stream, a);
  }
  return hipGetLastError() == hipSuccess ? EPIC_OK : EPIC_ERR_HIP;
}

}  // extern "C"
