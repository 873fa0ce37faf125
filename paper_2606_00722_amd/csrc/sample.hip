// Proposals from a denoiser's logits: epic_sample and epic_propose.
#include "rows.inc"

namespace epic_rows {

// ---------------------------------------------------------------- sampling
//
// One workgroup per row.  The row is read once into registers, J vectors a
// lane (J = 0, rows too long for that: every pass reads it again).  Two passes
// over the registers give the largest logit and the weights' sum W; without a
// filter one wavefront then finds the token.
//
// With a filter the tokens that it can keep are few in most rows, and end in a
// list in LDS, where one wavefront does the rest:
//  * top-k: those above a bound that follows from the lanes' largest logits;
//  * top-p: a histogram of the weights over the logits gives the step in which
//    the mass is reached, and those of that step are listed;
//  * min-p: those above the logit that it stands for.
// For top-k and min-p only the pairs of vectors whose largest logit is above the
// bound are read again, mostly none of a lane's.  If the list is too short for
// them (flat rows, a large k), a histogram gives the step of the border, the
// tokens of that step are listed and give the exact border, and one more pass
// sums what is kept.  If even those are too many (thousands of equal logits), the
// border is found by rounds of ever finer histograms.  The passes of top-p after
// the first read the row again, from L2: as unrolled code over registers they
// took as many registers as there are, and their arithmetic costs seven times the
// reading.
//
// Weights are whole numbers (2^31 for the likeliest token), so the order of
// the sums, the atomics' order among them, changes no result.
//
// Bound: without filters by the reading and the exponentials, about even (2048
// rows of 32768 bfloat16 logits, 80 % of them counted, in 32 us: 3.5 TB/s, vector
// units busy half of the time).  With top-k the list's latency is added (2867 rows, top-k 50:
// 60 us against 46), with top-p the arithmetic of two more passes (134 us;
// settings of all kinds take 23 vector instructions a logit, none 14).  Few rows are bound by the length of the chain:
// one row of 32768 takes 7 us without and 10 us with all filters.  Rows of 100003
// float32 logits are read by every pass: 158 of them with top-p take 60 us, of
// which four readings at a copy's 5.0 TB/s are 50.
constexpr float kOne = 2147483648.0f;

struct SampleArgs {
  const char* data;
  int64_t seq_stride, row_stride;  // bytes
  int rows, V;
  Window win;
  const float *uniform, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tok;
  float* conf;
  int spread;  // of how many rows those that count are dealt to the first workgroups (0: to their own)
  int first;   // row of the launch
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

// The exponent of a logit: its two roundings are part of the definition, so
// they may not be contracted into one.  Monotonic, and so are the steps that
// are counted of it.
EPIC_DEV float exponent(float l, float M, float c) { return __fmul_rn(__fsub_rn(l, M), c); }
EPIC_DEV float power(float l, float M, float c) { return __builtin_amdgcn_exp2f(exponent(l, M, c)); }
EPIC_DEV uint32_t weight_of(float x) {
  return to_u32(__builtin_fmaf(__builtin_amdgcn_exp2f(x), kOne, 0.5f));  // 2^31 e is exact: one rounding either way
}
EPIC_DEV uint32_t weight(float l, float M, float c) { return weight_of(exponent(l, M, c)); }
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
constexpr float kLowest = DT == EPIC_F16 ? -65504.f : DT == EPIC_BF16 ? -0x1.FEp127f : -0x1.FFFFFEp127f;  // finite

// A row read from memory by a pass; wavefronts have the same ids as the lanes
// that hold it in registers.
template <int DT>
struct Row {
  const char* base;
  int V, first, steps, lane;  // first vector of the wavefront; vectors a lane

  // id of element 0 of the lane's vector j
  EPIC_DEV int id(int j) const { return (first + j * 64 + lane) * kPer<DT>; }
  EPIC_DEV Vec load(int j) const {
    const int at = first + j * 64;
    return (at + 64) * kPer<DT> <= V ? load_whole<DT>(base, at + lane) : load_vec<DT>(base, at + lane, V);
  }
  // f(vector, j) for every j, G loads ahead
  template <int G = 2, class F>
  EPIC_DEV void vectors(F&& f) const {
    Vec a[G], b[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (g < steps) a[g] = load(g);
#pragma unroll 1
    for (int j = 0; j < steps; j += G) {
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (j + G + g < steps) b[g] = load(j + G + g);
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (j + g < steps) {
          f(a[g], j + g);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
      for (int g = 0; g < G; ++g) a[g] = b[g];
    }
  }
  template <int G = 2, class F>
  EPIC_DEV void elements(F&& f) const {
    vectors<G>([&](const Vec& x, int j) {
#pragma unroll
      for (int e = 0; e < kPer<DT>; ++e) f(elem<DT>(x, e), id(j) + e);
    });
  }
};

// BINS: of the histogram; room: of the list, the tokens that are put in order in
// LDS.  A step in which a border lies should hold no more than that: 33 doublings
// of weight in 1024 steps put 90 of 32768 normally distributed logits (deviation
// 2) in one, so longer rows have more steps.  That does not part equal logits, of
// which 131072 in bfloat16 have hundreds of a value: such rows go another way.
template <int BINS>
struct SampleLds {
  static constexpr int bins = BINS, room = 512;
  static constexpr int skew = BINS + BINS / 16;  // 17 words of 8 bytes every 16 bins
  uint64_t hist[skew];
  uint64_t list[room];  // entries, in no order
  uint32_t weights[room];
  uint64_t mass[kMaxWaves];
  float top[kMaxWaves];
  int listed;
  uint64_t before;  // mass (or tokens) above the chosen bin
  uint64_t inside;  // in it
  uint32_t lo, hi;  // keys of the bin
  uint64_t cut;
  int32_t id;
};
EPIC_DEV int slot(int bin) { return bin + (bin >> 4); }

// The sum of the wavefronts' masses.
EPIC_DEV uint64_t mass_of(const uint64_t* mass, int waves, int lane) {
  return wave_sum64(lane < waves ? mass[lane] : 0);
}
// The wavefront in which the running sum of `mass` exceeds target (-1: none),
// and what is left of the target there.
EPIC_DEV int owner_of(const uint64_t* mass, int waves, int lane, uint64_t target, uint64_t& left) {
  const uint64_t x = lane < waves ? mass[lane] : 0, upto = scan64(x);
  const uint64_t over = __ballot(upto > target);
  if (over == 0) return -1;
  const int w = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)over) - 1);
  left = target - lane64(upto - x, w);
  return w;
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
  uint64_t left = 0;
  if (owner_of(mass, waves, row.lane, target, left) != wave) return;
  bool open = true;
  row.vectors([&](const Vec& x, int j) {
    if (!open) return;
    uint64_t own = 0;
#pragma unroll
    for (int e = 0; e < kPer<DT>; ++e) own += part(elem<DT>(x, e), row.id(j) + e);
    const uint64_t all = wave_sum64(own);
    if (all > left) {
      open = false;
      find_element<DT>(x, row.id(j), own, left, row.lane, part, found);
    }
    left -= all;  // not read again once found
  });
}

// The bin in which the running sum of the histogram reaches `target` (-1:
// none), the sum before it and what is in it, by one wavefront.
template <int BINS>
EPIC_DEV int scan_bins(const uint64_t* hist, uint64_t target, int lane, uint64_t& before, uint64_t& inside) {
  constexpr int per = BINS / 64;  // a lane's
  uint64_t own = 0;
#pragma unroll 1
  for (int q = 0; q < per; q += 16) {
    const uint64_t* at = hist + slot(lane * per + q);  // 8 or 16 bins between two gaps
#pragma unroll 4
    for (int i = 0; i < (per < 16 ? per : 16); ++i) own += at[i];
  }
  const uint64_t upto = scan64(own);
  const uint64_t reach = __ballot(upto >= target);
  if (reach == 0) return -1;
  const int at = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)reach) - 1);
  const uint64_t base = lane64(upto - own, at);
  const uint64_t x = lane < per ? hist[slot(at * per + lane)] : 0;
  const uint64_t sum = base + scan64(x);
  const int i = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(sum >= target)) - 1);
  inside = lane64(x, i);
  before = lane64(sum, i) - inside;
  return at * per + i;
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

// scan_bins by one wavefront for the workgroup.
template <int BINS, class LDS>
EPIC_DEV int border_bin(LDS& s, uint64_t target, int wave, int lane, uint64_t& before) {
  if (wave == 0) {
    uint64_t under = 0, inside;  // no bin: nothing before
    const int bin = scan_bins<BINS>(s.hist, target, lane, under, inside);
    if (lane == 0) {
      s.id = bin;
      s.before = under;
    }
  }
  __syncthreads();
  const int bin = __builtin_amdgcn_readfirstlane(s.id);
  before = s.before;
  __syncthreads();
  return bin;
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
template <int DT, bool MASS, class LDS>
EPIC_DEV void find_cut(const Row<DT>& row, LDS& s, int wave, int waves, float M, float c, uint64_t target,
                       float least, float& cut, int& cut_id) {
  const int tid = (int)threadIdx.x, threads = waves * 64;
  uint32_t lo = key_of<DT>(least), hi = key_of<DT>(M);
  if (lo > hi) lo = hi;
  const float old_cut = cut;
  const int old_id = cut_id;
  while (true) {
    const float flo = of_key<DT>(lo), fhi = of_key<DT>(hi);
    const bool by_key = hi - lo < (uint32_t)LDS::bins;
    const float scale = (float)LDS::bins * 0.999f / (fhi - flo);
    // even steps of the logit need a finite, normal scale
    const bool even = !by_key && scale > 1e-30f && scale < 1e30f;
    int shift = 0;
    while (((hi - lo) >> shift) >= (uint32_t)LDS::bins) ++shift;
    auto bin_of = [&](float l, uint32_t k) {
      const int i = even ? (int)((fhi - l) * scale) : (int)((hi - k) >> shift);
      return i < 0 ? 0 : i < LDS::bins ? i : LDS::bins - 1;
    };
    for (int i = tid; i < LDS::skew; i += threads) s.hist[i] = 0;
    __syncthreads();
    row.elements([&](float l, int id) {
      if (!(l >= flo && l <= fhi)) return;
      if (!(l > old_cut || (l == old_cut && id <= old_id))) return;
      const uint64_t add = MASS ? (uint64_t)weight(l, M, c) : 1ull;
      atomicAdd((unsigned long long*)&s.hist[slot(bin_of(l, key_of<DT>(l)))], (unsigned long long)add);
    });
    __syncthreads();
    if (wave == 0) {
      const int lane = row.lane;
      uint64_t before, inside;
      const int bin = scan_bins<LDS::bins>(s.hist, target, lane, before, inside);
      if (bin < 0) {
        if (lane == 0) s.id = -1;
      } else {
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

// lane i's value in lane i ^ X
template <int X>
EPIC_DEV uint32_t swap32(uint32_t v) {
  if constexpr (X == 1) return dpp<0xB1>(0u, v);
  if constexpr (X == 2) return dpp<0x4E>(0u, v);
  if constexpr (X == 4) return dpp<0x1B>(0u, dpp<0x141>(0u, v));  // ^7, then ^3
  if constexpr (X == 8) return dpp<0x128>(0u, v);                 // rotate the row of 16 by 8
  if constexpr (X == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return __builtin_amdgcn_inverse_ballot_w64(0xFFFF0000FFFF0000ull) ? r[0] : r[1];
  }
  const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __builtin_amdgcn_inverse_ballot_w64(0xFFFFFFFF00000000ull) ? r[0] : r[1];
}
// lanes X apart in order: the larger key in the lanes of `up`
template <int X>
EPIC_DEV uint64_t order64(uint64_t v, uint64_t up) {
  const uint64_t o = ((uint64_t)swap32<X>((uint32_t)(v >> 32)) << 32) | swap32<X>((uint32_t)v);
  return (v > o) == __builtin_amdgcn_inverse_ballot_w64(up) ? v : o;
}
constexpr uint64_t lanes_without(int bit) {
  uint64_t m = 0;
  for (int i = 0; i < 64; ++i) m |= (uint64_t)((i & bit) == 0) << i;
  return m;
}
template <int K, int X>
EPIC_DEV uint64_t sort_step(uint64_t v) {
  constexpr uint64_t up = ~(lanes_without(K) ^ lanes_without(X));
  v = order64<X>(v, up);
  if constexpr (X > 1) return sort_step<K, X / 2>(v);
  return v;
}
// 64 keys, descending by lane (bitonic)
EPIC_DEV uint64_t sort64(uint64_t v) {
  v = sort_step<2, 1>(v);
  v = sort_step<4, 2>(v);
  v = sort_step<8, 4>(v);
  v = sort_step<16, 8>(v);
  v = sort_step<32, 16>(v);
  return sort_step<64, 32>(v);
}

// A token of a list: greater means earlier in the order.
EPIC_DEV uint64_t entry(uint32_t key, int id) { return ((uint64_t)key << 32) | (uint32_t)~id; }
EPIC_DEV uint32_t key_in(uint64_t e) { return (uint32_t)(e >> 32); }
EPIC_DEV int id_in(uint64_t e) { return (int)~(uint32_t)e; }

// the highest bit of an id
EPIC_DEV int top_bit(int V) { return V > 1 ? 1 << (31 - __clz(V - 1)) : 0; }

// What the lanes of a wavefront wrote to LDS, before others of its lanes read it.
EPIC_DEV void lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Lists in LDS (s.list, entries in no order), worked on by one wavefront.  Sums
// over the entries i of a list are of part(i).
template <class P>
EPIC_DEV uint64_t sum_list(int N, int lane, P&& part) {
  uint64_t sum = 0;
#pragma unroll 1
  for (int i = lane; i < N; i += 64) sum += part(i);
  return wave_sum64(sum);
}

// Where the running sum of part(i) reaches `target` >= 1, over the entries in
// the order of step(i) (0 to 511) and, within a step, of rank(i), greatest
// first.  Returns the rank of the entry that reaches it; 0 when the sum does not
// reach it, or when more than 64 entries are in its step, with crowded = true.
//
// A histogram over the steps and a sort of the entries of one: a few hundred
// clocks, where a search for the key bit by bit takes as many for every bit.
template <class LDS, class S, class K, class P>
EPIC_DEV uint64_t reach_by_steps(LDS& s, int N, int lane, uint64_t target, S&& step, K&& rank, P&& part,
                                 bool& crowded) {
  constexpr int bins = 512;
  crowded = false;
#pragma unroll 1
  for (int i = lane; i < bins + bins / 16; i += 64) s.hist[i] = 0;
  lds_fence();
#pragma unroll 1
  for (int i = lane; i < N; i += 64) {
    const uint64_t p = part(i);
    if (p) atomicAdd((unsigned long long*)&s.hist[slot(step(i))], (unsigned long long)p);
  }
  lds_fence();
  uint64_t before, inside;
  const int bin = scan_bins<bins>(s.hist, target, lane, before, inside);
  if (bin < 0) return 0;
  lds_fence();
  int count = 0;  // of the step's entries, whose numbers go to the histogram's place
#pragma unroll 1
  for (int i0 = 0; i0 < N; i0 += 64) {
    const int i = i0 + lane;
    const bool in = i < N && step(i) == bin && part(i) != 0;
    const uint64_t all = __ballot(in);
    const int to = count + __popcll((unsigned long long)(all & ((1ull << lane) - 1)));
    if (in && to < 64) s.hist[to] = (uint64_t)i;
    count += __popcll((unsigned long long)all);
  }
  lds_fence();
  if (count > 64) {
    crowded = true;
    return 0;
  }
  const int mine = lane < count ? (int)s.hist[lane] : 0;
  const uint64_t key = lane < count ? rank(mine) : 0, p = lane < count ? part(mine) : 0;
  lds_fence();
  // the parts in the order of the ranks, by the place of every entry in it
  const uint64_t ranked = sort64(key);
  int place = 0;
#pragma unroll 1
  for (int i = 0; i < count; ++i) place += lane64(ranked, i) > key ? 1 : 0;
  if (lane < count) s.hist[place] = p;
  lds_fence();
  const uint64_t upto = scan64(lane < count ? s.hist[lane] : 0);
  const int j = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(upto >= target - before)) - 1);
  return lane64(ranked, j);
}

// The lowest id at which the running sum of part(i), in the order of the ids,
// reaches `target` >= 1, into `id` (false: it does not).  If more than 64 are in
// one of the steps of the vocabulary, bit by bit.
template <class LDS, class P>
EPIC_DEV bool reach_id(LDS& s, int N, int lane, uint64_t target, int V, P&& part, int& id) {
  const float scale = 511.0f / (float)V;
  bool crowded;
  const uint64_t e = reach_by_steps(
      s, N, lane, target, [&](int i) { return (int)((float)id_in(s.list[i]) * scale); },
      [&](int i) { return (uint64_t)(uint32_t)s.list[i]; }, part, crowded);  // the id's complement
  id = id_in(e);
  if (!crowded) return e != 0;
  if (sum_list(N, lane, part) < target) return false;
  id = 0;
#pragma unroll 1
  for (int bit = top_bit(V); bit; bit >>= 1) {
    const int to = id + bit;
    if (sum_list(N, lane, [&](int i) { return id_in(s.list[i]) < to ? part(i) : 0; }) < target) id = to;
  }
  return true;
}

// The entry of s.list at which the running sum of part(i), in the order of the
// entries, reaches `target` >= 1 (0: it does not).  Steps are even in the logit;
// if too many entries are in one (equal logits), the key is searched by halves,
// then the id among equal keys.
template <int DT, class LDS, class P>
EPIC_DEV uint64_t reach_entry(LDS& s, int N, int lane, uint64_t target, int V, P&& part) {
  float top = -kInf, bottom = kInf;
#pragma unroll 1
  for (int i = lane; i < N; i += 64) {
    const float l = of_key<DT>(key_in(s.list[i]));
    top = fmaxf(top, l);
    bottom = fminf(bottom, l);
  }
  top = wave_max(top);
  bottom = -wave_max(-bottom);
  const float scale = 511.0f / (top - bottom);
  if (scale > 1e-30f && scale < 1e30f) {
    bool crowded;
    const uint64_t e = reach_by_steps(
        s, N, lane, target,
        [&](int i) { return min((int)((top - of_key<DT>(key_in(s.list[i]))) * scale), 511); },
        [&](int i) { return s.list[i]; }, part, crowded);
    if (!crowded) return e;
  }
  uint32_t key = key_of<DT>(bottom), over = key_of<DT>(top) + 1;  // the sum is reached at key, if at all, and not at over
#pragma unroll 1
  while (over - key > 1) {
    const uint32_t at = key + (over - key) / 2;
    if (sum_list(N, lane, [&](int i) { return key_in(s.list[i]) >= at ? part(i) : 0; }) >= target)
      key = at;
    else
      over = at;
  }
  const uint64_t above = sum_list(N, lane, [&](int i) { return key_in(s.list[i]) > key ? part(i) : 0; });
  auto equal = [&](int i) -> uint64_t { return key_in(s.list[i]) == key ? part(i) : 0; };
  const uint64_t with = above + sum_list(N, lane, equal);
  if (with < target) return 0;
  if (with == target) return entry(key, INT32_MAX);
  int at;
  const uint64_t found = reach_id(s, N, lane, target - above, V, equal, at);
  return found ? entry(key, at) : 0;
}

struct Draw {
  float M, c;
  int k;           // top-k, INT32_MAX: off
  uint32_t P;      // top-p in 2^24ths of the mass of the first k
  uint32_t least;  // min-p
  uint32_t U;
  int V;
};

// The token drawn from a list of N tokens, in which all that the filters can
// keep are found; by one wavefront.  Up to 64: a token a lane.
template <int DT, class LDS, class F>
EPIC_DEV void draw_from_short_list(LDS& s, int N, int lane, const Draw& d, F&& found) {
  const uint64_t e = lane < N ? s.list[lane] : 0;
  uint32_t w = e ? weight(of_key<DT>(key_in(e)), d.M, d.c) : 0;
  uint64_t cut = 0;
  if (d.k < N || d.P < 16777216u) {
    const uint64_t ranked = sort64(e);
    const uint64_t rw = ranked && lane < d.k ? (uint64_t)weight(of_key<DT>(key_in(ranked)), d.M, d.c) : 0;
    const uint64_t upto = scan64(rw);
    const uint64_t want = share(lane64(upto, 63), d.P), need = want > 0 ? want : 1;
    // the tokens whose mass before is short of the need: a prefix of the order
    const uint64_t prefix = __ballot(ranked != 0 && lane < d.k && upto - rw < need);
    cut = lane64(ranked, 63 - __clzll((long long)(prefix | 1)));
  }
  if (e < cut || w < d.least) w = 0;
  // in the order of the ids, the weights with them
  const uint64_t by_id = sort64(w ? ((uint64_t)(uint32_t)e << 32) | w : 0);
  const uint64_t upto = scan64((uint32_t)by_id);
  const uint64_t here = __ballot(upto > share(lane64(upto, 63), d.U));
  const int id = ~__builtin_amdgcn_readlane((int)(by_id >> 32), __ffsll((unsigned long long)here) - 1);
  if (w && id_in(e) == id) found(id, of_key<DT>(key_in(e)));
}
template <int DT, class LDS, class F>
EPIC_DEV void draw_from_list(LDS& s, int N, int lane, const Draw& d, F&& found) {
#pragma unroll 1
  for (int i = lane; i < N; i += 64) s.weights[i] = weight(of_key<DT>(key_in(s.list[i])), d.M, d.c);
  lds_fence();
  uint64_t cut = 0;
  if (d.k < N) cut = reach_entry<DT>(s, N, lane, (uint64_t)d.k, d.V, [&](int) -> uint64_t { return 1; });
  if (d.P < 16777216u) {
    auto in = [&](int i) -> uint64_t { return s.list[i] >= cut ? s.weights[i] : 0; };
    const uint64_t sum = sum_list(N, lane, in);
    const uint64_t want = share(sum, d.P), need = want > 0 ? want : 1;
    if (need < sum) cut = reach_entry<DT>(s, N, lane, need, d.V, in);
  }
  auto kept = [&](int i) -> uint64_t { return s.list[i] >= cut && s.weights[i] >= d.least ? s.weights[i] : 0; };
  // the lowest id at which the mass is over the target
  const uint64_t target = share(sum_list(N, lane, kept), d.U);
  int id;
  if (!reach_id(s, N, lane, target + 1, d.V, kept, id)) return;  // the kept mass is 2^31 at least
#pragma unroll 1
  for (int i = lane; i < N; i += 64)
    if (id_in(s.list[i]) == id) found(id, of_key<DT>(key_in(s.list[i])));
}

// A logit that at least k of the lanes' largest of their even and odd vectors
// reach, hence at least k logits: a lower bound of the k-th largest.  `none`
// when fewer than k of these have any weight.
template <class LDS>
EPIC_DEV float bound_of_top(LDS& s, float mine, float mine2, int wave, int waves, float M, float c, int k, float none) {
  const int tid = (int)threadIdx.x, lane = tid & 63;
  constexpr int bins = 512;
  const float scale = c * (bins / 33.0f);
  for (int i = tid; i < bins + bins / 16; i += waves * 64) s.hist[i] = 0;
  __syncthreads();
  const float at = (M - mine) * scale, at2 = (M - mine2) * scale;  // M is finite; a lane of nothing but -inf is out
  if (at < (float)bins) atomicAdd((unsigned long long*)&s.hist[slot((int)at)], 1ull);
  if (at2 < (float)bins) atomicAdd((unsigned long long*)&s.hist[slot((int)at2)], 1ull);
  __syncthreads();
  uint64_t before;
  const int bin = border_bin<bins>(s, (uint64_t)k, wave, lane, before);
  if (bin < 0) return none;
  // the lanes counted have (M - l) * scale < bin + 1; a little below that is below them all
  const float low = M - (float)(bin + 1) / scale;
  return fmaxf(low - fabsf(low) * 1e-6f - fabsf(M) * 1e-6f, none);
}

template <int DT, class LDS>
EPIC_DEV void list_token(LDS& s, float l, int id) {
  const int i = atomicAdd(&s.listed, 1);
  if (i < LDS::room) s.list[i] = entry(key_of<DT>(l), id);
}

// Those of a vector's tokens that reach `low`; false once the list is too short.
template <int DT, class LDS>
EPIC_DEV bool list_vector(LDS& s, const Vec& x, int id, float low) {
  uint32_t in = 0;
#pragma unroll
  for (int e = 0; e < kPer<DT>; ++e) in |= elem<DT>(x, e) >= low ? 1u << e : 0u;
  if (!in) return true;
  int at = atomicAdd(&s.listed, __popc(in));
  if (at + __popc(in) > LDS::room) return false;
#pragma unroll
  for (int e = 0; e < kPer<DT>; ++e)
    if (in & (1u << e)) s.list[at++] = entry(key_of<DT>(elem<DT>(x, e)), id + e);
  return true;
}

// The entry among the `count` <= LDS::room tokens of s.list at which the
// running sum of their numbers or weights reaches target >= 1; by the whole
// workgroup, of which one wavefront works.
template <int DT, bool MASS, class LDS>
EPIC_DEV uint64_t border_entry(LDS& s, int count, uint64_t target, int wave, int lane, int V, float M, float c) {
  if (wave == 0) {
    auto weigh = [&](uint64_t e) -> uint32_t {
      return e == 0 ? 0u : MASS ? weight(of_key<DT>(key_in(e)), M, c) : 1u;
    };
    uint64_t cut;
    if (count <= 64) {
      const uint64_t ranked = sort64(lane < count ? s.list[lane] : 0);
      const uint64_t reach = __ballot(scan64(weigh(ranked)) >= target);
      cut = lane64(ranked, __ffsll((unsigned long long)reach) - 1);
    } else {
#pragma unroll 1
      for (int i = lane; i < count; i += 64) s.weights[i] = weigh(s.list[i]);
      lds_fence();
      cut = reach_entry<DT>(s, count, lane, target, V, [&](int i) -> uint64_t { return s.weights[i]; });
    }
    if (lane == 0) s.cut = cut;
  }
  __syncthreads();
  const uint64_t cut = s.cut;
  __syncthreads();
  return cut;
}

// Where the order's running sum of numbers or weights reaches `target`, as an
// entry (0: nowhere).  Counts tokens of the order up to `old` only; logits
// below `low` are not looked at.  One pass for a histogram over even steps of
// the logit, one to collect the tokens of the step in which the target is
// reached, which a wavefront puts in order.
template <int DT, bool MASS, class LDS>
EPIC_DEV uint64_t border_of(const Row<DT>& row, LDS& s, int wave, int waves, float M, float c, uint64_t target,
                            float low, uint64_t old) {
  const int tid = (int)threadIdx.x, lane = row.lane;
  const float old_l = old ? of_key<DT>(key_in(old)) : -kInf;
  const int old_id = old ? id_in(old) : INT32_MAX;
  auto counts = [&](float l, int id) { return l >= low && (l > old_l || (l == old_l && id <= old_id)); };
  const float scale = (float)(LDS::bins - 1) / (M - low);
  if (scale > 1e-30f && scale < 1e30f) {
    for (int i = tid; i < LDS::skew; i += waves * 64) s.hist[i] = 0;
    if (tid == 0) s.listed = 0;
    __syncthreads();
    row.elements([&](float l, int id) {
      if (counts(l, id)) {
        const int bin = min((int)((M - l) * scale), LDS::bins - 1);
        atomicAdd((unsigned long long*)&s.hist[slot(bin)], MASS ? (unsigned long long)weight(l, M, c) : 1ull);
      }
    });
    __syncthreads();
    uint64_t before;
    const int bin = border_bin<LDS::bins>(s, target, wave, lane, before);
    if (bin < 0) return 0;
    row.elements([&](float l, int id) {
      if (counts(l, id) && min((int)((M - l) * scale), LDS::bins - 1) == bin) {
        list_token<DT>(s, l, id);
      }
    });
    __syncthreads();
    const int count = s.listed;
    __syncthreads();
    if (count <= LDS::room) return border_entry<DT, MASS>(s, count, target - before, wave, lane, row.V, M, c);
  }
  float cut_l = old_l;
  int cut_id = old_id;
  find_cut<DT, MASS>(row, s, wave, waves, M, c, target, low, cut_l, cut_id);
  return cut_l == -kInf ? 0 : entry(key_of<DT>(cut_l), cut_id);
}

// Row number x of all, those that count first and then the others, by the whole
// workgroup.  Rows that take a CU for themselves and are not many more than the
// CUs would else lie unevenly: workgroups go to the XCDs and their parts in
// turn, whether their row counts or not.  1055 rows of 100003 float32 logits of
// which 158 count, top-p 0.95: 67 us against 105; 1024 of 131072 float16, 212
// count: 66 against 110.  Where all rows count it costs (1024 rows of 65536
// bfloat16: 36.0 us without filters against 32.7, 136 with top-p against 134),
// and the positions of a window are mostly masked: calls with d_start do without.
constexpr int kSpread = 2048;  // rows at most
EPIC_DEV int nth_row(const SampleArgs& a, uint64_t* masks, int x, int wave, int waves, int lane) {
  const int chunks = (a.spread + 63) >> 6;
  for (int c = wave; c < chunks; c += waves) {
    const int r = c * 64 + lane, b = r / a.rows;
    const uint64_t in = __ballot(r < a.spread && row_counts(a.win, b, r - b * a.rows));
    if (lane == 0) masks[c] = in;
  }
  __syncthreads();
  uint64_t mine = lane < chunks ? masks[lane] : 0;
  uint64_t upto = scan64((uint64_t)__popcll((unsigned long long)mine));
  const int all = (int)lane64(upto, 63);
  if (x >= all) {
    x -= all;
    const int left = a.spread - lane * 64;
    mine = left <= 0 ? 0 : ~mine & (left < 64 ? (1ull << left) - 1 : ~0ull);
    upto = scan64((uint64_t)__popcll((unsigned long long)mine));
  }
  const int c = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot((int)upto > x)) - 1);
  const uint64_t in = lane64(mine, c);
  x -= (int)lane64(upto, c) - __popcll((unsigned long long)in);
  const bool here = (in >> lane & 1) && __popcll((unsigned long long)(in & ((1ull << lane) - 1))) == x;
  return c * 64 + __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(here)) - 1);
}

template <int DT, int J>
__global__ void __launch_bounds__(1024) sample_kernel(SampleArgs a) {
  using LDS = SampleLds<J == 0 || J == 16 ? 4096 : J == 8 ? 2048 : 1024>;
  __shared__ LDS s;
  constexpr int E = kPer<DT>;
  constexpr float kSteps = -(float)(LDS::bins / 33);  // steps of a doubling
  const int threads = (int)blockDim.x, waves = threads >> 6;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  int r = a.first + (int)blockIdx.x;
  if constexpr (J == 0 || J == 16)
    if (a.spread) r = nth_row(a, s.list, r, wave, waves, (int)threadIdx.x & 63);
  const int b = r / a.rows, i = r - b * a.rows;
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
  asm("" : "+s"(row.steps));  // not a constant: loops over it stay loops
  const int lane = row.lane;
  Vec v[J ? J : 1];
  if constexpr (J > 0) {
    if ((row.first + J * 64) * E <= a.V) {
#pragma unroll
      for (int j = 0; j < J; ++j) v[j] = load_whole<DT>(row.base, row.first + j * 64 + lane);
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) v[j] = row.load(j);
    }
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
      row.template vectors<8>(f);
    }
  };

  float mine = -kInf, mine2 = -kInf;  // of the lane's even and odd vectors
  float largest[J ? J / 2 : 1];       // of every pair of vectors
  each([&](const Vec& x, int j) {
    float m = -kInf;
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, elem<DT>(x, e));
    if constexpr (J > 0) largest[j / 2] = j & 1 ? fmaxf(largest[j / 2], m) : m;
    if (j & 1)
      mine2 = fmaxf(mine2, m);
    else
      mine = fmaxf(mine, m);
  });
  float M = wave_max(fmaxf(mine, mine2));
  if (lane == 0) s.top[wave] = M;
  __syncthreads();
  const float M_wave = M;
  M = wave_max(lane < waves ? s.top[lane] : -kInf);
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
  uint64_t sums[J > 1 ? J / 2 : 1] = {};  // the lane's, by pair of vectors
  uint64_t own_of_p = 0;
  const bool steps_of_p = by_p && !by_k;
  if (!steps_of_p) {
    each([&](const Vec& x, int j) {
      uint64_t w = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) w += weight(elem<DT>(x, e), M, c);
      sums[J ? j / 2 : 0] += w;
    });
  } else {
    // With it the weights by steps of the exponent, for top-p's border.  What
    // top-p leaves out weighs (1 - p) W at least, and W is 2^31 at least: steps
    // of which no token weighs the V-th part of that are not needed to get there.
    // A weight is up to 2^31 e + 1/2, and where less than a whole one is left of
    // that part without the half, no step is left out.  The border's step is then
    // always found: the steps counted weigh W - (1 - p) 2^31 >= p W.
    for (int i = (int)threadIdx.x; i < LDS::skew; i += threads) s.hist[i] = 0;
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
    const float light = (float)(16777216u - P) * (kOne / 16777216.f) / (float)a.V - 0.5f;
    const float all_steps = (float)LDS::bins;
    const float last = light > 1.f ? fminf(floorf(log2f(light / kOne) * kSteps) + 2.f, all_steps) : all_steps;
    row.template vectors<4>([&](const Vec& v, int) {
      uint64_t all = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float x = exponent(elem<DT>(v, e), M, c), step = x * kSteps;
        const uint32_t w = weight_of(x);
        all += w;
        if (step < last) atomicAdd((unsigned long long*)&s.hist[slot((int)step)], (unsigned long long)w);
      }
      own_of_p += all;
    });
  }
  uint64_t own = own_of_p;
#pragma unroll
  for (int j = 0; j < (J > 1 ? J / 2 : 1); ++j) own += sums[j];
  own = wave_sum64(own);
  if (lane == 0) s.mass[wave] = own;
  __syncthreads();
  const uint64_t W = mass_of(s.mass, waves, lane);
  auto found = [&](int id, float l) {
    a.tok[r] = id;
    a.conf[r] = power(l, M, c) * (kOne / (float)W);
  };

  if (!by_k && !by_p && !least) {
    auto part = [&](float l, int) { return (uint64_t)weight(l, M, c); };
    const uint64_t target = share(W, U);
    if constexpr (J > 0) {
      uint64_t left = 0;
      if (owner_of(s.mass, waves, lane, target, left) != wave) return;
      int j = -1;
#pragma unroll
      for (int t = 0; t < J / 2; ++t) {
        const uint64_t all = wave_sum64(sums[t]);
        if (j < 0) {
          if (all > left)
            j = 2 * t;
          else
            left -= all;
        }
      }
      j = __builtin_amdgcn_readfirstlane(j);
      Vec x = row.load(j);
      const Vec y = row.load(j + 1);
      uint64_t own_x = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) own_x += part(elem<DT>(x, e), 0);
      const uint64_t all = wave_sum64(own_x);
      if (all <= left) {
        left -= all;
        ++j;
        x = y;
        own_x = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) own_x += part(elem<DT>(x, e), 0);
      }
      find_element<DT>(x, row.id(j), own_x, left, lane, part, found);
    } else {
      locate(row, s.mass, wave, waves, target, part, found);
    }
    return;
  }

  // tokens further than 33 doublings below the largest weigh nothing; -inf is no token
  const float far = M - 33.0f / c;
  const float light = fmaxf(far - fabsf(far) * 1e-5f, kLowest<DT>);
  auto above = [&](float weighs) {  // a logit below all that weigh as much, which 2^31 e does from a half less on
    const float deep = M + (log2f((weighs - 0.5f) * (1.f / kOne)) - 0.01f) / c;
    return fmaxf(light, deep - fabsf(deep) * 1e-5f - fabsf(M) * 1e-5f);
  };
  uint64_t cut = 0;  // kept: entries not after it
  bool summed = false;
  if (steps_of_p) {
    const uint64_t want = share(W, P), need = want > 0 ? want : 1;
    uint64_t before;
    const int bin = border_bin<LDS::bins>(s, need, wave, lane, before);
    // one pass collects the tokens of the border's step and sums those before it
    const float first = (float)bin;
    uint64_t some = 0;
    row.template elements<4>([&](float l, int id) {
      const float x = exponent(l, M, c), step = x * kSteps;
      if (step < first) {
        const uint32_t w = weight_of(x);
        some += w >= least ? w : 0u;
      } else if (step < first + 1.f) {
        list_token<DT>(s, l, id);
      }
    });
    some = wave_sum64(some);
    __syncthreads();
    if (lane == 0) s.mass[wave] = some;
    const int count = s.listed;
    __syncthreads();
    if (count <= LDS::room) {
      cut = border_entry<DT, true>(s, count, need - before, wave, lane, a.V, M, c);
      // the border's own, to the wavefront that has their ids
      for (int i = (int)threadIdx.x; i < count; i += threads) {
        const uint64_t e = s.list[i];
        const uint32_t w = weight(of_key<DT>(key_in(e)), M, c);
        if (e >= cut && w >= least)
          atomicAdd((unsigned long long*)&s.mass[id_in(e) / (row.steps * 64 * E)], (unsigned long long)w);
      }
      __syncthreads();
      summed = true;
    } else {
      cut = border_of<DT, true>(row, s, wave, waves, M, c, need, fminf(light, M), 0);
    }
  } else {
    float low = light;
    if (k == 1)
      low = M;
    else if (by_k && k <= 2 * threads)
      low = bound_of_top(s, mine, mine2, wave, waves, M, c, k, light);
    else if (!by_k)
      low = above((float)least);
    low = fminf(low, M);  // rows of the type's lowest values
    if (!by_k || k <= 2 * threads) {
      if (threadIdx.x == 0) s.listed = 0;
      __syncthreads();
      if constexpr (J > 0) {
        // The lane's pairs of vectors that have one, mostly none, are read again.
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < J / 2; ++j) hits |= largest[j] >= low ? 1u << j : 0u;
        while (hits) {
          const int j = 2 * (__ffs(hits) - 1), at = row.first + j * 64 + lane;
          hits &= hits - 1;
          const Vec x = load_vec<DT>(row.base, at, a.V), y = load_vec<DT>(row.base, at + 64, a.V);
          if (!list_vector<DT>(s, x, row.id(j), low) || !list_vector<DT>(s, y, row.id(j + 1), low)) break;
        }
      } else if (M_wave >= low) {
        bool open = true;
        row.vectors([&](const Vec& x, int j) {
          float m = -kInf;
#pragma unroll
          for (int e = 0; e < E; ++e) m = fmaxf(m, elem<DT>(x, e));
          if (open && m >= low) open = list_vector<DT>(s, x, row.id(j), low);
        });
      }
      __syncthreads();
      const int N = __builtin_amdgcn_readfirstlane(s.listed);
      if (N <= LDS::room) {
        if (wave != 0) return;
        const Draw draw{M, c, k, P, least, U, a.V};
        if (N <= 64)
          draw_from_short_list<DT>(s, N, lane, draw, found);
        else
          draw_from_list<DT>(s, N, lane, draw, found);
        return;
      }
      __syncthreads();
    }
    if (by_k) cut = border_of<DT, false>(row, s, wave, waves, M, c, (uint64_t)k, low, 0);
    if (by_k && by_p) {
      const float cut_l = cut ? of_key<DT>(key_in(cut)) : -kInf;
      const int cut_id = cut ? id_in(cut) : INT32_MAX;
      uint64_t some = 0;
      row.elements([&](float l, int id) {
        const uint32_t w = weight(l, M, c);
        some += (l > cut_l || (l == cut_l && id <= cut_id)) ? w : 0u;
      });
      some = wave_sum64(some);
      __syncthreads();
      if (lane == 0) s.mass[wave] = some;
      __syncthreads();
      const uint64_t S = mass_of(s.mass, waves, lane);
      const uint64_t want = share(S, P);
      __syncthreads();
      cut = border_of<DT, true>(row, s, wave, waves, M, c, want > 0 ? want : 1, low, cut);
    }
  }
  const float cut_l = cut ? of_key<DT>(key_in(cut)) : -kInf;
  const int cut_id = cut ? id_in(cut) : INT32_MAX;
  auto kept = [&](float l, int id) -> uint64_t {
    const uint32_t w = weight(l, M, c);
    return (l > cut_l || (l == cut_l && id <= cut_id)) && w >= least ? w : 0u;
  };
  if (!summed) {  // the wavefronts' sums are still to be made
    uint64_t some = 0;
    row.elements([&](float l, int id) { some += kept(l, id); });
    some = wave_sum64(some);
    __syncthreads();
    if (lane == 0) s.mass[wave] = some;
    __syncthreads();
  }
  const uint64_t D = mass_of(s.mass, waves, lane);
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
//
// Bound by latency: 64 sequences of 1024 positions take 7.8 us on the GPU (0.5 MB,
// 0.1 us of reading), 8 of 128 take 4.9; the sort of 64 is 21 exchanges, a merge
// six, and each load of the counting is one trip to memory.
struct ProposeArgs {
  const int32_t* tok;
  const float* conf;
  const int32_t* start;
  int32_t *seq, *pos, *out_tok;
  float* out_conf;
  int32_t* offsets;
  int B, m, P;
  int first;  // sequence of the launch
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

EPIC_DEV uint64_t reversed(uint64_t v, int lane) {
  return ((uint64_t)(uint32_t)__shfl((int)(v >> 32), 63 - lane, 64) << 32) | (uint32_t)__shfl((int)v, 63 - lane, 64);
}
// the best 64 of two lists, a descending and b ascending, descending
EPIC_DEV uint64_t merge64(uint64_t a, uint64_t b) {
  // the greater of the first and the last, and so on, are the best 64, and bitonic
  return sort_step<64, 32>(a > b ? a : b);
}

// Adds the rows with a token among 64 H rows from `at` of eight sequences first,
// first + step, ..., whose loads are all in flight together, to n of lane 0, 1,
// ...; counts end at P.
constexpr int kCounts = 8;
template <int H>
EPIC_DEV void count_round(const ProposeArgs& a, int first, int step, int at, int lane, int& n) {
  int32_t t[kCounts][H];
  float f[kCounts][H];
#pragma unroll
  for (int g = 0; g < kCounts; ++g)
#pragma unroll
    for (int h = 0; h < H; ++h) {
      // never a branch around a load: they would wait for each other
      const int64_t row = (int64_t)min(first + g * step, a.B - 1) * a.m;
      const uint32_t i = (uint32_t)min(at + h * 64 + lane, a.m - 1);
      t[g][h] = (a.tok + row)[i];
      f[g][h] = (a.conf + row)[i];
    }
#pragma unroll
  for (int g = 0; g < kCounts; ++g) {
    int c = 0;
#pragma unroll
    for (int h = 0; h < H; ++h)
      c += __popcll((unsigned long long)__ballot(at + h * 64 + lane < a.m && proposes(t[g][h], f[g][h])));
    n += lane == g ? c : 0;
  }
  n = min(n, a.P);
}
// n and the rows with a token of sequence b from row `at` on, at most P, by one
// wavefront, 64 G rows at a time
template <int G>
EPIC_DEV int count_rows(const ProposeArgs& a, int b, int at, int lane, int n) {
  const int32_t* tok = a.tok + (int64_t)b * a.m;
  const float* conf = a.conf + (int64_t)b * a.m;
#pragma unroll 1
  for (at += lane; at - lane < a.m && n < a.P; at += 64 * G) {
    int32_t t[G];
    float f[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t i = (uint32_t)min(at + g * 64, a.m - 1);
      t[g] = tok[i];
      f[g] = conf[i];
    }
#pragma unroll
    for (int g = 0; g < G; ++g) n += __popcll((unsigned long long)__ballot(at + g * 64 < a.m && proposes(t[g], f[g])));
  }
  return min(n, a.P);
}
// min(P, rows with a token) of eight sequences first, first + step, ..., in lanes
// 0, 1, ... (0 past the last sequence and in the other lanes), by one wavefront.
// Most are settled by their first 64 rows.  Up to 320 rows the rest of more than
// two follows at once (64 sequences of 300 rows that have fewer than P: 8.9 us a
// call on the GPU), else one sequence after another (64 of 1024: 14.1 us; 4 of 130:
// 5.3, at once 5.9).  Counts stay in a register of one lane each: eight in every
// lane, and the loads beside them, took more registers than there are.  Batches
// counted by a launch of their own take 5.5 to 12.5 us (17 to 1024 sequences of up
// to 64 rows).
EPIC_DEV int count_eight(const ProposeArgs& a, int first, int step, int lane) {
  int n = 0;
  if (a.m <= 0 || first >= a.B) return n;
  const bool there = lane < kCounts && first + lane * step < a.B;
  count_round<1>(a, first, step, 0, lane, n);
  if (a.m > 64) {
    uint64_t open = __ballot(there && n < a.P);
    const bool few = a.m <= 64 + 256;
    if (few && __popcll((unsigned long long)open) > 2) {
      count_round<4>(a, first, step, 64, lane, n);
    } else {
      while (open) {
        const int g = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)open) - 1), b = first + g * step;
        open &= open - 1;
        const int so_far = __builtin_amdgcn_readlane(n, g);
        const int c = few ? count_rows<4>(a, b, 64, lane, so_far) : count_rows<16>(a, b, 64, lane, so_far);
        n = lane == g ? c : n;
      }
    }
  }
  return there ? n : 0;
}

// the offsets of a large batch: one workgroup, sequences dealt to wavefronts
__global__ void __launch_bounds__(1024) propose_count_kernel(ProposeArgs a) {
  __shared__ int n[1024];
  __shared__ int base;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (tid == 0) base = a.offsets[0] = 0;
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
#pragma unroll 1
    for (int k = wave * kCounts; k < 1024; k += 16 * kCounts) {
      const int c = count_eight(a, b0 + k, 1, lane);
      if (lane < kCounts) n[k + lane] = c;
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
  __shared__ int part[kMaxWaves], parts[kMaxWaves];
  const int b = a.first + (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = (int)blockDim.x >> 6;
  const int32_t* tok = a.tok + (int64_t)b * a.m;
  const float* conf = a.conf + (int64_t)b * a.m;
  uint64_t best = 0;
  for (int at = wave * 64; at < a.m; at += waves * 64) {
    const int i = at + lane;
    const uint64_t k = sort64(i < a.m ? propose_key(tok[i], conf[i], i) : 0);
    best = at == wave * 64 ? k : merge64(best, reversed(k, lane));
  }
  int off = 0, total = 0;
  if constexpr (!COUNTED) {
    int before = 0, all = 0;
#pragma unroll 1
    for (int o = wave; o < a.B; o += waves * kCounts) {
      const int c = count_eight(a, o, waves, lane);
      before += o + lane * waves < b ? c : 0;
      all += c;
    }
    before = (int)wave_sum64((uint64_t)before);
    all = (int)wave_sum64((uint64_t)all);
    if (lane == 0) {
      part[wave] = before;
      parts[wave] = all;
    }
  } else {
    off = a.offsets[b];
    total = a.offsets[a.B];
  }
  for (int half = 1; half < waves; half <<= 1) {
    list[wave][lane] = best;
    __syncthreads();
    if ((wave & (2 * half - 1)) == 0 && wave + half < waves) best = merge64(best, list[wave + half][63 - lane]);
    __syncthreads();
  }
  if constexpr (!COUNTED) {
    if (waves == 1) __syncthreads();
    off = (int)wave_sum64(lane < waves ? (uint64_t)part[lane] : 0);
    total = (int)wave_sum64(lane < waves ? (uint64_t)parts[lane] : 0);
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
epic_status launch_sample(SampleArgs a, int blocks, hipStream_t stream) {
  const int nvec = (a.V + kPer<DT> - 1) / kPer<DT>;
  auto threads = [&](int J) { return std::max(64, ((nvec + J - 1) / J + 63) / 64 * 64); };
#define EPIC_SAMPLE(J, NT)                                                                     \
  launches(blocks, NT, [&](int first, int count) {                                             \
    a.first = first;                                                                           \
    hipLaunchKernelGGL((sample_kernel<DT, J>), dim3(count), dim3(NT), 0, stream, a);           \
  })
  // Eight vectors a lane up to 768 lanes, which two workgroups of a CU can have:
  // 2048 rows of 49152 bfloat16 logits with top-p 0.9 154 us against 204 with
  // sixteen, 2867 of 32768 134 against 171 (46 without filters on either side).
  // Sixteen from there on: 2048 rows of 50304 with top-k 50 81 us against 103, of
  // 65536 76 against 106, as one workgroup of eight would take a CU.  Four and two
  // for short rows: 512 rows of 4096 float16 logits with top-p 0.9 16 us against
  // 23, with settings of all kinds 28 against 47.
  if (nvec <= 2 * 64)
    EPIC_SAMPLE(2, threads(2));
  else if (nvec <= 4 * 256)
    EPIC_SAMPLE(4, threads(4));
  else if (nvec <= 8 * 768)
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
               {d_seqs, d_start, n}, d_uniform, d_temperature, d_top_p, d_min_p, d_top_k, d_tok, d_conf, 0, 0};
  const int blocks = logits->batch * logits->rows;
  if (d_seqs && !d_start && blocks > 256 && blocks <= kSpread) a.spread = blocks;
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
  ProposeArgs a{d_tok, d_conf, d_start, d_cand_seq, d_cand_pos, d_cand_tok, d_cand_conf, d_offsets, batch, rows, per_seq, 0};
  const int threads = std::min(1024, std::max(64, (rows + 63) / 64 * 64));
  // in one launch while no wavefront has more than 16 sequences to count
  if (batch > 0 && batch <= 16 * (threads / 64)) {
    hipLaunchKernelGGL(propose_kernel<false>, dim3(batch), dim3(threads), 0, stream, a);
  } else {
    hipLaunchKernelGGL(propose_count_kernel, dim3(1), dim3(1024), 0, stream, a);
    launches(batch, threads, [&](int first, int count) {
      a.first = first;
      hipLaunchKernelGGL(propose_kernel<true>, dim3(count), dim3(threads), 0, stream, a);
    });
  }
  return hipGetLastError() == hipSuccess ? EPIC_OK : EPIC_ERR_HIP;
}

}  // extern "C"
