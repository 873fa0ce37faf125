// Distillation from a teacher's top logits: epic_distill_forward and
// epic_distill_backward.
#include "rows.inc"

namespace epic_rows {

struct DistillArgs {
  const char* data;
  int64_t seq_stride, row_stride;  // bytes
  int rows, V;
  Window win;
  const int32_t* idx;
  const float* logit;
  int K;
  int steps;  // vectors a lane
  const float* teacher_lse;
  float tau;
  float* loss;          // forward
  float* stats;         // written by forward, read by backward
  const float* weight;
  char* grad;
  int64_t grad_seq, grad_row;  // bytes
  int first;            // row of the launch
};

// Vector v of a gradient row, rounded to nearest even; nothing past its end.
template <int DT>
EPIC_DEV void store_vec(char* row, int v, int V, const float (&g)[kPer<DT>]) {
  constexpr int E = kPer<DT>;
  Loose16 x;
  if constexpr (DT == EPIC_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x.d[e] = __float_as_uint(g[e]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      typedef float f2 __attribute__((ext_vector_type(2)));
      typedef __bf16 b2 __attribute__((ext_vector_type(2)));
      typedef _Float16 h2 __attribute__((ext_vector_type(2)));
      const f2 p = {g[2 * k], g[2 * k + 1]};
      if constexpr (DT == EPIC_BF16)
        x.d[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, b2));
      else
        x.d[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, h2));
    }
  }
  const int t = v * E;
  if (t + E <= V) {
    *(Loose16*)(row + (int64_t)t * kSize<DT>) = x;
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (t + e >= V) continue;
      if constexpr (DT == EPIC_F32)
        *(uint32_t*)(row + 4 * (int64_t)(t + e)) = x.d[e];
      else
        *(uint16_t*)(row + 2 * (int64_t)(t + e)) = (uint16_t)((e & 1) ? x.d[e >> 1] >> 16 : x.d[e >> 1] & 0xFFFFu);
    }
  }
}
template <int DT>
EPIC_DEV void store_elem(char* row, int t, float g) {
  if constexpr (DT == EPIC_F32)
    *(float*)(row + 4 * (int64_t)t) = g;
  else if constexpr (DT == EPIC_BF16)
    *(uint16_t*)(row + 2 * (int64_t)t) = __builtin_bit_cast(uint16_t, (__bf16)g);
  else
    *(uint16_t*)(row + 2 * (int64_t)t) = __builtin_bit_cast(uint16_t, (_Float16)g);
}

template <int DT>
EPIC_DEV void zero_row(char* row, int V, int threads) {
  float g[kPer<DT>] = {};
  for (int v = (int)threadIdx.x; v * kPer<DT> < V; v += threads) store_vec<DT>(row, v, V, g);
}

// What a row's entries say, in LDS: ids, the teacher's shares, the student's
// scaled logits.
struct Entries {
  int32_t* id;
  float* q;
  float* z;
};

// The teacher's shares of the K entries into e.q and what it leaves to the
// rest, by one wavefront; e.q holds the scaled logits before.  `any`: whether
// there is an entry to go by.  Of +inf there is no share but NaN, of -inf always
// none, beside a logsumexp of -inf too.
EPIC_DEV float teacher_shares(const Entries& e, int K, bool has_lse, float lse, int lane, bool& any) {
  float top = -kInf;
  bool there = false;
  for (int k = lane; k < K; k += 64) {
    if (e.id[k] < 0) continue;
    there = there || has_lse || e.q[k] != -kInf;  // NaN is no absence
    top = fmaxf(top, e.q[k]);
  }
  any = __ballot(there) != 0;
  float base = lse < kInf ? lse : __builtin_nanf("");
  if (!has_lse) {
    top = wave_max(top);
    float s = 0.f;
    for (int k = lane; k < K; k += 64)
      if (e.id[k] >= 0) s += expf(e.q[k] - top);
    base = top + logf(wave_sum(s));
  }
  float s = 0.f;
  for (int k = lane; k < K; k += 64) {
    if (e.id[k] < 0) continue;
    const float t = e.q[k], q = !(t < kInf) ? __builtin_nanf("") : t == -kInf && base == -kInf ? 0.f : expf(t - base);
    e.q[k] = q;
    s += q;
  }
  s = wave_sum(s);
  const float left = 1.f - s;
  return !has_lse || left < 0.f ? 0.f : left;  // NaN stays
}

// Whether entry k is the first of its id; `twice`: some id is listed twice.
EPIC_DEV bool leads(const Entries& e, int k, bool twice) {
  if (!twice) return true;
  for (int j = 0; j < k; ++j)
    if (e.id[j] == e.id[k]) return false;
  return true;
}
EPIC_DEV float share_of(const Entries& e, int k, int K, bool twice) {
  if (!twice) return e.q[k];
  float s = 0.f;
  for (int j = 0; j < K; ++j) s += e.id[j] == e.id[k] ? e.q[j] : 0.f;
  return s;
}

struct DistillLds {
  float top[kMaxWaves], sum[kMaxWaves];
  int bad, twice;
  float scale;  // of the gradient outside the list: weight tau (p_rest - q_rest) / (sum of 2^((l - top) c))
  float base;   // the top it goes by
  float lse, pull;  // of listed tokens: pull (p - q)
  int dead;
};

// Forward: one workgroup per row, one reading of it.  Listed tokens are marked
// in a bitmap in LDS and made -inf as the vectors arrive, so that what is left
// is the rest, of which every lane keeps a running maximum and sum; the listed
// ones are summed by a wavefront.  With the gradient the row stays in registers
// (J vectors a lane; J = 0, rows too long for that: read again) and is written
// as the rest's derivative (0 where it was listed), then the listed ones over
// it.  The sums and shares are float32 relative to their largest; gradients are
// rounded once, to the logits' type.
//
// Bound by memory: losses and gradient of 2867 of 4096 rows of 32768 bfloat16
// logits take 103 us, 4.4 TB/s of what has to be read and written (a copy: 5.0);
// the vector units are busy half of the time.  Losses alone of 936 rows of 50021
// float16 logits take 33 us, 2.9 TB/s: less than four workgroups a CU in all.
template <int DT, int J, bool GRAD>
__global__ void __launch_bounds__(1024) distill_forward_kernel(DistillArgs a) {
  extern __shared__ uint32_t dyn[];
  __shared__ DistillLds s;
  constexpr int E = kPer<DT>;
  const int r = a.first + (int)blockIdx.x, b = r / a.rows, i = r - b * a.rows;
  const int tid = (int)threadIdx.x, threads = (int)blockDim.x, waves = threads >> 6, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* grow = GRAD ? a.grad + b * a.grad_seq + i * a.grad_row : nullptr;
  if (!row_counts(a.win, b, i)) {
    if (tid == 0) {
      a.loss[r] = 0.f;
      a.stats[2 * (int64_t)r] = a.stats[2 * (int64_t)r + 1] = 0.f;
    }
    if constexpr (GRAD) zero_row<DT>(grow, a.V, threads);
    return;
  }
  const char* row = a.data + b * a.seq_stride + i * a.row_stride;
  const int words = (a.V + 31) / 32, K = a.K;
  Entries ent{(int32_t*)dyn + words, (float*)dyn + words + K, (float*)dyn + words + 2 * K};
  const int steps = J ? J : a.steps;
  const int first = wave * steps * 64 + lane;
  Vec v[J ? J : 1];
  auto load = [&](int j) {
    const int at = first - lane + j * 64;  // of the wavefront
    return (at + 64) * E <= a.V ? load_whole<DT>(row, at + lane) : load_vec<DT>(row, at + lane, a.V);
  };
  if constexpr (J > 0) {
    if ((first - lane + J * 64) * E <= a.V) {
#pragma unroll
      for (int j = 0; j < J; ++j) v[j] = load_whole<DT>(row, first + j * 64);
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) v[j] = load(j);
    }
  }
  for (int w = tid; w < words; w += threads) dyn[w] = 0;
  if (tid == 0) s.bad = s.twice = 0;
  __syncthreads();
  const float inv_tau = 1.f / a.tau;
  for (int k = tid; k < K; k += threads) {
    const int id = a.idx[(int64_t)r * K + k];
    ent.id[k] = id;
    if (id >= a.V) {
      s.bad = 1;
    } else if (id >= 0) {
      if (atomicOr(&dyn[id >> 5], 1u << (id & 31)) & (1u << (id & 31))) s.twice = 1;
      ent.q[k] = a.logit[(int64_t)r * K + k] * inv_tau;
      ent.z[k] = load_elem<DT>(row, id) * inv_tau;
    }
  }
  __syncthreads();
  if (s.bad) {
    if (tid == 0) {
      a.loss[r] = __builtin_nanf("");
      a.stats[2 * (int64_t)r] = a.stats[2 * (int64_t)r + 1] = 0.f;
    }
    if constexpr (GRAD) zero_row<DT>(grow, a.V, threads);
    return;
  }
  const float c = kLog2e / a.tau;
  auto rest = [&](Vec x, int at) {
    const uint32_t t = (uint32_t)at * E;
    if (t >= (uint32_t)a.V) return x;
    const uint32_t bits = (dyn[t >> 5] >> (t & 31)) & ((1u << E) - 1u);
    if (bits) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (DT == EPIC_F32) {
          if (bits & (1u << k)) x.d[k] = kNegInf<DT>;
        } else {
          if (bits & (1u << (2 * k))) x.d[k] = (x.d[k] & 0xFFFF0000u) | (kNegInf<DT> & 0xFFFFu);
          if (bits & (2u << (2 * k))) x.d[k] = (x.d[k] & 0xFFFFu) | (kNegInf<DT> & 0xFFFF0000u);
        }
      }
    }
    return x;
  };
  // A running maximum and sum of the lane, one vector after another as they
  // arrive.
  float top = -kInf, sum = 0.f;
  auto add = [&](const Vec& x) {
    float m = top;
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, elem<DT>(x, e));
    const float by = m > -kInf ? m : 0.f;
    float some = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) some += __builtin_amdgcn_exp2f((elem<DT>(x, e) - by) * c);
    sum = sum * __builtin_amdgcn_exp2f((top - by) * c) + some;
    top = m;
  };
  if constexpr (J > 0) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      v[j] = rest(v[j], first + j * 64);
      add(v[j]);
      __builtin_amdgcn_sched_barrier(0);  // a vector's temporaries at a time
    }
  } else {
    constexpr int G = 4;  // loads ahead
    Vec x[G], y[G];
#pragma unroll
    for (int g = 0; g < G; ++g) x[g] = load(g < steps ? g : steps - 1);
#pragma unroll 1
    for (int j = 0; j < steps; j += G) {
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (j + G + g < steps) y[g] = load(j + G + g);
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (j + g < steps) add(rest(x[g], first + (j + g) * 64));
#pragma unroll
      for (int g = 0; g < G; ++g) x[g] = y[g];
    }
  }
  {
    const float m = wave_max(top), by = m > -kInf ? m : 0.f;
    sum = wave_sum(sum * __builtin_amdgcn_exp2f((top - by) * c));
    top = m;
  }
  if (lane == 0) {
    s.top[wave] = top;
    s.sum[wave] = sum;
  }
  __syncthreads();
  if (wave == 0) {
    const bool twice = s.twice != 0;
    float m = -kInf;
    for (int w = 0; w < waves; ++w) m = fmaxf(m, s.top[w]);
    const float by = m > -kInf ? m : 0.f;
    float S = 0.f;
    for (int w = 0; w < waves; ++w) S += s.sum[w] * __builtin_amdgcn_exp2f((s.top[w] - by) * c);
    const float lse_rest = m > -kInf || S != S ? by * inv_tau + logf(S) : -kInf;
    float zt = -kInf, zs = 0.f;
    for (int k = lane; k < K; k += 64)
      if (ent.id[k] >= 0) zt = fmaxf(zt, ent.z[k]);
    zt = wave_max(zt);
    const float zb = zt > -kInf ? zt : 0.f;
    for (int k = lane; k < K; k += 64)
      if (ent.id[k] >= 0 && leads(ent, k, twice)) zs += expf(ent.z[k] - zb);
    zs = wave_sum(zs);
    const float lse_top = zt > -kInf || zs != zs ? zb + logf(zs) : -kInf;
    const float both = fmaxf(lse_rest, lse_top);
    const bool empty = lse_rest == -kInf && lse_top == -kInf;
    const float lse = empty ? -kInf : both + logf(expf(lse_rest - both) + expf(lse_top - both));
    const bool has = a.teacher_lse != nullptr;
    bool any = false;
    float q_rest = teacher_shares(ent, K, has, has ? a.teacher_lse[r] : 0.f, lane, any);
    if (lse_rest == -kInf) q_rest = 0.f;
    float kl = 0.f;
    for (int k = lane; k < K; k += 64) {
      const float q = ent.id[k] >= 0 ? ent.q[k] : 0.f;
      if (q > 0.f || q != q) kl += q * (logf(q) - ent.z[k] + lse);
    }
    kl = wave_sum(kl);
    if (q_rest > 0.f || q_rest != q_rest) kl += q_rest * (logf(q_rest) - lse_rest + lse);
    if (lse != lse) kl = lse;  // also where the teacher has no share to multiply it with
    if (lane == 0) {
      const bool dead = !any || empty;
      a.loss[r] = dead ? 0.f : kl * a.tau * a.tau;
      a.stats[2 * (int64_t)r] = lse;
      a.stats[2 * (int64_t)r + 1] = lse_rest;
      if constexpr (GRAD) {
        const float pull = a.tau * (a.weight ? a.weight[r] : 1.f);
        s.dead = dead;
        s.pull = pull;
        s.lse = lse;
        s.base = by;
        s.scale = lse_rest == -kInf ? 0.f : pull * (expf(lse_rest - lse) - q_rest) / S;
      }
    }
  }
  if constexpr (GRAD) {
    __syncthreads();
    if (s.dead) {
      zero_row<DT>(grow, a.V, threads);
      return;
    }
    const float scale = s.scale, base = s.base;
    auto write = [&](const Vec& x, int at) {
      float g[E];
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = scale * __builtin_amdgcn_exp2f((elem<DT>(x, e) - base) * c);
      if (at * E < a.V) store_vec<DT>(grow, at, a.V, g);
    };
    if constexpr (J > 0) {
      // Without this the compiler keeps what the pass before computed of every
      // element, which takes more registers than there are.
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(v[j].d[k]));
#pragma unroll
      for (int j = 0; j < J; ++j) {
        write(v[j], first + j * 64);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      for (int j = 0; j < steps; ++j) write(rest(load(j), first + j * 64), first + j * 64);
    }
    __syncthreads();
    const bool twice = s.twice != 0;
    for (int k = tid; k < K; k += threads)
      if (ent.id[k] >= 0) store_elem<DT>(grow, ent.id[k], s.pull * (expf(ent.z[k] - s.lse) - share_of(ent, k, K, twice)));
  }
}

// Backward from a forward pass's stats: one workgroup per row, one reading and
// one writing of it.  Every element goes as one of the rest; then the listed
// ones are written over.  Bound by memory: 8192 rows of 32768 bfloat16 logits take
// 222 us, 4.85 TB/s (a copy: 5.0).
template <int DT>
__global__ void __launch_bounds__(1024) distill_backward_kernel(DistillArgs a) {
  extern __shared__ uint32_t dyn[];
  __shared__ DistillLds s;
  constexpr int E = kPer<DT>;
  const int r = a.first + (int)blockIdx.x, b = r / a.rows, i = r - b * a.rows;
  const int tid = (int)threadIdx.x, threads = (int)blockDim.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* grow = a.grad + b * a.grad_seq + i * a.grad_row;
  if (!row_counts(a.win, b, i)) {
    zero_row<DT>(grow, a.V, threads);
    return;
  }
  const char* row = a.data + b * a.seq_stride + i * a.row_stride;
  const int words = (a.V + 31) / 32, K = a.K;
  Entries ent{(int32_t*)dyn + words, (float*)dyn + words + K, (float*)dyn + words + 2 * K};
  for (int w = tid; w < words; w += threads) dyn[w] = 0;
  if (tid == 0) s.bad = s.twice = 0;
  __syncthreads();
  const float inv_tau = 1.f / a.tau;
  for (int k = tid; k < K; k += threads) {
    const int id = a.idx[(int64_t)r * K + k];
    ent.id[k] = id;
    if (id >= a.V) {
      s.bad = 1;
    } else if (id >= 0) {
      if (atomicOr(&dyn[id >> 5], 1u << (id & 31)) & (1u << (id & 31))) s.twice = 1;
      ent.q[k] = a.logit[(int64_t)r * K + k] * inv_tau;
      ent.z[k] = load_elem<DT>(row, id) * inv_tau;
    }
  }
  __syncthreads();
  const float lse = a.stats[2 * (int64_t)r], lse_rest = a.stats[2 * (int64_t)r + 1];
  if (wave == 0) {
    const bool has = a.teacher_lse != nullptr;
    bool any = false;
    float q_rest = teacher_shares(ent, K, has, has ? a.teacher_lse[r] : 0.f, lane, any);
    if (lse_rest == -kInf) q_rest = 0.f;
    if (lane == 0) {
      const float pull = a.tau * (a.weight ? a.weight[r] : 1.f);
      s.dead = s.bad || !any || lse == -kInf;
      s.pull = pull;
      s.scale = lse_rest == -kInf ? 0.f : pull * (expf(lse_rest - lse) - q_rest);
    }
  }
  __syncthreads();
  if (s.dead) {
    zero_row<DT>(grow, a.V, threads);
    return;
  }
  const float scale = s.scale, base = lse_rest == -kInf ? 0.f : lse_rest;
  for (int v = tid; v * E < a.V; v += threads) {
    const Vec x = load_vec<DT>(row, v, a.V);
    float g[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
      // the difference first: products of a mask's lowest values with log2(e) are no numbers
      g[e] = scale * __builtin_amdgcn_exp2f(__builtin_fmaf(elem<DT>(x, e), inv_tau, -base) * kLog2e);
    store_vec<DT>(grow, v, a.V, g);
  }
  __syncthreads();
  for (int k = tid; k < K; k += threads)
    if (ent.id[k] >= 0) store_elem<DT>(grow, ent.id[k], s.pull * (expf(ent.z[k] - lse) - share_of(ent, k, K, s.twice != 0)));
}

template <int DT, bool GRAD>
void launch_forward(DistillArgs a, int blocks, hipStream_t stream) {
  const int nvec = (a.V + kPer<DT> - 1) / kPer<DT>;
  const size_t lds = ((size_t)(a.V + 31) / 32 + 3 * (size_t)a.K) * 4;
  auto threads = [&](int J) { return std::max(64, ((nvec + J - 1) / J + 63) / 64 * 64); };
  // As many vectors a lane as keep two workgroups or more on a CU.  2048 rows of
  // 32768 bfloat16 logits, losses and gradient: eight 68 us, sixteen 71, none in
  // registers 91; of 65536: sixteen 123 us, eight 126 and none 157.
  const int J = nvec <= 2 * 64 ? 2 : nvec <= 4 * 256 ? 4 : nvec <= 8 * 512 ? 8 : nvec <= 16 * 1024 ? 16 : 0;
  const int NT = J ? threads(J) : 1024;
  // Losses alone keep nothing in registers, but deal the row to the lanes alike,
  // so that their bits are those of a call with the gradient.
  a.steps = J ? J : (nvec + NT - 1) / NT;
#define EPIC_DISTILL(J)                                                                                \
  launches(blocks, NT, [&](int first, int count) {                                                     \
    a.first = first;                                                                                   \
    hipLaunchKernelGGL((distill_forward_kernel<DT, J, GRAD>), dim3(count), dim3(NT), lds, stream, a);  \
  })
  if constexpr (!GRAD) {
    EPIC_DISTILL(0);
  } else {
    switch (J) {
      case 2: EPIC_DISTILL(2); break;
      case 4: EPIC_DISTILL(4); break;
      case 8: EPIC_DISTILL(8); break;
      case 16: EPIC_DISTILL(16); break;
      default: EPIC_DISTILL(0);
    }
  }
#undef EPIC_DISTILL
}

template <int DT>
void launch_distill(DistillArgs a, bool forward, int blocks, hipStream_t stream) {
  if (!forward) {
    const int nvec = (a.V + kPer<DT> - 1) / kPer<DT>;
    const int threads = std::min(512, std::max(64, (nvec + 255) / 256 * 64));
    const size_t lds = ((size_t)(a.V + 31) / 32 + 3 * (size_t)a.K) * 4;
    launches(blocks, threads, [&](int first, int count) {
      a.first = first;
      hipLaunchKernelGGL(distill_backward_kernel<DT>, dim3(count), dim3(threads), lds, stream, a);
    });
  } else if (a.grad) {
    launch_forward<DT, true>(a, blocks, stream);
  } else {
    launch_forward<DT, false>(a, blocks, stream);
  }
}

epic_status distill(const epic_rows_desc* logits, const int32_t* d_seqs, int32_t n, const int32_t* d_start,
                    const int32_t* d_top_idx, const float* d_top_logit, int32_t K, const float* d_teacher_lse, float tau,
                    float* d_loss, float* d_stats, const float* d_weight, const epic_rows_desc* grad, bool forward,
                    hipStream_t stream) {
  epic_status st = check_rows(logits, d_seqs, n);
  if (st != EPIC_OK) return st;
  if (K < 1 || K > 1024 || !(tau > 0.f) || !(tau < kInf) || !(kLog2e / tau < kInf)) return EPIC_ERR_ARG;
  if (!forward && !grad) return EPIC_ERR_NULL;
  if (grad) {
    if ((st = check_rows(grad, nullptr, 0)) != EPIC_OK) return st;
    if (grad->dtype != logits->dtype || grad->batch != logits->batch || grad->rows != logits->rows ||
        grad->vocab != logits->vocab)
      return EPIC_ERR_ARG;
  }
  if (logits->batch == 0 || logits->rows == 0) return EPIC_OK;
  if (grad && !rows_apart(grad)) return EPIC_ERR_ARG;
  if (!d_top_idx || !d_top_logit || !d_stats || (forward && !d_loss)) return EPIC_ERR_NULL;
  const int es = elem_size(logits->dtype);
  DistillArgs a{(const char*)logits->data, logits->seq_stride * es, logits->row_stride * es, logits->rows, logits->vocab,
                {d_seqs, d_start, n}, d_top_idx, d_top_logit, K, 0, d_teacher_lse, tau, d_loss, d_stats, d_weight,
                grad ? (char*)grad->data : nullptr, grad ? grad->seq_stride * es : 0, grad ? grad->row_stride * es : 0, 0};
  const int blocks = logits->batch * logits->rows;
  switch (logits->dtype) {
    case EPIC_F32: launch_distill<EPIC_F32>(a, forward, blocks, stream); break;
    case EPIC_F16: launch_distill<EPIC_F16>(a, forward, blocks, stream); break;
    default: launch_distill<EPIC_BF16>(a, forward, blocks, stream); break;
  }
  return hipGetLastError() == hipSuccess ? EPIC_OK : EPIC_ERR_HIP;
}

}  // namespace epic_rows

extern "C" {

epic_status epic_distill_forward(const epic_rows_desc* logits, const int32_t* d_seqs, int32_t n,
                                 const int32_t* d_start, const int32_t* d_top_idx, const float* d_top_logit, int32_t K,
                                 const float* d_teacher_lse, float tau, float* d_loss, float* d_stats,
                                 const float* d_weight, const epic_rows_desc* grad, hipStream_t stream) {
  return epic_rows::distill(logits, d_seqs, n, d_start, d_top_idx, d_top_logit, K, d_teacher_lse, tau, d_loss, d_stats,
                            d_weight, grad, true, stream);
}

epic_status epic_distill_backward(const epic_rows_desc* logits, const int32_t* d_seqs, int32_t n,
                                  const int32_t* d_start, const int32_t* d_top_idx, const float* d_top_logit,
                                  int32_t K, const float* d_teacher_lse, float tau, const float* d_stats,
                                  const float* d_weight, const epic_rows_desc* grad, hipStream_t stream) {
  return epic_rows::distill(logits, d_seqs, n, d_start, d_top_idx, d_top_logit, K, d_teacher_lse, tau, nullptr,
                            const_cast<float*>(d_stats), d_weight, grad, false, stream);
}

}  // extern "C"
