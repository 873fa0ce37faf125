// Between hidden states and logits: epic_quantize_rows, epic_logits_q8,
// epic_head_loss_forward and epic_head_loss_backward.
#include "product.inc"

namespace epic_rows {

// ------------------------------------------------------- rows that count
// Which rows of the window count, and what is kept of each, one after another
// (the count-th and later entries are not written): `src` the row's number.
struct Kept {
  int32_t* count;
  int32_t* src;
  int32_t* target;  // loss: the token, or -2 where it is no token
  float* lse;       // backward
  float* mul;       // backward: what the row's part of the gradient is multiplied with before it is rounded
  int32_t* exp;     // backward: and the power of two after the products
};

struct GatherArgs {
  const char* data;
  int64_t seq_stride, row_stride;  // bytes
  int batch, rows, d;
  Window win;
  const int32_t* target;
  const float* lse;
  const float* weight;
  float* loss;       // forward: 0 in rows that do not count
  float* lse_out;
  char* grad;        // backward: 0 in rows that do not count
  int64_t grad_seq, grad_row;
  Kept kept;
  char* out;         // packed rows
  char* out2;        // 16-bit numbers with the rows' powers of two, for the product over rows
  int64_t stride, plane;  // bytes
  float* scale;      // 8 bits: the rows' scales
  const float* tops; // 32 bits: largest magnitudes of hidden states and head, in parts
  int top_parts[2];
  int per;           // rows of a workgroup
  int V;
};

constexpr int kGather = 256;  // threads

template <int DT>
EPIC_DEV void load8(const char* row, int t, int d, float (&x)[8]) {
  if constexpr (DT == EPIC_F32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (t + 4 * h + 4 <= d) {
        const Vec v = load_whole<DT>(row, t / 4 + h);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * h + e] = elem<DT>(v, e);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * h + e] = t + 4 * h + e < d ? load_elem<DT>(row, t + 4 * h + e) : 0.f;
      }
    }
  } else if (t + 8 <= d) {
    const Vec v = load_whole<DT>(row, t / 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = elem<DT>(v, e);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = t + e < d ? load_elem<DT>(row, t + e) : 0.f;
  }
}

EPIC_DEV uint32_t pack_f16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16;
}
EPIC_DEV uint32_t pack_bf16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}
// A 32-bit number as the sum of two 16-bit ones.  With the tensor's largest
// magnitude scaled to [2^14, 2^15), numbers down to 2^-17 of it keep 22 bits and
// a sign (the second one's half step: 2^-24 of the number), smaller ones an
// error of 2^-40 of the largest.
EPIC_DEV void split_f16(float x, _Float16& a, _Float16& b) {
  a = (_Float16)x;
  const float r = x - (float)a;
  b = (_Float16)(r - r == 0.f ? r : 0.f);  // of an infinity there is no rest
}

// Eight numbers of packed row `row` at t.
template <int DT>
EPIC_DEV void store8(char* row, int64_t plane, int t, const float (&x)[8]) {
  uint4 a;
  if constexpr (DT == EPIC_F32) {
    uint4 b;
    _Float16 p[8], q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) split_f16(x[e], p[e], q[e]);
    a = __builtin_bit_cast(uint4, p);
    b = __builtin_bit_cast(uint4, q);
    *(uint4*)(row + plane + 2 * (int64_t)t) = b;
  } else if constexpr (DT == EPIC_F16) {
    a = make_uint4(pack_f16(x[0], x[1]), pack_f16(x[2], x[3]), pack_f16(x[4], x[5]), pack_f16(x[6], x[7]));
  } else {
    a = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
  *(uint4*)(row + 2 * (int64_t)t) = a;
}

// The power of two that scales a largest magnitude to [2^14, 2^15).
EPIC_DEV int scale_exp(float top) { return top > 0.f ? 15 - (__builtin_amdgcn_frexp_expf(top)) : 0; }

EPIC_DEV float block_max(float v, float* lds) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = lds[0];
  for (int w = 1; w < (int)blockDim.x >> 6; ++w) m = fmaxf(m, lds[w]);
  return m;
}

// The largest of a tensor's partial maxima, for all threads.
EPIC_DEV float top_of(const float* parts, int n, float* lds) {
  float m = 0.f;
  for (int i = (int)threadIdx.x; i < n; i += (int)blockDim.x) m = fmaxf(m, parts[i]);
  return block_max(m, lds);
}

EPIC_DEV bool kept_row(const GatherArgs& a, int r) {
  const int b = r / a.rows;
  return row_counts(a.win, b, r - b * a.rows) && (!a.target || a.target[r] >= 0);
}

// One row to 8 bits, by a wavefront: the scale is a 127th of the largest
// magnitude, ties go to the even number.  A row without a magnitude of 1e-30 has
// scale 0 and no number but 0, one with a NaN or an infinity scale NaN and 0.
template <int DT>
EPIC_DEV void quantize_row(const char* row, int d, int8_t* out, int stride, float* scale, int lane) {
  float top = 0.f;
  bool odd = false;
  for (int t = lane * 8; t < d; t += 512) {
    float x[8];
    load8<DT>(row, t, d, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      top = fmaxf(top, fabsf(x[e]));
      odd = odd || !(fabsf(x[e]) < kInf);
    }
  }
  top = wave_max(top);
  odd = __ballot(odd) != 0;
  const float inv = odd || top < 1e-30f ? 0.f : 127.f / top;
  if (lane == 0) *scale = odd ? __builtin_nanf("") : inv == 0.f ? 0.f : top / 127.f;
  for (int t = lane * 8; t < stride; t += 512) {
    float x[8];
    load8<DT>(row, t, d, x);
    uint32_t q[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int v = inv == 0.f ? 0 : (int)rintf(x[e] * inv);
      q[e >> 2] |= (uint32_t)(v & 255) << (8 * (e & 3));
    }
    *(uint2*)(out + t) = make_uint2(q[0], q[1]);
  }
}

enum GatherMode { kForward, kBackward, kQuantize };

// The rows that count, one after another, zeros behind them up to a multiple of
// 64.  Every workgroup counts the rows before its own itself (4 bytes a row from
// the L2), so that one launch does it.
template <int DT, int MODE>
__global__ void __launch_bounds__(kGather) gather_kernel(GatherArgs a) {
  __shared__ int lds_n[kGather / 64];
  __shared__ int lds_own[64];
  __shared__ float lds_f[kGather / 64];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int total = a.batch * a.rows, first = (int)blockIdx.x * a.per, last = min(total, first + a.per);
  constexpr bool kScaled = MODE == kBackward && DT != EPIC_BF16;
  int before = 0, top_exp = INT32_MIN;
  // (the powers of two of the rows' weights go by the largest one)
  for (int r = tid; r < (kScaled ? total : first); r += kGather)
    if (kept_row(a, r)) {
      before += r < first;
      if constexpr (kScaled) {
        const float w = a.weight ? a.weight[r] : 1.f;
        if (w != 0.f && fabsf(w) < kInf) top_exp = max(top_exp, __builtin_amdgcn_frexp_expf(w));
      }
    }
  before = (int)wave_sum((float)(before & 0xFFF)) + ((int)wave_sum((float)(before >> 12)) << 12);
  if constexpr (kScaled) top_exp = (int)wave_max((float)max(top_exp, -1000));
  if (lane == 0) {
    lds_n[wave] = before;
    lds_f[wave] = (float)top_exp;
  }
  __syncthreads();
  before = 0;
  for (int w = 0; w < kGather / 64; ++w) before += lds_n[w];
  if constexpr (kScaled)
    for (int w = 0; w < kGather / 64; ++w) top_exp = max(top_exp, (int)lds_f[w]);
  float mine = 1.f;
  int h_exp = 0;
  if constexpr (DT == EPIC_F32 && MODE != kQuantize) h_exp = scale_exp(top_of(a.tops, a.top_parts[0], lds_f));
  for (int base = first; base < last; base += 64) {
    const int n = min(64, last - base);
    __syncthreads();
    if (wave == 0) {
      const bool on = lane < n && kept_row(a, base + lane);
      const uint64_t all = __ballot(on);
      lds_own[lane] = on ? before + (int)__popcll(all & ((1ull << lane) - 1)) : -1;
      if (lane == 0) lds_n[0] = (int)__popcll(all);
    }
    __syncthreads();
    before += lds_n[0];
    for (int i = wave; i < n; i += kGather / 64) {
      const int r = base + i, at = __builtin_amdgcn_readfirstlane(lds_own[i]);
      const int b = r / a.rows, in = r - b * a.rows;
      if (at < 0) {
        if constexpr (MODE == kForward) {
          if (lane == 0) a.loss[r] = a.lse_out[r] = 0.f;
        } else if constexpr (MODE == kBackward) {
          if (a.grad) {
            char* g = a.grad + b * a.grad_seq + in * a.grad_row;
            constexpr int S = kSize<DT>;
            const float zero[kPer<DT>] = {};
            (void)zero;
            for (int t = lane * kPer<DT>; t < a.d; t += 64 * kPer<DT>) {
              if (t + kPer<DT> <= a.d) {
                *(Loose16*)(g + (int64_t)t * S) = Loose16{{0u, 0u, 0u, 0u}};
              } else {
                for (int e = t; e < a.d; ++e) {
                  if constexpr (S == 4)
                    *(uint32_t*)(g + 4 * (int64_t)e) = 0u;
                  else
                    *(uint16_t*)(g + 2 * (int64_t)e) = 0;
                }
              }
            }
          }
        }
        continue;
      }
      const char* row = a.data + b * a.seq_stride + in * a.row_stride;
      if (lane == 0) a.kept.src[at] = r;
      if constexpr (MODE == kQuantize) {
        quantize_row<DT>(row, a.d, (int8_t*)a.out + at * a.stride, (int)a.stride, a.scale + at, lane);
      } else {
        int y = a.target[r];
        if (y >= a.V) y = -2;
        if (lane == 0) a.kept.target[at] = y;
        int shift = 0;
        if constexpr (MODE == kBackward) {
          float w = a.weight ? a.weight[r] : 1.f;
          if (kScaled && w != 0.f && fabsf(w) < kInf) {
            const int e = __builtin_amdgcn_frexp_expf(w);
            shift = e - top_exp;
            w = __builtin_amdgcn_frexp_mantf(w);
            if (lane == 0) a.kept.exp[at] = e;
          } else if (lane == 0) {
            a.kept.exp[at] = 0;
          }
          if (lane == 0) {
            a.kept.mul[at] = y < 0 ? 0.f : w;
            a.kept.lse[at] = a.lse[r];
          }
        }
        for (int t = lane * 8; t < (int)(a.stride / 2); t += 512) {
          float x[8];
          load8<DT>(row, t, a.d, x);
          if constexpr (DT == EPIC_F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_ldexpf(x[e], h_exp);
          }
          store8<DT>(a.out + at * a.stride, a.plane, t, x);
          if constexpr (kScaled) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_ldexpf(x[e], shift);
            store8<DT>(a.out2 + at * a.stride, a.plane, t, x);
          }
        }
      }
    }
  }
  (void)mine;
  if (last == total) {
    if (tid == 0) *a.kept.count = before;
    if constexpr (kScaled)
      if (tid == 0) a.kept.count[1] = top_exp == -1000 ? 0 : top_exp;
    if constexpr (MODE == kBackward) {
      const int end = (before + 63) / 64 * 64, vecs = (int)(a.stride / 16);
      for (int i = tid; i < (end - before) * vecs; i += kGather) {
        const int64_t at = (int64_t)before * a.stride + (int64_t)i * 16;
        *(uint4*)(a.out + at) = make_uint4(0, 0, 0, 0);
        if constexpr (kScaled) *(uint4*)(a.out2 + at) = make_uint4(0, 0, 0, 0);
        if constexpr (DT == EPIC_F32) {
          *(uint4*)(a.out + a.plane + at) = make_uint4(0, 0, 0, 0);
          *(uint4*)(a.out2 + a.plane + at) = make_uint4(0, 0, 0, 0);
        }
      }
    }
  }
}

// Largest finite magnitudes of the hidden states' rows that count (the first
// workgroups) and of the head, one number a workgroup.
struct TopArgs {
  GatherArgs g;
  const char* head;
  int64_t head_row;
  float* tops;
};
__global__ void __launch_bounds__(256) top_kernel(TopArgs a) {
  __shared__ float lds[4];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  const bool head = (int)blockIdx.x >= a.g.top_parts[0];
  const int part = head ? (int)blockIdx.x - a.g.top_parts[0] : (int)blockIdx.x, parts = a.g.top_parts[head];
  const int total = head ? a.g.V : a.g.batch * a.g.rows;
  float top = 0.f;
  for (int r = part * 4 + wave; r < total; r += parts * 4) {
    const char* row;
    if (head) {
      row = a.head + r * a.head_row;
    } else {
      if (!kept_row(a.g, r)) continue;
      const int b = r / a.g.rows;
      row = a.g.data + b * a.g.seq_stride + (r - b * a.g.rows) * a.g.row_stride;
    }
    for (int t = lane * 8; t < a.g.d; t += 512) {
      float x[8];
      load8<EPIC_F32>(row, t, a.g.d, x);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (fabsf(x[e]) < kInf) top = fmaxf(top, fabsf(x[e]));
    }
  }
  top = block_max(top, lds);
  if (threadIdx.x == 0) a.tops[blockIdx.x] = top;
}

// Rows v0 .. of the head as the products read them, one wavefront a row: widths
// and numbers of rows filled up with zeros.
struct PackArgs {
  const char* head;
  int64_t head_row;  // bytes
  int V, d, v0, count;
  char* out;
  int64_t stride, plane;
  const float* tops;
  int top_parts[2];
};
template <int DT>
__global__ void __launch_bounds__(256) pack_kernel(PackArgs a) {
  __shared__ float lds[4];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  int e_head = 0;
  if constexpr (DT == EPIC_F32) e_head = scale_exp(top_of(a.tops + a.top_parts[0], a.top_parts[1], lds));
  for (int i = (int)blockIdx.x * 4 + wave; i < a.count; i += (int)gridDim.x * 4) {
    const char* row = a.head + (a.v0 + i) * a.head_row;
    const int d = a.v0 + i < a.V ? a.d : 0;
    for (int t = lane * 8; t < (int)(a.stride / 2); t += 512) {
      float x[8];
      load8<DT>(row, t, d, x);
      if constexpr (DT == EPIC_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_ldexpf(x[e], e_head);
      }
      store8<DT>(a.out + i * a.stride, a.plane, t, x);
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(256) quantize_kernel(const char* data, int64_t seq_stride, int64_t row_stride, int rows, int total,
                                                       int d, int8_t* q, int64_t stride, float* scale) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  for (int r = (int)blockIdx.x * 4 + wave; r < total; r += (int)gridDim.x * 4) {
    const int b = r / rows;
    quantize_row<DT>(data + b * seq_stride + (r - b * rows) * row_stride, d, q + r * stride, (int)stride, scale + r, lane);
  }
}

// ------------------------------------------------------------- products
struct HeadArgs {
  Operand H, W;      // rows that count [N, d], (a piece of) the head [v, d]
  Kept kept;
  int steps;         // of d
  uint32_t pairs;
  int planes;
  int v0, v1;        // tokens of the piece
  int V, d;
  int first;         // workgroup of the launch
  // losses
  float2* part;      // [rows][parts] maximum and sum of a tile's columns
  int64_t parts;
  float* at_target;
  const float* tops;
  int top_parts[2];
  // gradients
  Operand G;         // (p - y) of the piece [N, v] in 16 bits
  Operand H2;
  float* dh;         // [slices][rows][d] float32
  int64_t dh_slice;
  int slices, add;
  char* grad_head;
  int64_t grad_row;  // bytes
  // 8 bits
  const float* row_scale;
  const float* col_scale;
  char* logits;
  int64_t seq_stride, row_stride;  // bytes
  int rows;
};

// What sums of products are multiplied with to be logits.
template <bool SPLIT>
EPIC_DEV float unscale(const HeadArgs& a, float* lds) {
  if constexpr (!SPLIT) return 1.f;
  const int e = scale_exp(top_of(a.tops, a.top_parts[0], lds)) + scale_exp(top_of(a.tops + a.top_parts[0], a.top_parts[1], lds));
  return __builtin_amdgcn_ldexpf(1.f, -e);
}

// A tile's columns to a maximum and a sum for every row, over two wavefronts or
// more by LDS, and the logit of the row's token.
template <class T, bool SPLIT>
__global__ void __launch_bounds__(T::kThreads) lse_kernel(HeadArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float lds_top[4];
  const int count = *a.kept.count, m = (count + T::BM - 1) / T::BM, n = (a.v1 - a.v0 + T::BN - 1) / T::BN;
  const int id = a.first + (int)blockIdx.x;
  if (id >= m * n) return;
  int tm, tn;
  tile_of(id, m, n, tm, tn);
  T t;
  t.run(a.H, a.W, tm * T::BM, tn * T::BN, m * T::BM, a.v1 - a.v0, 0, a.steps, SPLIT ? 3 : 1, a.pairs, smem);
  const float by = unscale<SPLIT>(a, lds_top);
  __syncthreads();
  float2* part = (float2*)smem;  // [WN][BM]
  const int wn = T::wave() % T::WN, lane = (int)threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < T::MT; ++i) {
    const int r = T::row(i), at = tm * T::BM + r;
    const int y = at < count ? a.kept.target[at] : -1;
    float top = -kInf;
#pragma unroll
    for (int j = 0; j < T::NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = a.v0 + tn * T::BN + T::col(j) + e;
        float l = t.acc[i][j][e] * by;
        l = v < a.v1 ? l : -kInf;
        t.acc[i][j][e] = l;
        if (v == y) a.at_target[at] = l;
        top = fmaxf(top, l);
      }
    const float base = top > -kInf ? top : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < T::NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((t.acc[i][j][e] - base) * kLog2e);
    // the four lanes of a row
#pragma unroll
    for (int s = 16; s < 64; s *= 2) {
      const float t2 = __shfl_xor(top, s), s2 = __shfl_xor(sum, s);
      const float both = fmaxf(top, t2), b2 = both > -kInf ? both : 0.f;
      sum = sum * __builtin_amdgcn_exp2f((top - b2) * kLog2e) + s2 * __builtin_amdgcn_exp2f((t2 - b2) * kLog2e);
      top = both;
    }
    if (lane < 16) part[wn * T::BM + r] = make_float2(top, sum);
  }
  __syncthreads();
  for (int r = (int)threadIdx.x; r < T::BM; r += T::kThreads) {
    if (tm * T::BM + r >= count) continue;
    float2 p = part[r];
    for (int w = 1; w < T::WN; ++w) {
      const float2 q = part[w * T::BM + r];
      const float both = fmaxf(p.x, q.x), b2 = both > -kInf ? both : 0.f;
      p.y = p.y * __builtin_amdgcn_exp2f((p.x - b2) * kLog2e) + q.y * __builtin_amdgcn_exp2f((q.x - b2) * kLog2e);
      p.x = both;
    }
    a.part[(int64_t)(tm * T::BM + r) * a.parts + a.v0 / T::BN + tn] = p;
  }
}

// Losses from the tiles' maxima and sums, one wavefront a row.
__global__ void __launch_bounds__(256) loss_kernel(HeadArgs a, float* loss, float* lse_out) {
  const int at = a.first + (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  if (at >= *a.kept.count) return;
  const float2* p = a.part + at * a.parts;
  float top = -kInf;
  for (int64_t i = lane; i < a.parts; i += 64) top = fmaxf(top, p[i].x);
  top = wave_max(top);
  const float base = top > -kInf ? top : 0.f;
  float sum = 0.f;
  for (int64_t i = lane; i < a.parts; i += 64) sum += p[i].y * __builtin_amdgcn_exp2f((p[i].x - base) * kLog2e);
  sum = wave_sum(sum);
  if (lane == 0) {
    const int y = a.kept.target[at], r = a.kept.src[at];
    const float lse = base + logf(sum);
    lse_out[r] = lse;
    loss[r] = y < 0 ? __builtin_nanf("") : lse - a.at_target[at];
  }
}

// (p - y) times the rows' weights, in 16 bits (two planes where inputs have 32).
// float16 has few small numbers, so there p is multiplied with 2^14 and the
// weights are in [1/2, 1): 2^-24 of p = 1 is a normal number.  Rows past the last
// up to a multiple of 64 and columns past the vocabulary are zeros, which the
// products that follow sum over.
template <class T, bool SPLIT>
__global__ void __launch_bounds__(T::kThreads) excess_kernel(HeadArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float lds_top[4];
  const int count = *a.kept.count, m = (count + T::BM - 1) / T::BM, n = (a.v1 - a.v0 + T::BN - 1) / T::BN;
  const int id = a.first + (int)blockIdx.x;
  if (id >= m * n) return;
  int tm, tn;
  tile_of(id, m, n, tm, tn);
  T t;
  t.run(a.H, a.W, tm * T::BM, tn * T::BN, m * T::BM, a.v1 - a.v0, 0, a.steps, SPLIT ? 3 : 1, a.pairs, smem);
  const float by = unscale<SPLIT>(a, lds_top);
  constexpr float kScale = T::KIND == kF16 ? 16384.f : 1.f;
#pragma unroll
  for (int i = 0; i < T::MT; ++i) {
    const int at = tm * T::BM + T::row(i);
    const bool on = at < count;
    const int y = on ? a.kept.target[at] : -2;
    const float lse = on ? a.kept.lse[at] : 0.f, mul = on ? a.kept.mul[at] * kScale : 0.f;
    char* row = const_cast<char*>(a.G.data) + at * a.G.stride;
#pragma unroll
    for (int j = 0; j < T::NT; j += T::F) {
      float g[4 * T::F];
#pragma unroll
      for (int f = 0; f < T::F; ++f)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int v = a.v0 + tn * T::BN + T::col(j + f) + e;
          const float x = t.acc[i][j + f][e] * by - lse;
          float p = __builtin_amdgcn_exp2f(x * kLog2e);
          if (v == y) p = expm1f(x);  // 1 - p without what p = 1 rounds away
          g[4 * f + e] = y == -2 || v >= a.v1 ? 0.f : p * mul;
        }
      char* to = row + 2 * (tn * T::BN + T::col(j));
#pragma unroll
      for (int h = 0; h < 4 * T::F; h += 8) {
        if constexpr (T::F == 1) {
          static_assert(T::F > 1);
        } else {
          const float x[8] = {g[h], g[h + 1], g[h + 2], g[h + 3], g[h + 4], g[h + 5], g[h + 6], g[h + 7]};
          store8<SPLIT ? EPIC_F32 : T::KIND == kF16 ? EPIC_F16 : EPIC_BF16>(to, a.G.plane, h, x);
        }
      }
    }
  }
}

// A slice of the piece's part of the hidden states' gradient: G W, summed over
// pieces in float32.
template <class T, bool SPLIT>
__global__ void __launch_bounds__(T::kThreads) grad_hidden_kernel(HeadArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int count = *a.kept.count, m = (count + T::BM - 1) / T::BM, n = (a.d + T::BN - 1) / T::BN;
  int id = a.first + (int)blockIdx.x;
  if (id >= m * n * a.slices) return;
  const int slice = id / (m * n);
  id -= slice * m * n;
  int tm, tn;
  tile_of(id, m, n, tm, tn);
  const int all = (a.v1 - a.v0 + 63) / 64, k0 = (int)((int64_t)all * slice / a.slices), k1 = (int)((int64_t)all * (slice + 1) / a.slices);
  T t;
  t.run(a.G, a.W, tm * T::BM, tn * T::BN, m * T::BM, (int)(a.H.stride / 2), k0, k1 - k0, SPLIT ? 3 : 1, a.pairs, smem);
  const int dp = (int)(a.H.stride / 2);
#pragma unroll
  for (int i = 0; i < T::MT; ++i) {
    const int at = tm * T::BM + T::row(i);
    if (at >= count) continue;
#pragma unroll
    for (int j = 0; j < T::NT; ++j) {
      const int c = tn * T::BN + T::col(j);
      if (c >= dp) continue;
      f4* to = (f4*)(a.dh + slice * a.dh_slice + (int64_t)at * dp + c);
      *to = a.add ? *to + t.acc[i][j] : t.acc[i][j];
    }
  }
}

// Slices of the hidden states' gradient to its rows, one wavefront a row.
template <int DT>
__global__ void __launch_bounds__(256) scatter_kernel(HeadArgs a, char* grad, int64_t grad_seq, int64_t grad_row) {
  __shared__ float lds[4];
  int e_head = 0;
  if constexpr (DT == EPIC_F32) e_head = -scale_exp(top_of(a.tops + a.top_parts[0], a.top_parts[1], lds));
  const int at = a.first + (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  if (at >= *a.kept.count) return;
  const int r = a.kept.src[at], b = r / a.rows;
  char* row = grad + b * grad_seq + (r - b * a.rows) * grad_row;
  const int dp = (int)(a.H.stride / 2);
  const int e = DT == EPIC_BF16 ? 0 : a.kept.exp[at] - 14 + e_head;
  for (int t = lane * 8; t < a.d; t += 512) {
    float x[8] = {};
    for (int s = 0; s < a.slices; ++s) {
      const f4* p = (const f4*)(a.dh + s * a.dh_slice + (int64_t)at * dp + t);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] += p[k >> 2][k & 3];
    }
    if constexpr (DT != EPIC_BF16) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = __builtin_amdgcn_ldexpf(x[k], e);
    }
    if (t + 8 <= a.d) {
      if constexpr (DT == EPIC_F32) {
        Loose16 v[2];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k >> 2].d[k & 3] = __float_as_uint(x[k]);
        *(Loose16*)(row + 4 * (int64_t)t) = v[0];
        *(Loose16*)(row + 4 * (int64_t)t + 16) = v[1];
      } else {
        Loose16 v;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          v.d[k] = DT == EPIC_F16 ? pack_f16(x[2 * k], x[2 * k + 1]) : pack_bf16(x[2 * k], x[2 * k + 1]);
        *(Loose16*)(row + 2 * (int64_t)t) = v;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (t + k < a.d) {
          if constexpr (DT == EPIC_F32)
            *(float*)(row + 4 * (int64_t)(t + k)) = x[k];
          else
            *(uint16_t*)(row + 2 * (int64_t)(t + k)) = (uint16_t)(DT == EPIC_F16 ? pack_f16(x[k], 0.f) : pack_bf16(x[k], 0.f));
        }
    }
  }
}

// The head's gradient of a piece: G^T H over the rows that count, rounded once.
template <class T, bool SPLIT, int DT>
__global__ void __launch_bounds__(T::kThreads) grad_head_kernel(HeadArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float lds_top[4];
  const int count = *a.kept.count, m = (a.v1 - a.v0 + T::BM - 1) / T::BM, n = (a.d + T::BN - 1) / T::BN;
  const int id = a.first + (int)blockIdx.x;
  if (id >= m * n) return;
  int tm, tn;
  tile_of(id, m, n, tm, tn);
  T t;
  t.run(a.G, a.H2, tm * T::BM, tn * T::BN, m * T::BM, (int)(a.H.stride / 2), 0, (count + 63) / 64, SPLIT ? 3 : 1, a.pairs, smem);
  int e = 0;
  if constexpr (DT == EPIC_F16) e = a.kept.count[1] - 14;
  if constexpr (DT == EPIC_F32) e = a.kept.count[1] - 14 - scale_exp(top_of(a.tops, a.top_parts[0], lds_top));
#pragma unroll
  for (int i = 0; i < T::MT; ++i) {
    const int v = a.v0 + tm * T::BM + T::row(i);
    if (v >= a.v1) continue;
    char* row = a.grad_head + v * a.grad_row;
#pragma unroll
    for (int j = 0; j < T::NT; ++j) {
      const int c = tn * T::BN + T::col(j);
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = DT == EPIC_BF16 ? t.acc[i][j][k] : __builtin_amdgcn_ldexpf(t.acc[i][j][k], e);
      struct __attribute__((packed, aligned(2))) Loose8 {
        uint32_t d[2];
      };
      if (c + 4 <= a.d) {
        if constexpr (DT == EPIC_F32)
          *(Loose16*)(row + 4 * (int64_t)c) =
              Loose16{{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])}};
        else if constexpr (DT == EPIC_F16)
          *(Loose8*)(row + 2 * (int64_t)c) = Loose8{{pack_f16(x[0], x[1]), pack_f16(x[2], x[3])}};
        else
          *(Loose8*)(row + 2 * (int64_t)c) = Loose8{{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])}};
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + k < a.d) {
            if constexpr (DT == EPIC_F32)
              *(float*)(row + 4 * (int64_t)(c + k)) = x[k];
            else
              *(uint16_t*)(row + 2 * (int64_t)(c + k)) = (uint16_t)(DT == EPIC_F16 ? pack_f16(x[k], 0.f) : pack_bf16(x[k], 0.f));
          }
      }
    }
  }
}

// Logits of a head in 8 bits: sums of whole numbers, exact in 32 bits, times the
// row's and the token's scale.
template <class T, int DT>
__global__ void __launch_bounds__(T::kThreads) logits_kernel(HeadArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int count = *a.kept.count, m = (count + T::BM - 1) / T::BM, n = (a.V + T::BN - 1) / T::BN;
  const int id = a.first + (int)blockIdx.x;
  if (id >= m * n) return;
  int tm, tn;
  tile_of(id, m, n, tm, tn);
  T t;
  t.run(a.H, a.W, tm * T::BM, tn * T::BN, m * T::BM, a.V, 0, a.steps, 1, 0, smem);
#pragma unroll
  for (int i = 0; i < T::MT; ++i) {
    const int at = tm * T::BM + T::row(i);
    if (at >= count) continue;
    const int r = a.kept.src[at], b = r / a.rows;
    const float s = a.row_scale[at];
    char* row = a.logits + b * a.seq_stride + (r - b * a.rows) * a.row_stride;
#pragma unroll
    for (int j = 0; j < T::NT; j += T::F) {
      const int c = tn * T::BN + T::col(j);
#pragma unroll
      for (int h = 0; h < 4 * T::F; h += kPer<DT>) {
        float x[kPer<DT>];
        if (c + h >= a.V) continue;
#pragma unroll
        for (int k = 0; k < kPer<DT>; ++k)
          x[k] = (float)t.acc[i][j + (h + k) / 4][(h + k) & 3] * s * a.col_scale[min(c + h + k, a.V - 1)];
        if constexpr (DT == EPIC_F16) {
          // the product is a float32 number before it is rounded to float16: the compiler would join the two
#pragma unroll
          for (int k = 0; k < 8; ++k) asm volatile("" : "+v"(x[k]));
        }
        if (c + h + kPer<DT> <= a.V) {
          Loose16 v;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if constexpr (DT == EPIC_F32)
              v.d[k] = __float_as_uint(x[k]);
            else
              v.d[k] = DT == EPIC_F16 ? pack_f16(x[2 * k], x[2 * k + 1]) : pack_bf16(x[2 * k], x[2 * k + 1]);
          }
          *(Loose16*)(row + (int64_t)(c + h) * kSize<DT>) = v;
        } else {
#pragma unroll
          for (int k = 0; k < kPer<DT>; ++k)
            if (c + h + k < a.V) {
              if constexpr (DT == EPIC_F32)
                *(float*)(row + 4 * (int64_t)(c + h + k)) = x[k];
              else
                *(uint16_t*)(row + 2 * (int64_t)(c + h + k)) = (uint16_t)(DT == EPIC_F16 ? pack_f16(x[k], 0.f) : pack_bf16(x[k], 0.f));
            }
        }
      }
    }
  }
}

// ------------------------------------------------------------ host side
constexpr int64_t kMaxRows = 1 << 24;
constexpr int kMaxWidth = 65536;
constexpr int kTopParts = 256;  // workgroups that look for a tensor's largest magnitude, at most

inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

template <int KIND>
using Large = Tile<KIND, 256, 256, 2, 4, 2, true, true>;
template <int KIND>
using Small = Tile<KIND, 64, 64, 2, 2, 4, true, true>;

template <class T, class K>
epic_status launch_tiles(K kernel, HeadArgs a, int64_t blocks, hipStream_t stream) {
  // a launch needs to be told once that it may use more than 64 KiB of LDS
  if (T::kLds > 65536 && hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, T::kLds) != hipSuccess)
    return EPIC_ERR_HIP;
  if (blocks > INT32_MAX) return EPIC_ERR_UNSUPPORTED;
  launches((int)blocks, T::kThreads, [&](int first, int count) {
    a.first = first;
    hipLaunchKernelGGL(kernel, dim3(count), dim3(T::kThreads), T::kLds, stream, a);
  });
  return EPIC_OK;
}

// Where what a call keeps lies in its workspace.
struct Layout {
  int64_t rows, padded;  // rows of the window, and up to a multiple of 256
  int64_t width;         // of packed rows, in numbers
  int planes;
  bool direct;           // the head is read where it is
  int64_t piece;         // tokens of a piece
  int slices;            // of a piece, in the hidden states' gradient
  int64_t parts;
  int64_t count, src, target, lse, mul, exp, tops, at_target, part, H, H2, W, G, dh, bytes;
};

bool head_direct(const epic_rows_desc* head) {
  if (head->dtype == EPIC_F32) return false;
  return head->vocab % 64 == 0 && head->rows % 64 == 0 && head->row_stride % 8 == 0 && head->row_stride < (1 << 21) &&
         ((uintptr_t)head->data & 15) == 0;
}

Layout layout_of(const epic_rows_desc* hidden, const epic_rows_desc* head, bool backward) {
  Layout l{};
  const int64_t V = head->rows;
  l.rows = (int64_t)hidden->batch * hidden->rows;
  l.padded = up(l.rows, 256);
  l.width = up(hidden->vocab, 64);
  l.planes = hidden->dtype == EPIC_F32 ? 2 : 1;
  l.direct = head_direct(head);
  l.piece = up(V, 256);
  if (backward || !l.direct) {
    int64_t most = std::max<int64_t>(4096, (1 << 26) / std::max<int64_t>(1, std::max<int64_t>(l.direct ? 0 : l.width, backward ? l.padded : 0) * l.planes) / 256 * 256);
    const int64_t pieces = (V + most - 1) / most;
    l.piece = up((V + pieces - 1) / pieces, 256);
  }
  l.parts = up(V, 64) / 64;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t p = at;
    at += up(bytes, 256);
    return p;
  };
  l.slices = 1;
  l.count = take(8);
  l.src = take(4 * l.padded);
  l.target = take(4 * l.padded);
  l.lse = take(4 * l.padded);
  l.mul = take(4 * l.padded);
  l.exp = take(4 * l.padded);
  l.tops = take(8 * kTopParts);
  l.at_target = take(4 * l.padded);
  l.H = take(2 * l.planes * l.padded * l.width);
  if (!l.direct) l.W = take(2 * l.planes * l.piece * l.width);
  if (!backward) {
    l.part = take(8 * l.padded * l.parts);
  } else {
    if (hidden->dtype != EPIC_BF16) l.H2 = take(2 * l.planes * l.padded * l.width);
    else l.H2 = l.H;
    l.G = take(2 * l.planes * l.padded * l.piece);
    l.dh = take(4 * l.slices * l.padded * l.width);
  }
  l.bytes = at;
  return l;
}

epic_status check_hidden(const epic_rows_desc* hidden, const int32_t* d_seqs, int32_t n) {
  const epic_status st = check_rows(hidden, d_seqs, n);
  if (st != EPIC_OK) return st;
  if (hidden->vocab > kMaxWidth || (int64_t)hidden->batch * hidden->rows > kMaxRows) return EPIC_ERR_UNSUPPORTED;
  return EPIC_OK;
}

epic_status check_head(const epic_rows_desc* hidden, const epic_rows_desc* head) {
  const epic_status st = check_rows(head, nullptr, 0);
  if (st != EPIC_OK) return st;
  if (head->dtype != hidden->dtype || head->vocab != hidden->vocab || head->batch != 1 || head->rows < 1) return EPIC_ERR_ARG;
  if (head->rows > kMaxVocab) return EPIC_ERR_UNSUPPORTED;
  return EPIC_OK;
}

constexpr uint32_t kOnePair = 0;
constexpr uint32_t kThreePairs = 0x014;  // (0, 1), (1, 0), (0, 0): small products first

struct Call {
  const epic_rows_desc *hidden, *head;
  Layout l;
  GatherArgs g;
  HeadArgs a;
  hipStream_t stream;
};

template <int DT>
epic_status pack_head(const Call& c, int v0, int count) {
  PackArgs p{(const char*)c.head->data, c.head->row_stride * kSize<DT>, c.head->rows, c.head->vocab, v0, count,
             const_cast<char*>(c.a.W.data), c.a.W.stride, c.a.W.plane, c.a.tops, {c.a.top_parts[0], c.a.top_parts[1]}};
  hipLaunchKernelGGL(pack_kernel<DT>, dim3(std::min(2048, (count + 3) / 4)), dim3(256), 0, c.stream, p);
  return EPIC_OK;
}

template <int DT, int MODE>
void gather(Call& c) {
  c.g.per = (int)std::max<int64_t>(4, up((c.l.rows + 4095) / 4096, 4));
  if constexpr (DT == EPIC_F32 && MODE != kQuantize) {
    TopArgs t{c.g, (const char*)c.head->data, c.head->row_stride * 4, const_cast<float*>(c.a.tops)};
    hipLaunchKernelGGL(top_kernel, dim3(c.g.top_parts[0] + c.g.top_parts[1]), dim3(256), 0, c.stream, t);
  }
  hipLaunchKernelGGL((gather_kernel<DT, MODE>), dim3((int)std::max<int64_t>(1, (c.l.rows + c.g.per - 1) / c.g.per)), dim3(kGather), 0, c.stream, c.g);
}

// What both passes set up: operands, rows that count, the head's pieces.
template <int DT>
void set_up(Call& c, char* ws) {
  const Layout& l = c.l;
  Kept kept{(int32_t*)(ws + l.count), (int32_t*)(ws + l.src), (int32_t*)(ws + l.target), (float*)(ws + l.lse), (float*)(ws + l.mul),
            (int32_t*)(ws + l.exp)};
  const int64_t stride = 2 * l.width, plane = l.padded * stride;
  c.g.kept = c.a.kept = kept;
  c.g.out = ws + l.H;
  c.g.out2 = ws + l.H2;
  c.g.stride = stride;
  c.g.plane = plane;
  c.g.tops = c.a.tops = (float*)(ws + l.tops);
  c.g.top_parts[0] = c.a.top_parts[0] = (int)std::min<int64_t>(kTopParts, (l.rows + 3) / 4);
  c.g.top_parts[1] = c.a.top_parts[1] = std::min(kTopParts, (c.head->rows + 3) / 4);
  c.a.H = {ws + l.H, stride, plane};
  c.a.H2 = {ws + l.H2, stride, plane};
  if (l.direct)
    c.a.W = {(const char*)c.head->data, c.head->row_stride * 2, 0};
  else
    c.a.W = {ws + l.W, stride, l.piece * stride};
  c.a.G = {ws + l.G, 2 * l.piece, l.padded * l.piece * 2};
  c.a.steps = (int)(l.width / 64);
  c.a.planes = l.planes;
  c.a.pairs = l.planes == 2 ? kThreePairs : kOnePair;
  c.a.V = c.head->rows;
  c.a.d = c.head->vocab;
  c.a.at_target = (float*)(ws + l.at_target);
  c.a.part = (float2*)(ws + l.part);
  c.a.dh = (float*)(ws + l.dh);
  c.a.dh_slice = l.padded * l.width;
  c.a.slices = l.slices;
  c.a.rows = c.hidden->rows;
}

template <int DT, class T>
epic_status losses(Call& c, float* loss, float* lse) {
  constexpr bool kSplit = DT == EPIC_F32;
  gather<DT, kForward>(c);
  const int V = c.a.V;
  c.a.parts = (V + T::BN - 1) / T::BN;
  const Operand whole = c.a.W;
  for (int v0 = 0; v0 < V; v0 += (int)c.l.piece) {
    c.a.v0 = v0;
    c.a.v1 = (int)std::min<int64_t>(V, v0 + c.l.piece);
    if (c.l.direct)
      c.a.W.data = whole.data + v0 * whole.stride;
    else
      pack_head<DT>(c, v0, (int)up(c.a.v1 - v0, 64));
    const int64_t tiles = (c.l.rows + T::BM - 1) / T::BM * ((c.a.v1 - v0 + T::BN - 1) / T::BN);
    const epic_status st = launch_tiles<T>(lse_kernel<T, kSplit>, c.a, tiles, c.stream);
    if (st != EPIC_OK) return st;
  }
  c.a.first = 0;
  hipLaunchKernelGGL(loss_kernel, dim3((int)((c.l.rows + 3) / 4)), dim3(256), 0, c.stream, c.a, loss, lse);
  return EPIC_OK;
}

template <int DT, class T, class TH, class TW>
epic_status gradients(Call& c, const epic_rows_desc* gh, const epic_rows_desc* gw) {
  constexpr bool kSplit = DT == EPIC_F32;
  gather<DT, kBackward>(c);
  const int V = c.a.V, d = c.a.d;
  const Operand whole = c.a.W;
  for (int v0 = 0; v0 < V; v0 += (int)c.l.piece) {
    c.a.v0 = v0;
    c.a.v1 = (int)std::min<int64_t>(V, v0 + c.l.piece);
    const int count = c.a.v1 - v0;
    if (c.l.direct)
      c.a.W.data = whole.data + v0 * whole.stride;
    else
      pack_head<DT>(c, v0, (int)up(count, 64));
    epic_status st = launch_tiles<T>(excess_kernel<T, kSplit>, c.a, (c.l.rows + T::BM - 1) / T::BM * ((count + T::BN - 1) / T::BN), c.stream);
    if (st == EPIC_OK && gh) {
      c.a.add = v0 > 0;
      st = launch_tiles<TH>(grad_hidden_kernel<TH, kSplit>, c.a,
                            (c.l.rows + TH::BM - 1) / TH::BM * ((d + TH::BN - 1) / TH::BN) * c.a.slices, c.stream);
    }
    if (st == EPIC_OK && gw) {
      c.a.grad_head = (char*)gw->data;
      c.a.grad_row = gw->row_stride * kSize<DT>;
      st = launch_tiles<TW>(grad_head_kernel<TW, kSplit, DT>, c.a,
                            (int64_t)((count + TW::BM - 1) / TW::BM) * ((d + TW::BN - 1) / TW::BN), c.stream);
    }
    if (st != EPIC_OK) return st;
  }
  if (gh && c.l.rows > 0) {
    c.a.first = 0;
    hipLaunchKernelGGL(scatter_kernel<DT>, dim3((int)((c.l.rows + 3) / 4)), dim3(256), 0, c.stream, c.a, (char*)gh->data,
                       gh->seq_stride * kSize<DT>, gh->row_stride * kSize<DT>);
  }
  return EPIC_OK;
}

template <int DT>
epic_status run_losses(Call& c, char* ws, float* loss, float* lse) {
  constexpr int K = DT == EPIC_BF16 ? kBf16 : kF16;
  set_up<DT>(c, ws);
  if (c.l.rows * c.a.V <= 256 * 256 * 256) return losses<DT, Small<K>>(c, loss, lse);
  return losses<DT, Large<K>>(c, loss, lse);
}
template <int DT>
epic_status run_gradients(Call& c, char* ws, const epic_rows_desc* gh, const epic_rows_desc* gw) {
  constexpr int K = DT == EPIC_BF16 ? kBf16 : kF16;
  set_up<DT>(c, ws);
  if (c.l.rows * c.a.V <= 256 * 256 * 256)
    return gradients<DT, Small<K>, Tile<K, 64, 64, 2, 2, 4, true, false>, Tile<K, 64, 64, 2, 2, 4, false, false>>(c, gh, gw);
  return gradients<DT, Large<K>, Tile<K, 256, 256, 2, 4, 2, true, false>, Tile<K, 256, 256, 2, 4, 2, false, false>>(c, gh, gw);
}

epic_status head_loss(bool backward, const epic_rows_desc* hidden, const int32_t* d_seqs, int32_t n, const int32_t* d_start,
                      const epic_rows_desc* head, const int32_t* d_target, float* d_loss, float* d_lse, const float* d_weight,
                      const epic_rows_desc* grad_hidden, const epic_rows_desc* grad_head, void* d_workspace,
                      size_t workspace_bytes, hipStream_t stream) {
  epic_status st = check_hidden(hidden, d_seqs, n);
  if (st != EPIC_OK || (st = head ? check_head(hidden, head) : EPIC_ERR_NULL) != EPIC_OK) return st;
  if (grad_hidden) {
    if ((st = check_rows(grad_hidden, nullptr, 0)) != EPIC_OK) return st;
    if (grad_hidden->dtype != hidden->dtype || grad_hidden->batch != hidden->batch || grad_hidden->rows != hidden->rows ||
        grad_hidden->vocab != hidden->vocab)
      return EPIC_ERR_ARG;
    if (hidden->batch > 0 && hidden->rows > 0 && !rows_apart(grad_hidden)) return EPIC_ERR_ARG;
  }
  if (grad_head) {
    if ((st = check_rows(grad_head, nullptr, 0)) != EPIC_OK) return st;
    if (grad_head->dtype != head->dtype || grad_head->batch != 1 || grad_head->rows != head->rows || grad_head->vocab != head->vocab ||
        !rows_apart(grad_head))
      return EPIC_ERR_ARG;
  }
  const Layout l = layout_of(hidden, head, backward);
  if (l.rows == 0 && !grad_head) return EPIC_OK;
  if (backward && !grad_hidden && !grad_head) return EPIC_ERR_NULL;
  if (!d_workspace || (l.rows > 0 && (!d_target || !d_lse || (!backward && !d_loss)))) return EPIC_ERR_NULL;
  if (((uintptr_t)d_workspace & 255) != 0) return EPIC_ERR_ARG;
  if (workspace_bytes < (size_t)l.bytes) return EPIC_ERR_CAPACITY;
  const int es = elem_size(hidden->dtype);
  Call c{};
  c.hidden = hidden;
  c.head = head;
  c.l = l;
  c.stream = stream;
  c.g.data = (const char*)hidden->data;
  c.g.seq_stride = hidden->seq_stride * es;
  c.g.row_stride = hidden->row_stride * es;
  c.g.batch = hidden->batch;
  c.g.rows = hidden->rows;
  c.g.d = hidden->vocab;
  c.g.win = {d_seqs, d_start, n};
  c.g.target = d_target;
  c.g.lse = d_lse;
  c.g.weight = d_weight;
  c.g.loss = d_loss;
  c.g.lse_out = d_lse;
  c.g.V = head->rows;
  if (grad_hidden) {
    c.g.grad = (char*)grad_hidden->data;
    c.g.grad_seq = grad_hidden->seq_stride * es;
    c.g.grad_row = grad_hidden->row_stride * es;
  }
  char* ws = (char*)d_workspace;
  switch (hidden->dtype) {
    case EPIC_F32: st = backward ? run_gradients<EPIC_F32>(c, ws, grad_hidden, grad_head) : run_losses<EPIC_F32>(c, ws, d_loss, d_lse); break;
    case EPIC_F16: st = backward ? run_gradients<EPIC_F16>(c, ws, grad_hidden, grad_head) : run_losses<EPIC_F16>(c, ws, d_loss, d_lse); break;
    default: st = backward ? run_gradients<EPIC_BF16>(c, ws, grad_hidden, grad_head) : run_losses<EPIC_BF16>(c, ws, d_loss, d_lse); break;
  }
  if (st != EPIC_OK) return st;
  return hipGetLastError() == hipSuccess ? EPIC_OK : EPIC_ERR_HIP;
}

template <int DT>
void run_quantize(const epic_rows_desc* x, int8_t* q, int64_t stride, float* scale, hipStream_t stream) {
  const int total = x->batch * x->rows;
  hipLaunchKernelGGL(quantize_kernel<DT>, dim3(std::min(4096, (total + 3) / 4)), dim3(256), 0, stream, (const char*)x->data,
                     x->seq_stride * kSize<DT>, x->row_stride * kSize<DT>, x->rows, total, x->vocab, q, stride, scale);
}

struct LogitsLayout {
  int64_t rows, padded, stride, count, src, scale, H, bytes;
};
LogitsLayout logits_layout(const epic_rows_desc* hidden) {
  LogitsLayout l{};
  l.rows = (int64_t)hidden->batch * hidden->rows;
  l.padded = up(l.rows, 256);
  l.stride = up(hidden->vocab, 128);
  l.count = 0;
  l.src = 256;
  l.scale = l.src + 4 * l.padded;
  l.H = l.scale + 4 * l.padded;
  l.bytes = l.H + l.padded * l.stride;
  return l;
}

template <class T>
epic_status run_logits(const HeadArgs& a, int dtype, int64_t rows, hipStream_t stream) {
  const int64_t tiles = (rows + T::BM - 1) / T::BM * ((a.V + T::BN - 1) / T::BN);
  switch (dtype) {
    case EPIC_F32: return launch_tiles<T>(logits_kernel<T, EPIC_F32>, a, tiles, stream);
    case EPIC_F16: return launch_tiles<T>(logits_kernel<T, EPIC_F16>, a, tiles, stream);
    default: return launch_tiles<T>(logits_kernel<T, EPIC_BF16>, a, tiles, stream);
  }
}

}  // namespace epic_rows

extern "C" {

epic_status epic_quantize_rows(const epic_rows_desc* x, int8_t* d_q, int64_t q_stride, float* d_scale, hipStream_t stream) {
  using namespace epic_rows;
  const epic_status st = check_hidden(x, nullptr, 0);
  if (st != EPIC_OK) return st;
  if (q_stride < x->vocab || q_stride % 128 != 0 || q_stride > 2 * kMaxWidth) return EPIC_ERR_ARG;
  if (x->batch == 0 || x->rows == 0) return EPIC_OK;
  if (!d_q || !d_scale) return EPIC_ERR_NULL;
  if (((uintptr_t)d_q & 15) != 0) return EPIC_ERR_ARG;
  switch (x->dtype) {
    case EPIC_F32: run_quantize<EPIC_F32>(x, d_q, q_stride, d_scale, stream); break;
    case EPIC_F16: run_quantize<EPIC_F16>(x, d_q, q_stride, d_scale, stream); break;
    default: run_quantize<EPIC_BF16>(x, d_q, q_stride, d_scale, stream); break;
  }
  return hipGetLastError() == hipSuccess ? EPIC_OK : EPIC_ERR_HIP;
}

size_t epic_logits_q8_workspace_bytes(const epic_rows_desc* hidden) {
  using namespace epic_rows;
  if (check_hidden(hidden, nullptr, 0) != EPIC_OK) return 0;
  return (size_t)logits_layout(hidden).bytes;
}

epic_status epic_logits_q8(const epic_rows_desc* hidden, const int32_t* d_seqs, int32_t n, const int32_t* d_start,
                           const int8_t* d_q, int64_t q_stride, const float* d_q_scale, const epic_rows_desc* logits,
                           void* d_workspace, size_t workspace_bytes, hipStream_t stream) {
  using namespace epic_rows;
  epic_status st = check_hidden(hidden, d_seqs, n);
  if (st != EPIC_OK || (st = check_rows(logits, nullptr, 0)) != EPIC_OK) return st;
  const LogitsLayout l = logits_layout(hidden);
  if (logits->batch != hidden->batch || logits->rows != hidden->rows || q_stride != l.stride) return EPIC_ERR_ARG;
  if (l.rows == 0) return EPIC_OK;
  if (!rows_apart(logits)) return EPIC_ERR_ARG;
  if (!d_q || !d_q_scale || !d_workspace) return EPIC_ERR_NULL;
  if (((uintptr_t)d_q & 15) != 0 || ((uintptr_t)d_workspace & 255) != 0) return EPIC_ERR_ARG;
  if (workspace_bytes < (size_t)l.bytes) return EPIC_ERR_CAPACITY;
  char* ws = (char*)d_workspace;
  const int es = elem_size(hidden->dtype), eo = elem_size(logits->dtype);
  Call c{};
  c.hidden = hidden;
  c.l.rows = l.rows;
  c.stream = stream;
  c.g.data = (const char*)hidden->data;
  c.g.seq_stride = hidden->seq_stride * es;
  c.g.row_stride = hidden->row_stride * es;
  c.g.batch = hidden->batch;
  c.g.rows = hidden->rows;
  c.g.d = hidden->vocab;
  c.g.win = {d_seqs, d_start, n};
  c.g.kept = {(int32_t*)(ws + l.count), (int32_t*)(ws + l.src), nullptr, nullptr, nullptr, nullptr};
  c.g.out = ws + l.H;
  c.g.stride = l.stride;
  c.g.scale = (float*)(ws + l.scale);
  switch (hidden->dtype) {
    case EPIC_F32: gather<EPIC_F32, kQuantize>(c); break;
    case EPIC_F16: gather<EPIC_F16, kQuantize>(c); break;
    default: gather<EPIC_BF16, kQuantize>(c); break;
  }
  HeadArgs& a = c.a;
  a.kept = c.g.kept;
  a.H = {ws + l.H, l.stride, 0};
  a.W = {(const char*)d_q, q_stride, 0};
  a.steps = (int)(l.stride / 128);
  a.V = logits->vocab;
  a.row_scale = c.g.scale;
  a.col_scale = d_q_scale;
  a.logits = (char*)logits->data;
  a.seq_stride = logits->seq_stride * eo;
  a.row_stride = logits->row_stride * eo;
  a.rows = hidden->rows;
  if (l.rows * a.V <= 256 * 256 * 256)
    st = run_logits<Small<kI8>>(a, logits->dtype, l.rows, stream);
  else
    st = run_logits<Large<kI8>>(a, logits->dtype, l.rows, stream);
  if (st != EPIC_OK) return st;
  return hipGetLastError() == hipSuccess ? EPIC_OK : EPIC_ERR_HIP;
}

size_t epic_head_loss_workspace_bytes(const epic_rows_desc* hidden, const epic_rows_desc* head, int32_t backward) {
  using namespace epic_rows;
  if (check_hidden(hidden, nullptr, 0) != EPIC_OK || !head || check_head(hidden, head) != EPIC_OK) return 0;
  return (size_t)std::max(layout_of(hidden, head, false).bytes, backward ? layout_of(hidden, head, true).bytes : 0);
}

epic_status epic_head_loss_forward(const epic_rows_desc* hidden, const int32_t* d_seqs, int32_t n, const int32_t* d_start,
                                   const epic_rows_desc* head, const int32_t* d_target, float* d_loss, float* d_lse,
                                   void* d_workspace, size_t workspace_bytes, hipStream_t stream) {
  return epic_rows::head_loss(false, hidden, d_seqs, n, d_start, head, d_target, d_loss, d_lse, nullptr, nullptr, nullptr,
                              d_workspace, workspace_bytes, stream);
}

epic_status epic_head_loss_backward(const epic_rows_desc* hidden, const int32_t* d_seqs, int32_t n, const int32_t* d_start,
                                    const epic_rows_desc* head, const int32_t* d_target, const float* d_lse,
                                    const float* d_weight, const epic_rows_desc* grad_hidden, const epic_rows_desc* grad_head,
                                    void* d_workspace, size_t workspace_bytes, hipStream_t stream) {
  return epic_rows::head_loss(true, hidden, d_seqs, n, d_start, head, d_target, nullptr, const_cast<float*>(d_lse), d_weight,
                              grad_hidden, grad_head, d_workspace, workspace_bytes, stream);
}

}  // extern "C"
