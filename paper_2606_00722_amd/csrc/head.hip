// Between hidden states and logits: epic_quantize_rows, epic_logits_q8,
// epic_head_loss_forward and epic_head_loss_backward.
#include "product.inc"

namespace epic_rows {

// How numbers are multiplied.  float32 goes one of two ways: as it is, at a
// sixteenth of the rate of 16-bit numbers, or as the sum of two float16 numbers,
// three products of which keep 22 bits and a sign, at a third of it, for which
// hidden states and head have to be written out so first.
enum Form { kFormBf16, kFormF16, kFormF32, kFormSplit };
template <int FORM>
constexpr int kDtype = FORM == kFormBf16 ? EPIC_BF16 : FORM == kFormF16 ? EPIC_F16 : EPIC_F32;
template <int FORM>
constexpr int kKind = FORM == kFormBf16 ? kBf16 : FORM == kFormF32 ? kF32 : kF16;
template <int FORM>
constexpr int kPairs = FORM == kFormSplit ? 3 : 1;
constexpr uint32_t kThreePairs = 0x014;  // planes (0, 1), (1, 0), (0, 0): small products first
template <int FORM>
constexpr int kPacked = FORM == kFormF32 ? 4 : 2;  // bytes of a number that products read
template <int FORM>
constexpr bool kPacks = FORM != kFormF32;  // some heads are written out
template <int FORM>
constexpr bool kScaled = FORM == kFormF16 || FORM == kFormSplit;  // numbers are brought into float16's range

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
  int32_t* scale;   // 32 bits in two parts: the power of two of the packed row
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
  char* out2;        // with the rows' powers of two, for the product over rows
  int64_t stride, plane;  // bytes
  int width;         // of packed rows, in numbers
  int shift;         // of their last 64
  float* scale;      // 8 bits: the rows' scales
  int32_t* row_exp;  // 32 bits in two parts: powers of two of the rows' largest magnitudes, or NULL
  int per;           // rows of a workgroup
  int2* counts;      // of every 64 rows, or NULL
  int V;
};

constexpr int kGather = 256;  // threads

template <int DT>
EPIC_DEV void load8(const char* row, int t, int d, float (&x)[8]) {
  if (t >= d) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
  } else if constexpr (DT == EPIC_F32) {
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
// A 32-bit number as the sum of two 16-bit ones.  With the largest magnitude (of a
// row of hidden states, of the head) scaled to [2^14, 2^15), numbers down to 2^-17
// of it keep 22 bits and a sign (the second one's half step: 2^-24 of the number),
// smaller ones an error of 2^-40 of the largest.
EPIC_DEV void split_f16(float x, _Float16& a, _Float16& b) {
  a = (_Float16)x;
  const float r = x - (float)a;
  b = (_Float16)(r - r == 0.f ? r : 0.f);  // of an infinity there is no rest
}

// Eight numbers of packed row `row` at t.
template <int FORM>
EPIC_DEV void store8(char* row, int64_t plane, int t, const float (&x)[8]) {
  if constexpr (FORM == kFormF32) {
    *(float4*)(row + 4 * (int64_t)t) = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(row + 4 * (int64_t)t + 16) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint4 a;
    if constexpr (FORM == kFormSplit) {
      _Float16 p[8], q[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) split_f16(x[e], p[e], q[e]);
      a = __builtin_bit_cast(uint4, p);
      *(uint4*)(row + plane + 2 * (int64_t)t) = __builtin_bit_cast(uint4, q);
    } else if constexpr (FORM == kFormF16) {
      a = make_uint4(pack_f16(x[0], x[1]), pack_f16(x[2], x[3]), pack_f16(x[4], x[5]), pack_f16(x[6], x[7]));
    } else {
      a = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
    *(uint4*)(row + 2 * (int64_t)t) = a;
  }
}

struct __attribute__((packed, aligned(2))) Loose8 {
  uint32_t d[2];
};
// Four numbers at t of a row of d in the caller's memory; nothing past its end.
template <int DT>
EPIC_DEV void store4(char* row, int t, int d, const float (&x)[4]) {
  if (t + 4 <= d) {
    if constexpr (DT == EPIC_F32)
      *(Loose16*)(row + 4 * (int64_t)t) = Loose16{{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])}};
    else if constexpr (DT == EPIC_F16)
      *(Loose8*)(row + 2 * (int64_t)t) = Loose8{{pack_f16(x[0], x[1]), pack_f16(x[2], x[3])}};
    else
      *(Loose8*)(row + 2 * (int64_t)t) = Loose8{{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])}};
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (t + k < d) {
      if constexpr (DT == EPIC_F32)
        *(float*)(row + 4 * (int64_t)(t + k)) = x[k];
      else
        *(uint16_t*)(row + 2 * (int64_t)(t + k)) = (uint16_t)(DT == EPIC_F16 ? pack_f16(x[k], 0.f) : pack_bf16(x[k], 0.f));
    }
}
// Eight.
template <int DT>
EPIC_DEV void put8(char* row, int t, int d, const float (&x)[8]) {
  if (t + 8 <= d && DT != EPIC_F32) {
    Loose16 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v.d[k] = DT == EPIC_F16 ? pack_f16(x[2 * k], x[2 * k + 1]) : pack_bf16(x[2 * k], x[2 * k + 1]);
    *(Loose16*)(row + 2 * (int64_t)t) = v;
    return;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float y[4] = {x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
    store4<DT>(row, t + 4 * h, d, y);
  }
}

// e with 2^(e - 1) <= |x| < 2^e, kNoExp of 0; and the power of two that scales such a
// number to [2^14, 2^15).
constexpr int kNoExp = -1000;
EPIC_DEV int exp_of(float x) { return x != 0.f ? __builtin_amdgcn_frexp_expf(x) : kNoExp; }
EPIC_DEV int scale_exp(int e) { return e == kNoExp ? 0 : 15 - e; }

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
// Rows of up to 4096 numbers are read once.
template <int DT>
EPIC_DEV void quantize_row(const char* row, int d, int8_t* out, int stride, float* scale, int lane) {
  constexpr int N = 8;
  float x[N][8];
  float top = 0.f;
  bool odd = false;
  const auto load = [&](int t0) {
#pragma unroll
    for (int j = 0; j < N; ++j) load8<DT>(row, t0 + j * 512 + lane * 8, d, x[j]);
  };
  for (int t0 = 0; t0 < d; t0 += 512 * N) {
    load(t0);
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top = fmaxf(top, fabsf(x[j][e]));
        odd = odd || !(fabsf(x[j][e]) < kInf);
      }
  }
  top = wave_max(top);
  odd = __ballot(odd) != 0;
  const float inv = odd || top < 1e-30f ? 0.f : 127.f / top;
  if (lane == 0) *scale = odd ? __builtin_nanf("") : inv == 0.f ? 0.f : top / 127.f;
  for (int t0 = 0; t0 < stride; t0 += 512 * N) {
    if (t0 > 0 || d > 512 * N) load(t0);  // (zeros behind the row)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int t = t0 + j * 512 + lane * 8;
      uint32_t q[2] = {0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int v = inv == 0.f ? 0 : (int)rintf(x[j][e] * inv);
        q[e >> 2] |= (uint32_t)(v & 255) << (8 * (e & 3));
      }
      if (t < stride) *(uint2*)(out + t) = make_uint2(q[0], q[1]);
    }
  }
}

// A row to packed numbers, multiplied with 2^e; with TWO also with 2^(e + e2).  The
// last 64 are zeros and numbers `shift` further on where the row has so few that
// the head, read where it is, has to be read up to its end (a multiple of 8).
template <int FORM, bool TWO>
EPIC_DEV void pack_row(const char* row, int d, int width, int shift, char* out, int64_t plane, int e, char* out2, int64_t plane2, int e2, int lane) {
  constexpr int N = 4;  // loads ahead
  for (int t0 = 0; t0 < width; t0 += 512 * N) {
    float x[N][8];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      int t = t0 + j * 512 + lane * 8;
      if (t >= width - 64) t = t - shift < width - 64 ? d : t - shift;
      load8<kDtype<FORM>>(row, t, d, x[j]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int t = t0 + j * 512 + lane * 8;
      if (t >= width) continue;
      if constexpr (FORM == kFormSplit) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[j][k] = __builtin_amdgcn_ldexpf(x[j][k], e);
      }
      store8<FORM>(out, plane, t, x[j]);
      if constexpr (TWO) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[j][k] = __builtin_amdgcn_ldexpf(x[j][k], e2);
        store8<FORM>(out2, plane2, t, x[j]);
      }
    }
  }
}

template <int DT>
EPIC_DEV void zero_grad(char* row, int d, int lane) {
  const float zero[8] = {};
  for (int t = lane * 8; t < d; t += 512) put8<DT>(row, t, d, zero);
}

enum GatherMode { kForward, kBackward, kQuantize };

// The power of two of a row's weight, kNoExp where there is none: of 0, of what is no
// number, and in rows that add nothing.
EPIC_DEV int weight_exp(const GatherArgs& a, int r) {
  const float w = a.weight ? a.weight[r] : 1.f;
  return fabsf(w) < kInf && !(a.target && a.target[r] >= a.V) ? exp_of(w) : kNoExp;
}
// That of what the row brings to a sum over rows: of its weight, and where rows are
// scaled each by itself of its largest magnitude too.
EPIC_DEV int part_exp(const GatherArgs& a, int r) {
  const int e = weight_exp(a, r);
  if (!a.row_exp || e == kNoExp) return e;
  const int m = a.row_exp[r];
  return m == kNoExp ? kNoExp : e + m;
}

// Of every 64 rows of the window how many count, and the largest power of two of
// what they bring: one wavefront each.
__global__ void __launch_bounds__(256) count_kernel(GatherArgs a) {
  const int group = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  const int total = a.batch * a.rows, r = group * 64 + lane;
  if (group * 64 >= total) return;
  const bool on = r < total && kept_row(a, r);
  const int e = on ? part_exp(a, r) : kNoExp;
  const int n = (int)__popcll(__ballot(on));
  const float top = wave_max((float)e);
  if (lane == 0) a.counts[group] = make_int2(n, (int)top);
}

// The rows that count, one after another, zeros behind them up to a multiple of
// 64 (the gradients' products sum over them).  Every workgroup counts the rows
// before its own itself, so that one launch does it for up to 1024 rows; of more it
// adds up count_kernel's numbers of 64 rows each.
// Bound by latency and by memory: 2867 of 4096 rows of 2048 bfloat16 numbers 10 us,
// 8192 of 4096 33 us (134 MB: 4.1 TB/s), one row 5 us.
template <int FORM, int MODE>
EPIC_DEV void gather_rows(const GatherArgs& a, int group, int (&lds_n)[kGather / 64], int (&lds_own)[64], float (&lds_f)[kGather / 64]) {
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int total = a.batch * a.rows, first = group * a.per, last = min(total, first + a.per);
  constexpr int DT = kDtype<FORM>;
  constexpr bool kWeights = MODE == kBackward && kScaled<FORM>;
  int before = 0, top_exp = INT32_MIN;
  // (the powers of two of what the rows bring go by the largest one)
  if (a.counts) {
    const int mine = first / 64, groups = kWeights ? (total + 63) / 64 : mine;
    for (int g = tid; g < groups; g += kGather) {
      const int2 c = a.counts[g];
      before += g < mine ? c.x : 0;
      top_exp = max(top_exp, c.y);
    }
    if (wave == 0 && mine * 64 + lane < first) before += kept_row(a, mine * 64 + lane);
  } else {
    for (int r = tid; r < (kWeights ? total : first); r += kGather)
      if (kept_row(a, r)) {
        before += r < first;
        if constexpr (kWeights) top_exp = max(top_exp, part_exp(a, r));
      }
  }
  before = (int)wave_sum((float)(before & 0xFFF)) + ((int)wave_sum((float)(before >> 12)) << 12);
  if constexpr (kWeights) top_exp = (int)wave_max((float)max(top_exp, kNoExp));
  if (lane == 0) {
    lds_n[wave] = before;
    lds_f[wave] = (float)top_exp;
  }
  __syncthreads();
  before = 0;
  for (int w = 0; w < kGather / 64; ++w) before += lds_n[w];
  if constexpr (kWeights)
    for (int w = 0; w < kGather / 64; ++w) top_exp = max(top_exp, (int)lds_f[w]);
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
          if (a.grad) zero_grad<DT>(a.grad + b * a.grad_seq + in * a.grad_row, a.d, lane);
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
        int h_exp = 0, shift = 0;
        if constexpr (FORM == kFormSplit) h_exp = scale_exp(a.row_exp[r]);
        if (lane == 0) {
          a.kept.target[at] = y;
          if constexpr (FORM == kFormSplit) a.kept.scale[at] = h_exp;
        }
        if constexpr (MODE == kBackward) {
          float w = a.weight ? a.weight[r] : 1.f;
          int e = 0;
          if (kWeights && weight_exp(a, r) != kNoExp) {
            e = exp_of(w);
            shift = part_exp(a, r) == kNoExp ? 0 : part_exp(a, r) - top_exp;
            w = __builtin_amdgcn_frexp_mantf(w);
          }
          if (lane == 0) {
            a.kept.exp[at] = e;
            a.kept.mul[at] = y < 0 ? 0.f : w;
            a.kept.lse[at] = y < 0 ? 0.f : a.lse[r];
          }
        }
        // a row that adds nothing has no numbers
        pack_row<FORM, kWeights>(row, MODE == kBackward && y < 0 ? 0 : a.d, a.width, a.shift, a.out + at * a.stride, a.plane, h_exp,
                                        a.out2 + at * a.stride, a.plane, shift, lane);
      }
    }
  }
  if (last == total) {
    if (tid == 0) *a.kept.count = before;
    if constexpr (kWeights)
      if (tid == 0) a.kept.count[1] = top_exp == kNoExp ? 0 : top_exp;
    if constexpr (MODE == kBackward) {
      const int end = (before + 63) / 64 * 64, vecs = (int)(a.stride / 16);
      for (int i = tid; i < (end - before) * vecs; i += kGather) {
        char* to = a.out2 + (int64_t)before * a.stride + (int64_t)i * 16;
        *(uint4*)to = make_uint4(0, 0, 0, 0);
        if constexpr (FORM == kFormSplit) *(uint4*)(to + a.plane) = make_uint4(0, 0, 0, 0);
      }
    }
  }
}

// The largest finite magnitudes: of every row of hidden states that counts its power
// of two (the first workgroups), and of the head one number for each of the others.
struct TopArgs {
  GatherArgs g;
  const char* head;
  int64_t head_row;
  float* tops;
  int row_groups;
};
__global__ void __launch_bounds__(256) top_kernel(TopArgs a) {
  __shared__ float lds[4];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  const bool head = (int)blockIdx.x >= a.row_groups;
  const int part = head ? (int)blockIdx.x - a.row_groups : (int)blockIdx.x, parts = head ? (int)gridDim.x - a.row_groups : a.row_groups;
  const int total = head ? a.g.V : a.g.batch * a.g.rows;
  constexpr int N = 4;  // loads ahead
  float top = 0.f;
  for (int r = part * 4 + wave; r < total; r += parts * 4) {
    const char* row;
    if (head) {
      row = a.head + r * a.head_row;
    } else {
      if (!kept_row(a.g, r)) continue;
      const int b = r / a.g.rows;
      row = a.g.data + b * a.g.seq_stride + (r - b * a.g.rows) * a.g.row_stride;
      top = 0.f;
    }
    for (int t0 = 0; t0 < a.g.d; t0 += 512 * N) {
      float x[N][8];
#pragma unroll
      for (int j = 0; j < N; ++j) load8<EPIC_F32>(row, t0 + j * 512 + lane * 8, a.g.d, x[j]);
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (fabsf(x[j][e]) < kInf) top = fmaxf(top, fabsf(x[j][e]));
    }
    if (!head) {
      top = wave_max(top);
      if (lane == 0) a.g.row_exp[r] = exp_of(top);
    }
  }
  if (!head) return;
  top = block_max(top, lds);
  if (threadIdx.x == 0) a.tops[part] = top;
}

// Rows v0 .. of the head as the products read them, one wavefront a row: widths
// and numbers of rows filled up with zeros.
struct PackArgs {
  const char* head;
  int64_t head_row;  // bytes
  int V, d, v0, count;
  char* out;
  int64_t stride, plane;
  int width;
  const float* tops;  // 32 bits: the head's largest magnitudes, in parts
  int top_parts;
};
template <int FORM>
EPIC_DEV void pack_rows(const PackArgs& a, int group, int groups, float* lds) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  int e_head = 0;
  if constexpr (FORM == kFormSplit) e_head = scale_exp(exp_of(top_of(a.tops, a.top_parts, lds)));
  for (int i = group * 4 + wave; i < a.count; i += groups * 4)
    pack_row<FORM, false>(a.head + (a.v0 + i) * a.head_row, a.v0 + i < a.V ? a.d : 0, a.width, 0, a.out + i * a.stride, a.plane, e_head,
                                nullptr, 0, 0, lane);
}
template <int FORM>
__global__ void __launch_bounds__(256) pack_kernel(PackArgs a) {
  __shared__ float lds[4];
  pack_rows<FORM>(a, (int)blockIdx.x, (int)gridDim.x, lds);
}

// The rows that count by the first `groups` workgroups, and by the others the
// head's first piece where it has to be packed.
template <int FORM, int MODE>
__global__ void __launch_bounds__(kGather) gather_kernel(GatherArgs a, PackArgs p, int groups) {
  __shared__ int lds_n[kGather / 64];
  __shared__ int lds_own[64];
  __shared__ float lds_f[kGather / 64];
  if ((int)blockIdx.x < groups)
    gather_rows<FORM, MODE>(a, (int)blockIdx.x, lds_n, lds_own, lds_f);
  else if constexpr (kPacks<FORM> && MODE != kQuantize)
    pack_rows<FORM>(p, (int)blockIdx.x - groups, (int)gridDim.x - groups, lds_f);
}

// Bound by memory: 131072 rows of 4096 bfloat16 numbers 301 us (1.6 GB, 5.4 TB/s), of float32
// 516 (5.2); wider rows are read twice: 32768 of 8192 in bfloat16 210 us, 3.9 TB/s of one
// reading.
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
  Operand H2;        // the rows as the head's gradient reads them
  Kept kept;
  int steps;         // of d
  int piece;         // tokens of a whole piece
  int width;         // d up to a multiple of 64
  int shift;         // of the last 64 of hidden states: the head is read where it is, up to its rows' end
  bool direct;
  int v0, v1;        // tokens of the piece
  int V, d;
  // losses
  float2* part;      // [rows][parts] maximum and sum of a tile's columns
  int64_t parts;
  float* at_target;
  const float* tops;
  int top_parts;
  // gradients
  Operand G;         // (p - y) of the piece [N, v] in 16 bits
  float* dh;         // [slices][rows][d] float32
  int64_t dh_slice;
  int max_slices, add, last;  // last: the piece after which gradients are whole
  char* grad_hidden;
  int64_t gh_seq, gh_row;  // bytes
  char* grad_head;
  int64_t grad_row;  // bytes
  // 8 bits
  const float* row_scale;
  const float* col_scale;
  char* logits;
  int64_t seq_stride, row_stride;  // bytes
  int rows;
};

// ---- Tiles.  Three sizes, one workgroup of 512 threads a CU for all: the large
// one takes the least from LDS and memory for a product, the smaller ones cut a
// small result into more pieces and keep more loads of the head on their way.
// Which, the kernel decides, by how many rows count.  Losses of 32768 tokens of width
// 2048 in bfloat16, large, mid and few, in us: 16 rows 57, 34, 34; 128 rows 54, 35, 39;
// 256 rows 55, 51, 65; 512 rows 66, 89, 115.  Of the few rows that are multiplied in
// float32 the smallest tiles are best (16 rows 91 us, in mid tiles 152, large 484).
template <int KIND, bool A_ALONG, bool B_ALONG>
struct Sizes {
  typedef Tile<KIND, 256, 256, 2, 4, 2, A_ALONG, B_ALONG> Large;
  typedef Tile<KIND, 128, 128, 2, 4, 4, A_ALONG, B_ALONG> Mid;
  typedef Tile<KIND, 64, 128, 2, 4, 5, A_ALONG, B_ALONG> Few;
};
constexpr int kProductThreads = 512, kProductLds = 131072, kCus = 256;

EPIC_DEV int ceil_div(int a, int b) { return (a + b - 1) / b; }
// 0 large, 1 mid, 2 few: of a result of m x n sums, `copies` times.  The rounds
// that the CUs take, by what a round of each size costs (in bfloat16 products, as above;
// the other types go by the same numbers).
EPIC_DEV int tile_cost(int size) { return size == 0 ? 20 : size == 1 ? 9 : 6; }
template <int KIND>
EPIC_DEV int tile_size(int m, int n, int copies = 1) {
  if (KIND == kF32) return 2;
  const auto rounds = [&](int rows, int cols) { return ((int64_t)ceil_div(m, rows) * ceil_div(n, cols) * copies + kCus - 1) / kCus; };
  const int64_t c0 = rounds(256, 256) * tile_cost(0), c1 = rounds(128, 128) * tile_cost(1), c2 = rounds(64, 128) * tile_cost(2);
  return c2 < c1 && c2 < c0 ? 2 : c1 < c0 ? 1 : 0;
}
template <class S, class F>
EPIC_DEV void with_size(int size, F&& f) {
  if constexpr (S::Few::KIND != kF32) {
    if (size == 0) {
      typename S::Large t;
      f(t);
      return;
    }
    if (size == 1) {
      typename S::Mid t;
      f(t);
      return;
    }
  }
  typename S::Few t;
  f(t);
}

// The head's power of two.
template <int FORM>
EPIC_DEV int head_exp(const HeadArgs& a, float* lds) {
  if constexpr (FORM != kFormSplit) return 0;
  return scale_exp(exp_of(top_of(a.tops, a.top_parts, lds)));
}

// A row's sums without its and the head's power of two, which is taken out number by number:
// as a factor it could leave float32 where the logits do not.
template <int FORM, class T>
EPIC_DEV void unscale(T& t, int i, int e) {
  if constexpr (FORM == kFormSplit) {
#pragma unroll
    for (int j = 0; j < T::NT; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) t.acc[i][j][k] = __builtin_amdgcn_ldexpf(t.acc[i][j][k], e);
  }
}

constexpr float kFar = 16777216.f;  // of a logit in powers of two: it is rounded to whole numbers

// Losses: a tile's columns to a maximum and a sum for every row, over the wavefronts of a
// row of tiles by LDS, and the logit of the row's token.  exp2 takes one product
// and sum: with c = log2(e), t c is rounded to T, and the sum of 2^(l c - T) is too
// large by the factor 2^(t c - T), which is taken out.  Past 2^31 that factor can
// leave float32: from kFar on a term is 2^((l - t) c).
// 2867 rows of 32768 tokens, width 2048, in bfloat16: 333 us, 1.16 PFLOP/s (the ends
// of 32-step tiles take a tenth); 16 rows of 131072 tokens, width 4096: 180 us, bound
// by reading the head at 6.0 TB/s.
template <int FORM, class T>
EPIC_DEV void lse_tiles(const HeadArgs& a, T& t, int count, int e_head, char* smem, float2* part, int (&target)[2][256], int (&scale)[2][256]) {
  const int m = ceil_div(count, T::BM), n = ceil_div(a.v1 - a.v0, T::BN);
  constexpr float c = kLog2e;
  auto place = [&](int id, int& tm, int& tn) { tile_of(id, m, n, tm, tn); };
  every_tile<kPairs<FORM>>(
      t, smem, [&](int i) { return dealt(i, m * n); },
      [&](int id) {
        int tm, tn;
        place(id, tm, tn);
        t.template start<kPairs<FORM>>(a.H, a.W, tm * T::BM, tn * T::BN, m * T::BM, a.v1 - a.v0, 0, a.steps, kPairs<FORM> == 3 ? kThreePairs : 0,
                                         1 << 30, 2 * a.shift);
      },
      [&](int id, int k) {
        int tm, tn;
        place(id, tm, tn);
        for (int r = T::wave() * 64 + T::lane_now(); r < T::BM; r += T::kThreads) {
          const int at = tm * T::BM + r;
          target[k][r] = at < count ? a.kept.target[at] - a.v0 - tn * T::BN : -1;
          if constexpr (FORM == kFormSplit) scale[k][r] = at < count ? -(a.kept.scale[at] + e_head) : 0;
        }
      },
      [&](int id, int k) {
        int tm, tn;
        place(id, tm, tn);
        const int wn = T::wave() % T::WN, lane = T::lane_now();
        const int cols = a.v1 - a.v0 - tn * T::BN;  // that there are, from the tile's first on
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
          const int r = T::row(i, lane), y = target[k][r];
          if constexpr (FORM == kFormSplit) unscale<FORM>(t, i, scale[k][r]);
          if (cols < T::BN) {
#pragma unroll
            for (int j = 0; j < T::NT; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) t.acc[i][j][e] = T::col(j, lane) + e < cols ? t.acc[i][j][e] : -kInf;
          }
          if (__any((unsigned)(y - wn * (T::BN / T::WN)) < (unsigned)(T::BN / T::WN))) {
#pragma unroll
            for (int j = 0; j < T::NT; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (T::col(j, lane) + e == y) a.at_target[tm * T::BM + r] = t.acc[i][j][e];
          }
          float top = -kInf;
#pragma unroll
          for (int j = 0; j < T::NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, t.acc[i][j][e]);
          top = fmaxf(top, __shfl_xor(top, 16));  // the four lanes of a row
          top = fmaxf(top, __shfl_xor(top, 32));
          const float base = top > -kInf ? top : 0.f, tc = base * c;
          const bool far = fabsf(tc) >= kFar;
          float sum = 0.f;
          if (__any(far)) {  // (rows beside a far one as ever)
            const float b0 = far ? base : 0.f, t0 = far ? 0.f : tc;
#pragma unroll
            for (int j = 0; j < T::NT; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(t.acc[i][j][e] - b0, c, -t0));
          } else {
#pragma unroll
            for (int j = 0; j < T::NT; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(t.acc[i][j][e], c, -tc));
          }
          sum += __shfl_xor(sum, 16);
          sum += __shfl_xor(sum, 32);
          if (lane < 16) part[wn * T::BM + r] = make_float2(top, far ? sum : sum * __builtin_amdgcn_exp2f(-__builtin_fmaf(base, c, -tc)));
        }
        lds_barrier();
        for (int r = T::wave() * 64 + T::lane_now(); r < T::BM; r += T::kThreads) {
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
      });
}
template <int FORM>
__global__ void __launch_bounds__(kProductThreads) lse_kernel(HeadArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[kProductLds];
  __shared__ float lds_top[kProductThreads / 64];
  __shared__ float2 part[4 * 256];
  __shared__ int target[2][256], scale[2][256];
  const int count = *a.kept.count, e_head = head_exp<FORM>(a, lds_top);
  with_size<Sizes<kKind<FORM>, true, true>>(tile_size<kKind<FORM>>(count, a.piece), [&](auto& t) { lse_tiles<FORM>(a, t, count, e_head, smem, part, target, scale); });
}

// Losses from the tiles' maxima and sums, one wavefront a row.
template <int FORM>
__global__ void __launch_bounds__(256) loss_kernel(HeadArgs a, float* loss, float* lse_out) {
  const int at = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  if (at >= *a.kept.count) return;
  const float2* p = a.part + at * a.parts;
  const int parts = ceil_div(a.V, tile_size<kKind<FORM>>(*a.kept.count, a.piece) == 0 ? 256 : 128);
  float top = -kInf;
#pragma unroll 8
  for (int i = lane; i < parts; i += 64) top = fmaxf(top, p[i].x);
  top = wave_max(top);
  const float base = top > -kInf ? top : 0.f;
  float sum = 0.f;
#pragma unroll 8
  for (int i = lane; i < parts; i += 64) sum += p[i].y * __builtin_amdgcn_exp2f((p[i].x - base) * kLog2e);
  sum = wave_sum(sum);
  if (lane == 0) {
    const int y = a.kept.target[at], r = a.kept.src[at];
    const float lse = base + logf(sum);
    lse_out[r] = lse;
    loss[r] = y < 0 ? __builtin_nanf("") : lse - a.at_target[at];
  }
}

// (p - y) times the rows' weights, in 16 bits (two planes where inputs have 32): the
// matrix units' products with 16-bit hidden states and head take no wider numbers, and
// two planes would double them.  It is a second rounding beside the result's: bfloat16
// gradients are off by 2.4e-3 of their norm where one rounding leaves 1.7e-3, float16 by
// 3.3e-4 and 2.1e-4.
// float16 has few small numbers, so there p is multiplied with 2^14 and the
// weights are in [1/2, 1): 2^-24 of p = 1 is a normal number.  Numbers of rows past
// the last, of rows without a token (which have hidden states 0 and weight 0) and
// of columns past the vocabulary are 0: the products that follow sum over them.
// 8192 rows of 16384 tokens, width 4096, in bfloat16: 785 us, 1.40 PFLOP/s.
template <int FORM, class T>
EPIC_DEV void excess_tiles(const HeadArgs& a, T& t, int count, int e_head, char* smem, int (&target)[2][256], float2 (&factor)[2][256],
                           int (&scale)[2][256]) {
  constexpr float kScale = kScaled<FORM> ? 16384.f : 1.f;
  const int m = ceil_div(count, T::BM), n = ceil_div(a.v1 - a.v0, T::BN);
  constexpr float c = kLog2e;
  auto place = [&](int id, int& tm, int& tn) { tile_of(id, m, n, tm, tn); };
  every_tile<kPairs<FORM>>(
      t, smem, [&](int i) { return dealt(i, m * n); },
      [&](int id) {
        int tm, tn;
        place(id, tm, tn);
        t.template start<kPairs<FORM>>(a.H, a.W, tm * T::BM, tn * T::BN, m * T::BM, a.v1 - a.v0, 0, a.steps, kPairs<FORM> == 3 ? kThreePairs : 0,
                                         1 << 30, 2 * a.shift);
      },
      [&](int id, int k) {
        int tm, tn;
        place(id, tm, tn);
        for (int r = T::wave() * 64 + T::lane_now(); r < T::BM; r += T::kThreads) {
          const int at = tm * T::BM + r;
          int y = -1;
          float2 x = make_float2(0.f, 0.f);
          if (at < count) {
            y = a.kept.target[at] - a.v0 - tn * T::BN;
            const float lse = a.kept.lse[at];
            x.x = lse * kLog2e;  // rounded; the factor below has what is left out
            x.y = a.kept.mul[at] * kScale * __builtin_amdgcn_exp2f(-__builtin_fmaf(lse, kLog2e, -x.x));
          }
          target[k][r] = y;
          factor[k][r] = x;
          if constexpr (FORM == kFormSplit) scale[k][r] = at < count ? -(a.kept.scale[at] + e_head) : 0;
        }
      },
      [&](int id, int k) {
        int tm, tn;
        place(id, tm, tn);
        const int wn = T::wave() % T::WN, lane = T::lane_now();
        const int cols = a.v1 - a.v0 - tn * T::BN;
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
          const int r = T::row(i, lane), at = tm * T::BM + r, y = target[k][r];
          const float2 x = factor[k][r];
          if constexpr (FORM == kFormSplit) unscale<FORM>(t, i, scale[k][r]);
          char* row = const_cast<char*>(a.G.data) + at * a.G.stride + kPacked<FORM> * (int64_t)(tn * T::BN);
          const bool far = fabsf(x.x) >= kFar;
          const bool some = __any((unsigned)(y - wn * (T::BN / T::WN)) < (unsigned)(T::BN / T::WN));
#pragma unroll
          for (int j = 0; j < T::NT; j += T::F) {
            float g[4 * T::F];
#pragma unroll
            for (int f = 0; f < 4 * T::F; ++f)
              g[f] = x.y * __builtin_amdgcn_exp2f(__builtin_fmaf(t.acc[i][j + f / 4][f & 3], c, -x.x));
            if (__any(far)) {  // the factors' product could leave float32
              const float lse = at < count ? a.kept.lse[at] : 0.f, w = at < count ? a.kept.mul[at] * kScale : 0.f;
#pragma unroll
              for (int f = 0; f < 4 * T::F; ++f)
                g[f] = far ? w * __builtin_amdgcn_exp2f((t.acc[i][j + f / 4][f & 3] - lse) * kLog2e) : g[f];
            }
            const int c0 = T::col(j, lane);
            if (some && (unsigned)(y - c0) < (unsigned)(4 * T::F)) {  // 1 - p without what p = 1 rounds away
              float l = 0.f;
#pragma unroll
              for (int f = 0; f < 4 * T::F; ++f) l = c0 + f == y ? t.acc[i][j + f / 4][f & 3] : l;
              const float own = a.kept.mul[at] * kScale * expm1f(l - a.kept.lse[at]);
#pragma unroll
              for (int f = 0; f < 4 * T::F; ++f) g[f] = c0 + f == y ? own : g[f];
            }
            if (cols < T::BN || (tm + 1) * T::BM > count) {
#pragma unroll
              for (int f = 0; f < 4 * T::F; ++f) g[f] = c0 + f < cols && at < count ? g[f] : 0.f;
            }
#pragma unroll
            for (int h = 0; h < 4 * T::F; h += 8) {
              const float v[8] = {g[h], g[h + 1], g[h + 2], g[h + 3], g[h + 4], g[h + 5], g[h + 6], g[h + 7]};
              store8<FORM>(row + kPacked<FORM> * c0, a.G.plane, h, v);
            }
          }
        }
      });
}
template <int FORM>
__global__ void __launch_bounds__(kProductThreads) excess_kernel(HeadArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[kProductLds];
  __shared__ float lds_top[kProductThreads / 64];
  __shared__ int target[2][256];
  __shared__ float2 factor[2][256];  // lse in powers of two, and what 2^(l - lse) is multiplied with
  __shared__ int scale[2][256];
  const int count = *a.kept.count, e_head = head_exp<FORM>(a, lds_top);
  with_size<Sizes<kKind<FORM>, true, true>>(tile_size<kKind<FORM>>(count, a.piece), [&](auto& t) { excess_tiles<FORM>(a, t, count, e_head, smem, target, factor, scale); });
}

// ---- The two products with G, in one launch: the hidden states' gradient G W
// (few tiles, long sums over the piece's tokens, cut into slices) and the head's,
// G^T H (many tiles, sums over the rows that count).  Each workgroup takes its
// share of the first, and of the second those that had less before first one or
// more, so that all end at about the same time.
// 8192 rows of 16384 tokens, width 4096, in bfloat16: 1.69 ms, 1.30 PFLOP/s; 2867 of
// 32768, width 2048: 676 us, 1.14 (two launches, the first on 96 CUs, took 949).
struct Split {
  int size_h, size_w;    // tiles
  int m_h, n_h, m_w, n_w;
  int slices;            // of the sums over tokens
  int lead;              // tiles of the second that a workgroup with one less of the first takes before
};
template <int KIND>
EPIC_DEV Split split_of(const HeadArgs& a, int count) {
  Split s;
  s.size_h = tile_size<KIND>(count, a.d, min(a.max_slices, max(1, a.piece / 2048)));
  s.size_w = tile_size<KIND>(a.piece, a.d);
  const int hm = s.size_h == 0 ? 256 : s.size_h == 1 ? 128 : 64, hn = s.size_h == 0 ? 256 : 128;
  const int wm = s.size_w == 0 ? 256 : s.size_w == 1 ? 128 : 64, wn = s.size_w == 0 ? 256 : 128;
  s.m_h = ceil_div(count, hm);
  s.n_h = ceil_div(a.d, hn);
  s.m_w = ceil_div(a.v1 - a.v0, wm);
  s.n_w = ceil_div(a.d, wn);
  // by what a step of a tile costs; a tile's start and end are worth some steps
  const int k_h = ceil_div(a.piece, 64), k_w = ceil_div(count, 64) + 8, cost_h = tile_cost(s.size_h), cost_w = tile_cost(s.size_w);
  const int64_t all = (a.grad_hidden ? (int64_t)s.m_h * s.n_h * k_h * cost_h : 0) +
                      (a.grad_head ? (int64_t)ceil_div(a.piece, wm) * s.n_w * k_w * cost_w : 0);
  // Slices of no more than 4/5 of what each CU has to do (2867 rows of 32768 tokens,
  // width 2048, both passes: 1.05 ms; of 4/3 of it 1.18, of 2/5 1.07), and of at
  // least 1024 tokens.
  s.slices = 1;
  while (2 * s.slices <= a.max_slices && k_h >= 16 * s.slices && (int64_t)k_h * cost_h * 5 * kCus > 4 * all * s.slices) s.slices *= 2;
  s.lead = (int)(((int64_t)k_h / s.slices + 8) * cost_h / (k_w * cost_w));
  return s;
}

// Slices are float32, summed over pieces; of one slice, the last piece's end
// rounds and writes the gradient.
template <int FORM, class T>
EPIC_DEV void grad_hidden_tiles(const HeadArgs& a, T& t, const Split& s, int count, int e, char* smem) {
  constexpr int P = kPairs<FORM>, DT = kDtype<FORM>;
  const int m = s.m_h, n = s.n_h, all = ceil_div(a.v1 - a.v0, 64), dp = a.width;
  auto place = [&](int id, int& tm, int& tn) {
    const int slice = id / (m * n);
    tile_of(id - slice * m * n, m, n, tm, tn);
    return slice;
  };
  every_tile<P>(
      t, smem, [&](int i) { return dealt(i, m * n * s.slices); },
      [&](int id) {
        int tm, tn;
        const int slice = place(id, tm, tn);
        const int k0 = (int)((int64_t)all * slice / s.slices), k1 = (int)((int64_t)all * (slice + 1) / s.slices);
        t.template start<P>(a.G, a.W, tm * T::BM, tn * T::BN, m * T::BM, a.direct ? a.d : dp, k0, k1 - k0, P == 3 ? kThreePairs : 0,
                            a.direct ? a.v1 - a.v0 : 1 << 30);
      },
      [](int, int) {},
      [&](int id, int) {
        int tm, tn;
        const int slice = place(id, tm, tn), lane = T::lane_now();
        const bool whole = a.last && s.slices == 1;
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
          const int at = tm * T::BM + T::row(i, lane);
          if (at >= count) continue;
          char* row = nullptr;
          int x = 0;
          if (whole) {
            const int r = a.kept.src[at], b = r / a.rows;
            row = a.grad_hidden + b * a.gh_seq + (r - b * a.rows) * a.gh_row;
            if constexpr (kScaled<FORM>) x = a.kept.exp[at] + e;
          }
#pragma unroll
          for (int j = 0; j < T::NT; ++j) {
            const int c = tn * T::BN + T::col(j, lane);
            if (c >= dp) continue;
            f4* to = (f4*)(a.dh + slice * a.dh_slice + (int64_t)at * dp + c);
            f4 sum = t.acc[i][j];
            if (a.add) sum += *to;
            if (whole) {
              float g[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) g[k] = !kScaled<FORM> ? sum[k] : __builtin_amdgcn_ldexpf(sum[k], x);
              store4<DT>(row, c, a.d, g);
            } else {
              *to = sum;
            }
          }
        }
      });
}

// Rounded once.
template <int FORM, class T>
EPIC_DEV void grad_head_tiles(const HeadArgs& a, T& t, const Split& s, int count, int e, int first_tiles, char* smem) {
  constexpr int P = kPairs<FORM>, DT = kDtype<FORM>;
  const int m = s.m_w, n = s.n_w, grid = (int)gridDim.x, heavy = first_tiles % grid;
  // of the grid's workgroups, the first `heavy` have one tile more behind them:
  // the others take `lead` tiles each, then all in turn
  const int light = heavy ? grid - heavy : 0, lead = min(s.lead, light ? m * n / light : 0), base = light * lead;
  const int mine = (int)blockIdx.x - heavy;
  auto number = [&](int i) {
    int id;
    if (light && mine >= 0 && i < lead)
      id = mine + i * light;
    else
      id = base + (int)blockIdx.x + (i - (light && mine >= 0 ? lead : 0)) * grid;
    return id < m * n ? id : -1;
  };
  every_tile<P>(
      t, smem, number,
      [&](int id) {
        int tm, tn;
        tile_of(id, m, n, tm, tn);
        t.template start<P>(a.G, a.H2, tm * T::BM, tn * T::BN, m * T::BM, a.width, 0, ceil_div(count, 64), P == 3 ? kThreePairs : 0);
      },
      [](int, int) {},
      [&](int id, int) {
        int tm, tn;
        tile_of(id, m, n, tm, tn);
        const int lane = T::lane_now();
#pragma unroll
        for (int i = 0; i < T::MT; ++i) {
          const int v = a.v0 + tm * T::BM + T::row(i, lane);
          if (v >= a.v1) continue;
          char* row = a.grad_head + v * a.grad_row;
#pragma unroll
          for (int j = 0; j < T::NT; ++j) {
            int c = tn * T::BN + T::col(j, lane);
            if (c >= a.width - 64 && a.shift) {
              if (c - a.shift < a.width - 64) continue;  // zeros
              c -= a.shift;
            }
            float g[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) g[k] = !kScaled<FORM> ? t.acc[i][j][k] : __builtin_amdgcn_ldexpf(t.acc[i][j][k], e);
            store4<DT>(row, c, a.d, g);
          }
        }
      });
}

template <int FORM>
__global__ void __launch_bounds__(kProductThreads) grad_kernel(HeadArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[kProductLds];
  __shared__ float lds_top[kProductThreads / 64];
  constexpr int KIND = kKind<FORM>;
  const int count = *a.kept.count;
  const Split s = split_of<kKind<FORM>>(a, count);
  int e_h = 0, e_w = 0;  // what takes the scales out of the sums
  if constexpr (FORM == kFormF16) e_h = -14, e_w = a.kept.count[1] - 14;
  if constexpr (FORM == kFormSplit) {
    e_h = -14 - head_exp<FORM>(a, lds_top);
    e_w = a.kept.count[1] - 15 - 14;  // rows are scaled to 2^15, by the largest of what they bring
  }
  int first_tiles = 0;
  if (a.grad_hidden) {
    first_tiles = s.m_h * s.n_h * s.slices;
    with_size<Sizes<KIND, true, false>>(s.size_h, [&](auto& t) { grad_hidden_tiles<FORM>(a, t, s, count, e_h, smem); });
  }
  lds_barrier();  // the last tile's numbers are read
  if (a.grad_head)
    with_size<Sizes<KIND, false, false>>(s.size_w, [&](auto& t) { grad_head_tiles<FORM>(a, t, s, count, e_w, first_tiles, smem); });
}

// Slices of the hidden states' gradient to its rows, one wavefront a row.
template <int FORM>
__global__ void __launch_bounds__(256) scatter_kernel(HeadArgs a) {
  constexpr int DT = kDtype<FORM>;
  __shared__ float lds[4];
  const int slices = split_of<kKind<FORM>>(a, *a.kept.count).slices;
  if (slices == 1) return;  // written already
  int e_head = 0;
  if constexpr (FORM == kFormSplit) e_head = -head_exp<FORM>(a, lds);
  const int at = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  if (at >= *a.kept.count) return;
  const int r = a.kept.src[at], b = r / a.rows;
  char* row = a.grad_hidden + b * a.gh_seq + (r - b * a.rows) * a.gh_row;
  const int dp = a.width;
  const int e = !kScaled<FORM> ? 0 : a.kept.exp[at] - 14 + e_head;
  for (int t = lane * 8; t < a.d; t += 512) {
    float x[8] = {};
    for (int s = 0; s < slices; ++s) {
      const f4* p = (const f4*)(a.dh + s * a.dh_slice + (int64_t)at * dp + t);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] += p[k >> 2][k & 3];
    }
    if constexpr (kScaled<FORM>) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = __builtin_amdgcn_ldexpf(x[k], e);
    }
    put8<DT>(row, t, a.d, x);
  }
}

// ---- Both gradients of few float32 rows, on the vector units: G, hidden states
// and head as they are.  Every wavefront works by itself on 256 columns.  Bound by
// memory for some 16 rows (of 32768 tokens, width 2048: 145 us for 537 MB, a copy 110),
// by the vector units for more.
constexpr int kFewRows = 128, kFewCols = 256;

// 16 rows' gradient over the `per` tokens of a slice.
EPIC_DEV void few_hidden(const HeadArgs& a, int count, int id, int per, float* g, int lane) {
  const int chunks = ceil_div(a.d, kFewCols), c = id % chunks * kFewCols + lane * 4;
  // (the groups that there are one after another: every XCD has some)
  const int slices = ceil_div(a.V, per), slice = id / chunks % slices, group = id / chunks / slices;
  if (group * 16 >= count) return;
  const int j0 = slice * per, j1 = min(a.V, j0 + per), c_in = min(c, a.d - 4);
  const char* w_at = a.W.data + 4 * (int64_t)c_in;
  constexpr int N = 8;  // loads ahead
  f4 sum[16] = {}, w[N];
  if (j0 < j1) {
#pragma unroll
    for (int u = 0; u < N; ++u) w[u] = *(const f4*)(w_at + min(j0 + u, j1 - 1) * a.W.stride);
  }
  for (int t0 = j0; t0 < j1; t0 += 64) {
    const int n = min(64, j1 - t0);
    wait_lds();
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // 16 rows of 64 tokens
      const int r = k * 4 + (lane >> 4), t = (lane & 15) * 4;
      const f4 x = *(const f4*)(a.G.data + (group * 16 + r) * a.G.stride + 4 * (int64_t)(t0 + t));
#pragma unroll
      for (int e = 0; e < 4; ++e) g[(t + e) * 16 + r] = t + e < n ? x[e] : 0.f;
    }
    wait_lds();
    for (int t = 0; t < n; t += N) {
      f4 next[N];
#pragma unroll
      for (int u = 0; u < N; ++u) next[u] = *(const f4*)(w_at + min(t0 + t + N + u, j1 - 1) * a.W.stride);
      __builtin_amdgcn_sched_barrier(0);  // the loads first
      // (past the last token g is 0, and w the last token's)
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[r] += g[(t + u) * 16 + r] * w[u];
#pragma unroll
      for (int u = 0; u < N; ++u) w[u] = next[u];
    }
  }
  if (c >= a.d) return;  // (d is a multiple of 64)
#pragma unroll
  for (int r = 0; r < 16; ++r) *(f4*)(a.dh + slice * a.dh_slice + (int64_t)(group * 16 + r) * a.width + c) = sum[r];
}

// TOKENS tokens' gradient over all rows.
template <int TOKENS>
EPIC_DEV void few_head(const HeadArgs& a, int count, int id, float* g, int lane) {
  const int chunks = ceil_div(a.d, kFewCols), c = id % chunks * kFewCols + lane * 4, t0 = id / chunks * TOKENS;
  if (t0 >= a.V) return;
  const char* h_at = a.H.data + 4 * (int64_t)min(c, a.d - 4);
  constexpr int N = 8;  // rows ahead
  f4 sum[TOKENS] = {};
  for (int r1 = 0; r1 < count; r1 += 32) {
    wait_lds();
#pragma unroll
    for (int k = 0; k < TOKENS / 8; ++k) {  // 32 rows of so many tokens
      const int r = k * (256 / TOKENS) + lane / (TOKENS / 4), t = lane % (TOKENS / 4) * 4;
      const f4 x = *(const f4*)(a.G.data + min(r1 + r, count - 1) * a.G.stride + 4 * (int64_t)(t0 + t));
      *(f4*)(g + r * TOKENS + t) = r1 + r < count ? x : f4{};
    }
    wait_lds();
    for (int r0 = r1; r0 < min(count, r1 + 32); r0 += N) {  // (past the last row g is 0)
      f4 h[N];
#pragma unroll
      for (int u = 0; u < N; ++u) h[u] = *(const f4*)(h_at + min(r0 + u, count - 1) * a.H.stride);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sum[t] += g[(r0 - r1 + u) * TOKENS + t] * h[u];
    }
  }
  if (c >= a.d) return;
#pragma unroll
  for (int t = 0; t < TOKENS; ++t)
    if (t0 + t < a.V)
      *(Loose16*)(a.grad_head + (t0 + t) * a.grad_row + 4 * (int64_t)c) =
          Loose16{{__float_as_uint(sum[t][0]), __float_as_uint(sum[t][1]), __float_as_uint(sum[t][2]), __float_as_uint(sum[t][3])}};
}

// The first `hidden` wavefronts the one, the others the other.
template <int TOKENS>
__global__ void __launch_bounds__(256) few_kernel(HeadArgs a, int hidden, int per) {
  __shared__ __attribute__((aligned(16))) float g[4][1024];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  const int count = *a.kept.count, id = (int)blockIdx.x * 4 + wave;
  if (id < hidden)
    few_hidden(a, count, id, per, g[wave], lane);
  else if (a.grad_head)
    few_head<TOKENS>(a, count, id - hidden, g[wave], lane);
}

// The slices' sum to the hidden states' gradient: 256 columns of a row a
// workgroup, a fourth of the slices each wavefront.
__global__ void __launch_bounds__(256) few_sum_kernel(HeadArgs a, int slices) {
  __shared__ f4 part[4][64];
  const int chunks = ceil_div(a.d, 256), at = (int)blockIdx.x / chunks, lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int c = (int)blockIdx.x % chunks * 256 + lane * 4;
  if (at >= *a.kept.count) return;
  f4 sum = {};
  if (c < a.d) {
    const float* p = a.dh + (int64_t)at * a.width + c;
    for (int s0 = wave; s0 < slices; s0 += 32) {
      f4 x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = *(const f4*)(p + min(s0 + 4 * u, slices - 1) * a.dh_slice);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (s0 + 4 * u < slices) sum += x[u];
    }
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || c >= a.d) return;
  sum = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
  const int r = a.kept.src[at], b = r / a.rows;
  const float x[4] = {sum[0], sum[1], sum[2], sum[3]};
  store4<EPIC_F32>(a.grad_hidden + b * a.gh_seq + (r - b * a.rows) * a.gh_row, c, a.d, x);
}

// Logits of a head in 8 bits: sums of whole numbers, exact in 32 bits, times the
// row's and the token's scale.  2867 rows of 32768 tokens, width 4096, to bfloat16: 329
// us, 2.34 POP/s; one row of width 2048 13 us, bound by reading the head at 5.1 TB/s;
// 160 rows of 100003 tokens, width 1000, to float32: 58 us for 165 MB, bound by 391
// tiles on 256 CUs.
template <int DT, class T>
EPIC_DEV void logits_tiles(const HeadArgs& a, T& t, int count, char* smem, int64_t (&rows)[2][256], float (&row_scale)[2][256],
                           float (&col_scale)[2][256]) {
  const int m = ceil_div(count, T::BM), n = ceil_div(a.V, T::BN);
  auto place = [&](int id, int& tm, int& tn) { tile_of(id, m, n, tm, tn); };
  every_tile<1>(
      t, smem, [&](int i) { return dealt(i, m * n); },
      [&](int id) {
        int tm, tn;
        place(id, tm, tn);
        t.template start<1>(a.H, a.W, tm * T::BM, tn * T::BN, m * T::BM, a.V, 0, a.steps, 0);
      },
      [&](int id, int k) {
        int tm, tn;
        place(id, tm, tn);
        for (int r = T::wave() * 64 + T::lane_now(); r < T::BM; r += T::kThreads) {
          const int at = tm * T::BM + r;
          const int x = at < count ? a.kept.src[at] : 0, b = x / a.rows;
          rows[k][r] = at < count ? b * a.seq_stride + (x - b * a.rows) * a.row_stride : -1;
          row_scale[k][r] = at < count ? a.row_scale[at] : 0.f;
        }
        for (int r = T::wave() * 64 + T::lane_now(); r < T::BN; r += T::kThreads)
          col_scale[k][r] = tn * T::BN + r < a.V ? a.col_scale[tn * T::BN + r] : 0.f;
      },
      [&](int id, int k) {
        int tm, tn;
        place(id, tm, tn);
        const int lane = T::lane_now();
#pragma unroll
        for (int j = 0; j < T::NT; j += T::F) {
          float sc[4 * T::F];
#pragma unroll
          for (int f = 0; f < 4 * T::F; ++f) sc[f] = col_scale[k][T::col(j, lane) + f];
          const int c = tn * T::BN + T::col(j, lane);
#pragma unroll
          for (int i = 0; i < T::MT; ++i) {
            const int64_t at = rows[k][T::row(i, lane)];
            const float s = row_scale[k][T::row(i, lane)];
            if (at < 0) continue;
#pragma unroll
            for (int h = 0; h < 4 * T::F; h += 8) {
              float x[8];
#pragma unroll
              for (int f = 0; f < 8; ++f) {
                x[f] = (float)t.acc[i][j + (h + f) / 4][f & 3] * s * sc[h + f];
                // a float32 number before it is rounded to float16: the compiler would join the two
                if constexpr (DT == EPIC_F16) asm volatile("" : "+v"(x[f]));
              }
              put8<DT>(a.logits + at, c + h, a.V, x);
            }
          }
        }
      });
}
template <int DT>
__global__ void __launch_bounds__(kProductThreads) logits_kernel(HeadArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[kProductLds];
  __shared__ int64_t rows[2][256];
  __shared__ float row_scale[2][256], col_scale[2][256];
  const int count = *a.kept.count;
  with_size<Sizes<kI8, true, true>>(tile_size<kI8>(count, a.V), [&](auto& t) { logits_tiles<DT>(a, t, count, smem, rows, row_scale, col_scale); });
}

// ------------------------------------------------------------ host side
constexpr int64_t kMaxRows = 1 << 24;
constexpr int kMaxWidth = 65536;
constexpr int kTopParts = 2048;  // workgroups that look for largest magnitudes, of hidden states and of the head, at most

inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Workgroups that take one tile after another: one a CU.
template <class K>
void launch_product(K kernel, const HeadArgs& a, int64_t tiles, hipStream_t stream) {
  if (tiles > 0)
    hipLaunchKernelGGL(kernel, dim3((int)std::min<int64_t>(tiles, kCus)), dim3(kProductThreads), 0, stream, a);
}
// The smallest tiles of m x n sums.
inline int64_t most_tiles(int64_t m, int64_t n) { return (m + 63) / 64 * ((n + 127) / 128); }

// Where what a call keeps lies in its workspace.
struct Layout {
  int64_t rows, padded;  // rows of the window, and up to a multiple of 256
  int64_t width;         // of packed rows, in numbers
  int form;              // of the products
  bool direct;           // the head is read where it is
  int64_t piece;         // tokens of a piece
  int max_slices;        // of a piece's tokens, in the hidden states' gradient
  int64_t parts;
  int64_t counts, count, src, target, lse, mul, exp, scale, row_exp, tops, at_target, part, H, H2, W, G, dh, bytes;
};

// The products read a head in its place when its rows are vectors of 16 bytes.
bool head_direct(const epic_rows_desc* head) {
  const int per = 16 / elem_size(head->dtype);
  return head->vocab % 8 == 0 && head->vocab >= 64 && head->row_stride % per == 0 && head->row_stride < (1 << 20) &&
         ((uintptr_t)head->data & 15) == 0;
}

// Few float32 rows are multiplied as they are: finding the head's largest magnitude
// and writing it out in two parts takes longer than slower products.  Losses and
// gradients in us, so and in two parts: 32768 tokens of width 2048, 64 rows 82 + 412
// and 241 + 434, 128 rows 151 + 701 and 249 + 489.  Which is better near the bound goes
// by the width too, by a few us: 128 rows over heads of 2^18, 2^19, 2^20 and 2^21
// numbers of width 128 54, 55, 66, 78 and 61, 66, 76, 101 in all, of width 512 77, 80, 81,
// 91 and 60, 69, 75, 84 (64 rows of width 2048, 2^19 numbers: 169 and 103).
bool as_it_is(const epic_rows_desc* hidden, const epic_rows_desc* head) {
  const int64_t rows = (int64_t)hidden->batch * hidden->rows, size = (int64_t)head->rows * head->vocab;
  return hidden->dtype == EPIC_F32 && head_direct(head) && head->vocab % 64 == 0 && (rows <= 64 || (rows <= kFewRows && size <= 1 << 19));
}

Layout layout_of(const epic_rows_desc* hidden, const epic_rows_desc* head, bool backward) {
  Layout l{};
  const int64_t V = head->rows;
  l.rows = (int64_t)hidden->batch * hidden->rows;
  l.padded = up(l.rows, 256);
  l.width = up(hidden->vocab, 64);
  l.form = as_it_is(hidden, head) ? kFormF32 : hidden->dtype == EPIC_F32 ? kFormSplit : hidden->dtype == EPIC_F16 ? kFormF16 : kFormBf16;
  l.direct = l.form != kFormSplit && head_direct(head);
  const int planes = l.form == kFormSplit ? 2 : 1, es = l.form == kFormF32 ? 4 : 2;
  l.piece = up(V, 256);
  if (backward || !l.direct) {
    // 256 MiB of G (half of it: 2867 rows of 32768 tokens, width 2048, both passes
    // 1.39 ms, with this 1.32) and of the head, but not less than fills the CUs
    const int64_t wide = std::max<int64_t>(l.direct ? 0 : l.width, backward ? l.padded : 0);
    const int64_t most = std::max<int64_t>(4096, (1 << 27) / std::max<int64_t>(1, wide * planes) / 256 * 256);
    const int64_t pieces = (V + most - 1) / most;
    l.piece = up((V + pieces - 1) / pieces, 256);
  }
  l.parts = up(V, 128) / 128;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t p = at;
    at += up(bytes, 256);
    return p;
  };
  // slices of the hidden states' gradient: 128 MiB of them, or one
  l.max_slices = l.piece < 2048 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(16, (1 << 25) / std::max<int64_t>(1, l.padded * l.width)));
  if (l.form == kFormF32)  // wavefronts for every CU, of at least 16 tokens
    l.max_slices = (int)std::max<int64_t>(1, std::min<int64_t>((V + 15) / 16, 2048 / ((l.rows + 15) / 16 * ((l.width + kFewCols - 1) / kFewCols) + 1)));
  l.counts = take((l.padded + 63) / 64 * 8);
  l.count = take(8);
  l.src = take(4 * l.padded);
  l.target = take(4 * l.padded);
  l.lse = take(4 * l.padded);
  l.mul = take(4 * l.padded);
  l.exp = take(4 * l.padded);
  l.scale = take(4 * l.padded);
  l.row_exp = take(4 * l.padded);
  l.tops = take(4 * kTopParts);
  l.at_target = take(4 * l.padded);
  const int64_t whole = es * planes * l.width;  // bytes of a packed row in all its planes
  l.H = take(l.padded * whole);
  if (!l.direct) l.W = take(l.piece * whole);
  if (!backward) {
    l.part = take(8 * l.padded * l.parts);
  } else {
    l.H2 = l.form == kFormF16 || l.form == kFormSplit ? take(l.padded * whole) : l.H;
    l.G = take(es * planes * l.padded * l.piece);
    l.dh = take(4 * (l.form == kFormF32 ? l.max_slices * kFewRows : l.max_slices * l.padded) * l.width);
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

struct Call {
  const epic_rows_desc *hidden, *head;
  Layout l;
  GatherArgs g;
  HeadArgs a;
  hipStream_t stream;
};

template <int FORM>
PackArgs pack_args(const Call& c, int v0) {
  return {(const char*)c.head->data, c.head->row_stride * kSize<kDtype<FORM>>, c.head->rows, c.head->vocab, v0,
          (int)up(std::min<int64_t>(c.head->rows - v0, c.l.piece), 64), const_cast<char*>(c.a.W.data), c.a.W.stride, c.a.W.plane,
          (int)c.l.width, c.a.tops, c.a.top_parts};
}
inline int pack_groups(const PackArgs& p) { return std::min(2048, (p.count + 3) / 4); }

template <int FORM, int MODE>
void gather(Call& c) {
  c.g.per = (int)std::max<int64_t>(4, up((c.l.rows + 4095) / 4096, 4));
  const int groups = (int)std::max<int64_t>(1, (c.l.rows + c.g.per - 1) / c.g.per);
  PackArgs p{};
  int more = 0;
  if constexpr (FORM == kFormSplit && MODE != kQuantize) {
    const int row_groups = (int)std::min<int64_t>(kTopParts, (c.l.rows + 3) / 4);
    TopArgs t{c.g, (const char*)c.head->data, c.head->row_stride * 4, const_cast<float*>(c.a.tops), row_groups};
    hipLaunchKernelGGL(top_kernel, dim3(row_groups + c.a.top_parts), dim3(256), 0, c.stream, t);
  }
  if (c.l.rows <= 1024)
    c.g.counts = nullptr;
  else
    hipLaunchKernelGGL(count_kernel, dim3((int)((c.l.rows + 255) / 256)), dim3(256), 0, c.stream, c.g);
  if constexpr (kPacks<FORM> && MODE != kQuantize) {
    if (!c.l.direct) {
      p = pack_args<FORM>(c, 0);
      more = pack_groups(p);
    }
  }
  hipLaunchKernelGGL((gather_kernel<FORM, MODE>), dim3(groups + more), dim3(kGather), 0, c.stream, c.g, p, groups);
}

// The head's piece from token v0 on.
template <int FORM>
void piece(Call& c, int v0) {
  c.a.v0 = v0;
  c.a.v1 = (int)std::min<int64_t>(c.a.V, v0 + c.l.piece);
  c.a.last = c.a.v1 == c.a.V;
  c.a.add = v0 > 0;
  if (c.l.direct) {
    c.a.W.data = (const char*)c.head->data + v0 * c.a.W.stride;
  } else if constexpr (kPacks<FORM>) {
    if (v0 > 0) {
      const PackArgs p = pack_args<FORM>(c, v0);
      hipLaunchKernelGGL(pack_kernel<FORM>, dim3(pack_groups(p)), dim3(256), 0, c.stream, p);
    }
  }
}

// What both passes set up: operands, rows that count, the head's pieces.
template <int FORM>
void set_up(Call& c, char* ws) {
  const Layout& l = c.l;
  Kept kept{(int32_t*)(ws + l.count), (int32_t*)(ws + l.src), (int32_t*)(ws + l.target), (float*)(ws + l.lse), (float*)(ws + l.mul),
            (int32_t*)(ws + l.exp), (int32_t*)(ws + l.scale)};
  constexpr int64_t es = kPacked<FORM>;
  const int64_t stride = es * l.width, plane = l.padded * stride;
  c.g.kept = c.a.kept = kept;
  c.g.counts = (int2*)(ws + l.counts);
  c.g.out = ws + l.H;
  c.g.stride = stride;
  c.g.plane = plane;
  c.g.out2 = ws + l.H2;
  c.g.row_exp = FORM == kFormSplit ? (int32_t*)(ws + l.row_exp) : nullptr;
  c.a.tops = (float*)(ws + l.tops);
  c.a.top_parts = std::min(kTopParts, (c.head->rows + 3) / 4);
  c.a.H = {ws + l.H, stride, plane};
  c.a.H2 = {ws + l.H2, stride, plane};
  if (l.direct)
    c.a.W = {(const char*)c.head->data, c.head->row_stride * es, 0};
  else
    c.a.W = {ws + l.W, stride, l.piece * stride};
  c.a.G = {ws + l.G, es * l.piece, es * l.padded * l.piece};
  c.a.steps = (int)(stride / 128);
  c.a.V = c.head->rows;
  c.a.d = c.head->vocab;
  c.a.at_target = (float*)(ws + l.at_target);
  c.a.part = (float2*)(ws + l.part);
  c.a.dh = (float*)(ws + l.dh);
  c.a.dh_slice = l.padded * l.width;
  c.a.max_slices = l.max_slices;
  c.a.piece = (int)l.piece;
  c.a.width = c.g.width = (int)l.width;
  c.a.shift = c.g.shift = l.direct ? (int)(l.width - c.head->vocab) : 0;
  c.a.direct = l.direct;
  c.a.parts = l.parts;
  c.a.rows = c.hidden->rows;
}

template <int FORM>
void losses(Call& c, char* ws, float* loss, float* lse) {
  set_up<FORM>(c, ws);
  gather<FORM, kForward>(c);
  for (int64_t v0 = 0; v0 < c.a.V; v0 += c.l.piece) {
    piece<FORM>(c, (int)v0);
    launch_product(lse_kernel<FORM>, c.a, most_tiles(c.l.rows, c.a.v1 - c.a.v0), c.stream);
  }
  hipLaunchKernelGGL(loss_kernel<FORM>, dim3((int)((c.l.rows + 3) / 4)), dim3(256), 0, c.stream, c.a, loss, lse);
}

template <int FORM>
void gradients(Call& c, char* ws, const epic_rows_desc* gh, const epic_rows_desc* gw) {
  set_up<FORM>(c, ws);
  if (gh && c.l.rows > 0) {
    c.a.grad_hidden = (char*)gh->data;
    c.a.gh_seq = gh->seq_stride * kSize<kDtype<FORM>>;
    c.a.gh_row = gh->row_stride * kSize<kDtype<FORM>>;
  }
  if (gw) {
    c.a.grad_head = (char*)gw->data;
    c.a.grad_row = gw->row_stride * kSize<kDtype<FORM>>;
  }
  gather<FORM, kBackward>(c);
  const int d = c.a.d;
  if constexpr (FORM == kFormF32) {  // of so few rows G is one piece
    piece<FORM>(c, 0);
    launch_product(excess_kernel<FORM>, c.a, most_tiles(c.l.rows, c.a.V), c.stream);
    const int chunks = (d + kFewCols - 1) / kFewCols, per = (int)up((c.a.V + c.l.max_slices - 1) / c.l.max_slices, 16),
              slices = (c.a.V + per - 1) / per;
    c.a.dh_slice = kFewRows * c.l.width;
    const int waves = c.a.grad_hidden ? chunks * (kFewRows / 16) * slices : 0;
    // 32 tokens a wavefront take the least from LDS and the rows; of small heads 8, for
    // more wavefronts (64 rows, 512 tokens, width 128: 9 us, with 32 31)
    const bool wide = (int64_t)chunks * c.a.V >= 32 * 1024;
    const int tokens = wide ? 32 : 8, more = gw ? chunks * ((c.a.V + tokens - 1) / tokens) : 0;
    hipLaunchKernelGGL(wide ? few_kernel<32> : few_kernel<8>, dim3((waves + more + 3) / 4), dim3(256), 0, c.stream, c.a, waves, per);
    if (waves)
      hipLaunchKernelGGL(few_sum_kernel, dim3((int)c.l.rows * ((d + 255) / 256)), dim3(256), 0, c.stream, c.a, slices);
  } else {
    for (int64_t v0 = 0; v0 < c.a.V; v0 += c.l.piece) {
      piece<FORM>(c, (int)v0);
      const int count = c.a.v1 - c.a.v0;
      launch_product(excess_kernel<FORM>, c.a, most_tiles(c.l.rows, count), c.stream);
      launch_product(grad_kernel<FORM>, c.a, (gh ? most_tiles(c.l.rows, d) * c.a.max_slices : 0) + (gw ? most_tiles(count, d) : 0), c.stream);
    }
    if (c.a.grad_hidden && c.a.max_slices > 1)
      hipLaunchKernelGGL(scatter_kernel<FORM>, dim3((int)((c.l.rows + 3) / 4)), dim3(256), 0, c.stream, c.a);
  }
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
#define EPIC_HEAD(FORM) backward ? gradients<FORM>(c, ws, grad_hidden, grad_head) : losses<FORM>(c, ws, d_loss, d_lse)
  switch (l.form) {
    case kFormF32: EPIC_HEAD(kFormF32); break;
    case kFormSplit: EPIC_HEAD(kFormSplit); break;
    case kFormF16: EPIC_HEAD(kFormF16); break;
    default: EPIC_HEAD(kFormBf16);
  }
#undef EPIC_HEAD
  return hipGetLastError() == hipSuccess ? EPIC_OK : EPIC_ERR_HIP;
}

template <int DT>
void run_quantize(const epic_rows_desc* x, int8_t* q, int64_t stride, float* scale, hipStream_t stream) {
  const int total = x->batch * x->rows;
  hipLaunchKernelGGL(quantize_kernel<DT>, dim3(std::min(4096, (total + 3) / 4)), dim3(256), 0, stream, (const char*)x->data,
                     x->seq_stride * kSize<DT>, x->row_stride * kSize<DT>, x->rows, total, x->vocab, q, stride, scale);
}

struct LogitsLayout {
  int64_t rows, padded, stride, counts, count, src, scale, H, bytes;
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
  l.counts = l.H + l.padded * l.stride;
  l.bytes = l.counts + up((l.padded + 63) / 64 * 8, 256);
  return l;
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
  c.g.kept = {(int32_t*)(ws + l.count), (int32_t*)(ws + l.src), nullptr, nullptr, nullptr, nullptr, nullptr};
  c.g.out = ws + l.H;
  c.g.stride = l.stride;
  c.g.scale = (float*)(ws + l.scale);
  c.g.counts = (int2*)(ws + l.counts);
  switch (hidden->dtype) {
    case EPIC_F32: gather<kFormF32, kQuantize>(c); break;
    case EPIC_F16: gather<kFormF16, kQuantize>(c); break;
    default: gather<kFormBf16, kQuantize>(c); break;
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
  const int64_t tiles = most_tiles(l.rows, a.V);
  switch (logits->dtype) {
    case EPIC_F32: launch_product(logits_kernel<EPIC_F32>, a, tiles, stream); break;
    case EPIC_F16: launch_product(logits_kernel<EPIC_F16>, a, tiles, stream); break;
    default: launch_product(logits_kernel<EPIC_BF16>, a, tiles, stream); break;
  }
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
