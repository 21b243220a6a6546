// Paged cache operators for gfx950: token rows into pages of 16-bit or MXFP4 values with
// the position rotation applied on the way, the way back, and attention over the pages.
#include "paged.h"

#include <hip/hip_ext.h>

#include <algorithm>

#include "dev.h"

namespace mbp {
using namespace dev;
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename Kern, typename... Args>
hipError_t plaunch(Kern kernel, dim3 grid, dim3 block, hipStream_t st, hipEvent_t e0, hipEvent_t e1, Args... args) {
  if (e0 != nullptr || e1 != nullptr) hipExtLaunchKernelGGL(kernel, grid, block, 0, st, e0, e1, 0, args...);
  else hipLaunchKernelGGL(kernel, grid, block, 0, st, args...);
  return hipGetLastError();
}

// ---------------------------------------------------------- rows and elements ----
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

__device__ __forceinline__ float lo_bf16(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ float lo_f16(uint32_t u) { return (float)__builtin_bit_cast(f16x2, u)[0]; }
__device__ __forceinline__ float hi_f16(uint32_t u) { return (float)__builtin_bit_cast(f16x2, u)[1]; }

// Elements [at, at + 8) of rows of type t as they lie in memory (16-bit types: in u[0]),
// and their values: apart, so that several can be in flight.
struct Raw8 {
  uint4 u[2];
};
__device__ __forceinline__ void load_raw8(const void* p, int64_t at, int t, int vec, Raw8& r) {
  if (vec) {
    const char* c = reinterpret_cast<const char*>(p) + at * (t == PT_F32 ? 4 : 2);
    r.u[0] = *reinterpret_cast<const uint4*>(c);
    if (t == PT_F32) r.u[1] = *reinterpret_cast<const uint4*>(c + 16);
    return;
  }
  uint32_t w[8];
  if (t == PT_F32) {
    const uint32_t* f = reinterpret_cast<const uint32_t*>(p) + at;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = f[i];
    r.u[1] = make_uint4(w[4], w[5], w[6], w[7]);
  } else {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + at;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)h[2 * i] | (uint32_t)h[2 * i + 1] << 16;
  }
  r.u[0] = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void values8(const Raw8& r, int t, float (&x)[8]) {
  const uint32_t w[8] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w, r.u[1].x, r.u[1].y, r.u[1].z, r.u[1].w};
  if (t == PT_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = t == PT_BF16 ? lo_bf16(w[i]) : lo_f16(w[i]);
    x[2 * i + 1] = t == PT_BF16 ? hi_bf16(w[i]) : hi_f16(w[i]);
  }
}
__device__ __forceinline__ void load8(const void* p, int64_t at, int t, int vec, float (&x)[8]) {
  Raw8 r;
  load_raw8(p, at, t, vec, r);
  values8(r, t, x);
}

template <int N>
__device__ __forceinline__ void store_n(void* p, int64_t at, int t, int vec, const float (&x)[N]) {
  if (t == PT_F32) {
    float* f = reinterpret_cast<float*>(p) + at;
    if (vec && N % 4 == 0) {
#pragma unroll
      for (int i = 0; i + 3 < N; i += 4) *reinterpret_cast<float4*>(f + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = x[i];
    }
    return;
  }
  uint16_t* h = reinterpret_cast<uint16_t*>(p) + at;
  uint32_t u[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) u[i] = t == PT_BF16 ? pack_bf16(x[2 * i], x[2 * i + 1]) : pack_f16(x[2 * i], x[2 * i + 1]);
  if (vec && N % 8 == 0) {
#pragma unroll
    for (int i = 0; i + 3 < N / 2; i += 4) *reinterpret_cast<uint4*>(h + 2 * i) = make_uint4(u[i], u[i + 1], u[i + 2], u[i + 3]);
  } else if (vec && N % 4 == 0) {
#pragma unroll
    for (int i = 0; i + 1 < N / 2; i += 2) *reinterpret_cast<uint2*>(h + 2 * i) = make_uint2(u[i], u[i + 1]);
  } else if (vec) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) *reinterpret_cast<uint32_t*>(h + 2 * i) = u[i];
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      h[2 * i] = (uint16_t)u[i];
      h[2 * i + 1] = (uint16_t)(u[i] >> 16);
    }
  }
}

// The rows of sequence s, whatever row_start holds: [row0, row0 + n) within [0, n_rows).
struct SeqRows {
  int32_t row0, n, slot0;
};
__device__ __forceinline__ SeqRows seq_rows(const PagedRows& r, int s) {
  const int32_t a = min(max(r.row_start[s], 0), r.n_rows), b = min(max(r.row_start[s + 1], a), r.n_rows);
  return {a, b - a, r.first_slot[s]};
}

// The sequence that begins last at or before a row (which may lie behind its end), its
// rows and the slot of the first; s = -1: none does.
struct RowSeq {
  int32_t s, start, end, slot0;
};

// Of a row that all lanes of the wave agree on.  A wave looks through 64 sequences at a
// time, and their starts, ends and slots are loaded together: one load's latency, where a
// binary search would have one for each step.
__device__ __forceinline__ RowSeq seq_of(const PagedRows& r, int n_seqs, int row) {
  const int lane = threadIdx.x & 63;
  RowSeq f = {-1, 0, 0, 0};
  for (int at = 0; at < n_seqs; at += 64) {
    const int i = min(at + lane, n_seqs - 1);
    const int32_t start = r.row_start[i], end = r.row_start[i + 1], slot0 = r.first_slot[i];
    const int n = (int)__popcll(__ballot(at + lane < n_seqs && start <= row));
    if (n > 0) {
      f.s = at + n - 1;
      f.start = __builtin_amdgcn_readlane(start, n - 1);
      f.end = __builtin_amdgcn_readlane(end, n - 1);
      f.slot0 = __builtin_amdgcn_readlane(slot0, n - 1);
    }
  }
  return f;
}

// On to the sequence of a later row.
__device__ __forceinline__ void advance(const PagedRows& r, int n_seqs, int row, RowSeq* f) {
  while (row >= f->end && f->s + 1 < n_seqs && r.row_start[f->s + 1] <= row) {
    ++f->s;
    f->start = r.row_start[f->s];
    f->end = r.row_start[f->s + 1];
    f->slot0 = r.first_slot[f->s];
  }
}

// The slot of a row, -1 for one of no sequence.
__device__ __forceinline__ int32_t slot_of(const RowSeq& f, int row) {
  if (f.s < 0 || row < f.start || row >= f.end) return -1;
  return (int32_t)min(max((int64_t)f.slot0 + (row - max(f.start, 0)), (int64_t)-1), (int64_t)INT32_MAX);
}

// A wave's part of a call on token rows: 64 units of 8 channels each of the heads of one
// kind (queries, keys or values), in `rows` rows one after the other.  What belongs to a
// row (its sequence, slot, page, position) is then the same in all lanes and costs scalar
// instructions, what belongs to a lane (its head and channel) stays from row to row, and
// the slots that a wave writes lie side by side.
struct Tasks {
  int32_t first[3], chunks;  // chunks of 64 units before each kind, and of all
  int32_t per_shift;         // log2 of the units of a head
  int32_t rows;
};
struct Lane {
  int32_t which, h, c0, row0;
  bool live;
};
__device__ __forceinline__ Lane lane_of(const Tasks& tk, int heads0, int heads) {
  const int id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int group = id / tk.chunks, chunk = id - group * tk.chunks;
  Lane l;
  l.which = chunk < tk.first[1] ? 0 : chunk < tk.first[2] ? 1 : 2;
  const int unit = (chunk - tk.first[l.which]) * 64 + ((int)threadIdx.x & 63);
  l.h = unit >> tk.per_shift;
  l.c0 = (unit & ((1 << tk.per_shift) - 1)) * 8;
  l.live = l.h < (l.which == 0 ? heads0 : heads);
  l.row0 = group * tk.rows;
  return l;
}

// Byte offset of slot 0 of a page of head h, or -1 where the slot has no page.
__device__ __forceinline__ int64_t page_of(const PagedCache& c, int s, int32_t slot, int h) {
  if (slot < 0 || (slot >> c.shift) >= c.max_pages) return -1;
  const int32_t id = c.pages[(int64_t)s * c.max_pages + (slot >> c.shift)];
  if ((uint32_t)id >= (uint32_t)c.n_pages) return -1;
  return ((int64_t)id * c.hk + h) * c.page_bytes;
}

// Largest of four neighbouring lanes' values.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kDppXor2, 0xF, 0xF, false));
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kDppXor1, 0xF, 0xF, false));
}

// Scale exponent e of a block of 32 values from the largest biased exponent among them:
// floor(log2 amax) - 2, which puts amax into [4, 8) steps of the largest e2m1 binade.
// Returns 255 for a block with a NaN or an infinity.
__device__ __forceinline__ int scale_byte(int exponent, int special) {
  return exponent >= special ? 255 : min(max(exponent - special / 2 - 2, -127), 127) + 127;
}

// Codes of 8 values y (already divided by the scale), nearest-even, saturated at 6.
__device__ __forceinline__ uint32_t codes8(const float (&y)[8]) {
  uint32_t u = 0;
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[0], y[1], 1.0f, 0);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[2], y[3], 1.0f, 1);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[4], y[5], 1.0f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[6], y[7], 1.0f, 3);
}

// 8 codes of one scale block as bfloat16.
__device__ __forceinline__ u32x4 decode8(uint32_t u, uint32_t scale_byte) {
  const float sc = __uint_as_float(scale_byte << 23);
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, sc, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, sc, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, sc, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, sc, 3));
  return r;
}

// d as float32 whose last bit says whether something was cut off (round to odd): rounding
// that again to fewer bits gives what rounding d would give.
__device__ __forceinline__ float round_odd(double d) {
  const float f = (float)d;
  uint32_t u = __float_as_uint(f);
  const double back = (double)f;
  if (back != d) {
    if (fabs(back) > fabs(d)) u -= 1;
    u |= 1;
  }
  return __uint_as_float(u);
}

// ------------------------------------------------------------------- append ----
// Every value is read once and written once, so the copy rate bounds it (4.7 TB/s for a
// large copy): 4.6 to 5.4 TB/s with float32 rows, 4.1 from 16-bit rows into MXFP4.  The
// rotation is three operations a channel.  One row at a time: with two or four rows' loads
// in flight the code of the rows' cases, that many times unrolled, was slower (8 prompts
// of 32 + 2 x 8 heads of 128 bfloat16 channels into MXFP4: 127, 141 and 175 us).
template <int CT>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppend a, Tasks tk) {
  const Lane l = lane_of(tk, a.H, a.c.hk);
  const int dh = a.c.dh;
  if (l.row0 >= a.r.n_rows) return;
  const HeadRows src = l.which == 0 ? a.q : l.which == 1 ? a.k : a.v;
  const bool turn = l.which < 2 && a.rope != nullptr;
  const int64_t at_src = (int64_t)l.h * src.head + l.c0, at_out = (int64_t)l.h * a.qo.head + l.c0;
  const int64_t head = (int64_t)l.h * a.c.page_bytes;
  char* const pool = l.which == 1 ? a.c.k : a.c.v;
  const int es = src.type == PT_F32 ? 4 : 2;
  const int last = min(l.row0 + tk.rows, a.r.n_rows);
  // a row's values are loaded before its place is known, the next row's during this one
  Raw8 ahead;
  auto fetch = [&](int row) {
    if (l.live) load_raw8(reinterpret_cast<const char*>(src.p) + (int64_t)row * src.row * es, at_src, src.type, src.vec, ahead);
  };
  fetch(l.row0);
  RowSeq f = seq_of(a.r, a.c.n_seqs, l.row0);
  for (int row = l.row0; row < last; ++row) {
    const Raw8 raw = ahead;
    if (row + 1 < last) fetch(row + 1);
    advance(a.r, a.c.n_seqs, row, &f);
    if (f.s < 0 || row < f.start || row >= f.end) continue;
    const int32_t slot = slot_of(f, row);
    int32_t pos = slot, id = -1;
    if (a.rope != nullptr) {
      if (a.pos != nullptr) pos = a.pos[row];
      if ((uint32_t)pos >= (uint32_t)a.n_pos) continue;
    }
    if (l.which > 0) {
      if (slot >= 0 && (slot >> a.c.shift) < a.c.max_pages) id = a.c.pages[(int64_t)f.s * a.c.max_pages + (slot >> a.c.shift)];
      if ((uint32_t)id >= (uint32_t)a.c.n_pages) continue;
    }
    if (!l.live) continue;
    float4 cs[2];
    if (turn) {
      const float4* t = reinterpret_cast<const float4*>(a.rope + (int64_t)pos * (dh / 2)) + l.c0 / 4;
      cs[0] = t[0];
      cs[1] = t[1];
    }
    float x[8];
    values8(raw, src.type, x);
    if ((l.which == 0 || CT != PT_MXFP4) && turn) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float c = i & 1 ? cs[i >> 1].z : cs[i >> 1].x, sn = i & 1 ? cs[i >> 1].w : cs[i >> 1].y;
        const float r0 = x[2 * i] * c - x[2 * i + 1] * sn, r1 = x[2 * i] * sn + x[2 * i + 1] * c;
        x[2 * i] = r0;
        x[2 * i + 1] = r1;
      }
    }
    if (l.which == 0) {
      store_n(reinterpret_cast<char*>(a.qo.p) + (int64_t)row * a.qo.row * es, at_out, a.qo.type, a.qo.vec, x);
      continue;
    }
    char* page = pool + (int64_t)id * a.c.hk * a.c.page_bytes + head;
    const int at = slot & ((1 << a.c.shift) - 1);
    if constexpr (CT != PT_MXFP4) {
      if constexpr (CT == PT_F16) {  // finite values beyond the type's largest are held as that
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fabsf(x[i]) < INFINITY ? fminf(fmaxf(x[i], -65504.f), 65504.f) : x[i];
      }
      store_n(page, at * dh + l.c0, CT, 1, x);
    } else {
      // A value beside the middle of two codes has to go to the right one, and so has the
      // largest value beside a power of two: keys are rotated in float64, where the products
      // are exact, and reach the conversion through a float32 that is rounded to odd.
      float y[8];
      int byte;
      if (turn) {
        double d[8];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const double c = i & 1 ? cs[i >> 1].z : cs[i >> 1].x, sn = i & 1 ? cs[i >> 1].w : cs[i >> 1].y;
          d[2 * i] = (double)x[2 * i] * c - (double)x[2 * i + 1] * sn;
          d[2 * i + 1] = (double)x[2 * i] * sn + (double)x[2 * i + 1] * c;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, (uint32_t)(__builtin_bit_cast(uint64_t, d[i]) >> 32) & 0x7fffffffu);
        byte = scale_byte((int)(quad_max(top) >> 20), 2047);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = round_odd(ldexp(d[i], 127 - byte));
      } else {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
        byte = scale_byte((int)(quad_max(top) >> 23), 255);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = ldexpf(x[i], 127 - byte);
      }
      const uint32_t u = byte == 255 ? 0u : codes8(y);
      *reinterpret_cast<uint32_t*>(page + (at * dh + l.c0) / 2) = u;
      if ((l.c0 & 31) == 0) page[(dh / 2 << a.c.shift) + at * (dh >> 5) + (l.c0 >> 5)] = (char)byte;
    }
  }
}

// --------------------------------------------------------------------- read ----
template <int CT, int U>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedCache c, PagedRows r, HeadRows ko, HeadRows vo, Tasks tk) {
  const Lane l = lane_of(tk, 0, c.hk);
  const int dh = c.dh;
  if (l.row0 >= r.n_rows) return;
  RowSeq f = seq_of(r, c.n_seqs, l.row0);
  const HeadRows dst = l.which == 1 ? ko : vo;
  const char* const pool = l.which == 1 ? c.k : c.v;
  const int64_t at_dst = (int64_t)l.h * dst.head + l.c0, head = (int64_t)l.h * c.page_bytes;
  const int es = dst.type == PT_F32 ? 4 : 2;
  const int last = min(l.row0 + tk.rows, r.n_rows);
  u32x4 raw[U];
  uint32_t byte[U];
  auto fetch = [&](int row, int j) {
    raw[j] = u32x4{0, 0, 0, 0};
    byte[j] = 127;
    if (row >= last) return;
    advance(r, c.n_seqs, row, &f);
    const int32_t slot = slot_of(f, row);
    if (slot < 0 || (slot >> c.shift) >= c.max_pages) return;
    const int32_t id = c.pages[(int64_t)f.s * c.max_pages + (slot >> c.shift)];
    if ((uint32_t)id >= (uint32_t)c.n_pages || !l.live) return;
    const char* page = pool + (int64_t)id * c.hk * c.page_bytes + head;
    const int at = slot & ((1 << c.shift) - 1);
    if constexpr (CT != PT_MXFP4) {
      raw[j] = *reinterpret_cast<const u32x4*>(page + (at * dh + l.c0) * 2);
    } else {
      raw[j][0] = *reinterpret_cast<const uint32_t*>(page + (at * dh + l.c0) / 2);
      byte[j] = (uint8_t)page[(dh / 2 << c.shift) + at * (dh >> 5) + (l.c0 >> 5)];
    }
  };
  for (int row = l.row0; row < last; row += U) {
#pragma unroll
    for (int j = 0; j < U; ++j) fetch(row + j, j);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (row + j >= last || !l.live) continue;
      u32x4 u = raw[j];
      if constexpr (CT == PT_MXFP4) u = decode8(raw[j][0], byte[j]);
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = CT == PT_F16 ? lo_f16(u[i]) : lo_bf16(u[i]);
        x[2 * i + 1] = CT == PT_F16 ? hi_f16(u[i]) : hi_bf16(u[i]);
      }
      if (CT != PT_F16 && dst.type == PT_F16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fabsf(x[i]) < INFINITY ? fminf(fmaxf(x[i], -65504.f), 65504.f) : x[i];
      }
      store_n(reinterpret_cast<char*>(dst.p) + (int64_t)(row + j) * dst.row * es, at_dst, dst.type, dst.vec, x);
    }
  }
}

// ------------------------------------------------------------------- attend ----
// Products run on 16-bit matrix instructions with float32 sums: float16 for a float16
// cache, bfloat16 for the others (an e2m1 code times a power of two is a bfloat16 value).
// Queries and probabilities enter as one to three terms of that type, so that what they
// lose stays below the rounding of the output: kQ query terms, kP probability terms.
template <int CT, int QT>
struct Terms {
  static constexpr bool same = QT == CT || (CT == PT_MXFP4 && QT == PT_BF16);
  // float32 queries: float16 pairs hold 22 bits of a row scaled to its largest value,
  // bfloat16 triples 24; float16 queries over MXFP4 are exact as bfloat16 pairs
  static constexpr int kQ = same ? 1 : CT == PT_F16 || QT == PT_F16 ? 2 : 3;
  // probabilities: one term has half a step of the output's own type, float16 pairs 2^-22;
  // in bfloat16, a pair (2^-16) for float16 outputs and a triple (2^-24) for float32 ones
  static constexpr int kP = same ? 1 : CT == PT_F16 || QT == PT_F16 ? 2 : 3;
};

template <int CT>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
  if constexpr (CT == PT_F16) return pack_f16(a, b);
  else return pack_bf16(a, b);
}
template <int CT>
__device__ __forceinline__ float lo_of(uint32_t u) {
  if constexpr (CT == PT_F16) return lo_f16(u);
  else return lo_bf16(u);
}
template <int CT>
__device__ __forceinline__ float hi_of(uint32_t u) {
  if constexpr (CT == PT_F16) return hi_f16(u);
  else return hi_bf16(u);
}

// The exponent that brings a row whose largest magnitude is top into float16 as x 2^-e; its
// scores then count 2^e times as much, in a factor kept within float32's normal numbers
// (beyond them scores either differ by far too much or by nothing).  From 2^113 on the row
// rather fills float16.
__device__ __forceinline__ int fit16(float top) {
  return min(max((int)(__float_as_uint(top) >> 23) - 127, -126), 113);
}

// 8 values, times a power of two, as N terms of the product's type, each the rounded rest of
// the ones before.
template <int CT, int N>
__device__ __forceinline__ void split8(const float (&x)[8], u32x4 (&t)[N], float gain = 1.f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i] * gain, b = x[2 * i + 1] * gain;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint32_t u = pack_pair<CT>(a, b);
      t[n][i] = u;
      if (n + 1 < N) {
        a -= lo_of<CT>(u);
        b -= hi_of<CT>(u);
      }
    }
  }
}

template <int CT>
__device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (CT == PT_F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int CT>
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (CT == PT_F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The 4 x 16 tile of 16-bit values that the 16 lanes of a quarter wave point at (lane i:
// four values of row i / 4) turned round: lane i receives the four rows' values of
// column i.
__device__ __forceinline__ uint2 read_turned(const uint16_t* p) {
  return __builtin_bit_cast(
      uint2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(uintptr_t)lds_addr(p)));
}

// One element of a cache row.
template <int CT, int DH>
__device__ __forceinline__ float cache_at(const char* page, int shift, int at, int c) {
  if constexpr (CT == PT_BF16) return bf2f(reinterpret_cast<const uint16_t*>(page)[at * DH + c]);
  if constexpr (CT == PT_F16) return (float)reinterpret_cast<const _Float16*>(page)[at * DH + c];
  const uint32_t u = (uint8_t)page[(at * DH + c) / 2];
  const uint32_t s = (uint8_t)page[(DH / 2 << shift) + at * (DH / 32) + c / 32];
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, __uint_as_float(s << 23), 0);
  return c & 1 ? hi_bf16(__builtin_bit_cast(uint32_t, b)) : lo_bf16(__builtin_bit_cast(uint32_t, b));
}

// Largest and smallest over 16 neighbouring lanes (a row of the vector ALU).
template <int CTRL>
__device__ __forceinline__ int dpp_int(int x) {
  return __builtin_amdgcn_mov_dpp(x, CTRL, 0xF, 0xF, false);
}
__device__ __forceinline__ int min16(int x) {
  x = min(x, dpp_int<kDppXor1>(x));
  x = min(x, dpp_int<kDppXor2>(x));
  x = min(x, dpp_int<kDppMirror7>(x));
  return min(x, dpp_int<kDppMirror15>(x));
}
__device__ __forceinline__ int max16(int x) {
  x = max(x, dpp_int<kDppXor1>(x));
  x = max(x, dpp_int<kDppXor2>(x));
  x = max(x, dpp_int<kDppMirror7>(x));
  return max(x, dpp_int<kDppMirror15>(x));
}

// The value sums of N channels from c0 on, one visible slot after the other.  A matrix
// product adds 0 times the value of a slot that its row must not see, which is NaN when
// that value is an infinity or NaN; a row whose sum of probabilities is finite and whose
// output is not is summed again this way.  Never taken for finite caches.
template <int CT, int DH, int N>
__device__ __forceinline__ void sum_values(const PagedAttend& a, int s, int kvh, int row, int head, int lo, int hi, float m,
                                           float f, int c0, float (&o)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = 0.f;
#pragma unroll 1
  for (int slot = lo; slot < hi; ++slot) {
    const int64_t page = page_of(a.c, s, slot, kvh);
    if (page < 0) continue;
    const int at = slot & ((1 << a.c.shift) - 1);
    float dot = 0.f;
#pragma unroll 1
    for (int c = 0; c < DH; c += 8) {
      float q[8];
      load8(a.q.p, (int64_t)row * a.q.row + (int64_t)head * a.q.head + c, a.q.type, a.q.vec, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot += q[i] * cache_at<CT, DH>(a.c.k + page, a.c.shift, at, c + i);
    }
    const float p = __builtin_amdgcn_exp2f(dot * f - m);
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] += p * cache_at<CT, DH>(a.c.v + page, a.c.shift, at, c0 + i);
  }
}

// Slots [lo, hi) that row tok of its sequence sees; lo = cap, hi = 0 for none.
__device__ __forceinline__ void row_range(const PagedAttend& a, const SeqRows& sr, int tok, int cap, int* lo, int* hi) {
  const int row = sr.row0 + tok;
  *lo = a.lo != nullptr ? max(a.lo[row], 0) : 0;
  *hi = (int)min(a.hi != nullptr ? (int64_t)a.hi[row] : (int64_t)sr.slot0 + tok + 1, (int64_t)cap);
  if (*lo >= *hi) {
    *lo = cap;
    *hi = 0;
  }
}

struct Grid {  // of an attention launch: x is split fastest, then tile; y the KV head; z the sequence
  int32_t S, chunk, tiles, G;
};

// Probabilities are 2^(f s - f m) with a reference m that need not be the largest score:
// it follows once one is more than 2^kSlack times as probable, so that the sums are
// rescaled a few times in a row's life instead of at every block.  Float16 terms, and the
// value sums until the end, are kGain times larger: at most 2^15, within the type, whose
// smallest step is then 2^-31 of a probability of 1 (without it a million slots of 2^-25
// each, a thirtieth of the sum, would be left out).
constexpr float kSlack = 8.f;
constexpr float kFar = 1048576.f;  // f m whose rounding, 2^-4, is no more than its scores' own
template <int CT>
constexpr float kGain = CT == PT_F16 ? 128.f : 1.f;

// Where a row's channels go: the output, or this split's sums, at place `place` (its
// sequence's place times max_rows, plus the row's in that: known without a load).
template <int N>
__device__ __forceinline__ void put_out(const PagedAttend& a, int S, int split, int64_t place, int row, int head, int dh, int c0,
                                        float m, float l, float (&o)[N]) {
  if (S == 1) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = l == 0.f ? 0.f : o[i] * inv;
    store_n(a.o.p, (int64_t)row * a.o.row + (int64_t)head * a.o.head + c0, a.o.type, a.o.vec, o);
    return;
  }
  const int64_t rows = (int64_t)a.c.n_seqs * a.r.max_rows, i = ((int64_t)split * rows + place) * a.H + head, all = S * rows * a.H;
  store_n(a.work, i * dh + c0, PT_F32, 1, o);
  if (c0 == 0) reinterpret_cast<float2*>(a.work + all * dh)[i] = make_float2(m, l);
}

// Waves per SIMD that a step kernel's registers leave room for without spills.
constexpr int step_waves(int ct, int dh, int qt) {
  if (dh < 128) return 4;
  return ct != PT_MXFP4 || qt == PT_F32 ? 2 : qt == PT_BF16 ? 4 : 3;
}

// Up to 16 query rows of one sequence and KV head (its rows times the query heads of the
// group, row-major) against the slots of one split.  Four waves take blocks of KT slots in
// turn and join their softmax states at the end.  Computed transposed, so that lane l
// owns query l % 16 (16x16x32 products; lane l supplies row or column l % 16 and the 8
// positions 8 (l / 16).. of the contracted dimension, and receives rows 4 (l / 16).. of
// column l % 16):
//   S^T = K Q^T: keys come straight from the pages into the operand registers, a lane
//     holding DH / 4 consecutive channels of its key (the contraction may run over the
//     channels in any order, so the queries are held in the same one);
//   O^T += V^T P^T: the probabilities are already where the product wants them, values
//     go through the wave's own LDS tile and are read turned round.
// The next block's loads are in flight during a block's softmax and value product.
// Bound by the cache's stream: 5.4 TB/s over 64 float16 sequences of 1024 to 2048 slots, 5.8
// over 16 bfloat16 ones of 8192 (a large copy: 4.7); over MXFP4 by the instructions of
// decoding and softmax, 3.5 TB/s with float32 rows of d = 64, 4.9 with bfloat16 rows of d = 128.
template <int CT, int DH, int QT>
__global__ __launch_bounds__(256, step_waves(CT, DH, QT)) void paged_step_kernel(PagedAttend a, Grid gr) {
  using T = Terms<CT, QT>;
  constexpr bool F4 = CT == PT_MXFP4;
  constexpr int KT = DH == 32 ? 64 : 32;
  constexpr int NB = KT / 16, KS = DH / 32, CB = DH / 16;
  constexpr int PITCH = DH + 16;  // half a wave reads 32 bytes of 8 slots turned round: 8 x 32 bytes in different banks
  // values are loaded 16 slots or fewer at a time, so that a load's page is the same in all
  // lanes: VB bytes a lane, PER lanes a slot, VU loads a block
  constexpr int ROW = F4 ? DH / 2 : DH * 2, VB = ROW >= 64 ? 16 : ROW / 4, PER = ROW / VB, ROWS = 64 / PER, VU = KT / ROWS;
  static_assert(ROWS <= 16 && VB >= 4, "pieces");
  constexpr int TILE = KT * PITCH * 2, MERGE = 16 * (DH + 4) * 4;
  __shared__ __attribute__((aligned(16))) char lds[4 * (TILE > MERGE ? TILE : MERGE)];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int tile = gr.tiles == 1 ? 0 : blockIdx.x / gr.S, split = blockIdx.x - tile * gr.S, kvh = blockIdx.y, s = blockIdx.z;
  const int G = gr.G;
  const int cap = a.c.max_pages << a.c.shift;
  const int32_t* const ids = a.c.pages + (int64_t)s * a.c.max_pages;
  // The ids of a block's pages are fetched one block before its keys, so that no load waits
  // for the load of its address.
  // (a vector load, lane i the page of the block's 16-slot part i: scalar loads return out
  // of order, so that every wait for LDS would wait for them too.)
  int32_t ahead;
  auto fetch_ids = [&](int t) { ahead = ids[min((t + 16 * (lane & (NB - 1))) >> a.c.shift, a.c.max_pages - 1)]; };
  // without lower ends the split's first slots are known at once, and their pages' ids are
  // loaded beside the sequence's rows
  fetch_ids(a.lo == nullptr ? (int)min((int64_t)split * gr.chunk, (int64_t)cap) + wave * KT : 0);
  const SeqRows sr = seq_rows(a.r, s);
  const int nq = min(sr.n, a.r.max_rows) * G;
  if (tile * 16 >= nq) return;
  const int qi = tile * 16 + col, tok = G == 1 ? min(qi, nq - 1) : min(qi, nq - 1) / G,
            head = kvh * G + min(qi, nq - 1) - tok * G, row = sr.row0 + tok;
  float x[KS][8];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    load8(a.q.p, (int64_t)row * a.q.row + (int64_t)head * a.q.head + g * (DH / 4) + ks * 8, QT, a.q.vec, x[ks]);
  int lo = cap, hi = 0;
  if (qi < nq) row_range(a, sr, tok, cap, &lo, &hi);
  const int kmin = a.lo == nullptr ? 0 : __builtin_amdgcn_readfirstlane(min16(lo)), kmax = __builtin_amdgcn_readfirstlane(max16(hi));
  const int lo_all = __builtin_amdgcn_readfirstlane(max16(hi > 0 ? lo : 0)), hi_all = __builtin_amdgcn_readfirstlane(min16(hi > 0 ? hi : cap));
  const int64_t b0 = (int64_t)(kmin & ~(KT - 1)) + (int64_t)split * gr.chunk;
  const int begin = __builtin_amdgcn_readfirstlane((int)min(b0, (int64_t)cap));
  const int end = __builtin_amdgcn_readfirstlane(split == gr.S - 1 ? kmax : (int)min((int64_t)kmax, b0 + gr.chunk));

  f32x4 o[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) o[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  uint16_t* const vt = reinterpret_cast<uint16_t*>(lds + wave * TILE);
  constexpr int step = 4 * KT;
  u32x4 kr[NB][F4 ? 1 : KS], vr[VU];
  uint32_t ksc[NB], vsc[VU];
  const uint32_t in_page = (1u << a.c.shift) - 1;
  const uint32_t sc_off = DH / 2 << a.c.shift;
  // bytes of a page of all heads, and where this head's begin: both below 2^32
  const uint32_t stride = (uint32_t)(a.c.hk * a.c.page_bytes), head_at = (uint32_t)(kvh * a.c.page_bytes);
  const uint32_t k_off = col * ROW + g * (ROW / 4), ks_off = col * (DH / 32) + g * DH / 128;
  const uint32_t v_key = lane / PER, v_off = v_key * ROW + (lane % PER) * VB, vs_off = v_key * (DH / 32) + (lane % PER) * VB / 16;
  uint32_t valid = 0;  // of the block whose keys are in the registers: a bit for each 16 slots
  // Loads of the block at slot t.  16 slots never cross a page; slots at and behind kmax
  // are read from their page where there is one (any content is masked) and from page 0
  // where not.
  auto load = [&](int t) {
    uint64_t pg[NB];
    // parts behind kmax or without a page: page 0, and masked
    const bool there = t + 16 * lane < kmax && (uint32_t)ahead < (uint32_t)a.c.n_pages;
    valid = (uint32_t)__ballot(there) & ((1u << NB) - 1);
    const int32_t id = there ? ahead : 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) pg[b] = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(id, b) * stride + head_at;
    fetch_ids(t + step);
    // a scalar base and a lane's own offset, which stays from block to block
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const uint32_t at = (uint32_t)(t + 16 * b) & in_page;
      const char* kp = a.c.k + (pg[b] + at * ROW);
      if constexpr (F4) {
        if constexpr (DH == 128) {
          kr[b][0] = *reinterpret_cast<const u32x4*>(kp + k_off);
        } else if constexpr (DH == 64) {
          const uint2 u = *reinterpret_cast<const uint2*>(kp + k_off);
          kr[b][0][0] = u.x;
          kr[b][0][1] = u.y;
        } else {
          kr[b][0][0] = *reinterpret_cast<const uint32_t*>(kp + k_off);
        }
        ksc[b] = *reinterpret_cast<const uint8_t*>(a.c.k + (pg[b] + sc_off + at * (DH / 32)) + ks_off);
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kr[b][ks] = *reinterpret_cast<const u32x4*>(kp + (k_off + ks * 16));
      }
    }
#pragma unroll
    for (int u = 0; u < VU; ++u) {
      const uint32_t at = (uint32_t)(t + u * ROWS) & in_page;
      const uint64_t page = pg[u * ROWS / 16];
      const char* vp = a.c.v + (page + at * ROW);
      if constexpr (VB == 16) {
        vr[u] = *reinterpret_cast<const u32x4*>(vp + v_off);
      } else if constexpr (VB == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(vp + v_off);
        vr[u][0] = x.x;
        vr[u][1] = x.y;
      } else {
        vr[u][0] = *reinterpret_cast<const uint32_t*>(vp + v_off);
      }
      if constexpr (F4) vsc[u] = *reinterpret_cast<const uint8_t*>(a.c.v + (page + sc_off + at * (DH / 32)) + vs_off);
    }
  };
  int t = begin + wave * KT;
  if (a.lo != nullptr) fetch_ids(t);
  if (t < end) load(t);
  // queries: channels g DH / 4 + 8 ks .. +7 of row col in step ks
  float f = a.scale * 1.44269504f;
  float sign = f < 0.f ? -1.f : f == 0.f ? 0.f : 1.f;
  f = f == 0.f ? 1.f : fabsf(f);
  u32x4 q[KS][T::kQ];
  if constexpr (CT == PT_F16 && QT == PT_F32) {  // into the range of float16, by a power of two
    float top = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[ks][i]));
    top = across_max<16>(top);
    const int e = fit16(top);
    sign = ldexpf(sign, -e);
    f = fminf(fmaxf(ldexpf(f, e), 0x1p-126f), 0x1.fffffep127f);
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[ks][i] *= sign;
    split8<CT, T::kQ>(x[ks], q[ks]);
  }
  for (; t < end; t += step) {
    f32x4 sc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) sc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4 kf[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if constexpr (F4) kf[b] = decode8(kr[b][0][ks], ksc[b]);
        else kf[b] = kr[b][ks];
      }
#pragma unroll
      for (int n = 0; n < T::kQ; ++n)
#pragma unroll
        for (int b = 0; b < NB; ++b) sc[b] = mma16<CT>(kf[b], q[ks][n], sc[b]);
    }
    const uint32_t ok = valid;
    // blocks that every row sees whole need no mask
    const bool inner = t >= lo_all && t + KT <= hi_all && ok == (1u << NB) - 1;
    if (!inner) {  // values of slots that no row may see: zeros
      asm volatile("" ::: "memory");  // a branch, not selects in every block
#pragma unroll
      for (int u = 0; u < VU; ++u) {
        const int key = u * ROWS + (int)v_key;
        if (!(t + key >= kmin && t + key < kmax && ((ok >> (key >> 4)) & 1))) {
          vr[u] = u32x4{0, 0, 0, 0};
          vsc[u] = 127;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < VU; ++u) {
      uint16_t* d = vt + (u * ROWS + v_key) * PITCH + (lane % PER) * (DH / PER);
      if constexpr (F4) {
#pragma unroll
        for (int i = 0; i < VB / 4; ++i) reinterpret_cast<u32x4*>(d)[i] = decode8(vr[u][i], vsc[u]);
      } else {
        *reinterpret_cast<u32x4*>(d) = vr[u];
      }
    }
    if (t + step < end) load(t + step);
    if (!inner) {
      asm volatile("" ::: "memory");
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int slot = t + 16 * b + 4 * g + r;
          sc[b][r] = slot >= lo && slot < hi && ((ok >> b) & 1) ? sc[b][r] : -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[b][r]);
    mx = across_max<16>(mx);
    if (__any((mx - m) * f > kSlack || m == -INFINITY)) {
      const float mn = fmaxf(m, mx);
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * f);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) o[cb] *= alpha;
    }
    float ref = m == -INFINITY ? 0.f : m * f;
    if (__any(fabsf(ref) > kFar)) {  // the product's rounding would be taken for a score
      asm volatile("" ::: "memory");
      const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[b][r] -= off;
      ref = 0.f;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sc[b][r] = __builtin_amdgcn_exp2f(fmaf(sc[b][r], f, -ref));
        l += sc[b][r];
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int b = 0; b < NB; b += 2) {
      const float y[8] = {sc[b][0], sc[b][1], sc[b][2], sc[b][3], sc[b + 1][0], sc[b + 1][1], sc[b + 1][2], sc[b + 1][3]};
      u32x4 p[T::kP];
      split8<CT, T::kP>(y, p, kGain<CT>);
      const uint16_t* src = vt + (16 * b + 4 * g + (col >> 2)) * PITCH + (col & 3) * 4;
      u32x4 vf[CB];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const uint2 v0 = read_turned(src + cb * 16), v1 = read_turned(src + 16 * PITCH + cb * 16);
        vf[cb] = u32x4{v0.x, v0.y, v1.x, v1.y};
      }
#pragma unroll
      for (int n = 0; n < T::kP; ++n)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb] = mma16<CT>(vf[cb], p[n], o[cb]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  l = across_sum<16>(l);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) o[cb] *= 1 / kGain<CT>;
  if (hi == 0) {  // blocks that all other rows see whole were not masked for a row that sees none
    m = -INFINITY;
    l = 0.f;
  }
  // join the waves' states: [wave][query][max, sum, -, -, DH channels]
  __syncthreads();
  float* const mb = reinterpret_cast<float*>(lds);
  {
    float* w = mb + (wave * 16 + col) * (DH + 4);
    if (g == 0) {
      w[0] = m == -INFINITY ? m : m * f;  // in units of log 2
      w[1] = l;
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) *reinterpret_cast<float4*>(w + 4 + cb * 16 + g * 4) = make_float4(o[cb][0], o[cb][1], o[cb][2], o[cb][3]);
  }
  __syncthreads();
  // thread: query tid / 16, DH / 16 channels
  constexpr int N = DH / 16;
  const int qj = tid >> 4, c0 = (tid & 15) * N, q2 = tile * 16 + qj;
  if (q2 >= nq) return;
  float mj = -INFINITY, lj = 0.f, oj[N];
#pragma unroll
  for (int w = 0; w < 4; ++w) mj = fmaxf(mj, mb[(w * 16 + qj) * (DH + 4)]);
#pragma unroll
  for (int i = 0; i < N; ++i) oj[i] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float* p = mb + (w * 16 + qj) * (DH + 4);
    if (p[0] == -INFINITY && p[1] == 0.f) continue;  // saw nothing
    const float e = __builtin_amdgcn_exp2f(p[0] - mj);
    lj += p[1] * e;
#pragma unroll
    for (int i = 0; i < N; ++i) oj[i] += p[4 + c0 + i] * e;
  }
  const int tok2 = q2 / G, head2 = kvh * G + q2 - tok2 * G;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < N; ++i) odd |= !(fabsf(oj[i]) < INFINITY);
  if (odd && lj < INFINITY) {
    int lo2, hi2;
    row_range(a, sr, tok2, cap, &lo2, &hi2);
    sum_values<CT, DH>(a, s, kvh, sr.row0 + tok2, head2, max(lo2, begin), min(hi2, end), mj, a.scale * 1.44269504f, c0, oj);
  }
  put_out(a, gr.S, split, (int64_t)s * a.r.max_rows + tok2, sr.row0 + tok2, head2, DH, c0, mj, lj, oj);
}

// Many query rows: 128 per block (32 per wave, lane l owning query l % 32) against the
// slots of one split, 64 at a time.  The keys and values of the block's 64 slots lie in
// LDS for all four waves, the next 64 are loaded during the products.  32x32x16 products
// (lane l supplies row or column l % 32 and the 8 positions 8 (l / 32).. of the
// contracted dimension, and receives rows 8 (r / 4) + 4 (l / 32) + r % 4 of column l % 32);
// everything transposed and the values read turned round, as for few rows.  The matrix cores
// and the softmax's vector instructions share the time: causal prompts of 4 x 4096 rows and
// 32 heads over 8 run at 833 TFLOP/s (d = 128, bfloat16), 901 (MXFP4) and 768 (d = 64), where
// a library product reaches 1235.
template <int CT, int DH, int QT>
__global__ __launch_bounds__(256, 2) void paged_prompt_kernel(PagedAttend a, Grid gr) {
  using T = Terms<CT, QT>;
  constexpr bool F4 = CT == PT_MXFP4;
  // 64 slots a tile, 32 where two terms of 128 channels fill the registers
  constexpr int KT = DH == 128 && T::kQ > 1 ? 32 : 64, NB = KT / 32, NG = KT / 16, KS = DH / 16, CB = DH / 32;
  // distances of two slots in LDS: keys are read 16 bytes of 8 slots at a time; of values,
  // half a wave reads 64 bytes of 4 slots turned round: 64 bytes off a multiple of 256, they
  // lie in different banks
  constexpr int PITCH = DH + 8, VP = DH == 128 ? 160 : DH == 64 ? 96 : 32;
  // pieces of a tile: 16 bytes (16-bit types: 8 channels, codes: 16 channels of 8 bytes)
  constexpr int PER = F4 ? DH / 16 : DH / 8, PIECES = KT * PER, NP = PIECES < 256 ? 1 : PIECES / 256;
  // two tiles of keys and values; at the end each wave's outputs on their way to whole rows
  constexpr int CP = DH < 64 ? DH : 64, OUT = 32 * (CP + 4);  // channels at a time, floats of a wave
  constexpr int TILES = 2 * KT * (PITCH + VP) * 2;
  static_assert(4 * OUT * 4 <= TILES, "the outputs fit the tiles' place");
  __shared__ __attribute__((aligned(16))) char lds[TILES];
  uint16_t* const lds_k = reinterpret_cast<uint16_t*>(lds);
  uint16_t* const lds_v = lds_k + 2 * KT * PITCH;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
  // Blocks go to the 8 XCDs in turn.  With a multiple of 8 (sequence, KV head) pairs, a
  // pair's blocks all go to one, whose L2 then holds its keys and values (from four pairs
  // for each XCD on: with fewer, ragged sequences leave some XCDs without work).
  int bx = blockIdx.x, kvh = blockIdx.y, s = blockIdx.z;
  if (((gridDim.y * gridDim.z) & 7) == 0 && gridDim.y * gridDim.z >= 32) {
    const uint32_t id = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z), at = id >> 3, round = at / gridDim.x;
    const uint32_t pair = round * 8 + (id & 7);
    bx = (int)(at - round * gridDim.x);
    s = (int)(pair / gridDim.y);
    kvh = (int)(pair - s * gridDim.y);
  }
  // late rows see the most slots: they go first
  const int at_x = bx / gr.S, tile = gr.tiles - 1 - at_x, split = bx - at_x * gr.S;
  const int G = gr.G;
  const SeqRows sr = seq_rows(a.r, s);
  const int nq = min(sr.n, a.r.max_rows) * G;
  if (tile * 128 >= nq) return;
  const int cap = a.c.max_pages << a.c.shift;
  const int qi = tile * 128 + wave * 32 + col, tok = G == 1 ? min(qi, nq - 1) : min(qi, nq - 1) / G,
            head = kvh * G + min(qi, nq - 1) - tok * G, row = sr.row0 + tok;
  // the queries' loads go first; they are used once the first tile's are on their way
  Raw8 raw[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    load_raw8(a.q.p, (int64_t)row * a.q.row + (int64_t)head * a.q.head + ks * 16 + half * 8, QT, a.q.vec, raw[ks]);
  int lo = cap, hi = 0;
  if (qi < nq) row_range(a, sr, tok, cap, &lo, &hi);
  // the wave's extent: [wmin, wmax) holds every visible slot, all of [lo_all, hi_all) is
  // visible to every row that sees anything
  auto wide = [&](int x, bool largest) {
    x = largest ? max16(x) : min16(x);
    const int y = __shfl_xor(x, 16);
    return __builtin_amdgcn_readfirstlane(largest ? max(x, y) : min(x, y));
  };
  const int wmin = wide(lo, false), wmax = wide(hi, true);
  const int lo_all = wide(hi > 0 ? lo : 0, true), hi_all = wide(hi > 0 ? hi : cap, false);
  __shared__ int ext[4][2];
  if (lane == 0) {
    ext[wave][0] = wmin;
    ext[wave][1] = wmax;
  }
  __syncthreads();
  const int kmin = __builtin_amdgcn_readfirstlane(min(min(ext[0][0], ext[1][0]), min(ext[2][0], ext[3][0])));
  const int kmax = __builtin_amdgcn_readfirstlane(max(max(ext[0][1], ext[1][1]), max(ext[2][1], ext[3][1])));
  const int64_t b0 = (int64_t)(kmin & ~(KT - 1)) + (int64_t)split * gr.chunk;
  const int begin = __builtin_amdgcn_readfirstlane((int)min(b0, (int64_t)cap));
  const int end = __builtin_amdgcn_readfirstlane(split == gr.S - 1 ? kmax : (int)min((int64_t)kmax, b0 + gr.chunk));

  f32x16 o[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[cb][r] = 0.f;
  float m = -INFINITY, l = 0.f;

  const int32_t* const ids = a.c.pages + (int64_t)s * a.c.max_pages;
  const uint32_t in_page = (1u << a.c.shift) - 1;
  const uint32_t sc_off = DH / 2 << a.c.shift;
  const uint32_t stride = (uint32_t)(a.c.hk * a.c.page_bytes), head_at = (uint32_t)(kvh * a.c.page_bytes);
  u32x4 kr[NP], vr[NP];  // (codes: two words each)
  uint32_t ksc[NP], vsc[NP];
  // ids of the pages of a tile's 16-slot parts, in the first lanes, loaded a tile before they
  // are used
  int32_t ahead;
  auto fetch_ids = [&](int t) { ahead = ids[min((t + 16 * (lane & (NG - 1))) >> a.c.shift, a.c.max_pages - 1)]; };
  uint32_t valid = 0;  // parts with a page, of the tile in the registers
  auto load = [&](int t) {
    uint64_t pg[NG];
    const bool there = (uint32_t)ahead < (uint32_t)a.c.n_pages;
    valid = (uint32_t)__ballot(there) & ((1u << NG) - 1);
    const int32_t id = there ? ahead : 0;
#pragma unroll
    for (int b = 0; b < NG; ++b) pg[b] = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(id, b) * stride + head_at;
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      // a wave's 64 pieces lie within one part (or in two, for 32 channels of codes)
      const int i = min(u * 256 + tid, PIECES - 1), key = i / PER, piece = i % PER;
      uint64_t page = pg[min((u * 256 + wave * 64) / PER / 16, NG - 1)];
      if constexpr (PER < 4) page = (key >> 4) & 1 ? pg[min((u * 256 + wave * 64) / PER / 16 + 1, NG - 1)] : page;
      const uint32_t at = ((uint32_t)(t + (key & ~15)) & in_page) + (key & 15);
      if constexpr (F4) {
        const uint2 x = *reinterpret_cast<const uint2*>(a.c.k + page + (at * (DH / 2) + piece * 8));
        const uint2 y = *reinterpret_cast<const uint2*>(a.c.v + page + (at * (DH / 2) + piece * 8));
        kr[u][0] = x.x; kr[u][1] = x.y;
        vr[u][0] = y.x; vr[u][1] = y.y;
        ksc[u] = (uint8_t)a.c.k[page + (sc_off + at * (DH / 32) + piece / 2)];
        vsc[u] = (uint8_t)a.c.v[page + (sc_off + at * (DH / 32) + piece / 2)];
      } else {
        kr[u] = *reinterpret_cast<const u32x4*>(a.c.k + page + (at * (DH * 2) + piece * 16));
        vr[u] = *reinterpret_cast<const u32x4*>(a.c.v + page + (at * (DH * 2) + piece * 16));
      }
    }
    fetch_ids(t + KT);
  };
  // values of slots that no row of the block may see: zeros
  auto clean = [&](int t) {
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int key = min(u * 256 + tid, PIECES - 1) / PER;
      if (!(t + key >= kmin && t + key < kmax && ((valid >> (key >> 4)) & 1))) {
        vr[u] = u32x4{0, 0, 0, 0};
        vsc[u] = 127;
      }
    }
  };
  auto store = [&](int t, int buf) {
    if (t < kmin || t + KT > kmax || valid != (1u << NG) - 1) {
      asm volatile("" ::: "memory");
      clean(t);
    }
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int i = u * 256 + tid, key = i / PER, piece = i % PER;
      if (PIECES < 256 && i >= PIECES) continue;
      uint16_t* kd = lds_k + (buf * KT + key) * PITCH + piece * (DH / PER);
      uint16_t* vd = lds_v + (buf * KT + key) * VP + piece * (DH / PER);
      if constexpr (F4) {
        reinterpret_cast<u32x4*>(kd)[0] = decode8(kr[u][0], ksc[u]);
        reinterpret_cast<u32x4*>(kd)[1] = decode8(kr[u][1], ksc[u]);
        reinterpret_cast<u32x4*>(vd)[0] = decode8(vr[u][0], vsc[u]);
        reinterpret_cast<u32x4*>(vd)[1] = decode8(vr[u][1], vsc[u]);
      } else {
        *reinterpret_cast<u32x4*>(kd) = kr[u];
        *reinterpret_cast<u32x4*>(vd) = vr[u];
      }
    }
  };
  uint32_t ok = 0;
  fetch_ids(begin);
  if (begin < end) load(begin);
  float f = a.scale * 1.44269504f;
  float sign = f < 0.f ? -1.f : f == 0.f ? 0.f : 1.f;
  f = f == 0.f ? 1.f : fabsf(f);
  u32x4 q[KS][T::kQ];
  if constexpr (CT == PT_F16 && QT == PT_F32) {
    float top = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float x[8];
      values8(raw[ks], QT, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
    }
    top = pair_max<32>(top);
    const int e = fit16(top);
    sign = ldexpf(sign, -e);
    f = fminf(fmaxf(ldexpf(f, e), 0x1p-126f), 0x1.fffffep127f);
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    float x[8];
    values8(raw[ks], QT, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= sign;
    split8<CT, T::kQ>(x, q[ks]);
  }
  if (begin < end) {
    ok = valid;
    store(begin, 0);
  }
  int cur = 0;
  for (int t = begin; t < end; t += KT, cur ^= 1) {
    __syncthreads();  // the block's tile is complete, the other buffer is free
    const bool more = t + KT < end;
    if (more) load(t + KT);
    if (t < wmax && t + KT > wmin) {
      const uint16_t* kt = lds_k + cur * KT * PITCH;
      const uint16_t* vt = lds_v + cur * KT * VP;
      f32x16 sc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[b][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        u32x4 kf[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) kf[b] = *reinterpret_cast<const u32x4*>(kt + (32 * b + col) * PITCH + ks * 16 + half * 8);
#pragma unroll
        for (int n = 0; n < T::kQ; ++n)
#pragma unroll
          for (int b = 0; b < NB; ++b) sc[b] = mma32<CT>(kf[b], q[ks][n], sc[b]);
      }
      if (t < lo_all || t + KT > hi_all || ok != (1u << NG) - 1) {
        asm volatile("" ::: "memory");  // a branch, not selects in every tile
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int slot = t + 32 * b + 8 * (r >> 2) + 4 * half + (r & 3);
            sc[b][r] = slot >= lo && slot < hi && ((ok >> (2 * b + (r >> 3))) & 1) ? sc[b][r] : -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[b][r]);
      mx = pair_max<32>(mx);
      if (__any((mx - m) * f > kSlack || m == -INFINITY)) {
        const float mn = fmaxf(m, mx);
        const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * f);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb] *= alpha;
      }
      float ref = m == -INFINITY ? 0.f : m * f;
      if (__any(fabsf(ref) > kFar)) {  // the product's rounding would be taken for a score
        asm volatile("" ::: "memory");
        const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[b][r] -= off;
        ref = 0.f;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sc[b][r] = __builtin_amdgcn_exp2f(fmaf(sc[b][r], f, -ref));
          l += sc[b][r];
        }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          const float x[8] = {sc[b][8 * k2], sc[b][8 * k2 + 1], sc[b][8 * k2 + 2], sc[b][8 * k2 + 3],
                              sc[b][8 * k2 + 4], sc[b][8 * k2 + 5], sc[b][8 * k2 + 6], sc[b][8 * k2 + 7]};
          u32x4 p[T::kP];
          split8<CT, T::kP>(x, p, kGain<CT>);
          // lanes of a quarter wave: channels 16 (lane / 16 % 2) .., slots 4 half .. of the 8
          const uint16_t* src = vt + (32 * b + 16 * k2 + 4 * half + ((lane & 15) >> 2)) * VP + (lane & 16) + (lane & 3) * 4;
          u32x4 vf[CB];
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            const uint2 v0 = read_turned(src + cb * 32), v1 = read_turned(src + 8 * VP + cb * 32);
            vf[cb] = u32x4{v0.x, v0.y, v1.x, v1.y};
          }
#pragma unroll
          for (int n = 0; n < T::kP; ++n)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) o[cb] = mma32<CT>(vf[cb], p[n], o[cb]);
        }
    }
    ok = valid;
    if (more) store(t + KT, cur ^ 1);
  }
  l = pair_sum<32>(l);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) o[cb] *= 1 / kGain<CT>;
  if (hi == 0) {  // tiles that all other rows see whole were not masked for a row that sees none
    m = -INFINITY;
    l = 0.f;
  }
  m = m == -INFINITY ? m : m * f;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      float x[4] = {o[cb][4 * r4], o[cb][4 * r4 + 1], o[cb][4 * r4 + 2], o[cb][4 * r4 + 3]};
      const bool odd = !(fabsf(x[0]) < INFINITY && fabsf(x[1]) < INFINITY && fabsf(x[2]) < INFINITY && fabsf(x[3]) < INFINITY);
      if (odd && l < INFINITY) {
        sum_values<CT, DH>(a, s, kvh, row, head, max(lo, begin), min(hi, end), m, a.scale * 1.44269504f, 32 * cb + 8 * r4 + 4 * half, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[cb][4 * r4 + i] = x[i];
      }
    }
  // A lane holds 4 channels of its row here and there: through LDS they become whole rows,
  // of which 8 neighbouring channels are stored at a time.
  const int64_t place = ((int64_t)split * a.c.n_seqs + s) * a.r.max_rows, all = (int64_t)gr.S * a.c.n_seqs * a.r.max_rows * a.H;
  const float inv = l == 0.f ? 0.f : gr.S == 1 ? 1.0f / l : 1.0f;
  if (gr.S > 1 && half == 0 && qi < nq) reinterpret_cast<float2*>(a.work + all * DH)[(place + tok) * a.H + head] = make_float2(m, l);
  __syncthreads();  // the tiles are no longer read
  float* const ow = reinterpret_cast<float*>(lds) + wave * OUT;
#pragma unroll
  for (int c1 = 0; c1 < DH; c1 += CP) {
#pragma unroll
    for (int cb = c1 / 32; cb < (c1 + CP) / 32; ++cb)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (l != 0.f) x = make_float4(o[cb][4 * r4] * inv, o[cb][4 * r4 + 1] * inv, o[cb][4 * r4 + 2] * inv, o[cb][4 * r4 + 3] * inv);
        *reinterpret_cast<float4*>(ow + col * (CP + 4) + 32 * cb - c1 + 8 * r4 + 4 * half) = x;
      }
    __builtin_amdgcn_wave_barrier();
    constexpr int PR = CP / 8, RS = 64 / PR;  // lanes of a row, rows at a time
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += RS) {
      const int r = r0 + lane / PR, c = (lane % PR) * 8, tok2 = __shfl(tok, r), head2 = __shfl(head, r);
      const float4 x0 = *reinterpret_cast<const float4*>(ow + r * (CP + 4) + c), x1 = *reinterpret_cast<const float4*>(ow + r * (CP + 4) + c + 4);
      const float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
      if (tile * 128 + wave * 32 + r >= nq) continue;
      if (gr.S == 1) store_n(a.o.p, (int64_t)(sr.row0 + tok2) * a.o.row + (int64_t)head2 * a.o.head + c1 + c, QT, a.o.vec, x);
      else store_n(a.work, ((place + tok2) * a.H + head2) * DH + c1 + c, PT_F32, 1, x);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Joins up to 8 splits' sums: DH / 4 lanes per (row, head), 4 channels each.
constexpr int kFewSplits = 8;
template <int DH>
__global__ __launch_bounds__(256) void paged_join_few_kernel(PagedAttend a, int S) {
  constexpr int LR = DH / 4;
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LR;  // place of the row times heads, plus head
  const int64_t rows = (int64_t)a.c.n_seqs * a.r.max_rows * a.H;
  if (at >= rows) return;
  const int c0 = ((int)threadIdx.x & (LR - 1)) * 4;
  // everything that the sums take is loaded at once; rows that do not exist read what the
  // workspace holds, and write nothing
  const float2* ml = reinterpret_cast<const float2*>(a.work + rows * S * DH);
  float2 st[kFewSplits];
  float4 p[kFewSplits];
#pragma unroll
  for (int k = 0; k < kFewSplits; ++k) {
    if (k >= S) break;
    st[k] = ml[k * rows + at];
    p[k] = *reinterpret_cast<const float4*>(a.work + (k * rows + at) * DH + c0);
  }
  const int h = (int)(at % a.H), tok = (int)(at / a.H % a.r.max_rows), s = (int)(at / a.H / a.r.max_rows);
  const SeqRows sr = seq_rows(a.r, s);
  if (tok >= sr.n) return;
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int k = 0; k < kFewSplits; ++k) {
    if (k >= S) break;
    m = fmaxf(m, st[k].x);
  }
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int k = 0; k < kFewSplits; ++k) {
    if (k >= S) break;
    if (st[k].x == -INFINITY && st[k].y == 0.f) continue;  // saw nothing: may hold anything
    const float w = __builtin_amdgcn_exp2f(st[k].x - m);
    l += w * st[k].y;
    o.x += w * p[k].x; o.y += w * p[k].y; o.z += w * p[k].z; o.w += w * p[k].w;
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const float x[4] = {l == 0.f ? 0.f : o.x * inv, l == 0.f ? 0.f : o.y * inv, l == 0.f ? 0.f : o.z * inv, l == 0.f ? 0.f : o.w * inv};
  store_n(a.o.p, (int64_t)(sr.row0 + tok) * a.o.row + (int64_t)h * a.o.head + c0, a.o.type, a.o.vec, x);
}

// Joins more splits' sums, four waves per (row, head): lane i of each looks after split i's
// state; a wave's lanes take 4 channels each of 256 / DH splits at a time.
template <int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttend a, int S) {
  constexpr int LR = DH / 4, P = 64 / LR;  // lanes of a split's row, splits at a time
  __shared__ float4 part[4][LR];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t at = blockIdx.x;  // place of the row times heads, plus head
  const int64_t rows = (int64_t)a.c.n_seqs * a.r.max_rows * a.H;
  if (at >= rows) return;
  // everything that the sums take is loaded at once; rows that do not exist read what the
  // workspace holds, and write nothing
  const float2* ml = reinterpret_cast<const float2*>(a.work + rows * S * DH);
  float2 st = ml[min(lane, S - 1) * rows + at];
  if (lane >= S) st = make_float2(-INFINITY, 0.f);
  const int c0 = (lane & (LR - 1)) * 4, first = wave * P + lane / LR;
  constexpr int STEP = 4 * P, AHEAD = 4;
  float4 p[AHEAD];
#pragma unroll
  for (int j = 0; j < AHEAD; ++j)
    p[j] = *reinterpret_cast<const float4*>(a.work + ((int64_t)min(first + j * STEP, S - 1) * rows + at) * DH + c0);
  const int h = (int)(at % a.H), tok = (int)(at / a.H % a.r.max_rows);
  const int s = (int)(at / a.H / a.r.max_rows);
  const SeqRows sr = seq_rows(a.r, s);
  if (tok >= sr.n) return;
  const float m = wave_max(st.x);
  const bool used = !(st.x == -INFINITY && st.y == 0.f);
  const float w = used ? __builtin_amdgcn_exp2f(st.x - m) : 0.f;
  const float l = wave_sum(used ? w * st.y : 0.f);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < S; k0 += STEP * AHEAD) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int k = k0 + j * STEP + first;
      const float wk = __shfl(w, min(k, S - 1));
      if (k < S && wk != 0.f) {  // (a split that saw nothing may hold anything)
        o.x += wk * p[j].x; o.y += wk * p[j].y; o.z += wk * p[j].z; o.w += wk * p[j].w;
      }
      if (k0 + STEP * AHEAD < S) p[j] = *reinterpret_cast<const float4*>(a.work + ((int64_t)min(k + STEP * AHEAD, S - 1) * rows + at) * DH + c0);
    }
  }
  o.x = across_sum<LR>(o.x); o.y = across_sum<LR>(o.y); o.z = across_sum<LR>(o.z); o.w = across_sum<LR>(o.w);
  if (lane < LR) part[wave][lane] = o;
  __syncthreads();
  if (wave > 0) return;
  o = part[0][lane & (LR - 1)];
#pragma unroll
  for (int k = 1; k < 4; ++k) {
    const float4 p4 = part[k][lane & (LR - 1)];
    o.x += p4.x; o.y += p4.y; o.z += p4.z; o.w += p4.w;
  }
  if (lane >= LR) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const float x[4] = {l == 0.f ? 0.f : o.x * inv, l == 0.f ? 0.f : o.y * inv, l == 0.f ? 0.f : o.z * inv, l == 0.f ? 0.f : o.w * inv};
  store_n(a.o.p, (int64_t)(sr.row0 + tok) * a.o.row + (int64_t)h * a.o.head + c0, a.o.type, a.o.vec, x);
}

// Packed rows (rows of a sequence times query heads of a KV head) up to which the step
// kernel runs.  It reads the cache once for every 16 rows, the prompt kernel once for 128 but
// in tiles whose loads and products a block does in turn.  us in a graph, step and prompt:
// float16 d = 64, one sequence of 4096 slots, 32 rows 10.9 and 13.6, 33 rows 15.0 and 14.1;
// 16 of 2048, 16 rows 25.7 and 36.3, 32 rows 43 and 38, 64 rows 77 and 46; bfloat16 d = 128,
// 4 of 4096, 32 rows 18.9 and 23.4, 36 rows 34 and 24.  Over MXFP4, where reading again costs
// a quarter: d = 128, 4 of 8192, 32 rows 19 and 35, 128 rows 40 and 49; float32 rows, d = 64,
// 16 of 2048, 33 rows 28 and 46, 128 rows 63 and 63.
constexpr int step_rows(int type) { return type == PT_MXFP4 ? 128 : 32; }
constexpr int kMaxSplits = 64;
// blocks of a launch up to which the slots are split
constexpr int kStepBlocks = 1024, kPromptBlocks = 1024;

struct Plan {
  bool step;
  Grid g;
};

// Slots that a step block's waves take in one round.
int round_of(const PagedCache& c) { return c.dh == 32 ? 256 : 128; }

// A split costs a second launch (3 us) and its sums' way through memory, a block too few
// leaves compute units idle.  Step blocks: none up to 512 slots (us in a graph, one sequence
// of 16 heads of 64 float16 channels: 512 slots 6.4 alone, 7.5 split; 1024 9.3 and 7.3); behind them
// splits of one round or more, at most 32 (16384 slots of 8 heads of 128: bfloat16 16.8 with
// 32, 18.2 with 64; MXFP4 10.4 and 11.2) and 512 blocks (4 sequences of 2048 MXFP4 slots: 8.9
// with 512, 11.0 with 1024); and twice that once a split still has 1024 slots, where the
// stream of the cache is what counts.  Prompt blocks sit two to a compute unit: from 512 on
// all are busy.
Plan plan_of(const PagedCache& c, const PagedRows& r, int H) {
  Plan p;
  p.g.G = H / c.hk;
  const int64_t packed = (int64_t)r.max_rows * p.g.G;
  p.step = packed <= step_rows(c.type);
  const int64_t per = p.step ? 16 : 128;
  p.g.tiles = (int)((packed + per - 1) / per);
  const int64_t blocks = std::max<int64_t>((int64_t)p.g.tiles * c.n_seqs * c.hk, 1), slots = std::max(r.max_slots, 1);
  int64_t S = 1;
  if (p.step) {
    const int round = round_of(c);
    if (slots > 512) S = std::max<int64_t>({1, std::min<int64_t>({kStepBlocks / 2 / blocks, (slots + round - 1) / round, 32}),
                                            std::min<int64_t>({kStepBlocks / blocks, slots / 1024, kMaxSplits})});
  } else if (blocks < 512) {
    S = std::max<int64_t>(1, std::min<int64_t>({kPromptBlocks / blocks, slots / 256, kMaxSplits}));
  }
  p.g.chunk = (int)(((slots + S - 1) / S + 63) / 64 * 64);
  p.g.S = (int)((slots + p.g.chunk - 1) / p.g.chunk);
  return p;
}

template <int CT, int DH, int QT>
hipError_t attend_at(const PagedAttend& a, const Plan& p, hipStream_t st, const Ev& ev) {
  const dim3 grid((uint32_t)(p.g.S * p.g.tiles), (uint32_t)a.c.hk, (uint32_t)a.c.n_seqs);
  const bool join = p.g.S > 1;
  hipError_t e;
  if (p.step) e = plaunch(paged_step_kernel<CT, DH, QT>, grid, dim3(256), st, ev.start, join ? nullptr : ev.stop, a, p.g);
  else e = plaunch(paged_prompt_kernel<CT, DH, QT>, grid, dim3(256), st, ev.start, join ? nullptr : ev.stop, a, p.g);
  if (e != hipSuccess || !join) return e;
  const int64_t sums = (int64_t)a.c.n_seqs * a.r.max_rows * a.H;
  if (p.g.S <= kFewSplits)
    return plaunch(paged_join_few_kernel<DH>, dim3((uint32_t)((sums * (DH / 4) + 255) / 256)), dim3(256), st, nullptr, ev.stop, a, p.g.S);
  return plaunch(paged_join_kernel<DH>, dim3((uint32_t)sums), dim3(256), st, nullptr, ev.stop, a, p.g.S);
}

template <int CT, int DH>
hipError_t attend_dh(const PagedAttend& a, const Plan& p, hipStream_t st, const Ev& ev) {
  if (a.q.type == PT_F32) return attend_at<CT, DH, PT_F32>(a, p, st, ev);
  if constexpr (CT != PT_F16) {
    if (a.q.type == PT_BF16) return attend_at<CT, DH, PT_BF16>(a, p, st, ev);
  }
  if constexpr (CT != PT_BF16) {
    if (a.q.type == PT_F16) return attend_at<CT, DH, PT_F16>(a, p, st, ev);
  }
  return hipErrorInvalidValue;
}

template <int CT>
hipError_t attend_ct(const PagedAttend& a, const Plan& p, hipStream_t st, const Ev& ev) {
  switch (a.c.dh) {
    case 32: return attend_dh<CT, 32>(a, p, st, ev);
    case 64: return attend_dh<CT, 64>(a, p, st, ev);
    case 128: return attend_dh<CT, 128>(a, p, st, ev);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

size_t paged_work_bytes(const PagedCache& c, const PagedRows& r, int H) {
  const Plan p = plan_of(c, r, H);
  return p.g.S > 1 ? (size_t)p.g.S * c.n_seqs * r.max_rows * H * (c.dh + 2) * 4 : 0;
}

__global__ void paged_iota_kernel(int32_t* p, int64_t n) {
  const int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  if (i < n) p[i] = (int32_t)i;
}

hipError_t launch_paged_iota(int32_t* p, int64_t n, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  return plaunch(paged_iota_kernel, dim3((uint32_t)((n + 255) / 256)), dim3(256), st, nullptr, nullptr, p, n);
}

// A split launch has at most so many blocks, of 16 or 128 packed rows each.
size_t paged_work_most(int dh) {
  return (size_t)std::max(16 * kStepBlocks, 128 * kPromptBlocks) * (dh + 2) * 4;
}

// Rows of a wave: 4 where that leaves 8192 waves, 32 for each compute unit.
static Tasks tasks_of(int heads0, int heads, int dh, int n_rows, uint32_t* blocks) {
  Tasks t;
  t.per_shift = dh == 32 ? 2 : dh == 64 ? 3 : 4;
  const int c0 = ((heads0 << t.per_shift) + 63) / 64, c1 = ((heads << t.per_shift) + 63) / 64;
  t.first[0] = 0;
  t.first[1] = c0;
  t.first[2] = c0 + c1;
  t.chunks = c0 + 2 * c1;
  const int64_t waves = (int64_t)n_rows * t.chunks;
  t.rows = waves >= 4 * 8192 ? 4 : 1;
  *blocks = (uint32_t)(((int64_t)(n_rows + t.rows - 1) / t.rows * t.chunks + 3) / 4);
  return t;
}

template <int CT>
static hipError_t append_ct(const PagedAppend& a, hipStream_t st, const Ev& ev) {
  uint32_t blocks;
  const Tasks t = tasks_of(a.q.p != nullptr ? a.H : 0, a.c.hk, a.c.dh, a.r.n_rows, &blocks);
  return plaunch(paged_append_kernel<CT>, dim3(blocks), dim3(256), st, ev.start, ev.stop, a, t);
}

template <int CT>
static hipError_t read_ct(const PagedCache& c, const PagedRows& r, const HeadRows& k, const HeadRows& v, hipStream_t st, const Ev& ev) {
  uint32_t blocks;
  const Tasks t = tasks_of(0, c.hk, c.dh, r.n_rows, &blocks);
  if (t.rows == 1) return plaunch(paged_read_kernel<CT, 1>, dim3(blocks), dim3(256), st, ev.start, ev.stop, c, r, k, v, t);
  return plaunch(paged_read_kernel<CT, 2>, dim3(blocks), dim3(256), st, ev.start, ev.stop, c, r, k, v, t);
}

hipError_t launch_paged_append(const PagedAppend& a, hipStream_t st, const Ev& ev) {
  switch (a.c.type) {
    case PT_BF16: return append_ct<PT_BF16>(a, st, ev);
    case PT_F16: return append_ct<PT_F16>(a, st, ev);
    case PT_MXFP4: return append_ct<PT_MXFP4>(a, st, ev);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_paged_read(const PagedCache& c, const PagedRows& r, const HeadRows& k, const HeadRows& v, hipStream_t st,
                             const Ev& ev) {
  switch (c.type) {
    case PT_BF16: return read_ct<PT_BF16>(c, r, k, v, st, ev);
    case PT_F16: return read_ct<PT_F16>(c, r, k, v, st, ev);
    case PT_MXFP4: return read_ct<PT_MXFP4>(c, r, k, v, st, ev);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_paged_attend(const PagedAttend& a, hipStream_t st, const Ev& ev) {
  const Plan p = plan_of(a.c, a.r, a.H);
  switch (a.c.type) {
    case PT_BF16: return attend_ct<PT_BF16>(a, p, st, ev);
    case PT_F16: return attend_ct<PT_F16>(a, p, st, ev);
    case PT_MXFP4: return attend_ct<PT_MXFP4>(a, p, st, ev);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace mbp
