// Internal interface of the paged cache operators (paged.hip): appending rotated token
// rows, reading them back, and attention over the pages.  Not part of the public C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace mbp {

// Element types of a cache or of token rows; the values of mbp_dtype.
enum PagedType { PT_F32 = 0, PT_BF16 = 1, PT_F16 = 2, PT_MXFP4 = 3 };

// Pools [n_pages][hk][page], a page of one head being its slots' rows: dh 16-bit values,
// or (PT_MXFP4) dh / 2 bytes of codes per slot and behind all slots' codes dh / 32 scale
// bytes per slot.  pages [n_seqs][max_pages] holds each sequence's page ids; a slot
// whose id lies outside [0, n_pages) holds nothing.
struct PagedCache {
  char* k;
  char* v;
  const int32_t* pages;
  int32_t type, hk, dh, shift /* log2 of the slots of a page */, n_pages, n_seqs, max_pages;
  int64_t page_bytes;  // of one head
};

// Rows [row_start[i], row_start[i + 1]) belong to sequence i, row r at slot
// first_slot[i] + r - row_start[i].  max_rows bounds a sequence's rows, max_slots the
// slots that a row sees (a smaller value than the true one costs time, not results).
struct PagedRows {
  const int32_t* row_start;
  const int32_t* first_slot;
  int32_t n_rows, max_rows, max_slots;
};

// Rows of heads: element e of head h of row r at p + r * row + h * head + e; vec: every
// such head starts at a multiple of 16 bytes.
struct HeadRows {
  void* p;
  int64_t row, head;
  int32_t type, vec;
};

struct PagedAppend {
  PagedCache c;
  PagedRows r;
  HeadRows q, qo, k, v;  // q.p == nullptr: no queries
  int32_t H;
  const int32_t* pos;   // rotary position of each row, or nullptr: its slot
  const float2* rope;   // [n_pos][dh / 2] (cos, sin), or nullptr: no rotation
  int32_t n_pos;
};

struct PagedAttend {
  PagedCache c;
  PagedRows r;
  HeadRows q, o;  // of one type
  int32_t H;
  const int32_t* lo;  // first visible slot of each row, or nullptr: 0
  const int32_t* hi;  // end of the visible slots, or nullptr: the row's slot + 1
  float scale;
  // split sums (paged_work_bytes): [splits][n_seqs][max_rows][H] rows of dh floats, then as
  // many (max, sum) pairs
  float* work;
};

size_t paged_work_bytes(const PagedCache& c, const PagedRows& r, int H);
size_t paged_work_most(int dh);  // no call with a full row of heads in every tile needs more
hipError_t launch_paged_append(const PagedAppend& a, hipStream_t st, const Ev& ev = Ev());
// The inverse: all n_rows rows of k and v receive the values of their slots (0 for a row
// of no sequence or a slot without a page).
hipError_t launch_paged_read(const PagedCache& c, const PagedRows& r, const HeadRows& k, const HeadRows& v,
                             hipStream_t st, const Ev& ev = Ev());
hipError_t launch_paged_attend(const PagedAttend& a, hipStream_t st, const Ev& ev = Ev());

// p[i] = i: page tables whose rows' pages lie in order.
hipError_t launch_paged_iota(int32_t* p, int64_t n, hipStream_t st);

}  // namespace mbp
