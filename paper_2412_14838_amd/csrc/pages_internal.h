// Declarations shared by the translation units of the paged 8-bit cache and of the rotary positions.
#pragma once
#include "dkv_internal.h"

namespace dkv {

constexpr int kPagesTile = 64;              // cache rows a wavefront of the attention takes at a time
constexpr int kPagesMaxGroups = 4096;       // workgroups that an attention call is cut into at most

// What the kernels need of dkv_pages and the descriptor, by value.
struct PageArgs {
  int n_pages, page_rows, shift, table_len;      // page_rows = 1 << shift
  int L, Hkv, n_seqs, w, layer_max;
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  int32_t* table;
  int32_t* rows;
  int32_t* refs;
  int32_t* missing;
};

// Workspace (byte offsets, 256-byte aligned). The calls use it one at a time: the parts overlap.
struct PagesWorkspace {
  // resize
  size_t plan;        // int32 [n_seqs * L][6]   what the call plans for a (sequence, layer)
  size_t granted;     // int32 [n_pages]     the granted pages by rank
  size_t copies;      // int2 [n_seqs * L]   source and target page
  size_t n_copies;    // int32 [1]
  // fork
  size_t old_rows;    // int32 [n_seqs][L]
  size_t old_table;   // int32 [n_seqs][L][table_len]
  // attention
  size_t partials;    // float [pieces][Hq][d + 2]   maximum, sum, unnormalised output of every piece
  size_t total;
};

inline PagesWorkspace pages_workspace(const dkv_desc& d, const dkv_pages& p) {
  PagesWorkspace w{};
  const size_t pairs = size_t(d.n_seqs) * d.n_layers;
  size_t off = 0;
  w.plan = off;     off += align256(pairs * 6 * sizeof(int32_t));
  w.granted = off;  off += align256(size_t(p.n_pages) * sizeof(int32_t));
  w.copies = off;   off += align256(pairs * 2 * sizeof(int32_t));
  w.n_copies = off; off += 256;
  const size_t resize = off;
  off = 0;
  w.old_rows = off;  off += align256(pairs * sizeof(int32_t));
  w.old_table = off; off += align256(pairs * p.table_len * sizeof(int32_t));
  const size_t fork = off;
  w.partials = 0;
  const size_t attention = align256(size_t(kPagesMaxGroups) * (d.n_q_heads / d.n_kv_heads) * (d.head_dim + 2) * sizeof(float));
  w.total = resize > fork ? resize : fork;
  if (attention > w.total) w.total = attention;
  return w;
}

#if defined(__HIPCC__)
// Rows that (q, l) holds as the other kernels read them.
__device__ inline int held_rows(const PageArgs& a, int pair) {
  const int r = a.rows[pair], most = a.table_len << a.shift;
  return r < 0 ? 0 : (r < most ? r : most);
}
#endif

// How many workgroups share the rows of a head in an attention call (beside one more for each (layer, sequence)); 0: one workgroup
// per (layer, sequence, head). Two of the pieces' workgroups run on a compute unit at a time. The second kernel costs 3 us, balanced
// pieces are worth it for few heads of many rows, or for many rows whose number differs. One launch / pieces, us under graph replay, rows the
// same in all sequences (8 KV heads of 4 queries, d = 128), by sequences and rows:
//            512         1024        1536        2048        4096        8192
//    1    6.5 / 9.0   9.6 / 9.2  12.3 / 9.5  15.0 / 9.7 25.7 / 10.5  46.7 / 11.0
//    8    6.6 / 9.1   9.7 / 9.6 12.5 / 11.4 15.5 / 12.1 26.9 / 19.3  48.4 / 29.0
//   16    6.6 / 9.6  10.4 / 12.3 13.3 / 17.2 16.1 / 19.1 27.4 / 28.7  52.0 / 48.0
//   32   7.3 / 12.1  14.1 / 19.0 19.1 / 24.2 23.6 / 28.5 43.3 / 47.5  99.0 / 104
//   64  16.9 / 19.9  26.5 / 29.6 35.3 / 39.1 44.7 / 49.0  99.8 / 105   192 / 199
// With 16 sequences of 4 KV heads and 8192 to 32768 rows the longest decides: 101 / 65. For that the rule takes pieces for 65 to 512 items of
// 4096 rows and more although equal rows lose by it: 128 items 5 % at 4096 rows, 256 items 10 and 5 % at 4096 and 8192, 512 items 5 and 4 %.
inline int pages_groups(int Hkv, int pairs, int rows) {
  const int cus = device_cus(), resident = 2 * (cus < 1024 ? cus : 1024);
  const int64_t items = (int64_t)Hkv * pairs;
  if (rows <= 1024 || items > resident || (items > resident / 8 && rows < 4096)) return 0;
  return resident / Hkv;
}

hipError_t launch_pages_clear(const PageArgs& a, hipStream_t st);
hipError_t launch_pages_resize(const PageArgs& a, int layer, int n_layers, const int32_t* base, const int32_t* cu, int extra,
                               const int32_t* active, int head_dim, char* ws, const PagesWorkspace& wl, hipStream_t st);
hipError_t launch_pages_fork(const PageArgs& a, const int32_t* parents, char* ws, const PagesWorkspace& wl, hipStream_t st);
hipError_t launch_pages_store(const PageArgs& a, int dtype, int head_dim, int layer, int n_layers, const void* const* k_layers,
                              const void* const* v_layers, int64_t stride_token, int64_t stride_head, const int32_t* cu,
                              const int32_t* idx, int64_t idx_stride_layer, const int32_t* counts, hipStream_t st);
hipError_t launch_pages_append(const PageArgs& a, int dtype, int head_dim, int layer, int n_new, const void* k_new, const void* v_new,
                               int64_t stride_seq, int64_t stride_token, int64_t stride_head, const int32_t* active, hipStream_t st);
hipError_t launch_pages_attention(const PageArgs& a, int dtype, int head_dim, int G, float scale, int layer, int n_layers,
                                  int expected_rows, const void* q, float* out, float* lse, float* partials, hipStream_t st);

// One tensor of a rotation: strides in elements.
struct RotateHeads {
  const void* in;
  void* out;
  int n_heads;
  int64_t in_seq, in_token, in_head, out_seq, out_token, out_head;
};
// Whether the call's threads fit one grid.
bool rotate_fits(const dkv_rotary& r, int64_t tokens, const RotateHeads& q, const RotateHeads& k);
hipError_t launch_rotate(const dkv_rotary& r, int n_seqs, int n_tokens, const int32_t* positions, const RotateHeads& q,
                         const RotateHeads& k, hipStream_t st);

}  // namespace dkv
