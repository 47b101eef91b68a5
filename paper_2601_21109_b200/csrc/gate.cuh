// Per-row gate of the adapter: rank mask, scale and cross-fade weight of a row, looked up in a chunk table or given per row.
#pragma once

#include "cwl_common.cuh"

namespace cwl {

struct RowGate { float w_in, w_out; int r_in, r_out; };  // g[j] = w_in [j < r_in] + w_out [j < r_out]

// Gate of row t from the chunk table (Sec. III-C rank mask and scale, Sec. III-D cross-fade weight).  `Params` has T, R, window,
// window_mode and table.
template <typename Params>
__device__ __forceinline__ RowGate table_gate(int t, const Params& p) {
  RowGate g{0.f, 0.f, 0, 0};
  const cwl_chunk_table& tb = p.table;
  const int C = min(*tb.n_chunks, tb.capacity);
  if (t < p.T && C > 0 && t >= tb.offsets[0] && t < tb.offsets[C]) {
    int lo = 0, hi = C;                            // offsets[lo] <= t < offsets[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tb.offsets[mid] <= t) lo = mid; else hi = mid;
    }
    const int c = lo, j = t - tb.offsets[c];
    float lam = 1.f;
    int c_in = c, c_out = c;                       // configurations carrying lam and 1 - lam
    if (p.window_mode == CWL_WINDOW_CENTRED) {
      // the window lies around the join: floor(w/2) rows before it, ceil(w/2) rows after it; where a short chunk's
      // two windows meet, the rows belong to the join that opened the chunk
      const int before = p.window >> 1, after = p.window - before;
      const int len = tb.offsets[c + 1] - tb.offsets[c];
      if (c > 0 && !(tb.flags[c] & 1) && j < after) {
        lam = (float)(before + j + 1) / (float)(p.window + 1);
        c_out = c - 1;
      } else if (c + 1 < C && !(tb.flags[c + 1] & 1) && len - j <= before) {
        lam = (float)(before - (len - j) + 1) / (float)(p.window + 1);
        c_in = c + 1;
      }
    } else if (c > 0 && !(tb.flags[c] & 1) && j < p.window) {
      lam = (float)(j + 1) / (float)(p.window + 1);
      c_out = c - 1;
    }
    g.r_in = min(max(tb.rank[c_in], 0), p.R);
    g.w_in = lam * tb.scale[c_in];
    if (lam < 1.f) {
      g.r_out = min(max(tb.rank[c_out], 0), p.R);
      g.w_out = (1.f - lam) * tb.scale[c_out];
    }
  }
  return g;
}
// The same where rows may bring their own descriptors: `Params` also has row_gates, null unless every row does.
template <typename Params>
__device__ __forceinline__ RowGate row_gate(int t, const Params& p) {
  if (p.row_gates == nullptr) return table_gate(t, p);
  RowGate g{0.f, 0.f, 0, 0};
  if (t < p.T) {
    const cwl_row_gate d = p.row_gates[t];
    g.r_in = min(max(d.rank_in, 0), p.R);
    g.w_in = d.lambda * d.scale_in;
    if (d.lambda < 1.f) {
      g.r_out = min(max(d.rank_out, 0), p.R);
      g.w_out = (1.f - d.lambda) * d.scale_out;
    }
  }
  return g;
}
__device__ __forceinline__ float gate_at(const RowGate& g, int j) {
  return (j < g.r_in ? g.w_in : 0.f) + (j < g.r_out ? g.w_out : 0.f);
}

}  // namespace cwl
