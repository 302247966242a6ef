// Host stand-ins for the launchers of rotated appends, block-scaled caches and
// adjusted logits (see hip_stub.cpp).  Launches of attention are taken apart the way
// their kernels do it, workgroup by workgroup: every unit of work has to be done by
// exactly one of them, and every record (or output) written by exactly one part.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <tuple>
#include <vector>

#include "kvq_internal.h"

bool g_touch = true;       // "device" buffers are real ones
int64_t g_parts = 0;       // parts of attention launches that were checked
int g_block_launches = 0, g_tile_launches = 0, g_row_launches = 0;

namespace {

void rd(const void* p, size_t n) {
  static std::vector<uint8_t> sink;
  if (!g_touch) return;
  if (sink.size() < n) sink.resize(n);
  if (n) std::memcpy(sink.data(), p, n);
}
void wr(const void* p, size_t n) {
  if (g_touch && n) std::memset(const_cast<void*>(p), 0, n);
}
void bad(const char* what, int seq, int h, int group) {
  std::fprintf(stderr, "block check failed (%s): sequence %d, head %d, group %d\n", what, seq, h, group);
  std::abort();
}
using namespace kvq;
constexpr size_t kToken = kHeadDim * 2;

template <class Args, class F>
void packed(const Args& a, uint64_t head0, int seq, int h, int from, int to, F f) {
  for (int t = from; t < to; t += a.gk) {
    int in;
    const uint8_t* seg = a.arena + packed_seg(a.pm, head0, a.head_stride, seq, h, t, in);
    f(seg + region(a.kc) + (size_t)in * kHeadDim, (size_t)a.gk * kHeadDim);
    f(seg + region(a.km) + (size_t)(in / a.gk) * 8, 8);
    f(seg + region(a.vc) + (size_t)in * kHeadDim, (size_t)a.gk * kHeadDim);
  }
}
template <class Args, class F>
void ring(const Args& a, uint64_t head0, int h, int from, int to, F f) {
  const uint8_t* r = a.arena + head0 + (uint64_t)h * a.head_stride;
  for (int t = from; t < to; ++t) {
    f(r + region(a.tk) + (size_t)(t % a.W) * kToken, kToken);
    f(r + region(a.tv) + (size_t)(t % a.W) * kToken, kToken);
  }
}

// What an append reads and writes; block: a block-scaled cache's.
void touch_append(const AppendArgs& a, const RotaryArgs* rot, bool block, int bk, int bv) {
  for (int i = 0; i < a.nseq; ++i) {
    const AppendSeq& S = a.seq[i];
    const int n = S.L_new - S.L_old, packed_now = a.quantize ? S.n_quant * a.gk : 0;
    const int copy0 = std::max(S.Lq_new, S.L_old), copied = S.n_copy > 0 ? S.L_new - copy0 : 0;
    const int wgs = ((a.quantize ? S.n_quant : 0) + S.n_copy + S.n_query) * a.hkv;
    if ((i + 1 < a.nseq ? a.seq[i + 1].wg_begin : a.total_wg) - S.wg_begin != wgs) bad("append workgroups", S.seq, 0, 0);
    auto input = [&](int t, int h) {
      const size_t token = (size_t)S.seq * a.n_max + (t - S.L_old);
      rd(a.K + token * (rot ? rot->k_stride : a.hkv * kHeadDim) + (size_t)h * kHeadDim, kToken);
      rd(a.V + token * (rot ? rot->v_stride : a.hkv * kHeadDim) + (size_t)h * kHeadDim, kToken);
      if (!rot) return;
      if (rot->position) rd(rot->position + token, 4);
      else if (t >= rot->rows) bad("table row", S.seq, h, t);
      else {
        rd(rot->cos_ + (size_t)t * (rot->rot / 2), rot->rot / 2 * 4);
        rd(rot->sin_ + (size_t)t * (rot->rot / 2), rot->rot / 2 * 4);
      }
    };
    for (int h = 0; h < a.hkv; ++h) {
      ring(a, S.head0, h, S.Lq_old, std::min(S.L_old, S.Lq_old + packed_now), rd);
      for (int t = std::max(S.L_old, S.Lq_old); t < S.Lq_old + packed_now; ++t) input(t, h);
      if (block) packed(a, S.head0, S.seq, h, S.Lq_old, S.Lq_old + packed_now, wr);
      for (int t = copy0; t < copy0 + copied; ++t) input(t, h);
      ring(a, S.head0, h, copy0, copy0 + copied, wr);
    }
    if (rot && rot->q && S.n_query > 0) {
      if (S.n_query * kQueryTokens < n) bad("queries", S.seq, 0, 0);
      const size_t row = (size_t)a.hkv * rot->gqh * kHeadDim;
      for (int k = 0; k < n; ++k) {
        const size_t token = (size_t)S.seq * a.n_max + k;
        rd(rot->q + token * rot->q_stride, row * 2);
        wr(rot->q_out + token * row, row * 2);
      }
    }
  }
  (void)bk;
  (void)bv;
  ++g_block_launches;
}

// The parts of one (sequence, head, group): units done, records written.
struct Group {
  std::vector<char> unit, record;
};

// sequence that holds unit u
int sequence_at(const DecodeArgs& a, int u) {
  int si = 0;
  for (int i = 1; i < a.nseq; ++i) si = a.seq[i].wg_begin <= u ? i : si;
  return si;
}
void finish(const DecodeArgs& a, const std::map<std::tuple<int, int, int>, Group>& groups, size_t expected) {
  if (groups.size() != expected) bad("groups", -1, -1, (int)groups.size());
  for (auto& g : groups) {
    for (char x : g.second.unit)
      if (x != 1) bad("a unit of work is not done once", std::get<0>(g.first), std::get<1>(g.first), std::get<2>(g.first));
    for (char x : g.second.record)
      if (x != 1) bad("a record is not written once", std::get<0>(g.first), std::get<1>(g.first), std::get<2>(g.first));
  }
  const size_t rows = (size_t)a.hq * a.nqry;
  for (int i = 0; i < a.nseq; ++i) {
    const DecodeSeq& S = a.seq[i];
    rd(a.q + (size_t)S.seq * rows * kHeadDim, rows * kToken);
    if (S.nsplit == 1) wr(a.out + (size_t)S.seq * rows * kHeadDim, rows * kHeadDim * 4);
    else wr(a.ws + (size_t)S.ws_base * rows * kRecFloats, (size_t)S.nsplit * rows * kRecFloats * 4);
    for (int h = 0; h < a.hkv; ++h) {
      packed(a, S.head0, S.seq, h, 0, g_touch ? S.Lq : 0, rd);
      ring(a, S.head0, h, g_touch ? S.Lq : 0, g_touch ? S.L : 0, rd);
    }
  }
}
void take(Group& g, const DecodeSeq& S, int total, int from, int to, int split) {
  if (g.unit.empty()) {
    g.unit.assign(total, 0);
    g.record.assign(S.nsplit, 0);
  }
  if (from < 0 || to > total || split < 0 || split >= S.nsplit) bad("part", S.seq, split, to);
  for (int k = from; k < to; ++k) ++g.unit[k];
  ++g.record[split];
  for (int s = split + 1; to == total && s < S.nsplit; ++s) ++g.record[s];  // empty records
  ++g_parts;
}

}  // namespace

namespace kvq {

int launch_append_rotary(const AppendArgs& a, const RotaryArgs* rot, int bk, int bv, void*) { return touch_append(a, rot, false, bk, bv), 0; }
int launch_append_block(const AppendArgs& a, const RotaryArgs* rot, int tk, int tv, void*) { return touch_append(a, rot, true, tk, tv), 0; }

int launch_block_tiles(const DecodeArgs& a, int, int, int rows, void*) {
  if (a.total_wg <= 0) return 0;
  const int per = a.units_per_wg, gsh = a.gk == 32 ? 5 : a.gk == 64 ? 6 : 7;
  if (per < 1 || rows > 32 || a.qpr * a.gqh > rows || a.nrg != (a.nqry + a.qpr - 1) / a.qpr) bad("shape", -1, -1, -1);
  std::map<std::tuple<int, int, int>, Group> groups;
  size_t expected = 0;
  for (int i = 0; i < a.nseq; ++i) {
    const DecodeSeq& S = a.seq[i];
    expected += (size_t)a.hkv * a.nrg;
    if (S.L_old < 1 || S.L_old > S.nq) bad("units", S.seq, S.L_old, S.nq);
    for (int rg = 0; rg < a.nrg; ++rg) {  // the groups that a row group reads, and the tail, have their units
      const int first = S.L - a.nqry + 1 + std::min(rg * a.qpr, a.nqry - 1), last = S.L - a.nqry + 1 + std::min(rg * a.qpr + a.qpr - 1, a.nqry - 1);
      if (window_groups(first, last, S.Lq, gsh, a.window, a.sinks).count + (S.L > S.Lq ? 1 : 0) > S.L_old) bad("reach", S.seq, -1, rg);
    }
  }
  const int wgs = (a.total_wg + per - 1) / per;
  for (int w = 0; w < wgs; ++w) {
    const int end = std::min((w + 1) * per, a.total_wg);
    for (int u = w * per; u < end;) {
      const int si = sequence_at(a, u);
      const DecodeSeq& S = a.seq[si];
      const int seg = (u - S.wg_begin) / S.nq, begin = S.wg_begin + seg * S.nq, h = seg / a.nrg, rg = seg - h * a.nrg;
      if (h >= a.hkv) bad("head", S.seq, h, rg);
      const int u0 = u - begin, u1 = std::min(S.L_old, end - begin);
      if (u0 < u1) take(groups[{si, h, rg}], S, S.L_old, u0, u1, w - begin / per);
      u = begin + S.nq;
    }
  }
  finish(a, groups, expected);
  return ++g_tile_launches, 0;
}

int launch_block_rows(const DecodeArgs& a, int, int, int waves, void*) {
  if (a.total_wg <= 0) return 0;
  const int per = a.units_per_wg, gsh = a.gk == 32 ? 5 : a.gk == 64 ? 6 : 7, nrw = (a.nrg + waves - 1) / waves;
  if (per < 1 || a.qpr * a.gqh > 32 || a.nrg != (a.nqry + a.qpr - 1) / a.qpr || (waves != 4 && waves != 8)) bad("shape", -1, -1, -1);
  std::map<std::tuple<int, int, int>, Group> groups;
  size_t expected = 0;
  for (int i = 0; i < a.nseq; ++i) expected += (size_t)a.hkv * nrw;
  const int wgs = (a.total_wg + per - 1) / per;
  for (int w = 0; w < wgs; ++w) {
    const int end = std::min((w + 1) * per, a.total_wg);
    for (int u = w * per; u < end;) {
      const int si = sequence_at(a, u);
      const DecodeSeq& S = a.seq[si];
      const int h = (u - S.wg_begin) / S.nq;
      if (h >= a.hkv) bad("head", S.seq, h, -1);
      int begin = S.wg_begin + h * S.nq, rw = 0, units, total;
      for (;; ++rw) {
        const RowBlocks b = row_blocks(a.nqry, a.qpr * waves, S.L, S.Lq, gsh, a.window, a.sinks, rw);
        total = b.total;
        if (total < 1 || 32 * (b.tail0 + (b.total - b.packed)) >= S.L + 32) bad("blocks", S.seq, h, rw);
        units = total + a.extra_units;
        if (rw == nrw - 1 || u < begin + units) break;
        begin += units;
      }
      const int b0 = std::min(u - begin, total), b1 = std::min(end - begin, total);
      if (b0 < b1) take(groups[{si, h, rw}], S, total, b0, b1, w - begin / per);
      u = begin + units;
    }
  }
  finish(a, groups, expected);
  return ++g_row_launches, 0;
}

int launch_dequant_block(const DequantArgs& a, void*) {
  for (int h = 0; h < a.hkv; ++h) {
    packed(a, a.head0, a.seq, h, std::min(a.tok0, a.Lq) / a.gk * a.gk, std::min(a.tok0 + a.ntok, a.Lq), rd);
    ring(a, a.head0, h, std::max(a.tok0, a.Lq), a.tok0 + a.ntok, rd);
  }
  wr(a.K_out, (size_t)a.ntok * a.hkv * kHeadDim * 4);
  wr(a.V_out, (size_t)a.ntok * a.hkv * kHeadDim * 4);
  return ++g_block_launches, 0;
}
int launch_export_block(const ExportArgs& a, void*) {
  packed(a, a.head0, a.seq, a.h, 0, a.Lq, rd);
  ring(a, a.head0, a.h, a.Lq, a.Lq + a.ntail, rd);
  wr(a.kc_out, (size_t)a.Lq * kHeadDim);
  wr(a.km_out, (size_t)a.Lq / a.gk * 4);
  wr(a.vc_out, (size_t)a.Lq * kHeadDim);
  wr(a.vm_out, (size_t)a.Lq / a.gk * 4);
  wr(a.tk_out, a.ntail * kToken);
  wr(a.tv_out, a.ntail * kToken);
  return ++g_block_launches, 0;
}
int launch_adjust(const AdjustArgs& a, int type, void*) {
  const size_t size = type == 0 ? 4 : 2;
  for (int r = 0; r < a.batch; ++r) {
    rd(static_cast<const uint8_t*>(a.logits) + (size_t)r * a.row_stride * size, a.vocab * size);
    wr(static_cast<uint8_t*>(a.out) + (size_t)r * a.out_stride * size, a.vocab * size);
  }
  if (a.nchunk * kAdjustChunk < a.vocab + 7) std::abort();
  return ++g_block_launches, 0;
}

}  // namespace kvq
