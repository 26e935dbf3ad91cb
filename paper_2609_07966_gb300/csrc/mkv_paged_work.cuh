// Which chunks of 128 tokens a CTA of the paged attention kernels takes, found out by the warp that loads them.
//
// The chunks of all (entry, key head) units lie end to end and are cut into runs of one length, one a CTA, whatever the
// entries' lengths (which are read on the device).  A run's chunks of one unit are a piece; pieces of a unit that several
// runs share are added up by the CTA whose piece arrives last.  The other warps get what they have to know with each chunk.
#pragma once

#include "mkv_paged.cuh"
#include "mkv_paged_runs.h"

namespace mkv {

constexpr int kTokens = 128;        // of a chunk

struct WorkArgs {
  int log_page;                     // of the tokens of a page, which is a copy: 16 to 128, a chunk at most
  int parts;                        // CTAs a unit if each gets as many; 0: not to be done
  int lost;                         // so many chunks more a CTA are worth it
  int grid;
  float scale_log2;
};
// Where entries are equally long, every unit may be cut into equal parts, so that no CTA has pieces of two units.  That costs
// the CTAs that such a cut leaves without work: not taken beyond a fifth of them, or `lost` chunks a CTA.  (One token, where
// memory is the bound whatever the CTAs: 8 x 8K 32.2 -> 30.8 us, 16 x 32K, 256 of 304 CTAs, 164 -> 161.  Eight drafted tokens,
// 152 CTAs that are bound themselves: 8 x 8K, 5 chunks lost, 47 -> 44; 8 x 32K, 20 lost, 121 -> 129.)
constexpr int kAnyLost = 1 << 30;
inline WorkArgs work_args(const PagedAttnCall& c, int grid, int lost) {
  WorkArgs w{};
  while ((1 << w.log_page) < c.s.page) ++w.log_page;
  const int units = c.s.B * c.s.Hkv, parts = grid / units;
  w.parts = parts * units * 5 >= grid * 4 ? parts : 0;
  w.lost = lost;
  w.grid = grid;
  w.scale_log2 = c.scale * kLog2e;
  return w;
}

enum { kFirst = 1, kLast = 2, kWhole = 4, kEnd = 8 };     // of a piece; the piece is the whole unit; nothing comes any more
// What comes with a chunk, and what comes with the first one of a piece.
struct Chunk {
  int flags, chunk, copies, scales;  // copies: a bit for each page's copy that is there; scales: where the first one's are
};
struct Piece {
  int len, tokens, unit, kvh;      // tokens: the entry's new ones
  int row0, mine, first, place0;   // mine: this piece's place; the unit's pieces: the run of the first, its place,
  int count, pad[3];               // how many there are
  // place of the unit's piece i: runs have two, for their first piece and for their last
  __device__ __forceinline__ int place(int i) const { return i == 0 ? place0 : 2 * (first + i); }
};
struct Head {
  Chunk c;
  Piece p;
};
static_assert(sizeof(Head) == 64, "four 16-byte accesses");
// Scales of a batch of 32 copies lie together: key factor, log2 of the value scale.  Of several pieces as many
// batches are kept as chunks can be between the warp that loads and those that compute (a batch may hold one chunk alone).
constexpr int kBatches = 8;
constexpr int scale_bytes(int batches) { return batches * 32 * 8; }

struct Entry {
  int row0, tokens, len, chunks;   // its first row, new tokens, tokens held, chunks of a unit
};
__device__ __forceinline__ Entry entry_of(const PagedAttnCall& c, const WorkArgs& w, int b, uint32_t* report) {
  const EntryRows r = entry_rows(c.s, b);
  Entry e;
  e.row0 = r.first;
  e.tokens = (int)min((int64_t)r.count, c.max_rows + 1);
  e.len = (int)min((int64_t)max(c.T_len[b], 0), c.s.max_pages << w.log_page);
  if (e.tokens > c.max_rows) {
    if (report != nullptr) atomicOr(report, MKV_FLAG_BAD_INDEX);
    e.tokens = 0;
  }
  e.chunks = e.tokens > 0 ? max(1, (e.len + kTokens - 1) / kTokens) : 0;
  return e;
}

// A whole warp goes through chunks c0 .. c1 - 1 of entry b's key head.  It calls begin() once the first pages are being
// fetched, and for each chunk
//   copies(ch, mine, id, at)   lane: whether a copy of the chunk is its own, the copy's page, and its place in the chunk
//   publish(ch)                (after the scales are in place)
// of which the first two say whether to go on; whether all went through.  `batch`: how many batches were begun before.  Little
// is done a chunk: a warp alone takes 6 cycles an instruction.
template <int BATCHES, typename Begin, typename Copies, typename Publish>
__device__ __forceinline__ bool load_chunks(const PagedAttnCall& c, const WorkArgs& w, uint32_t* status, float2* held_scales,
                                            int lane, int& batch, int b, int kvh, int len, int c0, int c1, int flags,
                                            Begin begin, Copies copies, Publish publish) {
  // A batch is 32 copies' pages, a lane each: page and scales of the next batch are fetched during this one.
  const int log_per = 7 - w.log_page, span = 32 >> log_per; // copies a chunk, chunks a batch
  const int32_t* table = c.s.page_table + (int64_t)b * c.s.max_pages;
  auto exists = [&](int chunk) {                           // this lane's copy of the batch from `chunk` on
    return chunk + (lane >> log_per) < c1 && chunk * kTokens + (lane << w.log_page) < len;
  };
  auto fetch = [&](int chunk) {
    return exists(chunk) ? table[(chunk << (7 - w.log_page)) + lane] : -1;
  };
  auto check = [&](int chunk, int id) {                    // (a page outside the pool is not seen)
    if (!exists(chunk)) return -1;
    if (id >= 0 && id < c.s.num_pages) return id;
    atomicOr(status, MKV_FLAG_BAD_INDEX);
    return -1;
  };
  auto scales = [&](int id, float& ks, float& vs) {
    ks = 0.f;
    vs = 1.f;
    if (id >= 0) {
      ks = c.k_scale[(int64_t)id * c.s.Hkv + kvh];
      vs = c.v_scale[(int64_t)id * c.s.Hkv + kvh];
    }
  };
  int pid = fetch(c0), next = 0;
  if (!begin()) return false;
  pid = check(c0, pid);
  float ks, vs, nks = 0.f, nvs = 1.f;
  scales(pid, ks, vs);
  unsigned there = 0;                                      // copies of the batch
  int at = 0;                                              // its place among the scales
  for (int ch = c0; ch < c1; ++ch) {
    const int in = (ch - c0) & (span - 1);
    if (in == 0 && ch > c0) {
      pid = next;
      ks = nks;
      vs = nvs;
    }
    if (in == 0) next = fetch(ch + span);
    if (in == span / 2) {
      next = check(ch - in + span, next);
      scales(next, nks, nvs);
    }
    if (in == 0) {
      there = __ballot_sync(0xffffffffu, pid >= 0);
      at = batch++ % BATCHES * 32;
    }
    Chunk head;
    head.flags = (ch == c0 ? kFirst : 0) | (ch == c1 - 1 ? kLast : 0) | flags;
    head.chunk = ch;
    head.copies = (int)(there >> (in << log_per)) & ((1 << (1 << log_per)) - 1);
    head.scales = at + (in << log_per);
    if (!copies(head, pid >= 0 && lane >> log_per == in, pid, lane & ((1 << log_per) - 1))) return false;
    if (in == 0) {
      held_scales[at + lane] = make_float2(ks * w.scale_log2, __log2f(vs));
    }
    publish(head);
  }
  return true;
}

// A whole warp goes through this CTA's chunks: load_chunks for each piece, with begin(p), copies(ch, p, mine, id, at) and
// publish(ch, p); whether all went through.
template <typename Begin, typename Copies, typename Publish>
__device__ __forceinline__ bool work_through(const PagedAttnCall& c, const WorkArgs& w, uint32_t* status, float2* held_scales,
                                             int lane, Begin begin, Copies copies, Publish publish) {
  const int B = c.s.B, Hkv = c.s.Hkv;
  uint32_t* report = blockIdx.x == 0 ? status : nullptr;
  Entry held = {0, 0, 0, 0};                               // of entry `lane`
  if (lane < B) held = entry_of(c, w, lane, report);
  int upto = held.chunks * Hkv, total = 0;                 // inclusive prefix within the first 32 entries
  for (int b = lane + 32; b < B; b += 32) total += entry_of(c, w, b, report).chunks * Hkv;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += x;
  }
  const int upto32 = __shfl_sync(0xffffffffu, upto, 31);
  if (B > 32) {
#pragma unroll
    for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  }
  total += upto32;
  const int chunks0 = __shfl_sync(0xffffffffu, held.chunks, 0);
  const int part = w.parts > 0 ? (chunks0 + w.parts - 1) / w.parts : 0;  // chunks of each
  const bool even = B <= 32 && w.parts > 0 && part - total / w.grid <= w.lost &&
                    __all_sync(0xffffffffu, lane >= B || held.chunks == chunks0);
  Runs rs(total, w.grid);
  if (even) rs.runs = B * Hkv * w.parts;
  const int r = blockIdx.x;
  if (r >= rs.runs) return true;
  // the run's chunks, the entry that holds the first of them, and that entry's first chunk
  int b = 0, base = 0, cur = rs.start(r), end = rs.start(r + 1);
  if (even) {
    const int unit = r / w.parts, first = (r - unit * w.parts) * part;
    cur = unit * chunks0 + min(first, chunks0);
    end = unit * chunks0 + min(first + part, chunks0);
    b = unit / Hkv;
    base = b * Hkv * chunks0;
  } else if (cur < upto32) {
    b = __ffs(__ballot_sync(0xffffffffu, upto > cur)) - 1;
    base = __shfl_sync(0xffffffffu, upto - held.chunks * Hkv, b);
  } else {
    base = upto32;
    for (int b0 = 32;; b0 += 32) {
      const int mine = b0 + lane < B ? entry_of(c, w, b0 + lane, nullptr).chunks * Hkv : 0;
      int in = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, in, d);
        if (lane >= d) in += x;
      }
      const unsigned past = __ballot_sync(0xffffffffu, base + in > cur);
      if (past || b0 + 32 >= B) {
        const int l = past ? __ffs(past) - 1 : 0;
        b = b0 + l;
        base += __shfl_sync(0xffffffffu, in - mine, l);
        break;
      }
      base += __shfl_sync(0xffffffffu, in, 31);
    }
  }
  auto entry = [&](int i) {
    if (i >= 32) return entry_of(c, w, i, nullptr);
    Entry e;
    e.row0 = __shfl_sync(0xffffffffu, held.row0, i);
    e.tokens = __shfl_sync(0xffffffffu, held.tokens, i);
    e.len = __shfl_sync(0xffffffffu, held.len, i);
    e.chunks = __shfl_sync(0xffffffffu, held.chunks, i);
    return e;
  };
  int batch = 0;
  Entry e = entry(b);
  int of_entry = e.chunks * Hkv;
  while (cur < end) {
    if (!walk_to(cur, B, b, base, of_entry, [&](int i) {
          e = entry(i);
          return e.chunks * Hkv;
        })) {
      if (lane == 0) atomicOr(status, MKV_FLAG_BAD_INDEX); // (lengths changed under way)
      return true;
    }
    const int kvh = (cur - base) / e.chunks, unit0 = base + kvh * e.chunks;
    const int c0 = cur - unit0, c1 = min(e.chunks, c0 + (end - cur));
    cur += c1 - c0;
    const bool whole = c1 - c0 == e.chunks;
    Piece p;
    p.len = e.len;
    p.tokens = e.tokens;
    p.unit = b * Hkv + kvh;
    p.kvh = kvh;
    p.row0 = e.row0;
    p.first = p.place0 = p.count = p.mine = 0;
    const bool ok = load_chunks<kBatches>(
        c, w, status, held_scales, lane, batch, b, kvh, e.len, c0, c1, whole ? kWhole : 0, [&]() { return begin(p); },
        [&](const Chunk& ch, bool mine, int id, int at) { return copies(ch, p, mine, id, at); },
        [&](const Chunk& ch) {
          if (ch.chunk == c0 && !whole) {
            if (even) {
              p.first = p.unit * w.parts;
              p.place0 = 2 * p.first;
              p.count = (chunks0 + part - 1) / part;
            } else {
              const Shares sh(rs, unit0, e.chunks);
              p.first = sh.first;
              p.place0 = sh.place0;
              p.count = sh.count;
            }
            p.mine = r == p.first ? p.place0 : 2 * r;
          }
          publish(ch, p);
        });
    if (!ok) return false;
  }
  return true;
}

// The pieces' sums of one row, added up in the pieces' order: out = sum_i 2^(m2_i - M2) o_i, with M, sum and M2 of all.
// VL neighbouring dims a lane; part_o [place][rows][32 VL], part_st [place][rows].
template <int VL>
__device__ __forceinline__ float4 add_pieces(const Piece& hd, const float* part_o, const float4* part_st, int rows, int row,
                                             int lane, float& mx, float& sum, float& mx2) {
  mx = mx2 = kNoMax;
  sum = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = 0; i0 < hd.count; i0 += 8) {               // eight pieces' loads under way together
    float4 st[8], z[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t at = (int64_t)hd.place(min(i0 + k, hd.count - 1)) * rows + row;
      st[k] = __ldcg(part_st + at);
      const float* po = part_o + at * (32 * VL) + lane * VL;
      if constexpr (VL == 4) {
        z[k] = __ldcg(reinterpret_cast<const float4*>(po));
      } else {
        const float2 f = __ldcg(reinterpret_cast<const float2*>(po));
        z[k] = make_float4(f.x, f.y, 0.f, 0.f);
      }
      if (i0 + k >= hd.count) st[k] = make_float4(kNoMax, 0.f, kNoMax, 0.f);
    }
    float nm = mx, nm2 = mx2;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      nm = fmaxf(nm, st[k].x);
      nm2 = fmaxf(nm2, st[k].z);
    }
    sum *= ex2_approx(mx - nm);
    const float back = ex2_approx(mx2 - nm2);
    y = make_float4(y.x * back, y.y * back, y.z * back, y.w * back);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float f = i0 + k < hd.count ? ex2_approx(st[k].z - nm2) : 0.f;
      sum += st[k].y * ex2_approx(st[k].x - nm);
      y = make_float4(y.x + f * z[k].x, y.y + f * z[k].y, y.z + f * z[k].z, y.w + f * z[k].w);
    }
    mx = nm;
    mx2 = nm2;
  }
  return y;
}

}  // namespace mkv
