// Attention of tree nodes over a paged cache for gfx950 (tv_tree_attention, and over a
// cache of 4 bits tv_tree_attention_fp4).
//
// All nodes of a tree and all query heads of a key head read the same cached keys
// and values: these num_nodes * heads / kv_heads query rows are the columns of one
// matrix product with each key. Per 32 keys a wavefront forms S^T = K Q^T, takes
// 2^(s k - m k) with k = scale log2(e) in the frame of a running maximum m, and
// adds V^T P^T to its accumulators (16x16x32 products; out = sum p v / sum p).
// With keys as rows of S^T, a lane holds four consecutive keys of one query, which
// is how the second product wants its operand: P never leaves its lane, the keys
// of the two blocks taken in the order in which the lanes hold them. Values are
// read transposed from LDS.
//
// The frame is a maximum seen so far; it moves only once some score exceeds it by
// 8 in powers of two, so that most tiles rescale nothing (weights up to 2^8 in
// their frame, and 2^15 for fp16, which has few exponents below 1; sums in fp32). Weights are rounded to the type of the values, the
// operand type of the product, and summed as rounded: the quotient is off by at most
// half a step of sum p |v - out|, and nothing where one key holds all weight.
//
// Keys and values come through LDS, in 16-key halves (a page holds whole halves)
// by buffer loads that write LDS directly, chunks of 16 bytes of row r at position
// c ^ f(r) so that the reads touch all banks. A workgroup has RW row groups of 16 MT
// rows, a wavefront each: one with four groups of keys, which take the tiles in turn
// and are merged at the end, or two or four that share every tile.
//
// Work. The tiles of all trees and key heads form one line that is cut into equal
// parts, so ragged contexts keep every CU as busy as equal ones. A part is taken by
// a team of workgroups, one for each tile of rows, on one XCD at the same time, so
// that the keys leave HBM once. An item that is cut leaves its parts' (maximum, sum,
// accumulators) in the workspace, and a second kernel merges them.
//
// What bounds it. 256 trees of 65 nodes on contexts of 1000 to 2900, 32 heads over 8:
// 827 us, 640 TFLOP/s, 2.9 TB/s of keys and values, of which its three workgroups a tree
// bring every key into LDS once each. A wavefront's round of 32 keys takes 3900 to 4500
// cycles beside the other one of its SIMD (scores 620 to 940, weights 580 to 760, values
// 590 to 770, eight loads 620 to 1100, waits and barriers 620 to 1100, stamped): the issue
// of instructions bounds it, a quarter of them those that load. Single tokens of 64
// sequences: 288 us, 5.5 TB/s, near the rate of a large read (5.85). One tree: 31.6 us;
// a part of it takes 25 thousand cycles, of which its rounds take 6.5 (the cut 4.4, queries
// 1.8, the first loads' issue 1.6, links and words 1, the key groups' merge and the part's
// way out 10), and one that goes on in the next key head's item all but the cut again.
//
// Over a cache of 4 bits, which is 3.76 times smaller: 256 trees of 65 nodes 843 us, bound as
// above (widened values are written to LDS, keys go into the products from registers). Single
// tokens of 64 sequences, whose contexts are as long as those above are not: 174 us, 5.2 TB/s of
// blocks and exponents in the kernel itself; one tree 36, bound as above. In heads of 128 some
// registers do not fit into a lane's 256 and are spilled: 17 for 48 rows of a workgroup (one tree), 7
// for 96 (256 trees), 2 for 192; in heads of 64, and over 16 bits, none.
//
// Heads of 72 to 120 are computed as heads of 128, padded with zeros in LDS (what they
// read is not): where instructions bound it they cost what 128 cost.
//
// A common prefix is an item of its own whose rows are those of all trees; its
// (maximum, sum, accumulators) wait in the workspace for the trees' own parts.
#pragma once

#include <mutex>

#include "tv.h"
#include "tv_attention_common.h"
#include "tv_launch.h"

namespace {

constexpr int kMergeWaves = 4, kMergeAhead = 8;
constexpr int kKeys = 32, kHalf = 16;     // keys of a tile and of a half
constexpr int kXcds = 8, kMaxCus = 256;
constexpr int kWavesPerCu = 8;            // resident wavefronts, two on a SIMD
constexpr int kMaxTeam = 32;              // workgroups of a team: the CUs of an XCD
// Of a part: smaller parts use more CUs and leave more to merge. One tree of 65 nodes by
// rows of 96, parts of 2 / 4 / 8 / 16 tiles: 41 / 34 / 36 / 42 us (parts merged one after
// the other), 8 / 16 / 32: 34 / 41 / 50 (eight at a time); by rows of 48, 8 / 16: 32 / 33.
constexpr int kMinTiles = 8;
// Up to how many nodes the rows' paths are kept as words (in LDS, 32 bytes a node): 256
// trees of 65 nodes 831 us, walked per tile 839.
constexpr int kWordNodes = 256;

// One pass: the trees over their own positions, or all their rows over the prefix.
struct Pass {
  const uint16_t* q;
  const uint16_t* k_new;
  const uint16_t* v_new;
  const uint8_t* k_cache;
  const uint8_t* v_cache;
  const int32_t* parents;
  const int32_t* table;
  const int32_t* ctx_len;       // in the prefix pass NULL, or that of `trees` trees: the table's
  int trees;                    // row of the first one that has the prefix names its pages
  uint16_t* out;
  int64_t q_stride, kv_stride;  // elements
  int64_t page_stride;          // bytes
  int num_pages, page_shift, table_width;
  int batch, num_nodes, heads, kv_heads, head_dim;
  int group;                    // query heads of a key head
  int rows;                     // query rows of a tree and key head
  int prefix_len;
  bool prefix_pass;
  int team, chunks, teams;      // row tiles of a team, teams' worth of row tiles, teams
  float k;                      // scale log2(e)
  float slack;                  // how far a score may exceed its frame
  float* parts;                 // [team][2][member]: accumulators, then (maximum, sum) per row
  i32x4* desc;                  // [team]: tree, key head, chunk, parts of the item cut before it
  float* pre;                   // prefix accumulators [row][DP]
  f32x2* pre_ml;                // their (maximum, sum)
};

// Q4: the cache holds 4 bits (see the kernel's loop over such tiles).
template <int DP_, int MT_, int RW_, int KW_, bool Q4_ = false>
struct Shape {
  static constexpr bool Q4 = Q4_;
  static constexpr int DP = DP_, MT = MT_, RW = RW_, KW = KW_;
  static constexpr int WAVES = RW * KW, THREADS = 64 * WAVES, PER_CU = kWavesPerCu / WAVES;
  static constexpr int BM = 16 * MT * RW;         // rows of a workgroup
  static constexpr int CH = DP / 8;               // 16-byte chunks of a row
  static constexpr int DB = DP / 16;              // 16-wide blocks of the head
  static constexpr int ROW = DP * 2;
  static constexpr int HALF = kHalf * ROW;        // bytes
  static constexpr int LOADS = HALF / 1024;       // load instructions of a half
  // a tile's keys and, VALUES behind them, its values (in 4 bits: its values alone)
  static constexpr int MAT = 2 * HALF, VALUES = Q4 ? 0 : MAT, STAGE = VALUES + MAT;
  // loads of a wavefront per tile, of keys (or values)
  static constexpr int MINE = 2 * LOADS / RW;
  // tiles in LDS per key group
  static constexpr int S = Q4 ? (RW == 1 ? 1 : 2) : DP == 128 ? RW : RW == 1 ? 2 : 4;
  // Loads younger than those a round waits for, in units of MINE (see the tiles' loop)
  static constexpr int YOUNGER = 2 * (S - 1) + (RW == 1 ? 1 : 0);
  static constexpr int RING = KW * S * STAGE;
  // accumulators and (maximum, sum) of the other key groups
  static constexpr int ACC = (KW - 1) * RW * MT * DB * 1024;
  static constexpr int MERGE = ACC + (KW - 1) * RW * MT * 64 * 8;
  static constexpr int MAIN = RING > MERGE ? RING : MERGE;
  // Trees of up to kWordNodes nodes: a word per node of the row tile and 32 nodes says
  // which of these are on its path, and the links are needed only to find them.
  static constexpr int PARENTS = MAIN;            // int16 per node
  static constexpr int WORDS = PARENTS + 2 * kWordNodes;
  static constexpr int WORDS_END = WORDS + BM * (kWordNodes / 8);
  static constexpr int PARENTS_END = PARENTS + 2 * TV_MAX_NODES;
  static constexpr int WALK = WORDS_END > PARENTS_END ? WORDS_END : PARENTS_END;
  static constexpr int FLAGS = WALK + 2 * WAVES * 16 * MT;
  static constexpr int SCAN = FLAGS + 4 * WAVES;
  static constexpr int BYTES = SCAN + 8 * (WAVES + 2) + 16;
  // floats of a part in the workspace
  static constexpr int PART_ACC = RW * MT * DB * 256;
  static constexpr int PART = PART_ACC + BM * 2 + 4;   // the last: values that are not finite
  static_assert(BYTES <= 160 * 1024 / PER_CU, "that many workgroups on a CU");
  static_assert(YOUNGER * MINE < 64, "the count of loads in flight");
};

// Positions of tree b that this pass reads from pages, where they start, and whether
// its table cannot hold its context.
struct Reach {
  int from, len, tiles;   // first position, positions, tiles with those of the nodes
  bool bad, shared;
};
__device__ __forceinline__ Reach reach(const Pass& P, int ctx) {
  Reach r{};
  if (P.prefix_pass) {
    r.len = P.prefix_len;
    r.tiles = (r.len + kKeys - 1) / kKeys;
    return r;
  }
  if (ctx < 0) return r;
  r.shared = P.prefix_len > 0 && ctx >= P.prefix_len;
  r.from = r.shared ? P.prefix_len : 0;
  r.bad = ctx > static_cast<long long>(P.table_width) << P.page_shift ||
          (ctx > r.from && P.num_pages == 0);
  r.len = r.bad ? 0 : ctx - r.from;
  r.tiles = (r.len + kKeys - 1) / kKeys + (P.num_nodes + kKeys - 1) / kKeys;
  return r;
}
__device__ __forceinline__ int context(const Pass& P, int b) {
  return P.prefix_pass ? 0 : ((CONSTANT(int)*)P.ctx_len)[b];
}

// Where part `t` of `parts` begins on the line of `total` tiles. (In double precision,
// a tenth of the instructions of a 64-bit division: every workgroup computes the same
// cuts, which grow with t and end at the total.)
__device__ __forceinline__ long long cut(long long total, int t, int parts) {
  return static_cast<long long>(static_cast<double>(total) * t / parts);
}

// Output index of row r of an item: (node of the pass, head).
__device__ __forceinline__ size_t out_row(const Pass& P, int b, int kh, int r) {
  const int node = r / P.group, g = r - node * P.group;
  return (static_cast<size_t>(b) * P.num_nodes + node) * P.heads + kh * P.group + g;
}

template <class T, class SH>
__device__ __forceinline__ void write_out(const Pass& P, size_t row, int d, const f32x4& o) {
  if (d >= P.head_dim) return;
  *reinterpret_cast<u32x2*>(P.out + row * P.head_dim + d) =
      u32x2{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
}

// Adds to elements d .. d + 3 of an output what of the values of its row's path is not
// finite (written by this lane before, from sums without them).
template <class T, class SH>
__device__ __forceinline__ void add_odd(const Pass& P, int b, int kh, int r, size_t row, int d) {
  if (d >= P.head_dim) return;
  float add[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t tree = static_cast<int64_t>(b) * P.num_nodes;
  for (int x = r / P.group; x >= 0;) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(P.v_new + (tree + x) * P.kv_stride +
                                                    kh * P.head_dim + d);
    for (int e = 0; e < 4; ++e) {
      const uint32_t u = v[e >> 1] >> (16 * (e & 1)) & 0xffffu;
      if ((u & T::kExponent) == T::kExponent) add[e] += T::value(static_cast<uint16_t>(u));
    }
    const int p = P.parents && x > 0 ? P.parents[tree + x] : -1;
    x = p < x ? p : -1;
  }
  u32x2* const at = reinterpret_cast<u32x2*>(P.out + row * P.head_dim + d);
  const u32x2 o = *at;
  float s[4];
  for (int e = 0; e < 4; ++e)
    s[e] = T::value(static_cast<uint16_t>(o[e >> 1] >> (16 * (e & 1)))) + add[e];
  *at = u32x2{T::pack(s[0], s[1]), T::pack(s[2], s[3])};
}

template <class T, class SH>
__global__ void __launch_bounds__(SH::THREADS, 2) attention_kernel(Pass P) {
  constexpr int MT = SH::MT, RW = SH::RW, KW = SH::KW, DB = SH::DB, KK = SH::DP / 32;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[SH::BYTES];
  lds_byte* const lds = (lds_byte*)smem;
  const int lds0 = static_cast<int>(reinterpret_cast<uintptr_t>(lds));
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % RW, kg = wave / RW;
  const int n = lane & 15, g = lane >> 4;

  // This workgroup's team and row tile. Workgroups are dealt to the XCDs in turn, and
  // so are the teams (a team on one XCD), so that little work uses all of them.
  const int per_xcd = P.teams / kXcds;
  const int in_xcd = blockIdx.x / kXcds;
  const int of_xcd = uniform(in_xcd / P.team), member = in_xcd - of_xcd * P.team;
  const int team = of_xcd * kXcds + static_cast<int>(blockIdx.x % kXcds);
  if (of_xcd >= per_xcd) return;

  // The line of tiles: how long, and where this team's part begins.
  LDS(long long)* const scan = (LDS(long long)*)(lds + SH::SCAN);
  LDS(int)* const found = (LDS(int)*)(scan + SH::WAVES + 2);
  const long long per_tile = static_cast<long long>(P.kv_heads) * P.chunks;
  const int per = (P.batch + SH::THREADS - 1) / SH::THREADS;
  const int b_lo = min(tid * per, P.batch), b_hi = min(b_lo + per, P.batch);
  long long own = 0;
  for (int b = b_lo; b < b_hi; ++b)
    own += reach(P, P.prefix_pass ? 0 : P.ctx_len[b]).tiles * per_tile;
  long long upto = own;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long long o = __shfl_up(upto, off, 64);
    if (lane >= off) upto += o;
  }
  if (lane == 63) scan[wave] = upto;
  barrier();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < SH::WAVES; ++w) {
    if (w < wave) upto += scan[w];
    total += scan[w];
  }
  total = uniform(total);
  const long long room = total / kMinTiles;
  const int parts = uniform(static_cast<int>(max<long long>(1, min<long long>(P.teams, room))));
  const bool idle = team >= parts || total == 0;
  const long long begin = idle ? 0 : uniform(cut(total, team, parts));
  const long long end = idle ? 0 : uniform(cut(total, team + 1, parts));
  if (idle) {
    if (member == 0 && tid == 0) P.desc[team] = i32x4{0, 0, 0, 0};
    return;
  }
  if (upto - own <= begin && begin < upto) {
    long long at = upto - own;
    for (int b = b_lo; b < b_hi; ++b) {
      const long long t = reach(P, P.prefix_pass ? 0 : P.ctx_len[b]).tiles * per_tile;
      if (begin < at + t) {
        scan[SH::WAVES] = begin - at;
        found[0] = b;
        break;
      }
      at += t;
    }
  }
  barrier();
  int b = uniform(found[0]);
  long long in_tree = uniform(scan[SH::WAVES]);

  // Loads: instruction i of a half fills 1024 bytes, this lane the chunk at position
  // lane % CH of row i * 1024 / ROW + lane / CH. Swizzle: sixteen rows' reads of one
  // chunk, and eight rows' reads of two neighbouring ones, touch all banks once.
  constexpr int kRowsPer = 1024 / SH::ROW;
  auto swizzle = [](int r) {
    return SH::DP == 128 ? (r & 7) << 1 | (r >> 3 & 1) : (r & 6) | (r >> 3 & 1);
  };
  auto offset = [&](int ln, int i, int last, int stride) {
    const int r = i * kRowsPer + ln / SH::CH;
    const int c = ln % SH::CH ^ swizzle(r);
    return 8 * c < P.head_dim && r <= last ? r * stride + 16 * c : kPastRange;
  };
  const int dbytes = P.head_dim * 2;
  // this wavefront's halves of a tile, and its loads of a half
  constexpr int kHalves = RW == 1 ? 2 : 1, kIn = RW == 4 ? SH::LOADS / 2 : SH::LOADS;
  const int h0 = RW == 4 ? rg >> 1 : RW == 2 ? rg : 0, in0 = RW == 4 ? (rg & 1) * kIn : 0;
  int kv_off[kIn];
#pragma unroll
  for (int i = 0; i < kIn; ++i) kv_off[i] = offset(lane, in0 + i, kHalf - 1, dbytes);
  // Reads: keys, row n of a block and chunk 4 kk + g; values, four keys 4 g .. 4 g + 3
  // by sixteen of the head, lane n's eight bytes at key n / 4, transposed by the read.
  const int k_at = n * SH::ROW + (g ^ swizzle(n)) * 16;
  const int vrow = 4 * g + (n >> 2);
  const int v_at = vrow * SH::ROW + (((n & 3) >> 1) ^ swizzle(vrow)) * 16 + (n & 1) * 8;
  LDS(int16_t)* const par = (LDS(int16_t)*)(lds + SH::PARENTS);
  LDS(uint32_t)* const word = (LDS(uint32_t)*)(lds + SH::WORDS);
  LDS(int)* const flags = (LDS(int)*)(lds + SH::FLAGS);
  // the next node on the path of each of this wavefront's rows
  LDS(int16_t)* const walk = (LDS(int16_t)*)(lds + SH::WALK) + wave * 16 * MT;

  int table_row = 0;            // of the prefix
  if (P.prefix_pass && P.ctx_len) {
    for (int b0 = 0; b0 < P.trees; b0 += 64) {
      const int at = min(b0 + lane, P.trees - 1);
      const uint64_t has = __builtin_amdgcn_ballot_w64(P.ctx_len[at] >= P.prefix_len);
      if (has) {
        table_row = min(b0 + __builtin_ctzll(has), P.trees - 1);
        break;
      }
    }
    table_row = uniform(table_row);
  }

  bool opened = false;
  int word_tree = -1, word_chunk = -1;   // whose words are there
  for (long long pos = begin; pos < end;) {
    // the item at pos
    const int ctx = context(P, b);
    const Reach R = reach(P, ctx);
    const long long in_all = R.tiles * per_tile;
    if (in_tree >= in_all) {      // (also trees without tiles)
      in_tree -= in_all;
      if (++b >= P.batch) break;
      continue;
    }
    int item = uniform(static_cast<int>(static_cast<double>(in_tree) / R.tiles));
    if (static_cast<long long>(item) * R.tiles > in_tree) --item;   // (rounded up)
    item = uniform(item);
    const int t0 = static_cast<int>(in_tree - static_cast<long long>(item) * R.tiles);
    const int kh = uniform(item / P.chunks), chunk = item - kh * P.chunks;
    const int t1 = static_cast<int>(min<long long>(R.tiles, t0 + (end - pos)));
    if (!opened) {
      opened = true;
      if (member == 0 && tid == 0) {
        // the item this part cuts, if no earlier part cuts it too
        const long long s = begin - t0, e = s + R.tiles;
        int count = 0;
        if (team > 0 && t0 > 0 && cut(total, team - 1, parts) <= s) {
          count = 2;
          while (team + count - 1 < parts && cut(total, team + count - 1, parts) < e) ++count;
        }
        P.desc[team] = i32x4{b, kh, chunk, count};
      }
    }
    pos += t1 - t0;
    in_tree += t1 - t0;
    const int row_tile = chunk * P.team + member;
    const int r0 = row_tile * SH::BM;
    if (r0 >= P.rows) continue;   // (for the whole workgroup)
    const int nct = (R.len + kKeys - 1) / kKeys;

    barrier();                    // the last item's merge is done
    // queries
    const int rbase = r0 + rg * 16 * MT;
    s16x8 q[MT][KK];
    const int qn = here(n), qg = here(g);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int r = min(rbase + 16 * mt + qn, P.rows - 1);
      const int node = r / P.group;
      walk[16 * mt + qn] = static_cast<int16_t>(node);   // (the prefix pass walks no paths)
      const uint16_t* src = P.q + (static_cast<int64_t>(b) * P.num_nodes + node) * P.q_stride +
                            (kh * P.group + r - node * P.group) * P.head_dim;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const int d = SH::Q4 ? 8 * (KK * qg + kk) : 32 * kk + 8 * qg;
        q[mt][kk] = d < P.head_dim ? *reinterpret_cast<const s16x8*>(src + d) : s16x8{};
      }
    }
    // What the first tile needs besides: its queries, and which nodes the rows see.
    const bool words = P.num_nodes <= kWordNodes;
    const int node0 = r0 / P.group;                        // the row tile's first node
    auto prepare = [&] {
      const bool nodes = t1 > nct && !P.prefix_pass && !(words && b == word_tree && chunk == word_chunk);
      if (nodes) {
        for (int i = tid; i < P.num_nodes; i += SH::THREADS) {
          const int p = P.parents && i > 0
                            ? P.parents[static_cast<size_t>(b) * P.num_nodes + i] : -1;
          par[i] = static_cast<int16_t>(p >= 0 && p < i ? p : -1);
        }
      }
      // (left to the compiler, the queries' wait would be at the first product of every
      // tile, and one for all loads in flight)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(q[mt][kk]));
      if (!nodes) return;
      barrier();
      if (words) {
        word_tree = b;
        word_chunk = chunk;
        const int last = (min(r0 + SH::BM, P.rows) - 1) / P.group;
        for (int i = tid; i <= last - node0; i += SH::THREADS) {
          int y = node0 + i;
#pragma unroll 1
          for (int w = (P.num_nodes - 1) / kKeys; w >= 0; --w) {
            uint32_t on = 0;
            for (; y >= w * kKeys; y = par[y]) on |= 1u << (y - w * kKeys);
            word[i * (kWordNodes / kKeys) + w] = on;
          }
        }
        barrier();
      }
    };

    // Loads of tile t: this wavefront's part of its keys (0) and values (1).
    CONSTANT(int)* const pages =
        (CONSTANT(int)*)(P.table + static_cast<size_t>(b + table_row) * P.table_width);
    uint32_t worst = 0;           // the largest page number seen
    bool odd = false;             // a node's value that is not finite
    const int ring = kg * SH::S * SH::STAGE;
    const int in_page = (1 << P.page_shift) - 1, nfull = R.len / kKeys;
    // bytes of a cached row's elements (in 4 bits: 16 a block of 32, their exponents behind the
    // page's elements)
    const int row_bytes = SH::Q4 ? P.head_dim >> 1 : dbytes;
    const int64_t of_head = (static_cast<int64_t>(kh) << P.page_shift) *
                            (SH::Q4 ? row_bytes + (P.head_dim >> 5) : row_bytes);
    const uint64_t k_base = reinterpret_cast<uint64_t>(P.k_cache + of_head);
    const uint64_t v_base = reinterpret_cast<uint64_t>(P.v_cache + of_head);
    const uint32_t page_bytes = static_cast<uint32_t>(P.page_stride);
    const int mine = max(0, (t1 - t0 - kg + KW - 1) / KW);   // tiles of this key group
    const int tile0 = t0 + kg, tile_end = tile0 + mine * KW, last_key = R.from + R.len - 1;
    auto first_key = [&](int t, int h) { return R.from + t * kKeys + h * kHalf; };
    int page[kHalves] = {};       // of the tile to load next
    auto fetch = [&](int t) {
      if (t < min(nct, tile_end)) {
#pragma unroll
        for (int hh = 0; hh < kHalves; ++hh)
          page[hh] = pages[min(first_key(t, h0 + hh), last_key) >> P.page_shift];
      }
    };
    // Where the tile to load lies: each half's keys, how much further the values are, its
    // last row (below 0: none) and the rows' distance. Rows behind the last are zeros: their
    // weight 0 must not meet a value that is not finite. A tile behind the last has no range:
    // its loads write zeros and read nothing, so that every round has the same loads in flight.
    uint64_t at_k[kHalves] = {};
    uint64_t to_v = 0;
    int last[kHalves] = {}, stride = dbytes, range = 0;
    bool plain = true;            // two full halves of a page
    auto key_at = [&](int page, int key) {          // (a page that is none: any other, to report)
      const uint32_t pg = static_cast<uint32_t>(page);
      worst = max(worst, pg);
      return k_base + static_cast<uint64_t>(min(pg, static_cast<uint32_t>(P.num_pages - 1))) *
                          page_bytes + static_cast<uint32_t>((key & in_page) * row_bytes);
    };
    auto place = [&](int t) {
      plain = t < nfull || t >= tile_end;
      range = t < tile_end ? kRange : 0;
      if (t < nct && t < tile_end) {
        to_v = v_base - k_base;
        stride = dbytes;
#pragma unroll
        for (int hh = 0; hh < kHalves; ++hh) {
          const int key = first_key(t, h0 + hh);
          last[hh] = last_key - key;
          at_k[hh] = key_at(page[hh], min(key, last_key));
        }
      } else if (t < tile_end) {                    // nodes, the last ones first
        to_v = reinterpret_cast<uint64_t>(P.v_new) - reinterpret_cast<uint64_t>(P.k_new);
        stride = static_cast<int>(P.kv_stride) * 2;
#pragma unroll
        for (int hh = 0; hh < kHalves; ++hh) {
          const int half = (R.tiles - 1 - t) * kKeys + (h0 + hh) * kHalf;
          const int from = min(half, P.num_nodes - 1);
          last[hh] = P.num_nodes - 1 - half;
          at_k[hh] = reinterpret_cast<uint64_t>(
              P.k_new + (static_cast<int64_t>(b) * P.num_nodes + from) * P.kv_stride +
              kh * P.head_dim);
        }
      }
    };
    auto issue = [&](int stage, bool values) {      // of the tile at that place
      const int to = lds0 + stage + h0 * SH::HALF + in0 * 1024 + (values ? SH::MAT : 0);
#pragma unroll
      for (int hh = 0; hh < kHalves; ++hh) {
        const uint64_t a = at_k[hh] + (values ? to_v : 0);
        const i32x4 rs = {static_cast<int>(a), static_cast<int>(a >> 32) & 0xffff, range, 0x00020000};
        if (plain) {
          load_to_lds<kIn>(rs, kv_off, to + hh * SH::HALF);
        } else {
          const int ln = here(lane);
#pragma unroll 1
          for (int i = 0; i < kIn; ++i) {
            const int voff[1] = {offset(ln, in0 + i, last[hh], stride)};
            load_to_lds<1>(rs, voff, to + hh * SH::HALF + i * 1024);
          }
        }
      }
    };

    float m[MT], l[MT], c[MT];
    f32x4 acc[DB][MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt] = -INFINITY;
      l[mt] = c[mt] = 0.0f;
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Scores of a tile and their weights.
    auto scores = [&](int stage, f32x4 (&s)[MT][2]) {
      const int at = stage + k_at;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        s[mt][0] = s[mt][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      // operand i: chunk group i / 2 of block i % 2; all reads before the first product
      constexpr int kOps = 2 * KK, kAhead = kOps - 1;
      s16x8 a[kAhead + 1];
      auto read = [&](auto i) {
        a[i.value % (kAhead + 1)] =
            *(const LDS(s16x8)*)(lds + (at ^ (64 * (i.value / 2))) + i.value % 2 * SH::HALF);
      };
      unrolled<kAhead>(read);
      unrolled<kOps>([&](auto ic) {
        constexpr int i = ic.value, kb = i % 2, kk = i / 2;
        if constexpr (i + kAhead < kOps) read(std::integral_constant<int, i + kAhead>{});
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][kb] = T::mfma(a[i % (kAhead + 1)], q[mt][kk], s[mt][kb]);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // A tile with keys that some rows do not see.
    auto mask = [&](int t, f32x4 (&s)[MT][2]) {
      const int hn = here(n), hg = here(g);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t w = 0;
        if (t < nct) {
          w = (1u << (R.len - t * kKeys)) - 1;
        } else {
          const int tile = R.tiles - 1 - t, lo = tile * kKeys;
          int y = walk[16 * mt + hn];
          if (words) {
            w = word[(y - node0) * (kWordNodes / kKeys) + tile];
          } else {                // walk the path down to this tile, then through it
            while (y >= lo + kKeys) y = par[y];
            for (; y >= lo; y = par[y]) w |= 1u << (y - lo);
            walk[16 * mt + hn] = static_cast<int16_t>(y);
          }
        }
        w >>= 4 * hg;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[mt][kb][r] = w >> (16 * kb + r) & 1 ? s[mt][kb][r] : -INFINITY;
      }
    };
    auto weights = [&](f32x4 (&s)[MT][2], s16x8 (&p)[MT]) {
      float top[MT];
      bool moves = false;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        top[mt] = max3(s[mt][0][0], s[mt][0][1], s[mt][0][2]);
        top[mt] = max3(top[mt], s[mt][0][3], s[mt][1][0]);
        top[mt] = max3(top[mt], s[mt][1][1], s[mt][1][2]);
        top[mt] = __builtin_elementwise_maximum(top[mt], s[mt][1][3]);
        moves |= top[mt] > m[mt] + P.slack;
      }
      if (__builtin_amdgcn_ballot_w64(moves)) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          float u = fmaxf(m[mt], top[mt]);
          u = fmaxf(u, __shfl_xor(u, 16, 64));
          u = fmaxf(u, __shfl_xor(u, 32, 64));
          // (a row whose own scores do not ask for it stays, whatever its neighbours' do)
          u = u > m[mt] + P.slack ? u : m[mt];
          const float f = to_frame<T>(m[mt], u, P.k);
          m[mt] = u;
          c[mt] = frame<T>(u, P.k);
          l[mt] *= f;
#pragma unroll
          for (int db = 0; db < DB; ++db) acc[db][mt] *= f;
        }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[mt][kb][r] = __builtin_amdgcn_exp2f(fmaf(s[mt][kb][r], P.k, c[mt]));
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = T::pack(s[mt][i >> 1][2 * (i & 1)], s[mt][i >> 1][2 * (i & 1) + 1]);
          l[mt] = T::plus(l[mt], w[i]);
        }
        p[mt] = __builtin_bit_cast(s16x8, w);
      }
    };
    // Values: the first kAhead operands are read before the weights are formed.
    constexpr int kAhead = DB / 2;
    auto read_values = [&](int stage, auto dbc, s16x8 (&a)[kAhead + 1]) {
      constexpr int db = dbc.value;
      const int at = (stage + SH::VALUES + v_at) ^ (32 * db);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS(s16x4)*)(lds + at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS(s16x4)*)(lds + at + SH::HALF));
      a[db % (kAhead + 1)] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // Nodes that a row does not see may hold anything: their weight 0 times NaN or
    // infinity must not reach the row. Such values enter the product as 0 and are
    // added to the rows that see them once these are written.
    auto clean = [&](int stage) {
      const int mat = stage + SH::VALUES;
      // (a half word's exponent of ones, plus one, carries into its sign's place)
      constexpr uint32_t kExp = T::kExponent * 0x10001u, kOne = (0x8000u - T::kExponent) * 0x10001u;
      const int hl = here(lane);
      uint32_t ones = 0;
#pragma unroll 2
      for (int i = 0; i < SH::MAT / 1024; ++i) {
        const u32x4 w = *(const LDS(u32x4)*)(lds + mat + 1024 * i + 16 * hl);
#pragma unroll
        for (int j = 0; j < 4; ++j) ones |= (w[j] & kExp) + kOne;
      }
      const bool some = ones & 0x80008000u;
      if (__builtin_amdgcn_ballot_w64(some)) {
#pragma unroll 1
        for (int i = hl; i < SH::MAT / 4; i += 64) {
          LDS(uint32_t)* const at = (LDS(uint32_t)*)(lds + mat + 4 * i);
          const uint32_t w = *at;
          *at = ((w & T::kExponent) == T::kExponent ? 0 : w & 0xffffu) |
                ((w >> 16 & T::kExponent) == T::kExponent ? 0 : w & 0xffff0000u);
        }
      }
      odd |= __builtin_amdgcn_ballot_w64(some) != 0;
    };
    auto add_values = [&](int stage, const s16x8 (&p)[MT], s16x8 (&a)[kAhead + 1]) {
      unrolled<DB>([&](auto dbc) {
        constexpr int db = dbc.value;
        if constexpr (db + kAhead < DB) read_values(stage, std::integral_constant<int, db + kAhead>{}, a);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          acc[db][mt] = T::mfma(a[db % (kAhead + 1)], p[mt], acc[db][mt]);
        __builtin_amdgcn_sched_barrier(0);
      });
    };

    const int rounds = (t1 - t0 + KW - 1) / KW;              // of the whole workgroup
    // What a tile multiplied at `stage` does to the accumulators.
    auto multiply = [&](auto full, int stage, int t, f32x4 (&s)[MT][2]) {
      s16x8 p[MT];
      if constexpr (!full.value) {
        if (t >= nfull) {
          mask(t, s);
          if (t >= nct) clean(stage);
        }
      }
      s16x8 v[kAhead + 1];
      unrolled<kAhead>([&](auto db) { read_values(stage, db, v); });
      weights(s, p);
      add_values(stage, p, v);
    };
    if constexpr (SH::Q4) {
      // A cached tile of 4 bits is read into registers kDeep rounds ahead and widened there.
      // Keys need no LDS: the products take the head's elements in the order in which lanes hold
      // them, lane (n, g) elements 8 KK g .. 8 KK (g + 1) - 1 of key n, eight of them each (the
      // queries are loaded in that order), and wavefronts that share tiles each read all of their
      // keys. Values are shared, kWords words and their exponent a lane, and widened into the
      // tile's place in LDS. Tiles of wavefronts that share take two places in turn: a place is
      // written once all have passed the barrier behind the products of the tile before it.
      //
      // Keys through LDS too: single tokens of 64 sequences 190 us, 256 trees of 65 nodes 870, four
      // chains of 6 in heads of 64 with a prefix 89; so 173, 847 and 83. Rounds ahead 1 / 2 / 3 / 4:
      // the first 173 / 175 / 176 / 178, the last, whose tiles are half as large, 87 / 83 / 83 / 84;
      // rows of 48 in heads of 128 spill 17 registers with one, and 77 with two (one tree 37 and 47 us).
      // (Four wavefronts of 16 rows on a SIMD, in 128 registers each, spill: 254 us.)
      constexpr int kDeep = SH::DP == 64 ? 2 : 1;
      constexpr int kAll = kKeys * SH::DP / 8 / 64;          // a lane's words of the tile
      constexpr int kWords = kAll >= 4 * RW ? 4 : 2;
      constexpr int kUnits = kAll / kWords, kOwn = (kUnits + RW - 1) / RW;
      constexpr int kPieces = SH::DP / 8 / kWords, kUnitRows = 64 / kPieces;
      typedef __attribute__((ext_vector_type(KK))) uint32_t key_words;
      typedef __attribute__((ext_vector_type(kWords))) uint32_t value_words;
      const int blocks = P.head_dim >> 5;
      const bool k_in = 8 * KK * g < P.head_dim;             // (else the zeros behind a head)
      const int k_off = n * row_bytes + 4 * KK * g, ke_off = n * blocks + KK * g / 4;
      const int piece = lane % kPieces, row = lane / kPieces;
      const bool v_in = 8 * kWords * piece < P.head_dim;
      const int v_off = (row & (kHalf - 1)) * row_bytes + 4 * kWords * piece;
      const int ve_off = (row & (kHalf - 1)) * blocks + kWords * piece / 4;
      key_words kw[kDeep][2] = {};
      value_words vw[kDeep][kOwn] = {};
      uint32_t ke[kDeep][2] = {}, ve[kDeep][kOwn] = {};
      int next[2] = {};                                      // pages of the tile to load next
      uint64_t at[2] = {};                                   // its halves' first rows
      uint32_t to_e[2] = {};                                 // from there to their exponents
      auto fetch4 = [&](int t) {
        if (t < min(nct, tile_end)) {
#pragma unroll
          for (int h = 0; h < 2; ++h) next[h] = pages[min(first_key(t, h), last_key) >> P.page_shift];
        }
      };
      auto place4 = [&](int t) {
        if (t >= min(nct, tile_end)) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = min(first_key(t, h), last_key) & ~(kHalf - 1);
          at[h] = key_at(next[h], key);
          to_e[h] = (static_cast<uint32_t>(row_bytes) << P.page_shift) -
                    static_cast<uint32_t>((key & in_page) * (row_bytes - blocks));
        }
      };
      auto load_keys = [&](auto to, int t) {
        if (t >= min(nct, tile_end)) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint8_t* const from = reinterpret_cast<const uint8_t*>(at[h]);
          if (k_in) {
            kw[to.value][h] = *reinterpret_cast<const key_words*>(from + k_off);
            ke[to.value][h] = (from + to_e[h])[ke_off];
          }
        }
      };
      auto load_values = [&](auto to, int t) {
        if (t >= min(nct, tile_end)) return;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
          const int u = rg + j * RW;
          if (u >= kUnits) continue;
          const int first = u * kUnitRows;
          // (units of 32 rows: lanes of both halves)
          const int h = kUnitRows == kKeys ? row >> 4 : first >> 4;
          const uint32_t skip = first & (kHalf - 1);
          const uint8_t* const from = reinterpret_cast<const uint8_t*>((h ? at[1] : at[0]) + (v_base - k_base));
          if (v_in) {
            vw[to.value][j] = *reinterpret_cast<const value_words*>(from + skip * row_bytes + v_off);
            ve[to.value][j] = (from + (h ? to_e[1] : to_e[0]) + skip * blocks)[ve_off];
          }
        }
      };
      auto widen = [&](auto held, int stage, int t) {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
          const int u = rg + j * RW;
          if (u >= kUnits) continue;
          const int at_row = u * kUnitRows + row, r = at_row & (kHalf - 1);
          value_words w = vw[held.value][j];
          // rows behind the last are zeros: their weight 0 must not meet a value that is not finite
          uint32_t e = ve[held.value][j];
          if (t >= nfull && first_key(t, 0) + at_row > last_key) {
            w = 0;
            e = 0;
          }
          const float f = __uint_as_float(e << 23);
          const int to = stage + (at_row >> 4) * SH::HALF + r * SH::ROW;
#pragma unroll
          for (int i = 0; i < kWords; ++i)
            *(LDS(u32x4)*)(lds + to + ((kWords * piece + i) ^ swizzle(r)) * 16) =
                u32x4{T::template widen<0>(w[i], f), T::template widen<1>(w[i], f),
                      T::template widen<2>(w[i], f), T::template widen<3>(w[i], f)};
        }
      };
      // A tile of nodes, which are not in 4 bits.
      auto put_nodes = [&](int stage, int t) {
        const int first = (R.tiles - 1 - t) * kKeys;
#pragma unroll 4
        for (int i = rg * 64 + lane; i < kKeys * SH::CH; i += 64 * RW) {
          const int c = i % SH::CH, r = i / SH::CH;
          const int x = first + r;
          u32x4 w = {0, 0, 0, 0};
          if (x < P.num_nodes && 8 * c < P.head_dim)
            w = *reinterpret_cast<const u32x4*>(
                P.v_new + (static_cast<int64_t>(b) * P.num_nodes + x) * P.kv_stride +
                kh * P.head_dim + 8 * c);
          *(LDS(u32x4)*)(lds + stage + (r >> 4) * SH::HALF + (r & 15) * SH::ROW +
                         (c ^ swizzle(r & 15)) * 16) = w;
        }
      };
      // Scores of a tile, operand (half, step) of `key`.
      auto scores4 = [&](f32x4 (&s)[MT][2], auto key) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][0] = s[mt][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        unrolled<2 * KK>([&](auto ic) {
          constexpr int i = ic.value, kb = i % 2, kk = i / 2;
          const s16x8 a = key(kb, kk);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) s[mt][kb] = T::mfma(a, q[mt][kk], s[mt][kb]);
        });
      };
      auto cached_scores = [&](auto held, f32x4 (&s)[MT][2]) {
        const float f[2] = {__uint_as_float(ke[held.value][0] << 23),
                            __uint_as_float(ke[held.value][1] << 23)};
        scores4(s, [&](int kb, int kk) {
          const uint32_t w = kw[held.value][kb][kk];
          return __builtin_bit_cast(
              s16x8, u32x4{T::template widen<0>(w, f[kb]), T::template widen<1>(w, f[kb]),
                           T::template widen<2>(w, f[kb]), T::template widen<3>(w, f[kb])});
        });
      };
      auto node_scores = [&](int t, f32x4 (&s)[MT][2]) {
        const int first = (R.tiles - 1 - t) * kKeys + here(n);
        const int hg = here(g);
        scores4(s, [&](int kb, int kk) {
          const int x = first + 16 * kb, d = 8 * (KK * hg + kk);
          return x < P.num_nodes && d < P.head_dim
                     ? *reinterpret_cast<const s16x8*>(
                           P.k_new + (static_cast<int64_t>(b) * P.num_nodes + x) * P.kv_stride +
                           kh * P.head_dim + d)
                     : s16x8{};
        });
      };
      fetch4(tile0);
      unrolled<kDeep>([&](auto j) {
        place4(tile0 + j.value * KW);
        load_values(j, tile0 + j.value * KW);
        load_keys(j, tile0 + j.value * KW);
        fetch4(tile0 + (j.value + 1) * KW);
      });
      prepare();
      constexpr int kLast = (SH::S - 1) * SH::STAGE;
      int stage = ring;
      auto round = [&](auto full, auto held, int i, int t) {
        f32x4 s[MT][2];
        place4(t + kDeep * KW);
        if (full.value || t < nct) widen(held, stage, t);
        else if (t < tile_end) put_nodes(stage, t);
        load_values(held, t + kDeep * KW);
        if (full.value || t < nct) cached_scores(held, s);
        else if (t < tile_end) node_scores(t, s);
        load_keys(held, t + kDeep * KW);
        fetch4(t + (kDeep + 1) * KW);
        if constexpr (RW == 1) wait_reads();
        else barrier();
        if (full.value || KW == 1 || i < mine) multiply(full, stage, t, s);
        if constexpr (RW == 1) wait_reads();
        stage = stage == ring + kLast ? ring : stage + SH::STAGE;
      };
      int i = 0, t = tile0;
#pragma unroll 1
      for (const int lim = min(nfull, tile_end) - (kDeep - 1) * KW; t < lim; i += kDeep, t += kDeep * KW)
        unrolled<kDeep>([&](auto j) { round(std::true_type{}, j, i + j.value, t + j.value * KW); });
#pragma unroll 1
      for (; i < rounds; i += kDeep, t += kDeep * KW)
        unrolled<kDeep>([&](auto j) {
          if (j.value == 0 || i + j.value < rounds) round(std::false_type{}, j, i + j.value, t + j.value * KW);
        });
    } else {
      // Round i multiplies tile i. Its keys' place is free after the first product and its
      // values' after the second, once all wavefronts that share them are there, and is
      // refilled at once with those of tile i + S: loads are issued in the order K_0, V_0,
      // K_1, ..., V_{i-1+S} at the top of round i and K_{i+S} in its middle (a wavefront
      // that shares with none issues before it waits, the others after the barrier). All
      // but the YOUNGER newest have landed when tile i's are there.
      constexpr int kSteady = SH::YOUNGER * SH::MINE;
#pragma unroll 1
      for (int j = 0; j < SH::S; ++j) {
        fetch(tile0 + j * KW);
        place(tile0 + j * KW);
        issue(ring + j * SH::STAGE, false);
        if (j < SH::S - 1) issue(ring + j * SH::STAGE, true);
      }
      prepare();
      constexpr int kLast = (SH::S - 1) * SH::STAGE;
      int stage = ring, before = ring + kLast;                 // places of tiles i and i - 1
      // hot: the tile itself and those it loads are full and lie in pages. Such rounds run
      // without branches, of which every instruction counts (general rounds alone: 844 us
      // where 256 trees take 831).
      auto round = [&](auto hot_c, int i, int t) {
        constexpr bool kHot = hot_c.value;
        f32x4 s[MT][2];
        auto load = [&](int stage, bool values) {
          if constexpr (!kHot) {
            issue(stage, values);
          } else {
            const int to = lds0 + stage + h0 * SH::HALF + in0 * 1024 + (values ? SH::MAT : 0);
#pragma unroll
            for (int hh = 0; hh < kHalves; ++hh) {
              const uint64_t a = at_k[hh] + (values ? v_base - k_base : 0);
              load_to_lds<kIn>(i32x4{static_cast<int>(a), static_cast<int>(a >> 32) & 0xffff, kRange,
                                     0x00020000}, kv_off, to + hh * SH::HALF);
            }
          }
        };
        if constexpr (RW == 1) {
          wait_reads();
          load(before, true);
          wait_loads<kSteady>();
        } else {
          wait_loads<kSteady>();
          barrier();
          load(before, true);
        }
        if constexpr (kHot) {
#pragma unroll
          for (int hh = 0; hh < kHalves; ++hh)
            page[hh] = pages[first_key(t + SH::S * KW, h0 + hh) >> P.page_shift];
        } else {
          fetch(t + SH::S * KW);
        }
        scores(stage, s);           // (of a tile that is none, behind this group's last: unused)
        if constexpr (kHot) {
#pragma unroll
          for (int hh = 0; hh < kHalves; ++hh)
            at_k[hh] = key_at(page[hh], first_key(t + SH::S * KW, h0 + hh));
        } else {
          place(t + SH::S * KW);
        }
        if constexpr (RW == 1) {
          wait_reads();
          load(stage, false);
          wait_loads<kSteady>();
        } else {
          wait_loads<kSteady>();
          barrier();
          load(stage, false);
        }
        if (kHot || KW == 1 || i < mine) multiply(hot_c, stage, t, s);
        before = stage;
        stage = stage == ring + kLast ? ring : stage + SH::STAGE;
      };
      int i = 0, t = tile0;
#pragma unroll 1
      for (const int lim = min(nfull, tile_end) - SH::S * KW; t < lim; ++i, t += KW)
        round(std::true_type{}, i, t);
      // (what the first of these loads is placed by the last round above, or before them)
#pragma unroll 1
      for (; i < rounds; ++i, t += KW) round(std::false_type{}, i, t);
      wait_loads<0>();            // (zeros for tiles that are none)
    }

    // The key groups' parts, merged by group 0.
    const int el = here(lane), en = el & 15, eg = el >> 4;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      l[mt] += __shfl_xor(l[mt], 16, 64);
      l[mt] += __shfl_xor(l[mt], 32, 64);
    }
    barrier();                    // all have read their last tile
    if (el == 0) flags[wave] = (R.bad || (P.num_pages > 0 && worst >= static_cast<uint32_t>(P.num_pages))) | odd << 1;
    if (kg > 0) {
      const int w = (kg - 1) * RW + rg;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
          *(LDS(f32x4)*)(lds + ((w * MT + mt) * DB + db) * 1024 + el * 16) = acc[db][mt];
        *(LDS(f32x2)*)(lds + SH::ACC + (w * MT + mt) * 512 + el * 8) = f32x2{m[mt], l[mt]};
      }
    }
    barrier();
    int any = 0;
#pragma unroll
    for (int w = 0; w < SH::WAVES; ++w) any |= flags[w];
    if (kg == 0) {
      const bool whole = t0 == 0 && t1 == R.tiles;
      const size_t part = (static_cast<size_t>(team) * 2 + (t0 > 0 ? 0 : 1)) * P.team + member;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        f32x2 o[KW];
        float top = m[mt];
#pragma unroll
        for (int j = 1; j < KW; ++j) {
          o[j] = *(const LDS(f32x2)*)(lds + SH::ACC + (((j - 1) * RW + rg) * MT + mt) * 512 + el * 8);
          top = fmaxf(top, o[j][0]);
        }
        const float f = to_frame<T>(m[mt], top, P.k);
        m[mt] = top;
        l[mt] *= f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db][mt] *= f;
#pragma unroll
        for (int j = 1; j < KW; ++j) {
          const float fj = to_frame<T>(o[j][0], top, P.k);
          l[mt] += o[j][1] * fj;
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            acc[db][mt] += fj * *(const LDS(f32x4)*)(
                lds + ((((j - 1) * RW + rg) * MT + mt) * DB + db) * 1024 + el * 16);
            if (db % 4 == 3) __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (any & 1) {
          m[mt] = 0.0f;
          l[mt] = NAN;
        }
        const int r = rbase + 16 * mt + en;
        if (!whole) {
          float* const to = P.parts + part * SH::PART;
#pragma unroll
          for (int db = 0; db < DB; ++db)
            *reinterpret_cast<f32x4*>(to + ((rg * MT + mt) * DB + db) * 256 + el * 4) = acc[db][mt];
          if (eg == 0)
            *reinterpret_cast<f32x2*>(to + SH::PART_ACC + ((rg * MT + mt) * 16 + en) * 2) =
                f32x2{m[mt], l[mt]};
          if (mt == 0 && rg == 0 && el == 0) to[SH::PART - 1] = any & 2 ? 1.0f : 0.0f;
        } else if (r < P.rows) {
          const size_t row = out_row(P, b, kh, r);
          if (P.prefix_pass) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
              *reinterpret_cast<f32x4*>(P.pre + row * SH::DP + 16 * db + 4 * eg) = acc[db][mt];
            if (eg == 0) P.pre_ml[row] = f32x2{m[mt], l[mt]};
          } else {
            if (R.shared) {       // the prefix' part: all of it read before a row is written
              f32x4 pre[DB];
              const f32x2 ml = P.pre_ml[row];
#pragma unroll
              for (int db = 0; db < DB; ++db)
                pre[db] = *reinterpret_cast<const f32x4*>(P.pre + row * SH::DP + 16 * db + 4 * eg);
              const float both = fmaxf(m[mt], ml[0]);
              const float own = to_frame<T>(m[mt], both, P.k), theirs = to_frame<T>(ml[0], both, P.k);
              l[mt] = l[mt] * own + ml[1] * theirs;
#pragma unroll
              for (int db = 0; db < DB; ++db) acc[db][mt] = acc[db][mt] * own + pre[db] * theirs;
            }
            const float inv = 1.0f / l[mt];
#pragma unroll
            for (int db = 0; db < DB; ++db)
              write_out<T, SH>(P, row, 16 * db + 4 * eg, acc[db][mt] * inv);
          }
        }
      }
      if (whole && any & 2 && !P.prefix_pass) {
#pragma unroll 1
        for (int i = 0; i < MT * DB; ++i) {
          const int r = rbase + 16 * (i / DB) + en;
          if (r < P.rows) add_odd<T, SH>(P, b, kh, r, out_row(P, b, kh, r), 16 * (i % DB) + 4 * eg);
        }
      }
    }
  }
}

// Merges the parts of the item that team blockIdx.x's part cuts first: workgroup y
// one block of 16 rows of the item's, a wavefront a quarter of the head.
template <class T, class SH>
__global__ void __launch_bounds__(64 * kMergeWaves) merge_kernel(Pass P) {
  constexpr int DBW = SH::DB / kMergeWaves;     // blocks of the head per wavefront
  const int team = blockIdx.x;
  const i32x4 d = P.desc[team];
  const int count = d[3];
  if (count == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const int member = blockIdx.y / (SH::RW * SH::MT), block = blockIdx.y % (SH::RW * SH::MT);
  const int r = (d[2] * P.team + member) * SH::BM + 16 * block + n;
  if (r - n >= P.rows) return;
  // part i: the end of the team before, then the starts of this one and those behind
  auto part = [&](int i) {
    const size_t at = i == 0 ? (static_cast<size_t>(team - 1) * 2 + 1)
                             : static_cast<size_t>(team + i - 1) * 2;
    return P.parts + (at * P.team + member) * SH::PART;
  };
  // kMergeAhead parts at a time, all their loads in flight: a part comes from another
  // XCD, and one after the other 16 of them took 50 us.
  float m = -INFINITY, l = 0.0f;
  bool odd = false;
  f32x4 acc[DBW];
#pragma unroll
  for (int k = 0; k < DBW; ++k) acc[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int i0 = 0; i0 < count; i0 += kMergeAhead) {
    f32x2 ml[kMergeAhead];
    f32x4 of[kMergeAhead][DBW];
    float flag[kMergeAhead];
#pragma unroll
    for (int j = 0; j < kMergeAhead; ++j) {
      const float* const from = part(min(i0 + j, count - 1));
      ml[j] = *reinterpret_cast<const f32x2*>(from + SH::PART_ACC + (block * 16 + n) * 2);
      flag[j] = from[SH::PART - 1];
#pragma unroll
      for (int k = 0; k < DBW; ++k)
        of[j][k] = *reinterpret_cast<const f32x4*>(
            from + (block * SH::DB + wave * DBW + k) * 256 + lane * 4);
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < kMergeAhead; ++j) top = fmaxf(top, ml[j][0]);
    const float f = to_frame<T>(m, top, P.k);
    m = top;
    l *= f;
#pragma unroll
    for (int k = 0; k < DBW; ++k) acc[k] *= f;
#pragma unroll
    for (int j = 0; j < kMergeAhead; ++j) {
      if (i0 + j >= count) continue;
      const float fj = to_frame<T>(ml[j][0], top, P.k);
      l += ml[j][1] * fj;
      odd |= flag[j] != 0.0f;
#pragma unroll
      for (int k = 0; k < DBW; ++k) acc[k] += fj * of[j][k];
    }
  }
  if (r >= P.rows) return;
  const int b = d[0];
  const size_t row = out_row(P, b, d[1], r);
  const int db0 = wave * DBW;
  if (P.prefix_pass) {
    for (int k = 0; k < DBW; ++k)
      *reinterpret_cast<f32x4*>(P.pre + row * SH::DP + 16 * (db0 + k) + 4 * g) = acc[k];
    if (g == 0 && wave == 0) P.pre_ml[row] = f32x2{m, l};
    return;
  }
  f32x2 ml = {-INFINITY, 0.0f};
  const bool shared = P.prefix_len > 0 && P.ctx_len[b] >= P.prefix_len;
  if (shared) ml = P.pre_ml[row];
  const float both = fmaxf(m, ml[0]);
  const float own = to_frame<T>(m, both, P.k), pre = to_frame<T>(ml[0], both, P.k);
  const float inv = 1.0f / (l * own + ml[1] * pre);
  if (shared)
#pragma unroll
    for (int k = 0; k < DBW; ++k)
      acc[k] = acc[k] * own +
               pre * *reinterpret_cast<const f32x4*>(P.pre + row * SH::DP + 16 * (db0 + k) + 4 * g);
#pragma unroll
  for (int k = 0; k < DBW; ++k) {
    const int at = 16 * (db0 + k) + 4 * g;
    write_out<T, SH>(P, row, at, acc[k] * inv);
    if (odd) add_odd<T, SH>(P, b, d[1], r, row, at);
  }
}

// Rows per workgroup for `items` (trees times key heads) of `rows` query rows: 16, 32 or
// 48 of one wavefront's width, or two or four of 48, whichever pads less. A workgroup of
// 48 has four groups of keys, so a wavefront reads all its keys and values for 48 rows
// alone; one of 192 has one, which its wavefronts share, and a part is a wavefront's, not
// a workgroup's. Batch 256, contexts of 2048, 32 heads over 8, by 48 / 96 / 192 rows:
// 260 rows 1038 / 809 / 927 us, 192 rows 649 / 486 / 467, 128 rows 517 / 467 / 443.
// (Other contexts were not compared: on long ones few items have rounds enough that 96
// rows may be the better choice for them too.) Few items are cut into many parts, of which 48 rows leave a quarter as many to merge:
// contexts of 4096, by 48 or else, 260 rows of 8 / 16 / 32 / 64 items 33 or 47, 37 or 51,
// 55 or 57, 74 or 71 us; 192 rows of 32 / 64 / 128 items 41 or 81, 54 or 89, 75 or 92.
int block_rows(int64_t rows, int64_t items) {
  if (rows <= 16) return 16;
  if (rows <= 32) return 32;
  if (rows <= 48 || (rows + 47) / 48 * items <= kMaxCus) return 48;
  const int64_t two = (rows + 95) / 96 * 96, four = (rows + 191) / 192 * 192;
  return four <= two ? 192 : 96;
}

struct Plan {
  int rows_per_wg, team, chunks, teams;
  size_t parts_bytes;
};
Plan plan(int64_t rows, int64_t items, int padded, int cus) {
  Plan p{};
  p.rows_per_wg = block_rows(rows, items);
  const int64_t tiles = (rows + p.rows_per_wg - 1) / p.rows_per_wg;
  p.chunks = static_cast<int>((tiles + kMaxTeam - 1) / kMaxTeam);
  p.team = static_cast<int>((tiles + p.chunks - 1) / p.chunks);
  const int per_xcd = cus / kXcds * (p.rows_per_wg == 96 ? 4 : 2);   // workgroups resident
  p.teams = per_xcd / p.team * kXcds;
  p.parts_bytes = static_cast<size_t>(p.teams) * 2 * p.team *
                  (static_cast<size_t>(p.rows_per_wg) * (padded + 2) + 4) * sizeof(float);
  return p;
}

struct Layout {
  size_t desc, parts, pre, pre_ml, bytes;
};
Layout layout(int64_t batch, int num_nodes, int heads, int kv_heads, int head_dim, int prefix_len) {
  const int padded = head_dim <= 64 ? 64 : 128;
  const int64_t rows = static_cast<int64_t>(num_nodes) * (heads / kv_heads);
  Layout L{};
  L.desc = 0;
  L.parts = tv::align256(kMaxCus * kWavesPerCu * sizeof(i32x4));
  size_t parts = plan(rows, batch * kv_heads, padded, kMaxCus).parts_bytes;
  if (prefix_len > 0) {
    const size_t p = plan(rows * batch, kv_heads, padded, kMaxCus).parts_bytes;
    parts = parts > p ? parts : p;
  }
  L.pre = tv::align256(L.parts + parts);
  const size_t all = prefix_len > 0 ? static_cast<size_t>(batch) * num_nodes * heads : 0;
  L.pre_ml = tv::align256(L.pre + all * padded * sizeof(float));
  L.bytes = tv::align256(L.pre_ml + all * sizeof(f32x2));
  return L;
}

// CUs of the current device, in whole XCDs and at most kMaxCus; 0 on failure.
int device_cus() {
  constexpr int kMaxDevices = 64;
  static int cus[kMaxDevices];
  static std::mutex mu;
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
  std::lock_guard<std::mutex> lock(mu);
  if (dev < kMaxDevices && cus[dev]) return cus[dev];
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
  n = n > kMaxCus ? kMaxCus : n / kXcds * kXcds;
  // (fewer: the teams of an XCD still need room for the largest one)
  if (n < kMaxTeam / 2 * kXcds) n = kMaxTeam / 2 * kXcds;
  if (dev < kMaxDevices) cus[dev] = n;
  return n;
}

template <class T, class SH>
hipError_t run(const Pass& P, hipStream_t stream) {
  const unsigned wgs = static_cast<unsigned>(P.teams * P.team);
  // whole rounds over the XCDs: every XCD has teams / 8 teams
  hipLaunchKernelGGL((attention_kernel<T, SH>), dim3(wgs), dim3(SH::THREADS), 0, stream, P);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((merge_kernel<T, SH>),
                     dim3(static_cast<unsigned>(P.teams), static_cast<unsigned>(P.team * SH::RW * SH::MT)),
                     dim3(64 * kMergeWaves), 0, stream, P);
  return hipGetLastError();
}

template <class T, int DP, bool Q4>
hipError_t run_rows(const Pass& P, int rows_per_wg, hipStream_t stream) {
  switch (rows_per_wg) {
    case 16: return run<T, Shape<DP, 1, 1, 4, Q4>>(P, stream);
    case 32: return run<T, Shape<DP, 2, 1, 4, Q4>>(P, stream);
    case 48: return run<T, Shape<DP, 3, 1, 4, Q4>>(P, stream);
    case 96: return run<T, Shape<DP, 3, 2, 1, Q4>>(P, stream);
    default: return run<T, Shape<DP, 3, 4, 1, Q4>>(P, stream);
  }
}

template <bool Q4>
hipError_t run_pass(Pass P, int dtype, int cus, hipStream_t stream) {
  const int padded = P.head_dim <= 64 ? 64 : 128;
  const int64_t items = P.prefix_pass ? P.kv_heads : static_cast<int64_t>(P.batch) * P.kv_heads;
  const Plan p = plan(P.rows, items, padded, cus);
  P.team = p.team;
  P.chunks = p.chunks;
  P.teams = p.teams;
  if (dtype == TV_DTYPE_BF16)
    return padded == 64 ? run_rows<Bf16, 64, Q4>(P, p.rows_per_wg, stream)
                        : run_rows<Bf16, 128, Q4>(P, p.rows_per_wg, stream);
  return padded == 64 ? run_rows<F16, 64, Q4>(P, p.rows_per_wg, stream)
                      : run_rows<F16, 128, Q4>(P, p.rows_per_wg, stream);
}

// Enqueues the attention (page_stride in bytes).
template <bool Q4>
int launch(const tv::AttentionArgs& a, void* workspace, hipStream_t stream) {
  const int cus = device_cus();
  if (!cus) return TV_ERR_HIP;
  const Layout L = layout(a.batch, a.num_nodes, a.heads, a.kv_heads, a.head_dim, a.prefix_len);
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  Pass P{};
  P.q = static_cast<const uint16_t*>(a.q);
  P.k_new = static_cast<const uint16_t*>(a.k_new);
  P.v_new = static_cast<const uint16_t*>(a.v_new);
  P.k_cache = static_cast<const uint8_t*>(a.k_cache);
  P.v_cache = static_cast<const uint8_t*>(a.v_cache);
  P.parents = a.num_nodes > 1 ? a.parents : nullptr;
  P.table = a.block_table;
  P.ctx_len = a.ctx_len;
  P.out = static_cast<uint16_t*>(a.out);
  P.q_stride = a.q_stride;
  P.kv_stride = a.kv_stride;
  P.page_stride = a.page_stride;
  P.num_pages = a.num_pages;
  P.page_shift = 31 - __builtin_clz(static_cast<unsigned>(a.page_size));
  P.table_width = a.table_width;
  P.batch = a.batch;
  P.num_nodes = a.num_nodes;
  P.heads = a.heads;
  P.kv_heads = a.kv_heads;
  P.head_dim = a.head_dim;
  P.group = a.heads / a.kv_heads;
  P.rows = a.num_nodes * P.group;
  // (without pages a tree that has a context has bad ones, the prefix among them, and so has
  // a tree with a prefix that its table cannot hold)
  P.prefix_len = a.num_pages > 0 && a.prefix_len <= a.table_width * a.page_size ? a.prefix_len : 0;
  P.k = static_cast<float>(static_cast<double>(a.scale) * 1.4426950408889634);
  const double slack = 8.0 / static_cast<double>(P.k);
  P.slack = slack < 3.0e38 ? static_cast<float>(slack) : 3.0e38f;
  P.desc = reinterpret_cast<i32x4*>(ws + L.desc);
  P.parts = reinterpret_cast<float*>(ws + L.parts);
  P.pre = reinterpret_cast<float*>(ws + L.pre);
  P.pre_ml = reinterpret_cast<f32x2*>(ws + L.pre_ml);
  if (P.prefix_len > 0) {
    Pass X = P;
    X.prefix_pass = true;
    X.table = a.prefix_pages;
    X.table_width = 0;
    X.ctx_len = nullptr;
    if (a.prefix_pages == a.block_table) {
      X.table_width = a.table_width;
      X.ctx_len = a.ctx_len;
      X.trees = a.batch;
    }
    X.parents = nullptr;
    X.batch = 1;
    X.num_nodes = a.batch * a.num_nodes;
    X.rows = a.batch * P.rows;
    if (run_pass<Q4>(X, a.dtype, cus, stream) != hipSuccess) return TV_ERR_HIP;
  }
  return run_pass<Q4>(P, a.dtype, cus, stream) == hipSuccess ? TV_OK : TV_ERR_HIP;
}

}  // namespace
