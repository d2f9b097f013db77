// Arguments of the learning kernels (learn.hip), shared with their host driver (networks.cpp).
//
// Rows. A genome's edges are laid out four times, by destination ("in") and by source ("out"), the ones
// from input nodes apart from the others ("inp", "hid"): an input holds still over the steps, so its edges
// count once where the others count in every step. A row is a node with its edges of one kind. Rows
// lie in slices of sixteen places, the heavy ones first:
//   - a heavy slice holds one row of many edges (more than light_edges; the output nodes of "in" always),
//     its edge k at base + k: the lanes of a wave share it and add their sums at the end;
//   - a light slice holds sixteen rows, the edge k of its row r at base + 16 k + r, so that the
//     lanes of a wave, a row each, read sixteen edges side by side; rows come in falling order of
//     edges, which leaves few places empty.
// An empty place has the weight 0 and, as the other node, the one past the genome's last, whose values
// are zeros.
#pragma once
#include <stdint.h>

#include "network.h"

namespace emr {

// Gradients. The edges a second time, grouped by their source.
struct NetTurnArgs {
  const int64_t* in_offset;  // [nodes + 1]
  const uint32_t* in_src;    // [edges]
  uint32_t* key;             // [edges] source
  uint64_t* val;             // [edges] edge | destination << 32
  uint32_t* dst;             // [edges] destination
  const uint32_t* skey;      // sorted by source, each group in edge order
  int64_t* out_offset;       // [nodes + 1]
  int64_t nodes, edges;
};

// A genome that does not fit a workgroup: a launch per step, derivatives by the node sums ("gz") as
// [pblocks][its nodes] float4.
struct NetBackArgs {
  uint32_t genome;
  int64_t node0, size;         // its nodes
  int64_t edge0, edge1;        // its edges
  const int32_t* node_in;
  const int32_t* out_node;     // [n_outputs]
  const int64_t* in_offset;
  const uint32_t* in_src;
  const float* in_w;
  const uint32_t* dst;         // [edges]
  const int64_t* out_offset;   // [nodes + 1]
  const uint64_t* out_edge;    // [edges] edge | destination << 32
  const float* patterns;       // [n_patterns * n_inputs]
  const float* outputs;        // [n_genomes * n_patterns * n_outputs]
  const float* grad_outputs;   // the same
  const float* gz;             // derivatives after the step
  float* gz_before;            // before it
  float* grad_w;               // [edges]
  float* grad_inputs;          // [n_genomes * n_patterns * n_inputs] or NULL
  NetKept kept;
  int64_t nodes;               // of all genomes
  uint32_t n_inputs, n_outputs, n_patterns;
  uint32_t pblocks;
  uint32_t step;               // 1 .. steps: the step whose derivatives gz holds
  uint32_t last;               // whether it is the first one looked at: gradients are set, not added to
};

constexpr uint32_t kLayoutBins = 1024;  // of rows by edges (learn.hip)
// Edges of a light row, at most: four times the mean, so that no slice is much longer than the others. (Rows
// over the mean as heavy ones: a wave's sum and setup for each made the gradients three times as long.)
inline constexpr uint32_t light_edges(uint32_t edges, uint32_t rows) {
  const uint32_t four = 4u * (edges / (rows < 16u ? 16u : rows) + 1u);
  return four < 64u ? 64u : (four < kLayoutBins - 3u ? four : kLayoutBins - 3u);
}
constexpr uint32_t kLearnPad = 4;  // a slice's length is a multiple of this
constexpr int kInHid = 0, kInInp = 1, kOutHid = 2, kOutInp = 3, kSets = 4;
constexpr uint32_t kNoEdge = 0xFFFFFFFFu;

struct LearnSlice {
  uint32_t base;   // first place, from the genome's on
  uint32_t len;    // sixteens of places
  uint32_t first;  // (out) the sixteens that reach output nodes, which come first in a row
  uint32_t heavy;
};

// One of the four layouts; a genome's places start at place[g], its slices at slice[g].
struct LearnSet {
  uint2* ent;          // other node (local) | weight bits
  uint32_t* edge;      // edge number, or kNoEdge
  LearnSlice* slices;
  uint16_t* rows;      // [slice * 16] local nodes (heavy: the same one), kNoRow: none
  uint32_t* n_slices;  // [n_genomes]
  uint32_t* n_heavy;   // [n_genomes] of them
  uint32_t* n_places;  // [n_genomes]
};
constexpr uint32_t kNoRow = 0xFFFFu;

// A workgroup's block of patterns: a row has `lanes` lanes with four of them each. The values of a genome's
// nodes before a step lie in LDS, those after it and a third array (the input edges' sums, the sum of the
// steps' derivatives) there too (local), or in memory. With eight lanes a node's values are the 128 bytes
// that LDS delivers at a time, whatever nodes a wave's rows read.
struct LearnShape {
  uint32_t lanes, local;
};
constexpr LearnShape kLearnShapes[] = {{1, 1}, {1, 0}, {2, 1}, {2, 0}, {4, 1}, {4, 0}, {8, 1}, {8, 0}};
constexpr uint32_t kLearnLds = 160u * 1024u;
inline constexpr uint32_t learn_lds(uint32_t n, const LearnShape& S) {
  return (n + 1u) * 16u * S.lanes * (S.local ? 3u : 1u);
}
constexpr uint32_t kLearnNodes = kLearnLds / 16u - 1u;  // the most nodes of a genome that any shape takes

// Places and slices of one of a genome's layouts, at most: a slice's length is rounded up by up to kLearnPad - 1
// sixteens; a heavy row (of more than 64 edges) or an output leaves up to fifteen places more; falling rows
// leave sixteen times the first one's edges, of which light_edges is the bound.
inline constexpr int64_t learn_slices(int64_t n, int64_t e, int64_t n_out) {
  return n / 16 + 2 + e / 64 + n_out;
}
inline constexpr int64_t learn_places(int64_t n, int64_t e, int64_t n_out) {
  const int64_t most = e / 4 + 4 < (int64_t)kLayoutBins ? e / 4 + 4 : (int64_t)kLayoutBins;
  const int64_t light = e < (most < 64 ? 64 : most) ? e : (most < 64 ? 64 : most);
  const int64_t used = e < n ? e : n;  // (rows with edges)
  return (e + 15 * (e / 64 + n_out) + 16 * light + 16 * (kLearnPad - 1) * learn_slices(used, e, n_out) + 31) /
         16 * 16;
}
// Places of a genome's two layouts by source together, at most: what an item's sums take. Of a layout of E
// edges in R rows, h rows have more than L = light_edges(E, R); each takes up to 15 + 16 (kLearnPad - 1) places
// more than it has edges, and there are at most E / 65 of them, and at most R / 4 (R: 16 at least) + E / 1022.
// A light slice's rows have no more edges than any row of the slice before, so the light ones take their edges,
// 16 times the first slice's (L at most), and 16 (kLearnPad - 1) places for each slice that has edges. (A multiple
// of 64 floats: with sums of 64-byte alignment alone, three stepped genomes' gradients took 312 us for 306.)
inline constexpr int64_t learn_sums(int64_t n, int64_t e) {
  const int64_t by_edges = e / 65, by_rows = (n + 32) / 4 + e / 1022 + 2;
  const int64_t heavy = by_edges < by_rows ? by_edges : by_rows;
  const int64_t most = e / 4 + 4 < (int64_t)kLayoutBins - 3 ? e / 4 + 4 : (int64_t)kLayoutBins - 3;
  const int64_t first = 2 * (most < 64 ? 64 : most);
  const int64_t used = e < n ? e : n;  // (rows with edges)
  return (e + heavy * (15 + 16 * (kLearnPad - 1)) + 16 * (e < first ? e : first) +
          16 * (kLearnPad - 1) * (used / 16 + 2) + 63) / 64 * 64;
}
struct LearnRow {
  int64_t place;   // of its first edge
  uint32_t node0;  // the genome's first node
  uint32_t slice;  // of the genome (while rows are ranked: the row's rank); bit 31: heavy; kNoEdge: no row
};
struct LearnLayoutArgs {
  LearnSet set;
  int32_t which;
  uint32_t* key;               // [nodes] edges of the node's row, or kNoEdge
  LearnRow* row;               // [nodes]
  const uint32_t* genomes;     // [count]
  const int64_t* place;        // [n_genomes]
  const int64_t* slice;        // [n_genomes]
  const int64_t* node_offset;
  const int32_t* node_in;
  const int32_t* out_node;
  const int64_t* in_offset;
  const uint32_t* in_src;
  const float* in_w;
  const int64_t* out_offset;
  const uint64_t* out_edge;    // [edges] edge | destination << 32
  int64_t nodes;
  uint32_t count, n_outputs, n_sub;
};

// The weights of laid out places, after the edges' changed.
struct LearnWeightsArgs {
  LearnSet set[kSets];
  const uint32_t* genomes;
  const int64_t* place;
  const float* in_w;
  uint32_t count;
};

// A workgroup's share: blocks of patterns b0 .. b1 - 1 of one genome. The weights' derivatives of its share
// are summed at partial + part (places of kOutHid, then of kOutInp).
struct LearnItem {
  uint32_t genome, b0, b1;
  uint16_t shape;     // of kLearnShapes
  uint16_t alone;     // the genome has no other item: its derivatives go to grad_w directly
  int64_t part;
  int64_t values;     // (not local) in float4: [2][node][lanes]
};

// The genomes of more than one item.
struct LearnJoin {
  uint32_t genome, items;
  int64_t part, stride;  // its items' partial sums
};

struct LearnFillArgs {
  float* p;
  int64_t n;
};

// A workgroup of a step's launch: every chunks-th unit of rows of a genome for the blocks b0 .. b1 - 1 of 4
// `lanes` patterns.
struct LearnStepItem {
  uint32_t genome, b0, b1, chunk, chunks, lanes;
  int64_t values;  // of the genome's first block, in float4: [block][node][lanes] in each of the three arrays
  int64_t part;
};

// Kept states as numbers.
struct KeptValuesArgs {
  NetKept kept;
  int64_t nodes;
  uint32_t n_patterns;
  int32_t type;   // EMR_F32, EMR_BF16, EMR_F16
  void* out;      // [planes][nodes][n_patterns]
};

struct LearnArgs {
  LearnSet set[kSets];
  const LearnItem* items;
  const LearnJoin* joins;
  const int64_t* place;
  const int64_t* slice;
  const int64_t* node_offset;
  const int32_t* node_in;
  const int32_t* out_node;
  const float* patterns;       // [n_patterns * n_inputs]
  float* outputs;              // [n_genomes * n_patterns * n_outputs] (keep: written)
  const float* grad_outputs;
  float* partial;
  float* grad_w;
  float* grad_inputs;          // or NULL
  NetKept kept;
  int64_t nodes;
  uint32_t n_inputs, n_outputs, n_patterns, n_sub;
  uint32_t steps;
  uint32_t first_item, n_items, n_joins;
  uint32_t threads, lds_bytes;
  float4* values;              // (not local)
  // a step's launch
  const LearnStepItem* step_items;
  const float4 *cur;           // values before it (derivatives after it), and the others
  float4 *nxt, *held;          // held: the input edges' sums (the sum of the steps' derivatives)
  uint32_t step;               // 1 .. steps, or (gradients) 1: the input edges
};

}  // namespace emr
