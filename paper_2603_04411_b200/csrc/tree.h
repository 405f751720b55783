// Attention of drafted trees over the cache (tree_*.cu): one call's arguments, its tables and its buffers in the caller's workspace.
//
// A request is a sequence and the nodes of its tree.  The nodes' own states lie in two tiles of the workspace, one of keys and one
// of values, beside the sequence's tiles in the cache; a score row is a token's (or node's) scores with all query rows of the request:
//   column (g Rs + t rep + h): KV head g, node t, query head h of the group; Rs = max_nodes rep rounded up to 4, beyond 4 to 8
// and rows lie in the order of the request's V tiles (in the order of the sequence's list, the nodes' tile behind them), 128 a tile.
#pragma once
#include <cuda.h>
#include "twkv_dev.h"

namespace twkv {

// The tensor core cuts its fp32 sum toward zero after every instruction: an expected loss of half a unit in the last place, 0.36 x 2^-23 of the sum's
// size (averaged over mantissas), and of the final sum half of that per instruction, whether the sum grows steadily or wanders.  The kernels give that
// expected loss back as a factor 1 + TREE_CUT x instructions, of which only those count that can have cut something: a
// key's by its class, those of the last product by the widest class of the row's splits and by the parts that its components have.  Errors of fp32 outputs, without / with it for the keys alone: 4 sequences of 700 tokens
// 1.3e-6 / 5.2e-7 (plain fp32 sums: 6.8e-7), 2 of 8192 tokens 1.1e-6 / 6.9e-7 (1.7e-6).
constexpr float TREE_CUT = 2.15e-8f;
// Sums of weighted values lose a fifth less, and next to nothing to the largest of three bf16 parts, whose products have sixteen bits and mostly fit the
// sum: two instructions of sixteen tokens count, with two parts or three.  (With 2.15e-8 and every part counted, chains of 144 and 384 instructions
// of bf16 came out 1.4e-6 and 3.2e-6 too large, of 272 and 1024 of fp16 1.1e-6 and 4.6e-6.)
// Which of them count follows from the weights (tree_value.cu).  What it cannot see are values whose sums are exact (components that few tokens have): those
// come out too large by what is given back, 1.75e-8 for an instruction, up to the drain below.
constexpr float TREE_CUT_VALUES = 1.75e-8f;
// Boxes of sixteen tokens that an accumulator of the value kernel takes before it is emptied, for fp32 outputs (of bf16 caches, whose three parts lengthen the
// chains) and 16-bit ones: what the expectation leaves grows with the chain.  (By boxes, since the tiles of mixed ranks hold one or two of them: eight
// tiles of each took 313 us and 7.0e-7 for 48 x 100 tokens of any rank, 48 boxes 275 us and 7.3e-7.)  Error and time of fp32 outputs with 24 / 32 / 48:
// 64 x 1024 tokens fp16 5.5e-7 147 us / 7.1e-7 147 us / 8.9e-7 143 us (plain fp32 sums 7.4e-7), bf16 6.2e-7 161 us / 8.6e-7 160 us / 1.1e-6 152 us (6.5e-7);
// 16 x 2048 of any rank fp16 6.2e-7 198 us / 7.4e-7 192 us / 9.0e-7 181 us (1.1e-6), bf16 6.7e-7 237 us / 8.6e-7 227 us / 1.2e-6 211 us (9.4e-7).
constexpr int TREE_DRAIN_F32 = 48, TREE_DRAIN_F32_BF16 = 24, TREE_DRAIN_16 = 1024;
constexpr int TREE_MAX_RANGES = 4;               // ranges of panels whose sums a CTA of the value kernel keeps
constexpr int TREE_MAX_SPLITS = 64;              // of a request's V tiles
constexpr int TREE_PANEL_ROWS = 64;              // rows of a panel of the nodes' tiles
static_assert(TWKV_TREE_MAX_NODES <= TREE_PANEL_ROWS && TWKV_TREE_MAX_NODES <= 64, "a node is a bit of a 64-bit word, and a row of a panel");
// K list entry: .x tile in the cache / ~ number of a joint tile / score tile of the nodes, .y class | flags | tokens << 16, .z first block
// (nodes: first row of the panels), .w request
constexpr int TREE_NODES = 0x4000, TREE_FILLER = 0x8000, TREE_CLASS = 0x1f;

struct TreeCall {
  // the caller's
  const unsigned short *q, *K, *V, *levels;
  const int *req_seqs, *offsets, *positions;
  const unsigned long long* masks;
  void* out;
  int n_rows;           // rows of q, K, V, levels, positions, masks, out
  // this pass: requests r0 .. r0 + n_req - 1 of the call
  int r0, n_req;
  int T;                // most nodes of a request
  int R, Rs, Rp;        // query rows of a KV head: T rep; score columns; operand rows (R rounded up to 16)
  int C;                // columns of a score row, Hkv Rs
  int n_splits;
  int entries;          // room of a request in the K list
  int q_box;            // rows of qop that a CTA takes at a time
  int m_cluster, m_rows, m_comps;     // CTAs of a cluster of the merge, query rows of a cluster, components that each CTA takes at a time
  int n_parts;          // parts that a weight, and a component of the merge, goes into products as
  int drain;            // boxes of sixteen tokens that an accumulator of the value kernel takes before it is emptied
  int range;            // panels whose sums a CTA of the value kernel keeps
  int v_box;            // score columns that a CTA of the value kernel takes, at most 128
  // workspace
  unsigned short* qop;  // [n_req][Hkv][Rp][128] f16 queries in the order of the score contraction
  unsigned char *nk, *nv;     // [n_req][NC][64 rows][64] panels of the nodes' keys and values
  float* scores;        // [n_req][TPS + 1][128][C]
  int4* info;           // [n_req] first row, nodes, sequence (-1: refused), splits that hold tiles
  unsigned long long* bad;    // [n_req] nodes whose values are not finite
  unsigned long long* seers;  // [n_req][64] the nodes that see a node: bit t of entry k = bit k of node t's mask
  int4* klist;          // entries of all requests, a request's from an even place on
  int4* vmeta;          // [n_req][TPS + 1] V tiles in stride order: score tile, class, tokens, first block (-1: the nodes)
  int* vcut;            // [n_req][n_splits + 1]
  int *cta_start, *parts;     // [pieces + 1] first item part of a piece; parts of an item
  float* part_acc;      // [n_req][T][n_splits][Hq][d_kv]
  float4* part_m;       // [n_req][T][n_splits][Hq] what the split's weights are relative to (powers of two), per range of panels
  float* part_l;        // [n_req][T][n_splits][Hq] sum of the split's weights
  float4* part_x;       // [n_req][T][n_splits][Hq] size of the largest component of the split's sums, per range of panels (fp16 caches)
  int* part_cls;        // [n_req][n_splits] widest class of the split's tiles, 0: none
};

// The cache's blocks (whole panels, sixteen rows of one), the nodes' keys (128 rows) and values (sixteen rows), U_K^-1 (half panels), the
// queries, U_V^-1 (m_comps rows, 64 columns), the scores (a tile's rows or sixteen of them, v_box columns).
struct TreeMaps { CUtensorMap blocks, boxes, nodes, node_boxes, uinvT, q, uv, scores, score_boxes; };

// Two fp32 (packed) as three bf16 each: the nearest value, that of the rest, that of what is left then (24 bits in all).
__device__ __forceinline__ void tree_split3(uint64_t v, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  asm("{\n\t.reg .f32 a, b, c, d;\n\t.reg .b16 p, q, m;\n\tmov.b64 {a, b}, %3;\n\tmov.b16 m, 0xBF80;\n\t"
      "cvt.rn.bf16x2.f32 %0, b, a;\n\tmov.b32 {p, q}, %0;\n\tfma.rn.f32.bf16 c, p, m, a;\n\tfma.rn.f32.bf16 d, q, m, b;\n\t"
      "cvt.rn.bf16x2.f32 %1, d, c;\n\tmov.b32 {p, q}, %1;\n\tfma.rn.f32.bf16 a, p, m, c;\n\tfma.rn.f32.bf16 b, q, m, d;\n\t"
      "cvt.rn.bf16x2.f32 %2, b, a;\n\t}" : "=&r"(hi), "=&r"(mid), "=r"(lo) : "l"(v));
}

// Rows of tree i; false where the offsets do not describe at most max_nodes rows of n_rows.
__device__ __forceinline__ bool tree_rows(const int* offsets, int i, int n_rows, int max_nodes, int* first, int* n) {
  const int a = offsets[i], b = offsets[i + 1];
  const bool ok = a >= 0 && a <= b && b <= n_rows && b - a <= max_nodes;
  *first = ok ? a : 0;
  *n = ok ? b - a : 0;
  return ok;
}

cudaError_t launch_slot_map(const DevView& v, int layer, const int* req_seqs, const int* req_lens, const int* starts, int n_req, int max_rows,
                            int* offsets, int* seq_ids, int* positions, int sm_count, cudaStream_t st);
cudaError_t launch_tree_map(const DevView& v, const int* offsets, const int* parents, int n_req, int n_rows, int max_nodes, int* positions,
                            unsigned long long* masks, cudaStream_t st);
cudaError_t launch_tree_accept(const DevView& v, const int* offsets, const int* parents, const int* draft, const int* target, int n_req, int n_rows,
                               int max_nodes, int* n_accepted, int* rows, int* next_tokens, cudaStream_t st);
cudaError_t launch_tree_plan(const DevView& v, const TreeCall& a, int layer, int n_pieces, int sm_count, cudaStream_t st);
cudaError_t launch_tree_score(const DevView& v, const TreeCall& a, const TreeMaps& maps, int layer, int n_pieces, cudaStream_t st);
int tree_max_pairs(int sm_count);
int tree_query_box(const TreeCall& a);
int tree_merge_cluster(const DevView& v, const TreeCall& a, int sm_count, int* rows);
int tree_merge_comps(int d_kv, int cl, int parts);
int tree_value_range(int parts);
cudaError_t launch_tree_value(const DevView& v, const TreeCall& a, const TreeMaps& maps, cudaStream_t st);
cudaError_t launch_tree_merge(const DevView& v, const TreeCall& a, const TreeMaps& maps, cudaStream_t st);

}  // namespace twkv
