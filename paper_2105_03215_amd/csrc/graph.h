// Subgraph IR: the parsed and validated form of a serialized composite-op
// list (the JSON graph representation of Sec. 3.3, Option 1).  Host only;
// nothing here touches the device.
#pragma once

#include <cstdint>
#include <string>
#include <vector>

#include "../../include/byoc.h"

namespace byoc {

struct Status {
  byoc_status code = BYOC_OK;
  std::string msg;
  bool ok() const { return code == BYOC_OK; }
  static Status Ok() { return Status(); }
  static Status Err(byoc_status c, std::string m) {
    Status s;
    s.code = c;
    s.msg = std::move(m);
    return s;
  }
};

// I8: the compute type of a partially quantized graph (int8 codes with an
// affine scale and zero point per tensor); never an external dtype.
// I32: an index input (token positions, sequence lengths).
enum class DType { F32 = BYOC_F32, BF16 = BYOC_BF16, I8 = 2, I32 = BYOC_I32 };
enum class Act { None = 0, Relu = 1, Relu6 = 2, Gelu = 3, Leaky = 4 };
// AvgPool: global average pool; AvgPoolWin: windowed average pool.
enum class OpKind { Conv, Dense, MaxPool, AvgPool, Add, AvgPoolWin, Concat, QDense, Rotary, Attention,
                    MxDense, Logits };

// A named tensor of the graph: a subgraph input, a constant or a node output.
struct Value {
  std::string name;
  std::vector<int64_t> shape;  // external layout: NCHW or [M, K]
  DType dtype = DType::F32;
  enum Source { Input, Const, Node } source = Input;
  int index = -1;  // input number, constant index or node number
  // int8 graphs: affine codes of this tensor, value = qscale * (code - qzero)
  bool has_q = false;
  double qscale = 0.0;
  int qzero = 0;
  bool param = false;  // an f32 input that nodes read in place, whatever the graph's compute type
};

struct Node {
  std::string name;
  std::string composite;
  OpKind op = OpKind::Conv;
  bool has_bias = false;
  bool has_add = false;
  Act act = Act::None;
  float alpha = 0.1f;  // leaky ReLU slope (attrs.alpha)
  int data = -1, weight = -1, bias = -1, residual = -1, other = -1;  // value ids
  int out = -1;                                                      // value id
  int stride[2] = {1, 1};
  int pad[4] = {0, 0, 0, 0};  // top, left, bottom, right
  int pool[2] = {1, 1};
  int groups = 1;
  bool depthwise = false;
  bool count_include_pad = false;  // AvgPoolWin
  std::vector<int> cat;            // Concat: the joined values, in channel order
  // Rotary, Attention: packed heads (data: the rotated rows, or the queries)
  int index = -1;                  // value id of the positions or lengths (i32 input, -1: none)
  int parents = -1;                // Attention of a tree: value ids of the drafted tokens' parents,
  int key2 = -1, value2 = -1;      //   and of their keys and values (key, value: the cache)
  int key = -1, value = -1;        // Attention: value ids of keys and values
  int weight2 = -1;                // Rotary with norm: the key heads' weight (weight: the query heads')
  int heads = 0, kv_heads = 0, head_dim = 0;
  int batch = 1, q_len = 0, k_len = 0;
  int cols[5] = {0, 0, 0, 0, 0};   // Attention: first column of the queries, keys, values, drafted keys and values
  double scale = 0.0;              // Attention: of the scores
  bool causal = false;
  bool norm = false, interleaved = false;
  int rotary_dim = 0;
  double eps = 1e-6;
  std::vector<double> theta;       // Rotary: angle per position of each pair
  double mag = 1.0;                // factor on the rotated values
  // Logits: what is applied, and the value ids that it reads (-1: none); has_bias: the biases
  bool penalties = false, drafts = false, mask = false;
  int history = -1, prompts = -1, strengths = -1;  // lengths in index, the drafted tokens' parents in parents
  int draft_tokens = -1, bias_tokens = -1, bias_values = -1, mask_words = -1;
  int64_t macs = 0;

  // every value that the node reads as an activation or index, in no order
  std::vector<int> inputs() const {
    std::vector<int> r;
    for (int v : {data, residual, other, key, value, key2, value2, index, parents, history, prompts, strengths, draft_tokens,
                  bias_tokens, bias_values, mask_words})
      if (v >= 0) r.push_back(v);
    for (size_t k = 1; k < cat.size(); ++k) r.push_back(cat[k]);
    return r;
  }
};

struct IoDesc {
  int value = -1;
  DType dtype = DType::F32;
  byoc_layout layout = BYOC_NCHW;
};

struct Graph {
  std::vector<Value> values;
  std::vector<Node> nodes;
  std::vector<IoDesc> inputs;
  std::vector<IoDesc> outputs;
  std::vector<int> const_values;  // value id of constant index i
  DType compute = DType::BF16;
  int64_t macs = 0;
};

// Parses and validates text against the constants.  consts may be NULL when
// n_consts is 0.  Pure host code.
Status parse_graph(const char* json, size_t len, const byoc_const* consts, int32_t n_consts,
                   Graph* out);

const char* act_name(Act a);

}  // namespace byoc
