// Host run of the shared decode's plan (host_plan.cpp).
//
//   plan H DH DV DC DR DTYPE P B PAGES PREFIX
//       prints the plan: whether the decode of the layer runs on the 16-bit matrix cores, whether each part of the
//       shared one does, tiled, fused, splits of the prefix, its row blocks, workspace bytes
//   sizes H DH DV DC DR DTYPE P B PAGES PREFIX
//       batches, own pages and prefix pages up to these: fails where a smaller call asks for a larger workspace, or
//       where its partial rows leave it
//   layer H DH DV DC DR DTYPE
//       every batch up to 300 (and some larger): fails where a part's kernel family is not that of the layer's decode
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>
#include <vector>

#include "host_plan.h"

using namespace egmla;

namespace {

eg_mla_dims layer(char** v, int page) {
  eg_mla_dims d = {};
  d.num_heads = std::atoi(v[0]);
  d.head_dim = std::atoi(v[1]);
  d.v_head_dim = std::atoi(v[2]);
  d.latent_dim = d.gate_dim = std::atoi(v[3]);
  d.rope_dim = std::atoi(v[4]);
  d.dtype = std::atoi(v[5]);
  d.vocab_size = 1000;
  d.page_size = page;
  return d;
}

// 0: vector kernel, 1: fp32 matrix cores, 2: 16-bit matrix cores
int family(const DecodePlan& p) { return p.path == EG_MLA_PATH_MFMA ? 2 : p.f32_mfma ? 1 : 0; }

int plan(char** v) {
  const eg_mla_dims d = layer(v, std::atoi(v[6]));
  const int B = std::atoi(v[7]), pages = std::atoi(v[8]), prefix = std::atoi(v[9]);
  DecodePlan one;
  SharedPlan p;
  if (make_decode_plan(d, B, pages, nullptr, &one) != EG_MLA_OK || make_shared_plan(d, B, pages, prefix, &p) != EG_MLA_OK)
    return 2;
  std::printf("%d %d %d %d %d %d %d %zu\n", family(one), p.tiled ? 2 : family(p.pre), family(p.own), p.tiled ? 1 : 0,
              p.fused ? 1 : 0, p.splits, p.row_blocks, p.bytes);
  return 0;
}

// Whether what a plan lays out ends within its workspace.
bool fits(const eg_mla_dims& d, int B, const SharedPlan& p) {
  if (p.plain) return p.own.bytes <= p.bytes;
  const size_t rows = static_cast<size_t>(B) * d.num_heads, dc = d.latent_dim;
  const size_t n = p.tiled ? rows * p.splits : p.pre.capacity ? rows * p.pre.s_max : 0;
  const size_t pre_end = p.pre.off_o + n * dc * (p.half_rows ? 2 : 4);
  size_t own_end = 0;
  if (p.own.capacity && !p.fused) {
    const size_t m = p.own.balanced ? (static_cast<size_t>(kWideMaxGroups) + B) * d.num_heads : rows * p.own.s_max;
    own_end = p.own.off_o + m * dc * (p.own.balanced ? 2 : 4);
    if (p.pre.off_ml + n * 8 > p.pre.off_o || pre_end > p.own.off_ml || p.own.off_ml + m * 8 > p.own.off_o) return false;
  }
  const size_t tiles = p.tiled ? p.off_tiles + (static_cast<size_t>(p.pre.capacity) + p.keys - 1) / p.keys * p.keys *
                                                   (prefix_latent_row(d.latent_dim) + 128) : 0;
  return p.pre.off_ml + n * 8 <= p.pre.off_o && pre_end <= p.bytes && own_end <= p.bytes &&
         (!p.tiled || tiles <= (p.fused ? p.off_rows : p.pre.off_ml));
}

int sizes(char** v) {
  const eg_mla_dims d = layer(v, std::atoi(v[6]));
  const int B = std::atoi(v[7]), pages = std::atoi(v[8]), prefix = std::atoi(v[9]);
  // the largest of every (batch, pages, prefix) so far, along each of the three
  std::vector<int> ws, ps, bs;
  for (int w = 0; w <= pages; w += 1 + w / 5) ws.push_back(w);
  for (int x = 0; x <= prefix; x += 1 + x / 5) ps.push_back(x);
  for (int b = 1; b <= B; b += 1 + b / 40) bs.push_back(b);
  std::vector<size_t> most(ws.size() * ps.size(), 0);
  for (int b : bs)
    for (size_t i = 0; i < ws.size(); ++i)
      for (size_t j = 0; j < ps.size(); ++j) {
        SharedPlan p;
        if (make_shared_plan(d, b, ws[i], ps[j], &p) != EG_MLA_OK) return 2;
        size_t m = most[i * ps.size() + j];
        if (i) m = std::max(m, most[(i - 1) * ps.size() + j]);
        if (j) m = std::max(m, most[i * ps.size() + j - 1]);
        if (p.bytes < m || !fits(d, b, p)) {
          std::printf("%d sequences, %d pages, prefix of %d: %zu bytes, a smaller call %zu; %s\n", b, ws[i], ps[j],
                      p.bytes, m, fits(d, b, p) ? "fits" : "does not fit");
          return 1;
        }
        most[i * ps.size() + j] = p.bytes;
      }
  std::printf("0\n");
  return 0;
}

int families(char** v) {
  const eg_mla_dims d = layer(v, 64);
  for (int B = 1; B <= 300; ++B)
    for (int pages : {1, 4, 50})
      for (int prefix : {1, 7, 300}) {
        DecodePlan one;
        SharedPlan p;
        if (make_decode_plan(d, B, pages, nullptr, &one) != EG_MLA_OK || make_shared_plan(d, B, pages, prefix, &p) != EG_MLA_OK)
          return 2;
        if ((p.tiled ? 2 : family(p.pre)) != family(one) || family(p.own) != family(one)) {
          std::printf("%d sequences, %d pages, prefix of %d: decode %d, prefix %d, own tokens %d\n", B, pages, prefix,
                      family(one), p.tiled ? 2 : family(p.pre), family(p.own));
          return 1;
        }
      }
  std::printf("0\n");
  return 0;
}

}  // namespace

int main(int argc, char** argv) {
  if (argc == 12 && !std::strcmp(argv[1], "plan")) return plan(argv + 2);
  if (argc == 12 && !std::strcmp(argv[1], "sizes")) return sizes(argv + 2);
  if (argc == 8 && !std::strcmp(argv[1], "layer")) return families(argv + 2);
  return 2;
}
