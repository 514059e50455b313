// Host run of the shared decode's plan (host_plan.cpp).
//
//   plan H DH DV DC DR DTYPE P B PAGES PREFIX
//       prints the plan: whether the decode of the layer runs on the 16-bit matrix cores, whether each part of the
//       shared one does, tiled, fused, splits of the prefix, its row blocks, workspace bytes
//   layer H DH DV DC DR DTYPE
//       every batch up to 300 (and some larger): fails where a part's kernel family is not that of the layer's decode
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

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
  if (argc == 8 && !std::strcmp(argv[1], "layer")) return families(argv + 2);
  return 2;
}
