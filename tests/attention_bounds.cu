// Host program of tests/test_serving_edges.py: asks for the visible nodes of every row of every row tile, with the mask at
// the very end of a mapping (what lies behind it is not mapped, so a read past the mask ends the process).
//   attention_bounds N group B stride_per_sequence(0/1) with_mask(0/1)
// Prints, per (kernel, sequence, row, tile): nothing if all bits are as they should be; "wrong ..." otherwise.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <sys/mman.h>

#include "../paper_2506_04708_b200/csrc/attention_plain.cuh"
#include "../paper_2506_04708_b200/csrc/attention_tensor.cuh"

using namespace stand;

int main(int argc, char** argv) {
  if (argc != 6) return 2;
  AttnParams p = {};
  p.N = atoi(argv[1]);
  p.group = atoi(argv[2]);
  p.B = atoi(argv[3]);
  p.mask_words = (p.N + 31) / 32;
  const bool own = atoi(argv[4]) != 0, masked = atoi(argv[5]) != 0;
  const size_t per = (size_t)p.N * p.mask_words, words = per * (own ? p.B : 1), page = 4096;
  const size_t bytes = (words * 4 + page - 1) / page * page;
  char* at = (char*)mmap(nullptr, bytes + page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
  if (at == MAP_FAILED || mprotect(at + bytes, page, PROT_NONE) != 0) return 2;
  uint32_t* mask = (uint32_t*)(at + bytes) - words;
  srand(1);
  for (size_t i = 0; i < words; ++i) mask[i] = (uint32_t)rand() * 2654435761u;
  p.mask = masked ? mask : nullptr;
  p.mask_stride = own ? (long long)per : 0;

  int wrong = 0;
  auto walk = [&](const char* kernel, int tile_rows, int step) {  // rows in tiles of tile_rows, nodes `step` at a time
    const int rows = p.N * p.group;
    for (int b = 0; b < p.B; ++b)
      for (int row0 = 0; row0 < rows; row0 += tile_rows)
        for (int row = 0; row < tile_rows; ++row) {
          const int u = row0 / p.group + row / p.group;  // tiles of the first kernel begin with whole nodes
          const int node = step == 32 && tile_rows == PA_ROWS ? (row0 + row) / p.group : u;
          for (int first = 0; first < (p.N + TA_KT - 1) / TA_KT * TA_KT; first += step) {
            const uint32_t got = attn_nodes_seen(p, b, node, first);
            for (int i = 0; i < step; ++i) {
              const int v = first + i;
              bool want = node < p.N && v <= node;
              if (want && masked) want = mask[(own ? (size_t)b * per : 0) + (size_t)node * p.mask_words + v / 32] >> v % 32 & 1u;
              if ((got >> i & 1u) != (uint32_t)want && wrong++ < 5) printf("wrong %s b %d node %d sees %d\n", kernel, b, node, v);
            }
          }
        }
  };
  for (int step = 16; step <= 32 && p.group <= TA_ROWS; step += 16) walk("tensor", tensor_tile_rows(p.N, p.group), step);
  walk("plain", PA_ROWS, 32);
  return wrong ? 1 : 0;
}
