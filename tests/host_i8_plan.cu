// Host-only: which kernel and tile stb_gemm_i8 takes for each "n m T" among the arguments (compiled with nvcc, run on the CPU, no GPU needed).
// One line each: gemv split (0: another kernel), pair kernel or not, tokens of a tile, tiles along the tokens, log2 of the parts of K.
#include <cstdio>
#include <cstdlib>

#include "../paper_2408_01803_b200/csrc/stb_i8.cu"

int main(int argc, char** argv) {
  for (int i = 1; i + 2 < argc; i += 3) {
    const int n = atoi(argv[i]), m = atoi(argv[i + 1]), T = atoi(argv[i + 2]);
    const stb::I8Plan p = stb::i8_plan(n, m, T);
    printf("%d %d %d %d %d\n", stb::gemv_i8_split(n, m, T), p.pair ? 1 : 0, p.bn, p.ttiles, p.lks);
  }
  return 0;
}
