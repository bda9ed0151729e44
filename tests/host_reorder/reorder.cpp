// tss_seq_reorder and tss_get_beams on a context put together by hand (test only): what they answer
// without the operators' kernels (no argument), where no launch holds the work ("refuse") and where
// one does ("fit").  No device work: the launchers below report success and the pool is an address.
// Prints "status message" of each call, then the sequences' lengths.
#include <cstdio>
#include <cstring>

#include "tss_host.cpp"

#ifdef WITH_KERNELS
static bool g_fit = false;
namespace tss {
bool reorder_fits(const ReorderArgs&) { return g_fit; }
hipError_t launch_reorder(const ReorderArgs&, hipStream_t) { return hipSuccess; }
bool beams_fit(int, int, int) { return g_fit; }
size_t beams_bytes(int, int, int, int) { return (size_t)1 << 40; }
hipError_t launch_beams(const BeamArgs&, void*, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace tss
#endif

int main(int argc, char** argv) {
#ifdef WITH_KERNELS
  g_fit = argc > 1 && !std::strcmp(argv[1], "fit");
#endif
  (void)argc, (void)argv;
  static uint8_t pool[16];
  tss_ctx c;
  c.cfg.n_layers = 1;
  c.cfg.n_heads = 4;
  c.cfg.head_dim = 64;
  c.cfg.vocab = 100;
  c.kv = pool;
  c.kvl.pages_per_seq = 8;
  c.kvl.n_pages = 24;
  c.n_seqs = 3;
  c.n_kv = {40, 50, 60};
  c.kv_len = {{40}, {50}, {60}};
  c.mask = {{1}, {1}, {1}};
  c.window.resize(3);
  c.last_M = 4;
  const int32_t seqs[3] = {0, 1, 2}, parents[3] = {1, 1, 0};
  std::printf("%d %s\n", tss_seq_reorder(&c, seqs, parents, 3, 32), c.err.c_str());
  std::printf("%d %d %d\n", c.n_kv[0], c.n_kv[1], c.n_kv[2]);
  const float scores[4] = {};
  float score[2];
  int32_t parent[2], token[2];
  c.err.clear();
  std::printf("%d %s\n", tss_get_beams(&c, 1, 4, scores, nullptr, 0, 2, score, parent, token), c.err.c_str());
  return 0;
}
