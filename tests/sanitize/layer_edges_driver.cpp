// Plans of libsk_layer.so (layer_plan.cpp) at the ends of their ranges.
#include <cstdio>
#include <cstdlib>

#include "layer_internal.h"

static void need(bool ok, const char *what) {
  if (!ok) {
    std::printf("layer_edges_driver: %s\n", what);
    std::exit(1);
  }
}
static void *address(int i) { return (void *)(((uintptr_t)i + 1) << 44); }

// A chunk of several pieces is read by waves that take a row to have eight logits at least, and only a row that is longer than one piece has any use for it.
static void pieces_of_short_rows() {
  for (int vocab : {1, 2, 3, 5, 7, 8, 9, 100, 511, 512, 513, 1024, 1025, 2000, 2048, 2049, 50257})
    for (int rows : {1, 70, 1500, 2999, 3000, 3001, 5999, 6000, 6001, 24000, 100000, 1000000})
      for (int draft = 0; draft < 2; ++draft) {
        sk_verify_problem p{};
        p.dtype = SK_F32, p.sequences = 1, p.rows = rows, p.vocab = vocab;
        p.first_row = p.drafted = (const int32_t *)address(0), p.logits = address(0), p.accept_random = p.sample_random = (const float *)address(0);
        p.draft_logits = draft ? address(0) : nullptr;
        p.tokens = (int32_t *)address(1), p.accepted = (int32_t *)address(2);
        sk::VerifyPlanHost out;
        std::string err;
        need(sk::plan_verify(&p, 1, out, err) == SK_OK, err.c_str());
        const sk::VerifyDev &d = out.launches[0].table.problems[0];
        need(d.pieces == 1 || vocab >= 8, "chunks of several pieces for rows of fewer than eight logits");
        need(d.pieces == 1 || vocab > 256 * d.pieces, "chunks that are twice as long as the row or more");
        need((int64_t)d.chunks * d.pieces * 512 >= vocab && ((int64_t)d.chunks - 1) * d.pieces * 512 < vocab, "chunks");
      }
}

int main() {
  pieces_of_short_rows();
  std::printf("layer_edges_driver: ok\n");
  return 0;
}
