// Prints what the library's rules choose for cross entropies ("loss rows features classes bf16 piece") and updates
// ("update batch rows cols").  Loss: classes of a piece, sides of the tiles of the logits of the first and the last
// piece, of dl, of dh and of dW of both, ranges of dh and of dW, whether dl has two values.  Update: whether A and P take few
// tiles, side and ranges of A, side of X.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "wino_train_rules.hpp"

int main(int argc, char** argv) {
  using namespace wino;
  for (int i = 1; i < argc;) {
    int v[5] = {};
    const bool is_loss = !std::strcmp(argv[i], "loss");
    const int n = is_loss ? 5 : 3;
    if (i + n >= argc) return 1;
    for (int j = 0; j < n; ++j) v[j] = std::atoi(argv[i + 1 + j]);
    i += n + 1;
    if (is_loss) {
      LossArgs a{v[0], v[1], v[2], v[3], v[1], v[1], -100, v[4]};
      const LossLayout l = loss_layout(a, true);
      const int last = (a.classes - 1) % l.piece + 1;
      std::printf("%d %d %d %d %d %d %d %d %d %d\n", l.piece, loss::logits_side(a, l, l.piece), loss::logits_side(a, l, last), l.side,
                  l.dh_side, loss::dw_side(a, l, l.piece), loss::dw_side(a, l, last), l.splits, l.dw_splits, l.two);
    } else {
      UpdateArgs a{};
      a.batch = v[0], a.rows = v[1], a.cols = v[2];
      const UpdateLayout l = update_layout(a);
      std::printf("%d %d %d %d %d\n", update::few(l, a.batch, (int)up(l.c, 32)), update::few(l, a.batch, (int)up(l.r, 32)), l.side,
                  l.splits, update::next_side(l, a.batch));
    }
  }
  return 0;
}
