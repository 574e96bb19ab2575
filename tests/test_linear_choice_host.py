"""How the products with FB4 weights choose their cluster size, without a device: a size that does not fit (a count of 0) is never chosen, whatever the
sizes of the product, and where all fit the choice is among those of the rule."""
from test_attention_host import run

CHOICE = r"""
  const int32_t whole[9] = {0, 444, 222, 93, 107, 80, 66, 50, 48}, whole_tc[9] = {0, 148, 74, 48, 35, 26, 22, 17, 16};
  const int64_t Ns[] = {1, 32, 33, 128, 129, 1000, 4096, 12288, 49152, 1100000, 0x7fffffff}, Ks[] = {32, 64, 224, 256, 288, 1568, 4096, 12288, 16384, 65536, 1 << 21};
  const int64_t Ts[] = {1, 3, 8, 9, 16, 17, 64, 96, 97, 1000, 1 << 22};
  auto ok = [&](const int32_t* fit, int64_t T, int64_t N, int64_t K) {
    const int32_t s = fb4_linear_splits(fit, N, K);
    if (s < 1 || s > 8 || fit[s] == 0) return false;
    const Fb4LinearTcPlan p = fb4_linear_tc_plan(fit, T, N, K);
    if (p.splits < 1 || p.splits > 8 || fit[p.splits] == 0 || p.splits > (K / 32 + 7) / 8) return false;
    return p.rows >= 16 && p.rows <= 96 && p.rows % 16 == 0 && (T + 95) / 96 * p.rows >= T && p.quarters >= 1 && (p.quarters + 3) / 4 * p.rows <= 256;
  };
  for (int without = 0; without < 256; ++without) {              // bit s - 2: size s does not fit
    int32_t a[9], b[9];
    for (int s = 0; s < 9; ++s) {
      const bool fits = s == 1 || (s > 1 && !((without >> (s - 2)) & 1));
      a[s] = fits ? whole[s] : 0;
      b[s] = fits ? whole_tc[s] : 0;
    }
    for (int64_t T : Ts)
      for (int64_t N : Ns)
        for (int64_t K : Ks)
          if (!ok(a, T, N, K) || !ok(b, T, N, K)) return 1;
  }
  // few rows of W and many channels: the largest clusters, and the next smaller ones where those do not fit
  int32_t fit[9];
  memcpy(fit, whole_tc, sizeof fit);
  if (fb4_linear_tc_plan(fit, 1, 32, 16384).splits != 8 || fb4_linear_splits(fit, 32, 16384) != 8) return 2;
  fit[8] = 0;
  if (fb4_linear_tc_plan(fit, 1, 32, 16384).splits != 4 || fb4_linear_splits(fit, 32, 16384) != 7) return 3;
  fit[4] = fit[7] = 0;
  if (fb4_linear_tc_plan(fit, 1, 32, 16384).splits != 2 || fb4_linear_splits(fit, 32, 16384) != 6) return 4;
  for (int s = 2; s < 9; ++s) fit[s] = 0;
  if (fb4_linear_tc_plan(fit, 1, 32, 16384).splits != 1 || fb4_linear_splits(fit, 32, 16384) != 1) return 5;
  puts("ok");
  return 0;
}
"""


def test_sizes_that_do_not_fit_are_not_chosen(tmp_path):
    run(tmp_path, CHOICE)
