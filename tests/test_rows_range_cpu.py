"""Several rows per sequence of a cache in pages without a GPU: bounds that keep sums of large values finite."""
from tests.test_rows_cpu import _run


def test_lowered_weights_of_a_whole_sequence_add_up_to_less_than_a_half(tmp_path):
    """Each is 2^8 at most; the factor is a power of two; pieces below the limit stay finite whatever their number (places, of which there are at most 4 for each of 256 compute units, and one)."""
    _run(tmp_path, r"""
  for (int n : {1, 2, 3, 4, 5, 100, 1023, 1024, 1025, 9350, 131072, 131073, (1 << 30) - 1, 1 << 30}) {
    const float f = ckv::lowered_by(n);
    unsigned bits;
    __builtin_memcpy(&bits, &f, 4);
    if (bits & 0x7FFFFFu) return std::printf("%d: no power of two\n", n), 1;
    if ((double)n * 256 * f >= 0.5 || (double)n * 256 * f < 0.1) return std::printf("%d: %g\n", n, (double)n * 256 * f), 1;
  }
  if ((double)ckv::kLargeSum * ckv::kLargeSums != 0x1p128) return 1;
  if (ckv::rows_plan(1, 1, 1, 1 << 30, 256).places >= ckv::kLargeSums / 2) return 1;""")
