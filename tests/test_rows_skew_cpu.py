"""Several rows per sequence of a cache in pages without a GPU: how a call is cut where one sequence is much longer than the others."""
from tests.test_rows_cpu import _run

PLAN = r"""
  struct Cut {
    ckv::RowsPlan plan;
    int share, behind;
    double all, longest, piece;        // tiles of all blocks, of the longest, of the longest piece
  };
  // as paged_rows_cut_kernel has it: a row for each of `rows` per sequence, no window
  auto cut_of = [](const std::vector<int>& lengths, int hkv, int rows, int group, int most, int n_cu) {
    Cut c{};
    c.plan = ckv::rows_plan((long long)lengths.size() * hkv, rows, group, most, n_cu, (int)lengths.size());
    const int each = 32 * c.plan.wide, size = ckv::rows_tile(c.plan.wide);
    std::vector<int> blocks, tiles;
    float longest = 0;
    for (int n : lengths) {
      const int r = n < rows ? n : rows;
      blocks.push_back((r * group + each - 1) / each);
      tiles.push_back(r ? ckv::row_tiles(0, n, 0, size).count : 0);
      if (tiles.back() > longest) longest = (float)tiles.back();
    }
    auto sum = [&](auto f) {
      float s = 0;
      for (size_t b = 0; b < tiles.size(); ++b) s += blocks[b] * f((float)tiles[b]);
      return s * hkv;
    };
    c.share = ckv::rows_cut(ckv::RowsCost{each, c.plan.workers}, c.plan.least, c.plan.places, c.plan.more == 0, c.plan.more ? ckv::kMorePieces : 6, longest, sum);
    for (size_t b = 0; b < tiles.size(); ++b) {
      if (!blocks[b]) continue;
      const int behind = c.plan.more ? ckv::rows_behind(tiles[b], c.share, c.plan.places) : 0;
      c.behind += hkv * blocks[b] * behind;
      c.all += (double)hkv * blocks[b] * tiles[b];
      const int parts = ckv::unit_parts(tiles[b], ckv::rows_share(tiles[b], c.share, c.plan.places + behind));
      if ((double)tiles[b] / parts > c.piece) c.piece = (double)tiles[b] / parts;
    }
    c.longest = longest;
    return c;
  };
"""


def test_a_long_sequence_among_short_ones_is_cut_for_the_whole_chip(tmp_path):
    """Its pieces are no longer than twice what each compute unit would have of all the work dealt out evenly (and never shorter than a piece may be); all of them find a workgroup."""
    _run(tmp_path, PLAN + r"""
  for (int batch : {2, 3, 8, 16, 32, 64, 70, 128, 200, 600})
    for (int rows : {8, 25, 64})
      for (int hkv : {1, 2, 8})
        for (int longest : {30000, 131072, 1 << 20}) {
          std::vector<int> lengths(batch, 200);
          lengths[batch / 3] = longest;
          const Cut c = cut_of(lengths, hkv, rows, 4, longest, 256);
          const double even = c.all / 256, least = c.plan.least;
          if (c.behind > c.plan.more) return std::printf("%d x %d x %d: %d pieces behind places, %d workgroups\n", batch, rows, hkv, c.behind, c.plan.more), 1;
          const double most = 2 * (even > least ? even : least) + 1;
          if (c.piece > most && c.piece > ckv::kLongPiece) return std::printf("%d x %d x %d, one of %d: a piece of %g tiles, evenly %g\n", batch, rows, hkv, longest, c.piece, even), 1;
        }""")


def test_pieces_behind_places_find_workgroups_whatever_the_lengths(tmp_path):
    _run(tmp_path, PLAN + r"""
  unsigned state = 1;
  auto random = [&]() { return (state = state * 1664525u + 1013904223u) >> 8; };
  int cut = 0;
  for (int turn = 0; turn < 3000; ++turn) {
    const int batch = 2 + random() % 300, rows = 1 + random() % 100, hkv = 1 + random() % 8, group = 1 + random() % 16, most = 1 << (8 + random() % 12);
    std::vector<int> lengths;
    for (int b = 0; b < batch; ++b) lengths.push_back(random() % 3 ? random() % 300 % (most + 1) : random() % (most + 1));
    const Cut c = cut_of(lengths, hkv, rows, group, most, 256);
    if (c.behind > c.plan.more) return std::printf("%d pieces, %d workgroups\n", c.behind, c.plan.more), 1;
    cut += c.plan.more && c.behind;
  }
  if (cut < 100) return std::printf("only %d calls were cut like that\n", cut), 1;""")


def test_calls_of_the_gpu_tests_have_pieces_behind_places(tmp_path):
    """The sizes of tests/test_gpu_rows_skew.py are such that they go this way."""
    from tests.test_gpu_rows_skew import CASES
    for batch, hkv, g, rows, longest in [*(c[:5] for c in CASES), (200, 1, 4, 8, 40000), (80, 2, 4, 16, 60000)]:
        _run(tmp_path, PLAN + f"""
  std::vector<int> lengths({batch}, 300);
  lengths[1] = {longest};
  const Cut c = cut_of(lengths, {hkv}, {rows}, {g}, {longest}, 256);
  if (!c.plan.more || !c.behind) return std::printf("%d places of %g tiles, %d more\\n", c.plan.places, c.longest, c.plan.more), 1;""")


def test_blocks_that_read_the_same_entries_go_to_one_part_of_the_chip(tmp_path):
    _run(tmp_path, r"""
  for (int groups : {1, 7, 8, 9, 16, 63, 64, 250})
    for (int blocks : {1, 2, 3, 8, 13}) {
      std::vector<int> seen(groups * blocks, 0);
      for (int i = 0; i < groups * blocks; ++i) {
        const int piece = ckv::rows_behind_piece(i, groups, blocks);
        if (piece < 0 || piece >= groups * blocks || seen[piece]++) return std::printf("%d of %d x %d: piece %d\n", i, groups, blocks, piece), 1;
        if (piece / blocks < groups / 8 * 8 && piece / blocks % 8 != i % 8) return std::printf("group %d on part %d\n", piece / blocks, i % 8), 1;
      }
    }""")
