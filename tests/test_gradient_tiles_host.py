"""The tiles that the two gradients of an 8-bit layer are cut into, by their launches' sizes: the entry point, compiled for the host with stand-ins for the HIP
calls."""
from test_block_operators_host import BIG, compiled

PROGRAM = "#include <tuple>\n" + BIG.replace("static int launches,", "static unsigned grids[64];\nstatic int launches,").replace("  ++calls;", "  grids[calls++ & 63] = g.x;") + r"""
int main() {
  slim_ctx c;
  c.num_cus = 256;
  c.ws_external = true;
  alignas(256) static char buf[64];
  c.ws = buf;                      // (nothing is written: no launch runs)
  c.ws_bytes = SIZE_MAX;
  void* p = buf;
  const uint8_t* u = reinterpret_cast<const uint8_t*>(buf);
  const int64_t ld = 1 << 15;
  for (auto [n, m, t] : {SHAPES}) {
    calls = 0;
    const slim_status st = slim_fp8_linear_backward(&c, p, p, SLIM_BF16, t, ld, ld, u, ld, u, 512, n, m, p, ld, p, SLIM_BF16, ld);
    printf("%d", st);
    for (int i = 1; i < calls; ++i) printf(" %u", grids[i]);       // (the first one quantises)
    printf("\n");
  }
  return 0;
}
"""

# (n, m, tokens): in large tiles the rounds end at their last place, and what takes a little longer needs another one (22, 11, 9, 8, 4 and 4 % more than in
# medium ones, or in two launches)
NOT_LARGE = [(5504, 3584, 1792), (10492, 2375, 2589), (2465, 2455, 7850), (4096, 3328, 2119), (4992, 2560, 2560), (2021, 6252, 3571)]
# together in large tiles, 9 to 21 % less
LARGE = [(16384, 4096, 2048), (25053, 2798, 3193), (4480, 1536, 5632), (5248, 5120, 1681), (15616, 3584, 5456), (8704, 2816, 6685)]


def tiles(a, b, tile):
    return -(-a // tile) * -(-b // tile)


def test_large_tiles_together_only_with_room(tmp_path):
    shapes = NOT_LARGE + LARGE
    source = PROGRAM.replace("SHAPES", ", ".join("std::tuple<int, int, int>(%d, %d, %d)" % s for s in shapes))
    out = [tuple(map(int, line.split())) for line in compiled(tmp_path, source, "-O1")]
    assert len(out) == len(shapes)
    for (n, m, t), (status, *grids) in zip(shapes, out):
        large, medium = tiles(m, t, 256) + tiles(m, n, 256), tiles(m, t, 128) + tiles(m, n, 128)
        assert status == 0
        if (n, m, t) in LARGE:
            assert grids == [large], ((n, m, t), grids)
        else:
            assert grids == [medium] or len(grids) == 2, ((n, m, t), grids)


HEAD_PROGRAM = PROGRAM[:PROGRAM.index("  for (auto [n, m, t]")] + r"""
  for (auto [V, m, t] : {SHAPES}) {
    calls = 0;
    const int64_t ld = (V + 127) / 128 * 128 + 4096;
    const slim_status st = slim_head_loss_grad(&c, p, SLIM_BF16, t, ld, u, ld, u, 4096, u, ld, u, 4096, V, m, p, 1, reinterpret_cast<const float*>(p),
                                               reinterpret_cast<float*>(p), p, ld, nullptr, SLIM_F32, ld);
    printf("%d", st);
    for (int i = 0; i < calls; ++i) printf(" %u", grids[i]);
    printf("\n");
  }
  return 0;
}
"""


def test_logits_made_again_in_large_tiles(tmp_path):
    """Of the sizes of test_gpu_head_pieces.py: X quantised, the logits, their sums, then of every piece the gradients (kept, or made again) and dX."""
    sizes = [(40000, 2560, 2048, (32768,)), (16500, 2600, 8200, (7680, 15360))]
    source = HEAD_PROGRAM.replace("SHAPES", ", ".join("std::tuple<int, int, int>(%d, %d, %d)" % s[:3] for s in sizes))
    for (V, m, t, ends), line in zip(sizes, compiled(tmp_path, source, "-O1")):
        status, x, logits, sums, *grids = map(int, line.split())
        assert status == 0 and logits in (tiles(V, t, 256), tiles(V, t, 128)) and grids[0] == tiles(ends[0], t, 128), line
        for first, end in zip(ends, (*ends[1:], V)):
            assert tiles(end - first, t, 256) in grids[2:], (first, grids)
