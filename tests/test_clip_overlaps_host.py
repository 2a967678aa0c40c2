"""Which outputs the scaling of gradients may write: its own input, or memory that no input and no other output has a byte of.  The C entry point, compiled for the
host with stand-ins for the HIP calls, against a map of the bytes."""
import pytest

from test_block_operators_host import HEAD, compiled

PROGRAM = HEAD + r"""
#include <map>
#include <random>
int main() {
  slim_ctx c;
  c.num_cus = 256;
  static float space[1 << 14];
  char* const base = reinterpret_cast<char*>(space);
  float norm;
  std::mt19937 g(1);
  auto upto = [&](int n) { return (int)(g() % (unsigned)n); };
  const slim_dtype types[] = {SLIM_F16, SLIM_BF16, SLIM_F32};
  auto size = [](const slim_tensor& t) { return t.dtype == SLIM_F32 ? 4 : 2; };
  auto bytes = [&](const slim_tensor& t, auto use) {
    for (int64_t r = 0; r < t.rows; ++r)
      for (int64_t i = 0; i < t.cols * size(t); ++i) use((int64_t)(static_cast<char*>(t.data) - base) + r * t.ld * size(t) + i);
  };
  int refused = 0, taken = 0, wrong = 0, side_by_side = 0;
  for (int round = 0; round < 40000; ++round) {
    const int count = 1 + upto(5), grid = round % 3;              // what the tensors lie in: a common matrix, one of several widths, anything
    slim_tensor t[5], o[5];
    auto place = [&](slim_tensor& v) {
      const int width = grid == 0 ? 60 : grid == 1 ? 30 * (1 + upto(3)) : v.cols + upto(20);
      v.ld = v.rows > 1 ? width : v.cols;
      const int first = grid == 2 ? 2 * upto(1500) : grid == 1 ? 2 * upto(300) : 2 * upto(60);
      v.data = base + first * 2;
    };
    for (int i = 0; i < count; ++i) {
      t[i].dtype = types[grid == 2 ? upto(3) : 1];
      t[i].rows = upto(8) ? 1 + upto(6) : 0;
      t[i].cols = 1 + upto(12);
      place(t[i]);
      o[i] = t[i];
      if (upto(3) == 0) place(o[i]);
      if (upto(12) == 0 && i > 0 && t[i].rows == t[0].rows) o[i].data = t[0].data;
    }
    const bool in_place = round % 4 == 0;
    std::map<int64_t, int> writer, reader_other;
    bool bad = false;
    for (int i = 0; i < count; ++i) {
      const slim_tensor& w = in_place ? t[i] : o[i];
      bytes(w, [&](int64_t b) { bad |= !writer.emplace(b, i).second; });
    }
    for (int i = 0; i < count; ++i) {
      const slim_tensor& w = in_place ? t[i] : o[i];
      const bool same = w.data == t[i].data && (w.rows <= 1 || w.ld == t[i].ld);
      bytes(t[i], [&](int64_t b) {
        auto at = writer.find(b);
        bad |= at != writer.end() && !(same && at->second == i);
      });
    }
    launches = 0;
    const slim_status st = slim_clip_gradients(&c, t, in_place ? nullptr : o, count, 1.0, &norm);
    wrong += st != (bad ? SLIM_ERR_INVALID_ARG : SLIM_OK) || (bad && launches);
    (bad ? refused : taken) += 1;
    side_by_side += !bad && count > 1 && grid == 0;
  }
  printf("%d %d %d %d\n", wrong, refused, taken, side_by_side);
  slim_tensor v = {space, 4, 5, 9, SLIM_F32};
  v.ld = (int64_t)1 << 61;
  printf("%d %d\n", slim_clip_gradients(&c, &v, nullptr, 1, 1.0, &norm), slim_grad_norm(&c, &v, 1, &norm));
  return 0;
}
"""


def test_what_may_be_written(tmp_path):
    out = [tuple(map(int, line.split())) for line in compiled(tmp_path, PROGRAM, "-O1")]
    wrong, refused, taken, side_by_side = out[0]
    assert wrong == 0 and refused > 5000 and taken > 5000 and side_by_side > 500, out
    assert out[1:] == [(-1, -1)], out


def test_two_outputs_in_each_others_inputs(tmp_path):
    """a into b's place and b into a's: each is read and written by different workgroups, in no order."""
    source = HEAD + r"""
int main() {
  slim_ctx c;
  c.num_cus = 256;
  static float a[40], b[40], out[40];
  float norm;
  const slim_tensor A = {a, 4, 5, 10, SLIM_F32}, B = {b, 4, 5, 10, SLIM_F32}, C = {out, 4, 5, 10, SLIM_F32}, shifted = {a + 1, 4, 5, 10, SLIM_F32}, beside = {a + 5, 4, 5, 10, SLIM_F32};
  const slim_tensor in[2] = {A, B}, swapped[2] = {B, A}, one[2] = {A, C}, other[2] = {C, A};
  say("taken", slim_clip_gradients(&c, in, nullptr, 2, 1.0, &norm));
  say("taken", slim_clip_gradients(&c, in, one, 2, 1.0, &norm));
  say("taken", slim_clip_gradients(&c, &A, &beside, 1, 1.0, &norm));
  say("refused", slim_clip_gradients(&c, in, swapped, 2, 1.0, &norm));
  say("refused", slim_clip_gradients(&c, in, other, 2, 1.0, &norm));
  say("refused", slim_clip_gradients(&c, &A, &shifted, 1, 1.0, &norm));
  return 0;
}
"""
    for line in compiled(tmp_path, source, "-O0"):
        what, status, launches = line.split()
        assert (int(status), int(launches)) == ((0, 2) if what == "taken" else (-1, 0)), line
