"""What needs no GPU of the residual norm, the 8-bit layer's epilogue, the head's cross entropy and the clipping: the checks of arguments of the C entry
points (compiled for the host, with stand-ins for the HIP calls that count launches), those of the binding, and the workspace sizes."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2405_14917_amd import build
from test_operators_host import PROGRAM, SIZES, binding  # noqa: F401  (the fixture)

HEAD, BIG = PROGRAM[:PROGRAM.index("int main() {")], SIZES[:SIZES.index("int main() {")]

CHECKS = HEAD + r"""
int main() {
  slim_ctx c;
  c.num_cus = 256;
  alignas(64) static char buf[1 << 16];
  void* p = buf;
  uint8_t* u = reinterpret_cast<uint8_t*>(buf);
  float* f = reinterpret_cast<float*>(buf);
  const slim_dtype B = SLIM_BF16, F = SLIM_F32, D = SLIM_F64;
  auto norm = [&](int64_t rows, int cols, slim_dtype x, slim_dtype w, double eps, int64_t ldx, void* R, int64_t ldr, void* H, int64_t ldh, void* Y,
                  int64_t ldy, uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds) {
    return slim_add_norm(&c, p, R, x, rows, cols, ldx, ldr, p, nullptr, w, eps, 0, H, ldh, Y, ldy, q, ldq, s, lds, f, f);
  };
  say("one", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 256, u, 4));
  say("one", norm(3, 200, B, B, 0.0, 200, nullptr, 0, nullptr, 0, nullptr, 0, u, 256, u, 4));
  say("one", norm(3, 200, F, F, 1e-5, 200, p, 200, nullptr, 0, p, 200, nullptr, 0, nullptr, 0));
  say("none", norm(0, 200, B, F, 1e-5, 200, p, 200, p, 200, nullptr, 200, nullptr, 0, nullptr, 0));
  say("bad", norm(-1, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 256, u, 4));
  say("bad", norm(3, 0, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 256, u, 4));
  say("bad", norm(3, 200, B, F, -1.0, 200, p, 200, p, 200, p, 200, u, 256, u, 4));
  say("bad", norm(3, 200, B, F, 0.0 / 0.0, 200, p, 200, p, 200, p, 200, u, 256, u, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 199, p, 200, p, 200, p, 200, u, 256, u, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 199, p, 200, p, 200, u, 256, u, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 199, p, 200, u, 256, u, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 199, u, 256, u, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 128, u, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 250, u, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u + 8, 256, u, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 256, u, 2));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 256, u + 1, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 256, nullptr, 4));
  say("bad", norm(3, 200, B, F, 1e-5, 200, p, 200, p, 200, nullptr, 200, nullptr, 256, nullptr, 4));
  say("unsupported", norm(3, 200, D, F, 1e-5, 200, p, 200, p, 200, p, 200, u, 256, u, 4));
  say("unsupported", norm(3, 200, B, SLIM_F16, 1e-5, 200, p, 200, p, 200, p, 200, u, 256, u, 4));
  const int far = (1 << 30) + 1;
  say("unsupported", norm(3, far, B, F, 1e-5, far, p, far, p, far, p, far, nullptr, 0, nullptr, 0));
  say("unsupported", slim_add_norm_backward(&c, p, p, p, B, 3, far, far, far, far, p, F, nullptr, f, p, far, p, nullptr));
  auto back = [&](int64_t rows, const void* dY, const void* dH, const void* H, int64_t lddy, int64_t lddh, int64_t ldh, void* dX, int64_t lddx, void* dw) {
    return slim_add_norm_backward(&c, dY, dH, H, B, rows, 200, lddy, lddh, ldh, p, F, nullptr, f, dX, lddx, dw, nullptr);
  };
  say("one", back(3, p, p, p, 200, 200, 200, p, 200, p));
  say("one", back(3, p, nullptr, p, 200, 0, 200, p, 200, p));
  say("one", back(0, nullptr, p, nullptr, 200, 200, 200, nullptr, 200, p));
  say("bad", back(3, nullptr, p, p, 200, 200, 200, p, 200, p));
  say("bad", back(3, p, p, nullptr, 200, 200, 200, p, 200, p));
  say("bad", back(3, p, p, p, 199, 200, 200, p, 200, p));
  say("bad", back(3, p, p, p, 200, 199, 200, p, 200, p));
  say("bad", back(3, p, p, p, 200, 200, 199, p, 200, p));
  say("bad", back(3, p, p, p, 200, 200, 200, p, 199, p));
  say("bad", back(3, p, p, p, 200, 200, 200, p, 200, nullptr));

  slim_epilogue e = {p, F, SLIM_ACT_SILU, p, 130, p, 130};
  auto act = [&](int t, const void* X, slim_dtype x, const uint8_t* xq, const uint8_t* xs, slim_epilogue* ep, void* Y, slim_dtype y, int64_t ldx = 200,
                 int64_t ldxq = 256, int64_t ldxs = 4, int64_t ldy = 130) {
    return slim_fp8_linear_act(&c, X, x, t, ldx, xq, ldxq, xs, ldxs, u, 256, u, 4, 130, 200, ep, Y, y, ldy);
  };
  say("one", act(5, p, B, nullptr, nullptr, &e, p, F));
  say("one", act(5, nullptr, D, u, u, &e, p, F));
  say("one", act(5, nullptr, D, u, u, nullptr, p, B));
  say("none", act(0, nullptr, B, nullptr, nullptr, &e, nullptr, B));
  say("bad", act(-1, p, B, nullptr, nullptr, &e, p, F));
  say("bad", act(5, p, B, u, u, &e, p, F));
  say("bad", act(5, nullptr, B, nullptr, nullptr, &e, p, F));
  say("bad", act(5, nullptr, B, u, nullptr, &e, p, F));
  say("bad", act(5, p, B, nullptr, nullptr, &e, nullptr, F));
  say("bad", act(5, p, B, nullptr, nullptr, &e, p, F, 199));
  say("bad", act(5, nullptr, B, u, u, &e, p, F, 0, 200));
  say("bad", act(5, nullptr, B, u, u, &e, p, F, 0, 128));
  say("bad", act(5, nullptr, B, u, u, &e, p, F, 0, 256, 3));
  say("bad", act(5, nullptr, B, u + 4, u, &e, p, F));
  say("bad", act(5, p, B, nullptr, nullptr, &e, p, F, 200, 0, 0, 129));
  for (int a : {-1, 5}) {
    slim_epilogue x = e;
    x.act = a;
    say("bad", act(5, p, B, nullptr, nullptr, &x, p, F));
  }
  slim_epilogue x = e;
  x.ldr = 129;
  say("bad", act(5, p, B, nullptr, nullptr, &x, p, F));
  x = e;
  x.ldz = 129;
  say("bad", act(5, p, B, nullptr, nullptr, &x, p, F));
  x = e;
  x.bias_dtype = SLIM_F16;
  say("unsupported", act(5, p, B, nullptr, nullptr, &x, p, B));
  say("unsupported", act(5, p, F, nullptr, nullptr, &e, p, B));
  say("unsupported", act(5, p, B, nullptr, nullptr, &e, p, D));
  auto grad = [&](int t, const void* dY, const void* Z, int a, const void* X, void* dX, void* dW, void* db, slim_dtype dwt = SLIM_F32,
                  slim_dtype dbt = SLIM_F32, int64_t lddy = 130, int64_t ldz = 130, int64_t ldx = 200, int64_t lddx = 200, int64_t lddw = 200) {
    return slim_fp8_linear_act_backward(&c, dY, Z, a, X, B, t, lddy, ldz, ldx, u, 256, u, 4, 130, 200, dX, lddx, dW, dwt, lddw, db, dbt);
  };
  say("few", grad(5, p, p, 2, p, p, p, p));
  say("few", grad(5, p, nullptr, 0, p, p, p, p));
  say("few", grad(5, p, nullptr, 0, p, p, p, nullptr));
  say("few", grad(5, p, p, 4, nullptr, nullptr, nullptr, p));
  say("few", grad(0, nullptr, nullptr, 4, nullptr, p, p, p));
  say("bad", grad(5, p, p, 2, p, nullptr, nullptr, nullptr));
  say("bad", grad(5, nullptr, p, 2, p, p, p, p));
  say("bad", grad(5, p, nullptr, 2, p, p, p, p));
  say("bad", grad(5, p, p, 2, nullptr, p, p, p));
  say("bad", grad(5, p, p, 6, p, p, p, p));
  say("bad", grad(5, p, p, -1, p, p, p, p));
  say("bad", grad(-5, p, p, 2, p, p, p, p));
  say("bad", grad(5, p, p, 2, p, p, p, p, F, F, 129));
  say("bad", grad(5, p, p, 2, p, p, p, p, F, F, 130, 129));
  say("bad", grad(5, p, p, 2, p, p, p, p, F, F, 130, 130, 199));
  say("bad", grad(5, p, p, 2, p, p, p, p, F, F, 130, 130, 200, 199));
  say("bad", grad(5, p, p, 2, p, p, p, p, F, F, 130, 130, 200, 200, 199));
  say("unsupported", grad(5, p, p, 2, p, p, p, p, D));
  say("unsupported", grad(5, p, p, 2, p, p, p, p, F, D));

  auto head = [&](int t, const void* X, slim_dtype x, int64_t ldx, const uint8_t* q, int64_t ldq, int64_t lds, const void* labels, float* loss) {
    return slim_head_loss(&c, X, x, t, ldx, q, ldq, u, lds, 700, 200, labels, 1, loss);
  };
  say("few", head(5, p, B, 200, u, 256, 4, p, f));
  say("few", head(300, p, B, 200, u, 256, 4, p, f));
  say("none", head(0, nullptr, B, 200, u, 256, 4, nullptr, nullptr));
  say("bad", head(-1, p, B, 200, u, 256, 4, p, f));
  say("bad", head(5, p, B, 199, u, 256, 4, p, f));
  say("bad", head(5, nullptr, B, 200, u, 256, 4, p, f));
  say("bad", head(5, p, B, 200, nullptr, 256, 4, p, f));
  say("bad", head(5, p, B, 200, u, 255, 4, p, f));
  say("bad", head(5, p, B, 200, u, 256, 3, p, f));
  say("bad", head(5, p, B, 200, u, 256, 4, nullptr, f));
  say("bad", head(5, p, B, 200, u, 256, 4, p, nullptr));
  say("unsupported", head(5, p, F, 200, u, 256, 4, p, f));
  auto hgrad = [&](int t, const uint8_t* qt, int64_t ldqt, const float* dloss, void* dX, int64_t lddx, void* dW, int64_t lddw, slim_dtype dwt) {
    return slim_head_loss_grad(&c, p, B, t, 200, u, 256, u, 4, qt, ldqt, u, 8, 700, 200, p, 1, dloss, f, dX, lddx, dW, dwt, lddw);
  };
  say("few", hgrad(5, u, 768, f, p, 200, p, 200, F));
  say("few", hgrad(5, nullptr, 0, f, nullptr, 0, p, 200, B));
  say("few", hgrad(0, u, 768, nullptr, p, 200, p, 200, F));
  say("none", hgrad(0, u, 768, nullptr, p, 200, nullptr, 200, F));
  say("bad", hgrad(5, u, 768, f, nullptr, 200, nullptr, 200, F));
  say("bad", hgrad(5, nullptr, 768, f, p, 200, p, 200, F));
  say("bad", hgrad(5, u, 640, f, p, 200, p, 200, F));
  say("bad", hgrad(5, u, 768, nullptr, p, 200, p, 200, F));
  say("bad", hgrad(5, u, 768, f, p, 199, p, 200, F));
  say("bad", hgrad(5, u, 768, f, p, 200, p, 199, F));
  say("unsupported", hgrad(5, u, 768, f, p, 200, p, 200, D));

  slim_tensor t[3] = {{p, 5, 7, 9, B}, {buf + 512, 1, 100, 100, F}, {nullptr, 0, 5, 5, F}}, o[3];
  auto again = [&]() { memcpy(o, t, sizeof(t)); };
  again();
  say("one", slim_grad_norm(&c, t, 3, f) == 0 ? 0 : -9);
  say("few", slim_clip_gradients(&c, t, nullptr, 3, 1.0, f));
  say("few", slim_clip_gradients(&c, t, o, 3, 1.0, f));
  say("few", slim_clip_gradients(&c, nullptr, nullptr, 0, 1.0, f));
  say("bad", slim_clip_gradients(&c, t, nullptr, -1, 1.0, f));
  say("bad", slim_clip_gradients(&c, nullptr, nullptr, 2, 1.0, f));
  say("bad", slim_clip_gradients(&c, t, nullptr, 3, 1.0, nullptr));
  say("bad", slim_grad_norm(&c, t, 3, nullptr));
  say("bad", slim_clip_gradients(&c, t, nullptr, 3, -1.0, f));
  say("bad", slim_clip_gradients(&c, t, nullptr, 3, 0.0 / 0.0, f));
  o[0].rows = 4;
  say("bad", slim_clip_gradients(&c, t, o, 3, 1.0, f));
  again();
  o[1].dtype = B;
  say("bad", slim_clip_gradients(&c, t, o, 3, 1.0, f));
  again();
  o[1].data = p;
  say("bad", slim_clip_gradients(&c, t, o, 3, 1.0, f));
  again();
  o[0].ld = 6;
  say("bad", slim_grad_norm(&c, o, 3, f));
  again();
  o[0].rows = -1;
  say("bad", slim_grad_norm(&c, o, 3, f));
  again();
  o[1].data = nullptr;
  say("bad", slim_grad_norm(&c, o, 3, f));
  again();
  o[0].rows = o[0].cols = 1ll << 40;
  o[0].ld = 1ll << 41;
  say("bad", slim_grad_norm(&c, o, 3, f));
  again();
  o[1].dtype = D;
  say("unsupported", slim_grad_norm(&c, o, 3, f));
  return 0;
}
"""

ENOUGH = "#include <cmath>\n" + BIG + r"""
#include <random>
int main() {
  slim_ctx c;
  c.num_cus = 256;
  c.ws_external = true;
  alignas(256) static char buf[64];
  c.ws = buf;                      // (nothing is written: no launch runs)
  void* p = buf;
  float* f = reinterpret_cast<float*>(buf);
  uint8_t* u = reinterpret_cast<uint8_t*>(buf);
  std::mt19937 g(1);
  auto size = [&](int hi) { return (int)std::exp(std::uniform_real_distribution<double>(0.0, std::log((double)hi))(g)); };
  int bad = 0, pieces = 0;
  const int64_t ld = 1 << 18;
  for (int i = 0; i < 20000; ++i) {
    const int n = size(200000), m = size(30000), t = size(i % 2 ? 3000 : 60000), x = i % 3, w = i / 3 % 3;
    const slim_dtype d = i % 4 < 2 ? SLIM_F32 : SLIM_BF16;
    const slim_epilogue e = {p, SLIM_F32, 1, p, ld, p, ld};
    c.ws_bytes = slim_fp8_linear_act_workspace(n, m, t, i & 1, d, 256);
    bad += slim_fp8_linear_act(&c, i & 1 ? nullptr : p, SLIM_BF16, t, ld, i & 1 ? u : nullptr, ld, i & 1 ? u : nullptr, 2048, u, ld, u, 2048, n, m, &e, p, d,
                               ld) != 0;
    c.ws_bytes = slim_fp8_linear_act_backward_workspace(n, m, t, x != 0, w != 0 || x == 0, d, i & 1, 256);
    bad += slim_fp8_linear_act_backward(&c, p, p, 2, p, SLIM_BF16, t, ld, ld, ld, u, ld, u, 2048, n, m, x != 0 ? p : nullptr, ld, w != 0 || x == 0 ? p : nullptr,
                                        d, ld, i & 1 ? p : nullptr, SLIM_F32) != 0;
    c.ws_bytes = slim_head_loss_workspace(n, m, t, 256);
    bad += slim_head_loss(&c, p, SLIM_BF16, t, ld, u, ld, u, 2048, n, m, p, 1, f) != 0;
    c.ws_bytes = slim_head_loss_grad_workspace(n, m, t, x != 0, w != 0 || x == 0, d, 256);
    calls = 0;
    bad += slim_head_loss_grad(&c, p, SLIM_BF16, t, ld, u, ld, u, 2048, u, ld, u, 2048, n, m, p, 1, f, f, x != 0 ? p : nullptr, ld, w != 0 || x == 0 ? p : nullptr, d,
                               ld) != 0;
    pieces += calls > 8;
  }
  printf("%d %d %d\n", bad, pieces, large);
  large = calls = 0;
  c.ws_bytes = SIZE_MAX;
  for (int t : {(1 << 23) - 64, 1 << 23}) {
    printf("%d %d ", slim_head_loss(&c, p, SLIM_BF16, t, 128, u, 128, u, 4, 8192, 128, p, 1, f), calls != 0);
    printf("%d\n", large);
    calls = 0;
  }
  return 0;
}
"""


def compiled(tmp_path, source, level):
    src, exe = tmp_path / "t.hip", tmp_path / "t"
    src.write_text(source)
    jobs, objs = [], []
    for f in [str(src)] + [os.path.join(build.CSRC, f) for f in build.SOURCES if f.startswith(("ctx", "fp8_", "norm", "add_norm", "head_", "clip"))]:
        objs.append(str(tmp_path / (os.path.basename(f) + ".o")))
        jobs.append(subprocess.Popen([build.hipcc(), "--offload-host-only", level, "-fPIC", "-std=c++17", "-I" + build.INCLUDE, "-I" + build.CSRC, "-c", f,
                                      "-o", objs[-1]], stderr=subprocess.DEVNULL))
    assert not any(j.wait() for j in jobs)
    subprocess.run(["g++", *objs, "-o", str(exe), "-pthread", "-Wl,--unresolved-symbols=ignore-in-object-files"], check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]


def test_arguments_are_checked_before_anything_is_launched(tmp_path):
    out = compiled(tmp_path, CHECKS, "-O0")
    assert len(out) > 110
    want = {"one": (0, (1, 2)), "few": (0, range(1, 9)), "none": (0, (0,)), "bad": (-1, (0,)), "unsupported": (-5, (0,))}
    for k, line in enumerate(out):
        what, status, launches = line.split()
        assert int(status) == want[what][0] and int(launches) in want[what][1], (k, line)


def test_the_queried_workspace_holds_every_shapes_parts(tmp_path):
    """20000 shapes in workspaces of exactly the queried sizes; more tokens than a launch has threads for are refused."""
    out = [tuple(map(int, line.split())) for line in compiled(tmp_path, ENOUGH, "-O1")]
    assert out[0][0] == 0 and out[0][1] > 100 and out[0][2] == 0, out
    assert out[1] == (0, 1, 0) and out[2] == (-5, 0, 0), out


@pytest.mark.parametrize("V,m,tokens", [(32000, 4096, 2048), (50257, 1501, 700), (1003, 384, 300), (131072, 256, 400), (700, 130, 20000)])
def test_a_workspace_is_enough_for_fewer_tokens(binding, V, m, tokens):
    from paper_2405_14917_amd import tuning
    bf16, f32 = torch.bfloat16, torch.float32
    needs = lambda t: (binding.head_loss_workspace(V, m, t, 256), binding.head_loss_grad_workspace(V, m, t, num_cus=256),
                       binding.head_loss_grad_workspace(V, m, t, True, False, f32, 256), binding.fp8_linear_act_workspace(V, m, t, True, bf16, 256),
                       binding.fp8_linear_act_workspace(V, m, t, False, f32, 256), binding.fp8_linear_act_backward_workspace(V, m, t, num_cus=256),
                       binding.fp8_linear_act_backward_workspace(V, m, t, True, True, f32, True, 256),
                       tuning.block_workspace_query(V, m, 3 * m, t, num_cus=256))
    whole = needs(tokens)
    for t in list(range(1, min(tokens, 600))) + list(range(600, tokens, 37)) + [tokens]:
        now = needs(t)
        assert all(a <= b for a, b in zip(now, whole)), (t, now, whole)


def test_workspace_sizes(binding):
    assert binding.fp8_linear_act_workspace(4096, 4096, 16) == 0 == binding.fp8_linear_act_workspace(4096, 4096, 16, True)
    assert binding.fp8_linear_act_workspace(4096, 4096, 2048, True) + 2048 * 4096 <= binding.fp8_linear_act_workspace(4096, 4096, 2048, False)
    for q in (binding.head_loss_workspace, binding.head_loss_grad_workspace):
        assert q(0, 1, 1) == q(1, 0, 1) == q(1, 1, 0) == 0
    # a piece of the logits, not all of them
    assert binding.head_loss_grad_workspace(131072, 4096, 16384) < 4 * 131072 * 16384 // 8
    assert binding.grad_norm_workspace(-1) == 0 and binding.grad_norm_workspace(1000) > binding.grad_norm_workspace(10) > 0


def test_null_contexts_are_rejected(binding):
    lib = binding.load()
    for name in ("slim_add_norm", "slim_add_norm_backward", "slim_fp8_linear_act", "slim_fp8_linear_act_backward", "slim_head_loss", "slim_head_loss_grad",
                 "slim_grad_norm", "slim_clip_gradients"):
        fn = getattr(lib, name)
        assert name in binding.EXPORTS
        assert fn(*[None if a is ctypes.c_void_p else a(0).value for a in fn.argtypes]) == binding.ERR_INVALID_ARG, name


def test_the_epilogues_bytes_are_the_structure(binding):
    assert binding._EPILOGUE.size == ctypes.sizeof(binding.SlimEpilogue)
    e = binding.SlimEpilogue.from_buffer_copy(binding._EPILOGUE.pack(11, 2, 4, 13, 14, 15, 16))
    assert (e.bias, e.bias_dtype, e.act, e.R, e.ldr, e.Z, e.ldz) == (11, 2, 4, 13, 14, 15, 16)


def test_lists_of_tensors(binding):
    a = torch.zeros((4, 10))
    d = list(binding._tensor_list([a, a[:, 2:7], a[1], torch.zeros(()), torch.zeros((0, 3)).half()], "t"))
    assert d[1:5] == [1, 40, 40, 2] and d[6:10] == [4, 5, 10, 2] and d[11:15] == [1, 10, 10, 2] and d[16:20] == [1, 1, 1, 2] and d[21:25] == [1, 0, 0, 0]
    assert list(binding._tensor_rows([a, a[1]], "t"))[1:5] == [4, 10, 10, 2]
    for bad in (a.t(), a.double(), a[:, ::2], torch.zeros((2, 3, 4))[:, :, :2], torch.zeros(1, 10).expand(4, 10)):
        with pytest.raises(ValueError):
            binding._tensor_list([bad], "t")


def test_a_gradient_is_not_lost_silently(binding):
    slim = object.__new__(binding.Slim)                          # (no context: the check comes first)
    slim.ctx = None
    x, w = torch.ones(2, 8), torch.ones(8)
    leaf = lambda t: t.clone().requires_grad_()
    for call in (lambda: slim.add_norm(leaf(x), None, w), lambda: slim.add_norm(x, leaf(x), w), lambda: slim.add_norm(x, x, leaf(w)),
                 lambda: slim.add_norm(x, x, w, leaf(w)), lambda: slim.fp8_linear_act(leaf(x), w, w), lambda: slim.fp8_linear_act(x, w, w, leaf(w)),
                 lambda: slim.fp8_linear_act(x, w, w, residual=leaf(x)), lambda: slim.head_loss(leaf(x), w, w, w),
                 lambda: slim.add_norm(x, x, w, stats=True, H=leaf(x)), lambda: slim.grad_norm([x, leaf(x)]), lambda: slim.clip_gradients([x, leaf(x)], 1.0),
                 lambda: slim.clip_gradients([x], 1.0, out=[leaf(x)])):
        with pytest.raises(ValueError, match="graph"):
            call()
    with pytest.raises(ValueError, match="act"):
        binding._check_act("tanh")
