"""Host side of layer norm, dense layers and the vocabulary losses (no GPU):
workspace sizes, refusals of the C entry points under AddressSanitizer and
UndefinedBehaviorSanitizer, and refusals of the binding."""
import os
import shutil
import subprocess

import pytest
import torch

from test_sanitizers import ROOT, TESTS, run_clean


def test_layer_entry_points_under_asan_and_ubsan(tmp_path):
    from paper_2403_17607_amd import build
    llvm = "/opt/rocm/llvm/bin"
    if not (os.path.exists(f"{llvm}/clang++") and shutil.which(build.HIPCC)):
        pytest.skip("ROCm clang not found")
    mine = ("api.hip", "layers.hip")
    objs = [os.path.join(build.BUILD, os.path.splitext(s)[0] + ".o") for s in build.SOURCES if s not in mine]
    if not all(os.path.exists(o) for o in objs):
        build.build()
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
           "-fno-omit-frame-pointer"]
    flags = [f for f in build.FLAGS if f != "-O3"]
    for s in mine:
        objs.append(str(tmp_path / (s + ".o")))
        subprocess.run([build.HIPCC, *flags, "-O1", "-g", *san, "-c", os.path.join(build.CSRC, s), "-o", objs[-1]],
                       check=True, capture_output=True)
    main_o = str(tmp_path / "main.o")
    subprocess.run([f"{llvm}/clang", "-std=c11", "-O1", "-g", "-fsanitize=address,undefined", "-fno-omit-frame-pointer",
                    "-I", os.path.join(ROOT, "include"), "-c", os.path.join(TESTS, "asan_layers_main.c"), "-o", main_o],
                   check=True)
    exe = str(tmp_path / "layers_asan")
    subprocess.run([f"{llvm}/clang++", "-fsanitize=address,undefined", main_o, *objs, "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True)
    assert "layers ok" in run_clean(exe)


def test_shapes_the_binding_refuses(ffmlp):
    for bad in [lambda: ffmlp.LayerNorm(0), lambda: ffmlp.LayerNorm(8, eps=0.0), lambda: ffmlp.LayerNorm(8, eps=float("nan")),
                lambda: ffmlp.LayerNorm(8.0), lambda: ffmlp.Dense(0, 8), lambda: ffmlp.Dense(8, ffmlp.MLP_MAX_DIM + 1),
                lambda: ffmlp.Dense(8, 8, "tanh"), lambda: ffmlp.Dense(8, 8, 6), lambda: ffmlp.SoftmaxHead(8, 0),
                lambda: ffmlp.SoftmaxHead(True, 8)]:
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ffmlp.FFMLPError):
        ffmlp.FusedMLP(64, 2, 64, 16, 4)  # GELU is not an activation of the fused nets


def test_binding_refuses_host_tensors(ffmlp):
    X, W = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, 16, dtype=torch.bfloat16)
    t = torch.zeros(4, dtype=torch.int64)
    for f in [lambda: ffmlp.LayerNorm(8).forward(X), lambda: ffmlp.Dense(8, 16).forward(W, X),
              lambda: ffmlp.SoftmaxHead(8, 16).cross_entropy(W, X, t, None),
              lambda: ffmlp.SoftmaxHead(8, 16).distill(W, X, t[:, None], X[:, :1], None)]:
        with pytest.raises(ValueError, match="GPU"):
            f()


def test_workspace_sizes(ffmlp):
    d = ffmlp.Dense(1024, 4096, "gelu")
    assert d.workspace_bytes(8192) >= 8192 * 4096 * 2  # the rounded delta
    assert ffmlp.Dense(8, 8).workspace_bytes(8, ffmlp.MLP_MODE_INFER) == 0
    h = ffmlp.SoftmaxHead(2048, 1 << 17)
    # the logits of 16384 tokens would take 8 GiB; a piece of them takes 1 GiB
    assert h.workspace_bytes(16384) < 3 << 29
    # without gradients: sums per row and run, and where each 128 columns begin
    assert h.workspace_bytes(16384, ffmlp.MLP_MODE_INFER) < 64 << 20
    assert h.workspace_bytes(64, top=1024) > h.workspace_bytes(64)
    assert ffmlp.LayerNorm(512).workspace_bytes(100, ffmlp.MLP_MODE_INFER) == 0


def test_a_workspace_size_is_that_of_its_own_call(ffmlp):
    """The remembered size may be replaced by another thread's call at any
    moment: a call never checks its workspace against that one's."""
    class Racing(ffmlp.SoftmaxHead):
        mine, reads = ((8, ffmlp.MLP_MODE_TRAIN, 1), 12345), 0

        @property
        def _need(self):
            self.reads += 1
            return self.mine if self.reads == 1 else ((1, ffmlp.MLP_MODE_INFER, 1), 0)

    assert Racing(16, 32)._ws_bytes(8, ffmlp.MLP_MODE_TRAIN, 1) == 12345


def test_the_two_sides_of_a_step_keep_their_workspace_sizes(ffmlp):
    """A forward call's size does not replace the backward call's."""
    asked = []

    class Counting(ffmlp.Dense):
        def workspace_bytes(self, M, mode=ffmlp.MLP_MODE_TRAIN):
            asked.append((M, mode))
            return super().workspace_bytes(M, mode)

    d = Counting(512, 512, "gelu")
    for _ in range(3):
        infer, train = d._ws_bytes(64, ffmlp.MLP_MODE_INFER), d._ws_bytes(64)
        assert infer == d.workspace_bytes(64, ffmlp.MLP_MODE_INFER) and train == d.workspace_bytes(64)
    # three times by the test itself, once by the layer
    assert asked.count((64, ffmlp.MLP_MODE_INFER)) == 4 and asked.count((64, ffmlp.MLP_MODE_TRAIN)) == 4


def test_a_piece_is_as_large_as_it_may_be(ffmlp):
    """Where the logits outgrow one piece by a little, only a little of them is
    left to further pieces (and computed again): the first keeps its size."""
    h = ffmlp.SoftmaxHead(64, 40000)
    whole, more = h.workspace_bytes(13400), h.workspace_bytes(13500)
    assert 13400 * 40000 < 1 << 29 < 13500 * 40000
    assert 0.98 * whole < more < 1.05 * whole
