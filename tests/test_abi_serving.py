"""Refusals of the serving entry points (CPU: every call fails validation or has
nothing to do, so none reaches a GPU)."""
import ctypes as C

import pytest
import torch

from paper_2608_28511_amd import _lib as L
from paper_2608_28511_amd import layer

P = C.c_void_p(0x10000)
ODD = C.c_void_p(0x10002)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return L.load(build_if_missing=True)


def test_quant(lib):
    rows, weights = lib.moe_quant_rows_i8, lib.moe_quant_weights_i8
    assert rows(P, 0, 16, P, P, None) == 0
    for D in (0, 8, 24, 65552, -16):
        assert rows(P, 4, D, P, P, None) == -2
    assert rows(P, -1, 16, P, P, None) == -2 and rows(P, 1 << 31, 16, P, P, None) == -2
    assert rows(None, 4, 16, P, P, None) == -1 and rows(P, 4, 16, None, P, None) == -1
    assert rows(P, 4, 16, P, None, None) == -1
    assert rows(ODD, 4, 16, P, P, None) == -3 and rows(P, 4, 16, C.c_void_p(0x10008), P, None) == -3
    assert weights(P, 0, 16, 8, P, P, None) == -2 and weights(P, 1025, 16, 8, P, P, None) == -2
    assert weights(P, 2, 24, 8, P, P, None) == -2 and weights(P, 2, 16, 12, P, P, None) == -2
    assert weights(P, 2, 65536, 16384, P, P, None) == -6
    assert weights(P, 2, 16, 8, P, None, None) == -1 and weights(P, 2, 16, 8, P, C.c_void_p(0x10004), None) == -3


def test_grouped_gemm_i8(lib):
    f = lib.moe_grouped_gemm_i8
    assert f(P, P, P, 2, 0, 16, 8, P, P, 0, P, None) == 0
    assert f(P, P, P, 2, 4, 24, 8, P, P, 0, P, None) == -2 and f(P, P, P, 2, 4, 16, 12, P, P, 0, P, None) == -2
    assert f(P, P, P, 2, -1, 16, 8, P, P, 0, P, None) == -2
    assert f(P, P, P, 2, 4, 16, 8, P, P, 2, P, None) == -6
    assert f(P, P, None, 2, 4, 16, 8, P, P, 0, P, None) == -1      # only one dense weight goes without a schedule
    assert f(P, None, P, 2, 4, 16, 8, P, P, 0, P, None) == -1
    assert f(C.c_void_p(0x10008), P, P, 2, 4, 16, 8, P, P, 0, P, None) == -3
    assert f(P, P, P, 2, 4, 16, 8, P, C.c_void_p(0x10004), 0, P, None) == -3


def test_latent_and_ffn_i8(lib):
    assert lib.moe_latent_proj_i8_workspace_bytes(5, 24) == 0
    assert lib.moe_latent_proj_i8_workspace_bytes(-1, 16) == 0
    assert lib.moe_latent_proj_i8_workspace_bytes(32, 4096) == 0    # a small call needs none
    n = lib.moe_latent_proj_i8_workspace_bytes(33, 2688)
    assert n >= 33 * 2688 + 33 * 4
    assert lib.moe_latent_proj_i8_workspace_bytes(5, 4112) >= 5 * 4112 + 20
    f = lib.moe_latent_proj_i8
    assert f(P, P, P, 33, 2688, 8, P, P, n - 1, None) == -4 and f(P, P, P, 33, 2688, 8, P, None, n, None) == -4
    assert f(P, P, P, 33, 2688, 8, P, C.c_void_p(0x10010), n, None) == -3
    assert f(P, P, P, 33, 2680, 8, P, P, n, None) == -2 and f(P, P, None, 33, 2688, 8, P, P, n, None) == -1
    assert f(P, P, P, 5, 2680, 8, P, None, 0, None) == -2 and f(P, P, P, -1, 2688, 8, P, None, 0, None) == -2
    assert f(ODD, P, P, 5, 2688, 8, P, None, 0, None) == -3 and f(P, P, P, 0, 2688, 8, P, None, 0, None) == 0
    g = lib.moe_grouped_ffn_i8
    n = lib.moe_grouped_ffn_i8_workspace_bytes(8, 1000, 64, 48)
    assert n >= 1000 * (64 + 2 * 48)
    assert lib.moe_grouped_ffn_i8_workspace_bytes(8, 1000, 64, 40) == 0
    assert g(P, P, 8, 1000, 64, 48, P, P, P, P, P, P, n - 1, None) == -4
    assert g(P, P, 8, 1000, 64, 40, P, P, P, P, P, P, n, None) == -2
    assert g(P, P, 8, 1000, 65536, 16384, P, P, P, P, P, P, BIG, None) == -6
    assert g(P, P, 8, 1000, 64, 48, P, P, P, None, P, P, n, None) == -1
    assert g(P, P, 8, 0, 64, 48, P, P, P, P, P, P, n, None) == 0


def _few(**kw):
    a = L.LayerFewArgs()
    a.struct_size = C.sizeof(L.LayerFewArgs)
    a.S, a.D, a.E, a.K, a.F = 3, 32, 8, 2, 48
    for n in ("x", "Wr", "W1", "W2", "y"):
        setattr(a, n, 0x10000)
    a.ws, a.ws_bytes = 0x10000, BIG
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change, code", [
    (dict(struct_size=8), -2), (dict(S=65), -2), (dict(S=-1), -2), (dict(K=9), -2), (dict(E=1025), -2),
    (dict(D=20), -2), (dict(F=0), -2), (dict(Fs=12, Ws1=0x10000, Ws2=0x10000), -2), (dict(score_fn=2), -2),
    (dict(weights=2), -2), (dict(sel_bias=0x10000), -2), (dict(s1=0x10000), -2), (dict(Ws1=0x10000), -2),
    (dict(Fs=16), -1), (dict(x=None), -1), (dict(W2=None), -1), (dict(y=0x10008), -3), (dict(W1=0x10008), -3),
    (dict(weights=1), -1), (dict(weights=1, F=40), -2), (dict(weights=1, s1=0x10000, s2=0x10004), -3),
    (dict(ws=None), -4), (dict(ws_bytes=64), -4), (dict(ws=0x10010), -3), (dict(topk_idx=0x10002), -3),
    (dict(D=65536, F=16384), -6), (dict(S=0), 0)])
def test_layer_few(lib, change, code):
    assert lib.moe_layer_few(C.byref(_few(**change)), None) == code


def test_layer_few_workspace(lib):
    assert lib.moe_layer_few(None, None) == -1
    assert lib.moe_layer_few_workspace_bytes(C.byref(_few(S=65))) == 0
    assert lib.moe_layer_few_workspace_bytes(C.byref(_few(S=0))) == 0
    n = lib.moe_layer_few_workspace_bytes(C.byref(_few()))
    assert n > 0
    assert lib.moe_layer_few(C.byref(_few(ws_bytes=n - 1)), None) == -4


@pytest.mark.parametrize("weights", [0, 1])
@pytest.mark.parametrize("sizes", [dict(D=32, E=8, K=2, F=48), dict(D=2688, E=512, K=22, F=1344, Fs=2688),
                                   dict(D=4096, E=64, K=32, F=16)])
def test_layer_few_workspace_serves_fewer_tokens(lib, sizes, weights):
    n = [lib.moe_layer_few_workspace_bytes(C.byref(_few(S=S, weights=weights, **sizes))) for S in range(1, 65)]
    assert n == sorted(n) and n[0] > 0


def test_few_struct_layout(tmp_path):
    """The ctypes mirror has the C layout (offsets printed by a C program)."""
    import shutil
    import subprocess
    from pathlib import Path
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    root = Path(__file__).resolve().parents[1]
    names = [f for f, _ in L.LayerFewArgs._fields_]
    src = tmp_path / "off.c"
    src.write_text('#include <stdio.h>\n#include "moe.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu\\n", offsetof(moe_layer_few_args, {f}));\n' for f in names) +
                   '  printf("%zu %d\\n", sizeof(moe_layer_few_args), MOE_FEW_MAX_TOKENS);\n  return 0;\n}\n')
    exe = tmp_path / "off"
    subprocess.run(["gcc", "-std=c99", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", str(root / "include"),
                    str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [getattr(L.LayerFewArgs, f).offset for f in names] + [
        C.sizeof(L.LayerFewArgs), L.FEW_MAX_TOKENS]


def test_python_layer_refuses(lib):
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    i8 = lambda *s: torch.zeros(s, dtype=torch.int8)  # noqa: E731
    f32 = lambda *s: torch.zeros(s)  # noqa: E731
    with pytest.raises(ValueError):
        layer.quant_rows_i8(bf(4, 32))                                   # a host tensor
    with pytest.raises(ValueError):
        layer.latent_proj_i8(bf(4, 32), i8(8, 48), f32(8))
    with pytest.raises(ValueError):
        layer.grouped_ffn_i8(bf(4, 32), torch.zeros(3, dtype=torch.int32), i8(2, 16, 32), f32(2, 16), i8(2, 16, 32),
                             f32(2, 32))
    ok = dict(S=4, Wr=f32(32, 8), W1=bf(8, 32, 48), W2=bf(8, 48, 32), K=2)
    for bad in (dict(W2=bf(8, 32, 48)), dict(Wr=f32(8, 32)), dict(s2=f32(8, 32)), dict(Ws1=bf(32, 16)),
                dict(bias=f32(7))):
        with pytest.raises(ValueError):
            layer.LayerFew(**{**ok, **bad})
    with pytest.raises(ValueError):
        layer.LayerFew(**ok)                                             # host tensors
