"""Host-only checks of the 8-bit operators: what they refuse, before anything touches a device, and the 64-bit oracle."""
import ctypes
import re
import struct
import subprocess
import types

import numpy as np
import pytest
import torch

import oracle.scaled as ref
from paper_2510_25977_amd import binding as B
from tests.conftest import ROOT

OK, BAD, UNSUPPORTED, SMALL = B.SVDMLP_OK, B.SVDMLP_INVALID_ARGUMENT, B.SVDMLP_UNSUPPORTED, B.SVDMLP_WORKSPACE_TOO_SMALL
BF16, F32, F8 = B.SVDMLP_BF16, B.SVDMLP_F32, B.SVDMLP_F8

# the fields of the header's argument structures with a call that is right in everything but that it has no rows
QUANTIZE = dict(rows=0, cols=256, type=BF16, block_rows=1, x=0x1000, gated=0, x_ld=256, gated_ld=0, codes=0x2000, scales=0x3000,
                codes_ld=256, scales_ld=64)
NORM = dict(rows=0, d=256, type=BF16, stream_type=BF16, out_type=F8, kind=B.NORM_RMS, next_kind=B.NORM_RMS, gate_act=0, gate_rows=4,
            eps=1e-6, next_eps=1e-6, weight_plus=0.0, residual_scale=1.0, residual=0x1000, branch=0x2000, residual_ld=256,
            branch_ld=256, weight=0x3000, bias=0x3000, branch_scale=0x3000, gate=0x4000, gate_ld=256, next_weight=0x3000,
            next_bias=0x3000, h=0x5000, h_ld=256, out=0x6000, out_ld=256, out_scales=0x7000, out_scales_ld=64)
MATMUL = dict(M=0, N=64, K=256, out_type=F8, gated=0, a=0x1000, a_scales=0x2000, a_ld=256, a_scales_ld=64, w=0x3000, w_scales=0x4000,
              w_ld=256, c=0x5000, c_scales=0x6000, c_ld=64, c_scales_ld=64, workspace=0x7000, workspace_bytes=1 << 30)
CALLS = {"svdmlp_quantize": (QUANTIZE, struct.Struct("=qqiiQQqqQQqq")),
         "svdmlp_norm": (NORM, struct.Struct("=qqiiiiiiqffffQQqqQQQQqQQQqQqQq")),
         "svdmlp_scaled_matmul": (MATMUL, struct.Struct("=qqqiiQQqqQQqQQqqQQ"))}


def status(name, **changed):
    fields, layout = CALLS[name]
    assert set(changed) <= set(fields)
    return getattr(B.lib(), name)(layout.pack(*{**fields, **changed}.values()), None)


def test_overlap_of_matrices_byte_for_byte(tmp_path):
    """The host's check for shared memory against sets of bytes, over all small matrices of a buffer: no overlap is missed and
    none is seen where rows of one lie in the gaps of the other."""
    (tmp_path / "t.cpp").write_text(r"""
#include <cstdio>
#include "rows.h"
using namespace svdmlp;
int main() {
  static char buf[1];
  const int64_t base = (int64_t)(uintptr_t)buf;      // addresses only, nothing is read
  long cases = 0, wrong = 0, shared = 0;
  auto at = [&](int64_t x) { return (const void*)(uintptr_t)(base + x); };
  for (int ra = 1; ra <= 4; ++ra) for (int wa = 1; wa <= 4; ++wa) for (int la = wa; la <= 7; ++la)
  for (int rb = 1; rb <= 4; ++rb) for (int wb = 1; wb <= 4; ++wb) for (int lb = wb; lb <= 7; ++lb)
  for (int off = 0; off < 30; ++off) {
    unsigned long long a = 0, b = 0;
    for (int r = 0; r < ra; ++r) for (int e = 0; e < wa; ++e) a |= 1ull << (r * la + e);
    for (int r = 0; r < rb; ++r) for (int e = 0; e < wb; ++e) b |= 1ull << (off + r * lb + e);
    const Rows x{at(0), ra, wa, la}, y{at(off), rb, wb, lb};
    const bool want = a & b;
    wrong += overlap(x, y) != want;
    wrong += overlap(y, x) != want;
    shared += want;
    ++cases;
  }
  wrong += overlap({at(0), 1, 4, 0}, {at(4), 1, 4, -9}) + !overlap({at(0), 1, 4, 0}, {at(3), 1, 4, 0});      // one row: no stride
  wrong += overlap({nullptr, 4, 4, 4}, {at(0), 4, 4, 4}) + overlap({at(0), 0, 4, 4}, {at(0), 4, 4, 4});
  std::printf("%ld %ld %ld", cases, shared, wrong);
}
""")
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{ROOT}/paper_2510_25977_amd/csrc", "t.cpp", "-o", "t"], cwd=tmp_path, check=True)
    cases, shared, wrong = map(int, subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split())
    assert wrong == 0 and 0 < shared < cases == 30 * (4 * (7 + 6 + 5 + 4)) ** 2


@pytest.mark.parametrize("name,changed", [
    # rows of 512 bytes of x, 256 of codes; each call shares memory between what it writes and something else
    ("svdmlp_quantize", dict(codes=0x1100)), ("svdmlp_quantize", dict(codes=0xF00)), ("svdmlp_quantize", dict(scales=0x1700)),
    ("svdmlp_quantize", dict(gated=0x8000, gated_ld=256, codes=0x8010)), ("svdmlp_quantize", dict(scales=0x2100)),
    ("svdmlp_quantize", dict(block_rows=128, scales=0x17FC)),
    ("svdmlp_norm", dict(h=0x1200)), ("svdmlp_norm", dict(h=0xE00)), ("svdmlp_norm", dict(h=0x2004)), ("svdmlp_norm", dict(h=0x2E02)),
    ("svdmlp_norm", dict(h=0x41FE)), ("svdmlp_norm", dict(out=0x1100)), ("svdmlp_norm", dict(out=0x2700)), ("svdmlp_norm", dict(out=0x5100)),
    ("svdmlp_norm", dict(out_scales=0x30FE)), ("svdmlp_norm", dict(out_scales=0x6080)), ("svdmlp_norm", dict(out_scales=0x5100)),
    ("svdmlp_norm", dict(out_type=BF16, out=0x6000, h=0x6100)), ("svdmlp_norm", dict(bias=0x5010)), ("svdmlp_norm", dict(next_bias=0x6010)),
    ("svdmlp_scaled_matmul", dict(c=0x1100)), ("svdmlp_scaled_matmul", dict(c=0x10010)), ("svdmlp_scaled_matmul", dict(c=0x2080)),
    ("svdmlp_scaled_matmul", dict(c=0x20000)), ("svdmlp_scaled_matmul", dict(c_scales=0x50C0)), ("svdmlp_scaled_matmul", dict(c_scales=0x10100)),
])
def test_outputs_that_share_memory_are_refused(name, changed):
    matmul = name == "svdmlp_scaled_matmul"
    four = dict(M=4, w=0x10000, w_scales=0x20000) if matmul else dict(rows=4)       # all apart but for what is changed
    assert status(name, **four, **changed) == BAD


@pytest.mark.parametrize("workspace", [0x1000010, 0x1100000, 0x2000000, 0x2800000, 0x3000000 - 16, 0x3100000])
def test_a_workspace_that_shares_memory_is_refused(workspace):
    args = dict(M=16, N=512, K=14336, a=0x1000000, a_ld=14336, a_scales=0x1100000, w=0x2000000, w_ld=14336, w_scales=0x2800000,
                c=0x3000000, c_ld=512, c_scales=0x3100000, workspace=workspace)
    assert B.svdmlp_scaled_matmul_workspace_bytes(16, 512, 14336, F8) > 16
    assert status("svdmlp_scaled_matmul", **args) == BAD


def test_packed_arguments_are_the_headers_structures():
    """The struct formats of these tests field for field against the header: order, kind and size."""
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "svdmlp.h").read_text(), flags=re.S)
    for name, (fields, layout) in CALLS.items():
        body = re.search(r"typedef struct \{([^}]*)\}\s*" + name + "_args;", text).group(1)
        names, fmt = [], ""
        for line in body.split(";"):
            if not line.strip():
                continue
            kind, rest = re.match(r"\s*(const void|void|const float|float|int64_t|int32_t|size_t)\b(.*)", line, flags=re.S).groups()
            for f in rest.split(","):
                fmt += "Q" if "*" in f or kind == "size_t" else {"int64_t": "q", "int32_t": "i", "float": "f"}[kind]
                names.append(f.strip(" *\n"))
        assert names == list(fields), name
        assert "=" + fmt == layout.format, name
        native = ctypes.sizeof(type("S", (ctypes.Structure,), {"_fields_": [
            (f"f{i}", {"q": ctypes.c_int64, "i": ctypes.c_int32, "f": ctypes.c_float, "Q": ctypes.c_void_p}[c]) for i, c in enumerate(fmt)]}))
        assert native == layout.size, name                 # the C layout has no gaps


@pytest.mark.parametrize("name", CALLS)
def test_no_rows_are_accepted_and_null_arguments_refused(name):
    assert status(name) == OK
    assert getattr(B.lib(), name)(None, None) == BAD


@pytest.mark.parametrize("changed,want", [
    (dict(rows=-1), BAD), (dict(cols=0), BAD), (dict(type=F8), BAD), (dict(type=7), BAD), (dict(block_rows=64), BAD),
    (dict(x=0), BAD), (dict(x=0x1001), BAD), (dict(x_ld=255), BAD), (dict(gated=0x1001, gated_ld=256), BAD), (dict(gated=0x1100, gated_ld=10), BAD),
    (dict(codes=0), BAD), (dict(codes=0x2008), BAD), (dict(codes_ld=264), BAD), (dict(codes_ld=240), BAD), (dict(scales=0), BAD),
    (dict(scales=0x3001), BAD), (dict(block_rows=128, scales=0x3002), BAD), (dict(codes=0x1000), BAD), (dict(rows=65), BAD), (dict(codes_ld=1 << 23), UNSUPPORTED),
    (dict(block_rows=128, gated=0x1100, gated_ld=256), BAD), (dict(rows=1 << 24, scales_ld=1 << 24), UNSUPPORTED),
    (dict(cols=1 << 23, x_ld=1 << 23, codes_ld=(1 << 23) - 16), BAD), (dict(block_rows=128, scales_ld=0), OK), (dict(gated=0x1100, gated_ld=300), OK),
])
def test_quantize_refuses(changed, want):
    assert status("svdmlp_quantize", **changed) == want


@pytest.mark.parametrize("changed,want", [
    (dict(rows=-1), BAD), (dict(d=0), BAD), (dict(type=F8), BAD), (dict(stream_type=5), BAD), (dict(out_type=F32), BAD),
    (dict(kind=3), BAD), (dict(next_kind=-1), BAD), (dict(gate_act=3), BAD), (dict(residual=0, branch=0), BAD), (dict(out=0), BAD),
    (dict(next_kind=B.NORM_NONE), BAD),                                             # an out that nothing makes
    (dict(next_kind=B.NORM_NONE, out=0, h=0), BAD), (dict(next_kind=B.NORM_NONE, out=0), BAD),      # next_weight without a norm
    (dict(next_kind=B.NORM_NONE, out=0, next_weight=0, next_bias=0), OK),
    (dict(branch=0), BAD), (dict(kind=B.NORM_NONE), BAD), (dict(kind=B.NORM_NONE, weight=0, bias=0), OK), (dict(eps=0.0), BAD),
    (dict(eps=float("nan")), BAD), (dict(next_eps=-1.0), BAD), (dict(gate_rows=0), BAD), (dict(gate_ld=255), BAD), (dict(gate=0, gate_rows=0), OK),
    (dict(residual_ld=255), BAD), (dict(branch_ld=10), BAD), (dict(h_ld=255), BAD), (dict(weight=0x3001), BAD), (dict(h=0x5001), BAD),
    (dict(stream_type=F32, residual=0x1002), BAD), (dict(out=0x6008), BAD), (dict(out_ld=264), BAD), (dict(out_scales=0), BAD),
    (dict(rows=65), BAD), (dict(out_type=BF16, out_ld=255), BAD), (dict(out_type=BF16, out=0x6001), BAD), (dict(out_type=BF16, out_scales=0), OK),
    (dict(h=0x1000), OK), (dict(h=0x1000, h_ld=300), BAD), (dict(h=0x2000), BAD), (dict(out=0x1000), BAD), (dict(out=0x5000), BAD),
    (dict(type=F32, stream_type=BF16, out_type=F32), UNSUPPORTED), (dict(stream_type=F32), OK), (dict(residual=0), OK), (dict(h=0), OK),
    (dict(d=32769, residual_ld=40000, branch_ld=40000, gate_ld=40000, h_ld=40000, out_ld=40000), UNSUPPORTED),
    (dict(rows=1 << 25, out_scales_ld=1 << 25), UNSUPPORTED),
    (dict(rows=1 << 21, d=16385, residual_ld=40000, branch_ld=40000, gate_ld=40000, h_ld=40000, out_ld=40000, out_scales_ld=1 << 21),
     UNSUPPORTED),
])
def test_norm_refuses(changed, want):
    assert status("svdmlp_norm", **changed) == want


@pytest.mark.parametrize("changed,want", [
    (dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(out_type=3), BAD), (dict(out_type=F32), BAD), (dict(gated=2), BAD), (dict(gated=-1), BAD),
    (dict(gated=1), OK), (dict(gated=1, K=128), BAD), (dict(gated=1, K=384, a_ld=384, w_ld=384), BAD), (dict(gated=1, out_type=BF16), OK),
    (dict(a=0), BAD),
    (dict(a=0x1008), BAD), (dict(a_ld=248), BAD), (dict(a_ld=240), BAD), (dict(w=0), BAD), (dict(w=0x3001), BAD), (dict(w_ld=255), BAD),
    (dict(a_scales=0), BAD), (dict(w_scales=0), BAD), (dict(a_scales=0x2001), BAD), (dict(M=65), BAD), (dict(c=0), BAD), (dict(c=0x5004), BAD),
    (dict(c_ld=56), BAD), (dict(c_scales=0), BAD), (dict(c=0x1000), BAD), (dict(c=0x3000), BAD), (dict(out_type=BF16, c=0x5001), BAD),
    (dict(out_type=BF16, c=0x5002, c_ld=65), OK), (dict(out_type=BF16, c_ld=63), BAD), (dict(out_type=BF16, c_scales=0), OK),
    (dict(a_ld=1 << 23), UNSUPPORTED), (dict(w_ld=1 << 23), UNSUPPORTED), (dict(M=1 << 24), UNSUPPORTED), (dict(N=(1 << 22) + 1), UNSUPPORTED),
    (dict(K=(1 << 22) + 1), UNSUPPORTED),
    (dict(M=1 << 23, N=1 << 16, c_ld=1 << 16, a_scales_ld=1 << 23, c_scales_ld=1 << 23), UNSUPPORTED),
])
def test_scaled_matmul_refuses(changed, want):
    assert status("svdmlp_scaled_matmul", **changed) == want


def test_scaled_matmul_workspace():
    """Extents that need a workspace say so, and a call without it is refused; bad extents need none."""
    need = B.svdmlp_scaled_matmul_workspace_bytes(16, 512, 14336, F8)
    assert need >= 16 * 512 * 4
    args = dict(M=16, N=512, K=14336, a_ld=14336, w_ld=14336, c_ld=512)
    assert status("svdmlp_scaled_matmul", **args, workspace_bytes=need - 1) == SMALL
    assert status("svdmlp_scaled_matmul", **args, workspace=0) == BAD
    assert status("svdmlp_scaled_matmul", **args, workspace=0x7008) == BAD
    for bad in ((-1, 1, 1, F8), (1, 0, 1, F8), (1, 1, 0, BF16), (1, 1, 1, F32)):
        assert B.svdmlp_scaled_matmul_workspace_bytes(*bad) == 0
        with pytest.raises(B.SvdMlpError):
            B.svdmlp_scaled_matmul_describe(*bad)


def test_the_gpu_tests_sizes_reach_every_kernel_of_the_product():
    """Every kernel, with whole and cut contractions, into bf16 and 8 bits, as far as the planner takes them at all."""
    from tests.test_gpu_scaled import MATMULS
    seen = set()
    for M, N, K in MATMULS:
        for out in (BF16, F8):
            d = B.svdmlp_scaled_matmul_describe(M, N, K, out)
            seen.add((re.match(r"k_mm_\w+\[tile=\d+x\d+", d).group(0), "ranges=1 " in d, out))
            assert ("k_mm_join" in d) == (B.svdmlp_scaled_matmul_workspace_bytes(M, N, K, out) > 0)
    kernels = ["k_mm_few[tile=16x16", "k_mm_ring[tile=32x64", "k_mm_ring[tile=64x64", "k_mm_ring[tile=64x128", "k_mm_tile[tile=128x256",
               "k_mm_tile[tile=256x256"]
    assert seen == {(k, whole, out) for k in kernels for whole in (True, False) for out in (BF16, F8)}


@pytest.mark.parametrize("M,N,K,kernel", [
    (1, 4096, 4096, "few"), (16, 4096, 4096, "few"), (1, 14336, 4096, "ring[tile=32x64"), (16, 14336, 4096, "ring[tile=32x64"),
    (128, 8192, 2048, "ring[tile=32x64"), (256, 4096, 4096, "ring[tile=32x64"), (300, 4096, 8192, "ring[tile=64x64"),
    (1024, 4096, 4096, "ring[tile=64x128"), (512, 14336, 4096, "tile[tile=128x256"), (2048, 4096, 4096, "tile[tile=128x256"),
    (1777, 7301, 2687, "tile[tile=256x256"), (4096, 16384, 8192, "tile[tile=256x256"), (286, 7424, 13184, "tile[tile=256x256 tiles=58 ranges=4"),
])
def test_the_products_planner_takes_what_measured_fastest(M, N, K, kernel):
    assert B.svdmlp_scaled_matmul_describe(M, N, K, BF16).startswith("k_mm_" + kernel)


def test_gated_products_have_three_kernels():
    """Sizes of the GPU tests reach all; none cuts the contraction."""
    from tests.test_gpu_scaled import GATED
    seen = {B.svdmlp_scaled_matmul_describe(M, N, K, F8, True).split(" ")[0] for M, N, K in GATED}
    assert seen == {"k_mm_ring[tile=32x128", "k_mm_ring[tile=64x128", "k_mm_tile[tile=128x256"}
    for M, N, K in GATED:
        assert "ranges=1 " in B.svdmlp_scaled_matmul_describe(M, N, K, F8, True)
    for K in (16, 128, 384):
        with pytest.raises(B.SvdMlpError):
            B.svdmlp_scaled_matmul_describe(64, 64, K, F8, True)


class _OnDevice(torch.Tensor):
    """A CPU tensor that says it lies on the GPU: the binding's checks need no more."""
    is_cuda = property(lambda self: True)


def fake(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape).to(dtype).as_subclass(_OnDevice)


def test_the_binding_checks_tensors(monkeypatch):
    monkeypatch.setattr(B, "_run", lambda *a: None)
    x = fake(4, 256)
    good = B.empty_scaled(4, 256, "cpu")
    weights = B.empty_scaled(64, 256, "cpu", 128)
    pair = (good.codes.as_subclass(_OnDevice), good.scales)
    assert good.codes.shape == (4, 256) and good.scales.shape == (2, 4) and weights.scales.shape == (1, 2)
    assert B.empty_scaled(3, 33, "cpu").codes.stride() == (48, 1)
    assert B.quantize(x, out=good).codes is good.codes
    for call in (lambda: B.quantize(torch.zeros(4, 256)),                                     # not on the GPU
                 lambda: B.quantize(fake(4, 256, dtype=torch.float16)), lambda: B.quantize(fake(4, 4, 4)),
                 lambda: B.quantize(x.t()),                                                   # columns in one piece, not rows
                 lambda: B.quantize(x, fake(4, 255)), lambda: B.quantize(x, fake(4, 256, dtype=torch.float32)),
                 lambda: B.quantize(x, out=B.empty_scaled(4, 255, "cpu")), lambda: B.quantize(x, out=weights),
                 lambda: B.quantize(x, block_rows=128, out=(weights.codes[:4], good.scales)),
                 lambda: B.norm_in(x, fake(255)), lambda: B.norm_in(x, fake(256, dtype=torch.float16)),
                 lambda: B.norm_in(x, add=fake(5, 256)), lambda: B.norm_in(x, h=fake(4, 256, dtype=torch.float32)),
                 lambda: B.norm_in(x, out=fake(4, 256, dtype=torch.float32)), lambda: B.norm_out(x, x, gate=fake(3, 256)),
                 lambda: B.norm_out(x, x, out=x.clone(), next_kind=B.NORM_NONE), lambda: B.norm_in(x, kind=B.NORM_NONE, scaled=True),
                 lambda: B.quantize(x, out=(good.codes, None)), lambda: B.norm_in(x, [1.0], out=x.clone()),
                 lambda: B.quantize(x, block_rows=1 << 40, out=weights), lambda: B.norm_in(x, kind=1 << 35),
                 lambda: B.norm_out(x, x, gate=x, gate_rows=0), lambda: B.norm_out(x, x, gate=x, gate_rows=2),
                 lambda: B.scaled_matmul(pair, B.empty_scaled(64, 128, "cpu", 128)),
                 lambda: B.scaled_matmul(pair, (weights.codes, weights.scales.t())),
                 lambda: B.scaled_matmul(pair, weights, out_dtype=torch.float32),
                 lambda: B.scaled_matmul(pair, weights, out=fake(4, 64, dtype=torch.float32)),
                 lambda: B.scaled_matmul(pair, weights, out=fake(4, 63)),
                 lambda: B.scaled_matmul((x, good.scales), weights)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        B.SvdMlpF8(Ug=fake(256, 64), Vg=fake(64, 512))                                        # four factors missing
    with pytest.raises(ValueError):
        B.SvdMlpF8(Ug=fake(256, 64), Vg=fake(65, 512), kind=B.SVDMLP_LINEAR)


def test_a_plain_buffer_for_an_8_bit_result_is_refused(monkeypatch):
    """A call that asks for codes and hands over a plain tensor would get the plain result without a word."""
    monkeypatch.setattr(B, "_run", lambda *a: None)
    x, plain = fake(4, 256), fake(4, 256)
    a, w = B.empty_scaled(4, 256, "cpu"), B.empty_scaled(256, 256, "cpu", 128)
    a = (a.codes.as_subclass(_OnDevice), a.scales)
    codes = B.empty_scaled(4, 256, "cpu")
    for call in (lambda out: B.norm_in(x, out=out, scaled=True), lambda out: B.norm_out(x, x.clone(), out=out, scaled=True)[1],
                 lambda out: B.scaled_matmul(a, w, out=out, out_dtype=torch.float8_e4m3fn)):
        with pytest.raises(ValueError, match="8-bit"):
            call(plain)
        assert call(codes) is codes and type(call(None)) is B.Scaled
    assert B.scaled_matmul(a, w, out=codes) is codes and B.scaled_matmul(a, w, out=plain) is plain


def fields_of(monkeypatch, call):
    """The argument structure that a call of the binding hands over, by field."""
    got = []
    monkeypatch.setattr(B, "_run", lambda name, args, device: got.append((name, args, device)))
    call()
    (name, args, device), = got
    names, layout = CALLS[name]
    assert device == -1
    return None if args is None else dict(zip(names, layout.unpack(args)))


def test_what_the_binding_hands_over(monkeypatch):
    """Every field of every structure, from tensors whose addresses and strides all differ."""
    def strided(rows, cols, dtype, pad):
        return torch.zeros(rows, cols + pad).to(dtype)[:, :cols].as_subclass(_OnDevice)

    def f8(rows, cols, pad, spad):
        return strided(rows, cols, torch.float8_e4m3fn, pad), strided(-(-cols // 128), rows, torch.bfloat16, spad)

    bf, f32 = torch.bfloat16, torch.float32
    x, u, (c, s) = strided(5, 300, f32, 3), strided(5, 300, f32, 7), f8(5, 300, 20, 2)
    want = dict(rows=5, cols=300, type=F32, block_rows=1, x=x.data_ptr(), gated=u.data_ptr(), x_ld=303, gated_ld=307, codes=c.data_ptr(),
                scales=s.data_ptr(), codes_ld=320, scales_ld=7)
    assert fields_of(monkeypatch, lambda: B.quantize(x, u, out=(c, s))) == want
    w = B.empty_scaled(5, 300, "cpu", 128)
    got = fields_of(monkeypatch, lambda: B.quantize(x, block_rows=128, out=w))
    assert got == {**want, "gated": 0, "gated_ld": 0, "block_rows": 128, "codes": w.codes.data_ptr(), "codes_ld": 304,
                   "scales": w.scales.data_ptr(), "scales_ld": 0}
    one = fields_of(monkeypatch, lambda: B.quantize(x[2:3], out=(c[:1], s[:, 3:4])))       # one row: its stride says nothing
    assert one == {**want, "rows": 1, "x": x.data_ptr() + 2 * 303 * 4, "x_ld": 300, "gated": 0, "gated_ld": 0, "codes_ld": 304,
                   "scales": s.data_ptr() + 6}

    res, br, h, gate = strided(5, 300, f32, 1), strided(5, 300, bf, 2), strided(5, 300, f32, 4), strided(3, 300, bf, 5)
    v = [torch.zeros(300, dtype=bf).as_subclass(_OnDevice) for _ in range(5)]
    norm = dict(rows=5, d=300, type=BF16, stream_type=F32, out_type=F8, kind=B.NORM_LAYER, next_kind=B.NORM_RMS, gate_act=B.GATE_TANH,
                gate_rows=2, eps=0.5, next_eps=0.25, weight_plus=1.0, residual_scale=2.0, residual=res.data_ptr(), branch=br.data_ptr(),
                residual_ld=301, branch_ld=302, weight=v[0].data_ptr(), bias=v[1].data_ptr(), branch_scale=v[2].data_ptr(),
                gate=gate.data_ptr(), gate_ld=305, next_weight=v[3].data_ptr(), next_bias=v[4].data_ptr(), h=h.data_ptr(), h_ld=304,
                out=c.data_ptr(), out_ld=320, out_scales=s.data_ptr(), out_scales_ld=7)
    assert fields_of(monkeypatch, lambda: B.norm_out(
        br, res, v[0], bias=v[1], kind=B.NORM_LAYER, eps=0.5, weight_plus=1.0, residual_scale=2.0, branch_scale=v[2], gate=gate, gate_rows=2,
        gate_act=B.GATE_TANH, next_weight=v[3], next_bias=v[4], next_kind=B.NORM_RMS, next_eps=0.25, h=h, out=(c, s))) == norm
    n = strided(5, 300, bf, 6)
    got = fields_of(monkeypatch, lambda: B.norm_in(res, v[3], bias=v[4], add=br, kind=B.NORM_LAYER, eps=0.25, weight_plus=1.0,
                                                   residual_scale=2.0, h=h, out=n))
    assert got == {**norm, "kind": 0, "next_kind": B.NORM_LAYER, "gate_act": 0, "gate_rows": 1, "eps": 0.25, "weight": 0, "bias": 0,
                   "branch_scale": 0, "gate": 0, "gate_ld": 0, "out_type": BF16, "out": n.data_ptr(), "out_ld": 306, "out_scales": 0,
                   "out_scales_ld": 0}

    (a, sa), o = f8(5, 300, 36, 1), strided(5, 70, bf, 9)
    w = B.Scaled(strided(70, 300, torch.float8_e4m3fn, 4), torch.zeros(1, 3))
    mm = dict(M=5, N=70, K=300, out_type=BF16, gated=0, a=a.data_ptr(), a_scales=sa.data_ptr(), a_ld=336, a_scales_ld=6,
              w=w.codes.data_ptr(), w_scales=w.scales.data_ptr(), w_ld=304, c=o.data_ptr(), c_scales=0, c_ld=79, c_scales_ld=0,
              workspace=0, workspace_bytes=B.svdmlp_scaled_matmul_workspace_bytes(5, 70, 300, BF16))
    got = fields_of(monkeypatch, lambda: B.scaled_matmul((a, sa), w, out=o))
    assert {**got, "workspace": 0} == mm and bool(got["workspace"]) == bool(mm["workspace_bytes"])
    q, sq = f8(5, 70, 10, 3)
    got = fields_of(monkeypatch, lambda: B.scaled_matmul((a, sa), w, out=(q, sq)))
    assert {**got, "workspace": 0} == {**mm, "out_type": F8, "c": q.data_ptr(), "c_ld": 80, "c_scales": sq.data_ptr(), "c_scales_ld": 5,
                                       "workspace_bytes": B.svdmlp_scaled_matmul_workspace_bytes(5, 70, 300, F8)}
    g8, gw = f8(5, 512, 0, 0), B.empty_scaled(70, 512, "cpu", 128)
    got = fields_of(monkeypatch, lambda: B.scaled_matmul(g8, gw, gated=True))
    assert (got["gated"], got["out_type"], got["K"], got["workspace"], got["workspace_bytes"]) == (1, BF16, 512, 0, 0)
    a8, w8 = f8(16, 14336, 0, 0), B.empty_scaled(512, 14336, "cpu", 128)
    got = fields_of(monkeypatch, lambda: B.scaled_matmul(a8, w8, out_dtype=torch.float8_e4m3fn))
    assert got["workspace"] and got["workspace_bytes"] == B.svdmlp_scaled_matmul_workspace_bytes(16, 512, 14336, F8) > 0
    for call in (lambda: B.quantize(x[:0]), lambda: B.norm_in(res[:0]), lambda: B.scaled_matmul((a[:0], sa[:, :0]), w)):
        assert fields_of(monkeypatch, call) is None


def test_scales_that_a_stride_repeats_are_refused(monkeypatch):
    """Scales [blocks, rows] whose blocks lie less than `rows` apart (one per row, expanded over the blocks; a buffer of fewer
    rows seen through strides) are not what the kernels read: their stride reaches the C entry, which refuses it."""
    monkeypatch.setattr(B, "_current_device", lambda: -1)
    monkeypatch.setattr(B, "_current_raw_stream", lambda index: 0)
    good = B.empty_scaled(4, 256, "cpu")
    codes = good.codes.as_subclass(_OnDevice)
    per_row = torch.zeros(1, 4, dtype=torch.bfloat16).expand(2, 4)
    weights = B.empty_scaled(64, 256, "cpu", 128)
    out = torch.empty(4, 64, dtype=torch.bfloat16)
    for scales in (per_row, torch.zeros(7, dtype=torch.bfloat16).as_strided((2, 4), (3, 1))):
        with pytest.raises(B.SvdMlpError) as e:
            B.scaled_matmul((codes, scales), weights, out=out)
        assert e.value.status == B.SVDMLP_INVALID_ARGUMENT
        with pytest.raises(B.SvdMlpError):
            B.quantize(fake(4, 256), out=(good.codes, scales))
        with pytest.raises(B.SvdMlpError):
            B.norm_in(fake(4, 256), out=(good.codes, scales))


def test_a_missing_build_is_an_error(monkeypatch, tmp_path):
    monkeypatch.setattr(B, "_checks", None)
    monkeypatch.setattr(B, "TENSORS_PATH", tmp_path / "nope.so")
    with pytest.raises(FileNotFoundError):
        B.quantize(fake(4, 256), out=B.empty_scaled(4, 256, "cpu"))


def test_a_build_for_another_torch_is_an_error(monkeypatch):
    """The tensor checks read torch's own structures, so those compiled for another version are refused and not called."""
    monkeypatch.setattr(B, "_checks", None)
    monkeypatch.setattr(torch, "__version__", "0.0.0")
    for _ in range(2):
        with pytest.raises(ImportError, match="0.0.0"):
            B.quantize(fake(4, 256), out=B.empty_scaled(4, 256, "cpu"))


def test_a_call_on_another_device_makes_it_current(monkeypatch):
    """Kernels go to the current device, so an operator whose tensors lie elsewhere switches to theirs and back, and asks for
    the current stream of that device."""
    now, seen = [0], []

    class on:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *e):
            now[0] = self.before

    monkeypatch.setattr(B, "_current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(B, "_current_raw_stream", lambda index: 100 + index)
    monkeypatch.setattr(B, "lib", lambda: types.SimpleNamespace(op=lambda args, stream: seen.append((now[0], stream)) or 0))
    B._run("op", b"", 1)
    B._run("op", b"", 0)
    B._run("op", None, 0)          # a call of no rows
    assert seen == [(1, 101), (0, 100)] and now == [0]


def test_what_a_call_on_a_stream_makes_is_that_streams(monkeypatch):
    """Results and workspaces are allocated while the given stream is the current one; one of another device is refused."""
    current, made = [None], []

    class on:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            current[0] = self.stream

        def __exit__(self, *e):
            current[0] = None

    empty = torch.empty

    def seen_empty(*args, **kw):
        made.append(current[0])
        return empty(*args, **kw)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", seen_empty)
    monkeypatch.setattr(B, "_run", lambda *a: made.append(current[0]))
    a, w = B.empty_scaled(8, 4096, "cpu"), B.empty_scaled(4096, 4096, "cpu", 128)
    a = (a.codes.as_subclass(_OnDevice), a.scales)
    there, elsewhere = types.SimpleNamespace(device_index=-1), types.SimpleNamespace(device_index=0)
    calls = [(3, lambda s: B.quantize(fake(4, 256), stream=s)), (2, lambda s: B.norm_in(fake(4, 256), stream=s)),
             (3, lambda s: B.norm_in(fake(4, 256), scaled=True, stream=s)), (2, lambda s: B.norm_out(fake(4, 256), stream=s)),
             (3, lambda s: B.norm_out(fake(4, 256), fake(4, 256), next_kind=B.NORM_RMS, stream=s)),
             (4, lambda s: B.scaled_matmul(a, w, out_dtype=torch.float8_e4m3fn, stream=s))]      # with partial sums
    for count, call in calls:
        made.clear()
        call(there)
        assert len(made) == count and all(m is there for m in made)
        with pytest.raises(ValueError):
            call(elsewhere)


@pytest.mark.parametrize("kind,quantised", [(B.SVDMLP_GATED, 4), (B.SVDMLP_LINEAR, 2)])
def test_a_block_is_quantised_when_its_constructor_returns(monkeypatch, kind, quantised):
    """A forward may run on any stream: the constructor waits for its own, where the factors are quantised, after the last of
    them and before a forward can be called.  While that stream is captured nothing runs that could be waited for."""
    done, capturing = [], [False]

    class on:
        def __init__(self, where):
            pass

        def __enter__(self):
            pass

        def __exit__(self, *e):
            pass

    stream = types.SimpleNamespace(synchronize=lambda: done.append("synchronize"))
    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    monkeypatch.setattr(B, "_run", lambda name, *a: done.append(name))
    monkeypatch.setattr(B, "_device_of", lambda t, what: -1)       # what is made between the products lies on the CPU here
    f = dict(Ug=fake(256, 64), Vg=fake(64, 512), Uu=fake(256, 64), Vu=fake(64, 512), Ud=fake(512, 40), Vd=fake(40, 256))
    mlp = B.SvdMlpF8(kind=kind, **f)
    assert done == ["svdmlp_quantize"] * quantised + ["synchronize"]
    mlp.forward(fake(4, 256), stream=types.SimpleNamespace(device_index=-1))
    assert done[quantised + 1:] == ["svdmlp_quantize"] + ["svdmlp_scaled_matmul"] * quantised      # as many products as operands
    done.clear()
    capturing[0] = True
    B.SvdMlpF8(kind=kind, **f)
    assert done == ["svdmlp_quantize"] * quantised


def test_the_e4m3_table_of_the_oracle():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.E4M3, want, equal_nan=True)
    assert np.nanmax(ref.E4M3) == ref.LARGEST and np.isnan(ref.E4M3).sum() == 2


def test_the_oracles_scales_on_a_case_by_hand():
    v = np.zeros((3, 130))
    v[0, 0], v[0, 129], v[1, 5], v[2, 128] = 448.0, -896.0, 44.8, 1e-40
    s = ref.scales_of(v)
    assert s.shape == (2, 3)
    assert np.allclose(s, [[1.0, 0.1, 2.0 ** -100], [2.0, 2.0 ** -100, 2.0 ** -100]], rtol=1e-15)
    assert np.allclose(ref.scales_of(v, 128), [[1.0, 2.0]], rtol=1e-15)
    codes = np.full((3, 130), 0x38, np.uint8)                                       # 1.0
    assert np.allclose(ref.activations(codes, s)[:, [0, 127, 128]], s.T[:, [0, 0, 1]])
    assert np.allclose(ref.weights(codes, np.array([[1.0, 2.0]]))[1, [127, 129]], [1.0, 2.0])
