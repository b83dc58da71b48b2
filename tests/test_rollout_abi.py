"""The entry points of the rollout's last stage without a GPU: struct layouts, and argument errors before any CUDA call."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2512_23087_b200 import build, binding
    build.build()
    return binding.load_library()


def _structs():
    from paper_2512_23087_b200 import binding as b
    return {"dvp_rms_norm_args": b.RmsNormArgs, "dvp_rms_norm_backward_args": b.RmsNormBackwardArgs,
            "dvp_quantize_fp8_args": b.QuantizeFp8Args, "dvp_gemm_fp8_args": b.GemmFp8Args,
            "dvp_sample_args": b.SampleArgs}


def test_struct_layout_matches_the_header(tmp_path):
    structs = _structs()
    lines = []
    for cname, cls in structs.items():
        lines.append(f'printf("{cname} %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname}.{f[0]} %zu\\n", offsetof({cname}, {f[0]}));' for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "dvp.h"\nint main(void){' + "".join(lines) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for cname, cls in structs.items():
        assert int(out[cname]) == ctypes.sizeof(cls), cname
        for f in cls._fields_:
            assert int(out[f"{cname}.{f[0]}"]) == getattr(cls, f[0]).offset, f"{cname}.{f[0]}"


def _filled(cls, **fields):
    a = cls()
    a.struct_size = ctypes.sizeof(cls)
    for name, value in fields.items():
        setattr(a, name, value)
    return a


def _refused(fn, cls, good, cases):
    """Every case differs from `good`, which would be launched, in what makes it wrong."""
    for status, change in cases:
        assert fn(ctypes.byref(_filled(cls, **{**good, **change}))) == status, change


def test_norm_refusals(lib):
    from paper_2512_23087_b200 import binding as b
    bad, unsupported = b.DVP_ERR_INVALID_ARG, b.DVP_ERR_UNSUPPORTED
    fn = ctypes.CDLL(b.LIB_PATH).dvp_rms_norm
    good = dict(x_dtype=b.DVP_BF16, weight_dtype=b.DVP_BF16, out_dtype=b.DVP_E4M3, T=4, H=300, ld_x=300, ld_residual=300,
                ld_residual_out=300, ld_out=300, ld_scale=3, eps=1e-6, x=0x1000, residual=0x2000, weight=0x3000,
                residual_out=0x4000, out=0x5000, scale=0x6000, rstd=0x7000)
    assert fn(None) == bad
    _refused(fn, b.RmsNormArgs, good, [
        (bad, dict(struct_size=8)), (bad, dict(T=-1)), (bad, dict(H=0)), (bad, dict(eps=-1.0)), (bad, dict(eps=float("nan"))),
        (bad, dict(eps=float("inf"))), (bad, dict(x=None)), (bad, dict(weight=None)), (bad, dict(out=None)), (bad, dict(scale=None)),
        (bad, dict(out_dtype=b.DVP_BF16)), (bad, dict(ld_x=299)), (bad, dict(ld_residual=299)), (bad, dict(ld_residual_out=299)),
        (bad, dict(ld_out=299)), (bad, dict(ld_scale=2)), (unsupported, dict(x_dtype=b.DVP_E4M3)), (unsupported, dict(x_dtype=9)),
        (unsupported, dict(weight_dtype=b.DVP_F16)), (unsupported, dict(out_dtype=4)), (unsupported, dict(T=1 << 31)),
        (b.DVP_OK, dict(T=0))])


def test_norm_backward_refusals(lib):
    from paper_2512_23087_b200 import binding as b
    bad, unsupported = b.DVP_ERR_INVALID_ARG, b.DVP_ERR_UNSUPPORTED
    fn = ctypes.CDLL(b.LIB_PATH).dvp_rms_norm_backward
    good = dict(h_dtype=b.DVP_BF16, weight_dtype=b.DVP_F32, dy_dtype=b.DVP_F32, T=4, H=300, ld_dy=300, ld_h=300, ld_d_residual=300,
                ld_d_x=300, dy=0x1000, h=0x2000, weight=0x3000, rstd=0x4000, d_residual=0x5000, d_x=0x6000, d_weight=0x7000,
                workspace=0x8000, workspace_bytes=1 << 30)
    need = lib.dvp_workspace_bytes(b.DVP_ENTRY_RMS_NORM_BACKWARD, ctypes.byref(_filled(b.RmsNormBackwardArgs, **good)))
    assert 4 * 300 * 4 <= need < 1 << 20
    _refused(fn, b.RmsNormBackwardArgs, good, [
        (bad, dict(struct_size=8)), (bad, dict(T=-1)), (bad, dict(H=0)), (bad, dict(dy=None)), (bad, dict(h=None)),
        (bad, dict(weight=None)), (bad, dict(rstd=None)), (bad, dict(d_x=None, d_weight=None)), (bad, dict(ld_dy=299)),
        (bad, dict(ld_h=299)), (bad, dict(ld_d_residual=299)), (bad, dict(ld_d_x=299)), (unsupported, dict(h_dtype=b.DVP_E4M3)),
        (unsupported, dict(dy_dtype=5)), (unsupported, dict(weight_dtype=b.DVP_F16)), (unsupported, dict(H=1 << 31)),
        (b.DVP_ERR_WORKSPACE, dict(workspace=None)), (b.DVP_ERR_WORKSPACE, dict(workspace=0x8010)),
        (b.DVP_ERR_WORKSPACE, dict(workspace_bytes=need - 1)), (b.DVP_OK, dict(T=0, accumulate_dw=1))])


@pytest.mark.parametrize("T,H", [(1, 1), (7, 64), (591, 96), (592, 96), (593, 64), (100000, 4096), (3, 20011)])
def test_norm_backward_workspace_holds_every_partial_row(lib, T, H):
    """Blocks of up to eight rows side by side, 592 rows of partial sums at most."""
    from paper_2512_23087_b200 import binding as b
    a = _filled(b.RmsNormBackwardArgs, T=T, H=H, d_weight=0x1000)
    need = lib.dvp_workspace_bytes(b.DVP_ENTRY_RMS_NORM_BACKWARD, ctypes.byref(a))
    for rpb in (1, 2, 4, 8):
        blocks = min(-(-T // rpb), 592 // rpb)
        assert need >= blocks * rpb * H * 4
    a.d_weight = None
    assert lib.dvp_workspace_bytes(b.DVP_ENTRY_RMS_NORM_BACKWARD, ctypes.byref(a)) == 0


def test_quantiser_refusals(lib):
    from paper_2512_23087_b200 import binding as b
    bad, unsupported = b.DVP_ERR_INVALID_ARG, b.DVP_ERR_UNSUPPORTED
    fn = ctypes.CDLL(b.LIB_PATH).dvp_quantize_fp8
    good = dict(x_dtype=b.DVP_F16, rows=5, cols=200, ld_x=200, ld_out=208, ld_scale=2, x=0x1000, out=0x2000, scale=0x3000,
                block_rows=128)
    _refused(fn, b.QuantizeFp8Args, good, [
        (bad, dict(struct_size=0)), (bad, dict(rows=-1)), (bad, dict(cols=0)), (bad, dict(block_rows=64)), (bad, dict(x=None)),
        (bad, dict(out=None)), (bad, dict(scale=None)), (bad, dict(ld_x=199)), (bad, dict(ld_out=199)), (bad, dict(ld_scale=1)),
        (unsupported, dict(x_dtype=b.DVP_E4M3)), (unsupported, dict(rows=1 << 31)),
        (unsupported, dict(rows=1 << 30, cols=1 << 30, ld_x=1 << 30, ld_out=1 << 30, ld_scale=1 << 23)), (b.DVP_OK, dict(rows=0))])


def test_product_refusals(lib):
    from paper_2512_23087_b200 import binding as b
    bad, unsupported = b.DVP_ERR_INVALID_ARG, b.DVP_ERR_UNSUPPORTED
    fn = ctypes.CDLL(b.LIB_PATH).dvp_gemm_fp8
    good = dict(c_dtype=b.DVP_BF16, M=5, N=300, K=200, lda=208, ldb=208, ldc=300, ld_a_scale=2, ld_b_scale=2, a=0x1000, b=0x2000,
                a_scale=0x3000, b_scale=0x4000, c=0x5000, status=0x6000)
    _refused(fn, b.GemmFp8Args, good, [
        (bad, dict(struct_size=0)), (bad, dict(M=-1)), (bad, dict(N=-1)), (bad, dict(K=0)), (bad, dict(launch_hint=3)),
        (bad, dict(launch_hint=2, M=65)), (bad, dict(a=None)), (bad, dict(b=None)), (bad, dict(a_scale=None)),
        (bad, dict(b_scale=None)), (bad, dict(c=None)), (bad, dict(status=None)), (bad, dict(lda=192)), (bad, dict(ldb=192)),
        (bad, dict(ldc=299)), (bad, dict(ld_a_scale=1)), (bad, dict(ld_b_scale=1)), (unsupported, dict(c_dtype=b.DVP_E4M3)),
        (unsupported, dict(lda=200)), (unsupported, dict(ldb=200)), (unsupported, dict(a=0x1008)), (unsupported, dict(b=0x2004)),
        (unsupported, dict(N=1 << 31)), (unsupported, dict(M=0x7fffff00, N=0x7fffff00)), (b.DVP_OK, dict(M=0)),
        (b.DVP_OK, dict(N=0))])


def test_sample_refusals(lib):
    from paper_2512_23087_b200 import binding as b
    bad, unsupported, nan = b.DVP_ERR_INVALID_ARG, b.DVP_ERR_UNSUPPORTED, float("nan")
    fn = ctypes.CDLL(b.LIB_PATH).dvp_sample
    good = dict(logits_dtype=b.DVP_BF16, id_dtype=b.DVP_ID_I64, T=3, V=100, ld=100, logits=0x1000, uniform=0x2000, temperature=1.0,
                top_p=0.9, rho=0.1, top_k=5, ids=0x3000, logp=0x4000, logp_mp=0x5000, count=0x6000)
    _refused(fn, b.SampleArgs, good, [
        (bad, dict(struct_size=0)), (bad, dict(T=-1)), (bad, dict(V=0)), (bad, dict(ld=99)), (bad, dict(logits=None)),
        (bad, dict(uniform=None)), (bad, dict(ids=None)), (bad, dict(temperature=-0.5)), (bad, dict(temperature=nan)),
        (bad, dict(temperature=float("inf"))), (bad, dict(temperature=1e-31)), (bad, dict(temperature=1e31)), (bad, dict(rho=-0.1)),
        (bad, dict(rho=1.5)), (bad, dict(rho=nan)), (bad, dict(top_p=-0.1)), (bad, dict(top_p=nan)), (bad, dict(launch_hint=3)),
        (bad, dict(launch_hint=16)), (unsupported, dict(logits_dtype=b.DVP_E4M3)), (unsupported, dict(id_dtype=2)),
        (unsupported, dict(T=1 << 28)), (unsupported, dict(V=0x7fff0001, ld=0x7fff0001)), (b.DVP_OK, dict(T=0)),
        (b.DVP_OK, dict(T=0, temperature=nan, temperature_rows=0x7000))])
