"""What the entry points of layer norm, the gated recurrence and the 8-bit products refuse, on the host, before any device call."""
import ctypes
import os
import subprocess

import pytest

from paper_2312_00752_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000001000   # non-null, 4096-byte aligned, never dereferenced

STRUCTS = {"ss_norm_params": B.NormParams, "ss_norm_bwd_params": B.NormBwdParams, "ss_gate_params": B.GateParams,
           "ss_gate_bwd_params": B.GateBwdParams, "ss_gate_step_params": B.GateStepParams, "ss_quant_params": B.QuantParams,
           "ss_qlinear_params": B.QLinearParams}


def test_structs_match_the_headers(tmp_path):
    """Size and last field of every struct, as the C compiler lays it out."""
    src = tmp_path / "s.c"
    lines = ["printf(\"%s %%zu %%zu\\n\", sizeof(%s), offsetof(%s, %s));" % (n, n, n, c._fields_[-1][0]) for n, c in STRUCTS.items()]
    src.write_text("#include <stdio.h>\n#include \"ss_norm.h\"\n#include \"ss_gate.h\"\n#include \"ss_quant.h\"\nint main(void) { %s return 0; }" % " ".join(lines))
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", exe, str(src)], check=True)
    for line in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines():
        name, size, off = line.split()
        c = STRUCTS[name]
        assert (ctypes.sizeof(c), getattr(c, c._fields_[-1][0]).offset) == (int(size), int(off)), name


def expect(call, make, changes, code):
    for change in changes:
        p = make()
        for k, v in change.items():
            o = p
            while "." in k:
                head, k = k.split(".", 1)
                o = getattr(o, head)
            setattr(o, k, v)
        assert call(ctypes.byref(p), None) == code, (change, code)


def norm():
    p = B.NormParams()
    p.rows, p.width, p.io_dtype, p.eps = 4, 32, B.SS_BF16, 1e-5
    p.flags = B.SS_NORM_HAS_WEIGHT | B.SS_NORM_HAS_BIAS | B.SS_NORM_HAS_RESIDUAL | B.SS_NORM_SAVE_STATS
    for f in ("x", "residual", "weight", "bias", "out", "summed", "stats"):
        setattr(p, f, FAKE)
    return p


def norm_bwd():
    p = B.NormBwdParams()
    p.fwd = norm()
    for f in ("dout", "dsummed", "dx", "dweight", "dbias", "workspace"):
        setattr(p, f, FAKE)
    p.workspace_bytes = B.ss_norm_workspace_bytes(4, 32)
    return p


def test_norm():
    call = B.lib().ss_norm_fwd
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, norm, [{f: None} for f in ("x", "residual", "weight", "bias", "out", "summed", "stats")], B.SS_ERR_NULL)
    expect(call, norm, [dict(rows=-1), dict(width=0)], B.SS_ERR_SHAPE)
    expect(call, norm, [dict(io_dtype=2), dict(flags=32), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(width=2 ** 31 - 1),
                        dict(rows=2 ** 31 - 1)], B.SS_ERR_UNSUPPORTED)
    expect(call, norm, [dict(x=FAKE + 1), dict(residual=FAKE + 1), dict(weight=FAKE + 2), dict(bias=FAKE + 1), dict(out=FAKE + 1), dict(stats=FAKE + 2),
                        dict(summed=FAKE + 1), dict(flags=norm().flags | B.SS_NORM_RESIDUAL_F32, residual=FAKE + 2)], B.SS_ERR_ALIGN)
    expect(call, norm, [dict(rows=0, x=None, out=None)], B.SS_OK)
    call = B.lib().ss_norm_bwd
    assert call(None, None) == B.SS_ERR_NULL
    two = norm().flags | B.SS_NORM_RESIDUAL_F32
    expect(call, norm_bwd, [{"fwd.summed": None}, {"fwd.stats": None}, {"dout": None}, {"dx": None}, {"dweight": None}, {"dbias": None},
                            {"fwd.flags": two}], B.SS_ERR_NULL)
    expect(call, norm_bwd, [dict(dout=FAKE + 1), dict(dx=FAKE + 1), dict(dsummed=FAKE + 1), dict(dweight=FAKE + 2), dict(workspace=FAKE + 64),
                            {"fwd.flags": two, "dresidual": FAKE + 2}], B.SS_ERR_ALIGN)
    expect(call, norm_bwd, [dict(workspace=None), dict(workspace_bytes=norm_bwd().workspace_bytes - 1)], B.SS_ERR_WORKSPACE)
    assert B.ss_norm_workspace_bytes(0, 32) == 0 and B.ss_norm_workspace_bytes(4, 32) > 0


def gate():
    p = B.GateParams()
    p.batch, p.dim, p.seqlen, p.io_dtype = 2, 4, 96, B.SS_BF16
    p.flags = (B.SS_GATE_HAS_I | B.SS_GATE_HAS_Z | B.SS_GATE_HAS_F_BIAS | B.SS_GATE_HAS_I_BIAS | B.SS_GATE_HAS_RESET
               | B.SS_GATE_HAS_H0 | B.SS_GATE_WRITE_H_LAST | B.SS_GATE_SAVE_FOR_BWD)
    for f in ("x", "f", "i", "z", "rate", "f_bias", "i_bias", "reset", "h0", "out", "h_last", "workspace"):
        setattr(p, f, FAKE)
    p.x_batch = p.f_batch = p.i_batch = p.z_batch = 4 * 96
    p.workspace_bytes = B.ss_gate_workspace_bytes(2, 4, 96)
    return p


def gate_bwd():
    p = B.GateBwdParams()
    p.fwd = gate()
    for f in ("dout", "dh_last", "dx", "df", "di", "dz", "drate", "df_bias", "di_bias", "dh0"):
        setattr(p, f, FAKE)
    p.dx_batch = p.df_batch = p.di_batch = p.dz_batch = 4 * 96
    return p


def gate_step():
    p = B.GateStepParams()
    p.batch, p.dim, p.io_dtype = 2, 4, B.SS_BF16
    p.flags = B.SS_GATE_HAS_I | B.SS_GATE_HAS_Z | B.SS_GATE_HAS_F_BIAS | B.SS_GATE_HAS_I_BIAS | B.SS_GATE_HAS_RESET
    for f in ("h", "x_t", "f_t", "i_t", "z_t", "rate", "f_bias", "i_bias", "reset_t", "out_t"):
        setattr(p, f, FAKE)
    p.x_batch = p.f_batch = p.i_batch = p.z_batch = 4
    return p


def test_gate():
    call = B.lib().ss_gate_fwd
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, gate, [{f: None} for f in ("x", "f", "i", "z", "rate", "f_bias", "i_bias", "reset", "h0", "out", "h_last")], B.SS_ERR_NULL)
    expect(call, gate, [dict(batch=0), dict(dim=0), dict(seqlen=-1), dict(x_batch=383), dict(z_batch=0)], B.SS_ERR_SHAPE)
    expect(call, gate, [dict(io_dtype=2), dict(flags=256), dict(flags=B.SS_GATE_HAS_I_BIAS), dict(batch=1 << 16, dim=1 << 16), dict(seqlen=2 ** 31 - 1)],
           B.SS_ERR_UNSUPPORTED)
    expect(call, gate, [dict(x=FAKE + 1), dict(i=FAKE + 1), dict(out=FAKE + 1), dict(rate=FAKE + 2), dict(h0=FAKE + 2), dict(h_last=FAKE + 1),
                        dict(workspace=FAKE + 16), dict(io_dtype=B.SS_F32, f=FAKE + 2)], B.SS_ERR_ALIGN)
    expect(call, gate, [dict(workspace=None), dict(workspace_bytes=gate().workspace_bytes - 1)], B.SS_ERR_WORKSPACE)
    call = B.lib().ss_gate_bwd
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, gate_bwd, [{f: None} for f in ("dout", "dx", "df", "di", "dz", "drate", "df_bias", "di_bias")], B.SS_ERR_NULL)
    expect(call, gate_bwd, [dict(dx_batch=1), dict(dz_batch=383), {"fwd.f_batch": 5}], B.SS_ERR_SHAPE)
    expect(call, gate_bwd, [dict(dout=FAKE + 1), dict(df=FAKE + 1), dict(drate=FAKE + 1), dict(dh0=FAKE + 2), dict(dh_last=FAKE + 2),
                            {"fwd.workspace": FAKE + 16}], B.SS_ERR_ALIGN)
    expect(call, gate_bwd, [{"fwd.workspace": None}, {"fwd.workspace_bytes": gate().workspace_bytes - 1}], B.SS_ERR_WORKSPACE)
    call = B.lib().ss_gate_step
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, gate_step, [{f: None} for f in ("h", "x_t", "f_t", "i_t", "z_t", "rate", "f_bias", "i_bias", "reset_t", "out_t")], B.SS_ERR_NULL)
    expect(call, gate_step, [dict(batch=0), dict(dim=-1), dict(f_batch=3)], B.SS_ERR_SHAPE)
    expect(call, gate_step, [dict(io_dtype=7), dict(flags=B.SS_GATE_HAS_H0), dict(flags=B.SS_GATE_HAS_I_BIAS), dict(batch=1 << 15, dim=1 << 16)],
           B.SS_ERR_UNSUPPORTED)
    expect(call, gate_step, [dict(h=FAKE + 2), dict(x_t=FAKE + 1), dict(out_t=FAKE + 1), dict(f_bias=FAKE + 2)], B.SS_ERR_ALIGN)


def test_gate_workspace():
    assert B.ss_gate_workspace_bytes(0, 4, 96) == 0
    assert B.ss_gate_workspace_bytes(8, 4096, 2048, for_backward=False) == 0      # rows enough: nothing to split
    assert B.ss_gate_workspace_bytes(1, 16, 1 << 20, for_backward=False) > 0
    # a state for every 512 steps of a row, and three sums
    assert B.ss_gate_workspace_bytes(8, 4096, 2048) >= 8 * 4096 * (4 + 3) * 4


def quant():
    p = B.QuantParams()
    p.batch, p.seqlen, p.dim, p.io_dtype, p.flags = 2, 5, 40, B.SS_BF16, B.SS_Q_X_SEQ_LAST
    for f in ("x", "q", "scale", "scratch"):
        setattr(p, f, FAKE)
    p.scratch_bytes = B.lib().ss_quant_rows_scratch_bytes(ctypes.byref(p))
    return p


def linear():
    p = B.QLinearParams()
    p.batch, p.seqlen, p.dim, p.features, p.io_dtype = 2, 5, 40, 24, B.SS_BF16
    p.flags = B.SS_Q_HAS_BIAS | B.SS_Q_OUT_SEQ_LAST
    for f in ("x", "x_scale", "weight", "scale", "bias", "out", "scratch"):
        setattr(p, f, FAKE)
    p.scratch_bytes = B.ss_qlinear_scratch_bytes(2, 5, 40, 24)
    return p


def test_quant():
    assert [B.ss_quant_pitch(n) for n in (-1, 0, 1, 128, 129)] == [0, 0, 128, 128, 256]
    call = B.lib().ss_quant_rows
    assert call(None, None) == B.SS_ERR_NULL and quant().scratch_bytes > 0
    expect(call, quant, [{f: None} for f in ("x", "q", "scale")], B.SS_ERR_NULL)
    expect(call, quant, [dict(batch=-1), dict(seqlen=-1), dict(dim=0)], B.SS_ERR_SHAPE)
    expect(call, quant, [dict(dim=B.SS_QUANT_MAX_DIM + 1), dict(io_dtype=3), dict(flags=2), dict(batch=1 << 16, seqlen=1 << 15)], B.SS_ERR_UNSUPPORTED)
    expect(call, quant, [dict(x=FAKE + 1), dict(q=FAKE + 8), dict(scale=FAKE + 2), dict(scratch=FAKE + 128)], B.SS_ERR_ALIGN)
    expect(call, quant, [dict(scratch=None), dict(scratch_bytes=quant().scratch_bytes - 1)], B.SS_ERR_WORKSPACE)
    expect(call, quant, [dict(batch=0, x=None), dict(seqlen=0, q=None)], B.SS_OK)
    call = B.lib().ss_qlinear
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, linear, [{f: None} for f in ("x", "weight", "scale", "bias", "out")] + [dict(flags=B.SS_Q_X_QUANTISED, x_scale=None)], B.SS_ERR_NULL)
    expect(call, linear, [dict(batch=-1), dict(seqlen=-1), dict(dim=0), dict(features=0)], B.SS_ERR_SHAPE)
    expect(call, linear, [dict(dim=B.SS_QUANT_MAX_DIM + 1), dict(io_dtype=3), dict(flags=16), dict(flags=B.SS_Q_X_QUANTISED | B.SS_Q_X_SEQ_LAST),
                          dict(features=2 ** 31 - 1), dict(batch=1 << 16, seqlen=1)], B.SS_ERR_UNSUPPORTED)
    expect(call, linear, [dict(x=FAKE + 1), dict(weight=FAKE + 8), dict(scale=FAKE + 2), dict(bias=FAKE + 2), dict(out=FAKE + 1), dict(scratch=FAKE + 128),
                          dict(flags=B.SS_Q_X_QUANTISED, x=FAKE + 8), dict(flags=B.SS_Q_X_QUANTISED, x_scale=FAKE + 2)], B.SS_ERR_ALIGN)
    expect(call, linear, [dict(scratch=None), dict(scratch_bytes=linear().scratch_bytes - 1)], B.SS_ERR_WORKSPACE)
    expect(call, linear, [dict(batch=0, x=None), dict(seqlen=0, out=None)], B.SS_OK)


@pytest.mark.parametrize("name", sorted(STRUCTS))
def test_headers_stand_alone(name, tmp_path):
    """Each header compiles by itself as C."""
    header = {"ss_norm": "ss_norm.h", "ss_gate": "ss_gate.h", "ss_quan": "ss_quant.h", "ss_qlin": "ss_quant.h"}[name[:7]]
    src = tmp_path / "h.c"
    src.write_text("#include \"%s\"\n%s p;\n" % (header, name))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)], check=True)


def test_gate_rows_of_one_launch():
    big = lambda dim, seqlen: dict(batch=1 << 13, dim=dim, seqlen=seqlen, x_batch=dim * seqlen, f_batch=dim * seqlen, i_batch=dim * seqlen, z_batch=dim * seqlen)
    expect(B.lib().ss_gate_fwd, gate, [big(1 << 13, 200), big(1 << 15, 128), big(1 << 17, 9)], B.SS_ERR_UNSUPPORTED)
    expect(B.lib().ss_gate_fwd, gate, [dict(workspace=None, **big((1 << 13) - 64, 200))], B.SS_ERR_WORKSPACE)
