"""What the entry points of RMS norm with its 8-bit result refuse, on the host, before any device call; and their structs as the C compiler lays them out."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2312_00752_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000001000   # non-null, 4096-byte aligned, never dereferenced
MANY = 2 ** 32 + 5

STRUCTS = {"ss_norm_quant_params": B.NormQuantParams}
HEADERS = ["ss_norm.h"]


def t(*shape, dtype=torch.bfloat16):
    """A tensor without memory."""
    return torch.empty(shape, dtype=dtype, device="meta")


def test_structs_match_the_headers(tmp_path):
    """Size and last field of every struct, as the C compiler lays it out."""
    src = tmp_path / "s.c"
    lines = ["printf(\"%s %%zu %%zu\\n\", sizeof(%s), offsetof(%s, %s));" % (n, n, n, c._fields_[-1][0]) for n, c in STRUCTS.items()]
    src.write_text("#include <stdio.h>\n%sint main(void) { %s return 0; }" % ("".join("#include \"%s\"\n" % h for h in HEADERS), " ".join(lines)))
    exe = str(tmp_path / "s")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", exe, str(src)], check=True)
    seen = 0
    for line in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines():
        name, size, off = line.split()
        c = STRUCTS[name]
        assert (ctypes.sizeof(c), getattr(c, c._fields_[-1][0]).offset) == (int(size), int(off)), name
        seen += 1
    assert seen == len(STRUCTS)


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


# ---- norm in 8 bits -----------------------------------------------------------------------------------
def norm_quant():
    p = B.NormQuantParams()
    p.fwd.rows, p.fwd.width, p.fwd.io_dtype, p.fwd.eps = 4, 32, B.SS_BF16, 1e-5
    p.fwd.flags = B.SS_NORM_HAS_WEIGHT | B.SS_NORM_HAS_BIAS | B.SS_NORM_HAS_RESIDUAL | B.SS_NORM_RMS
    for f in ("x", "residual", "weight", "bias", "summed"):
        setattr(p.fwd, f, FAKE)
    p.q = p.scale = FAKE
    return p


def test_norm_quant():
    call = B.lib().ss_norm_quant
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, norm_quant, [{f: None} for f in ("fwd.x", "fwd.residual", "fwd.weight", "fwd.bias", "fwd.summed", "q", "scale")], B.SS_ERR_NULL)
    expect(call, norm_quant, [{"fwd.rows": -1}, {"fwd.width": 0}], B.SS_ERR_SHAPE)
    flags = norm_quant().fwd.flags
    expect(call, norm_quant, [{"fwd.io_dtype": 2}, {"fwd.flags": flags | 32}, {"fwd.flags": flags | 128}, {"fwd.flags": flags | B.SS_NORM_SAVE_STATS}, {"fwd.eps": -1.0},
                              {"fwd.eps": float("nan")}, {"fwd.width": B.SS_QUANT_MAX_DIM + 1}, {"fwd.rows": 2 ** 31 - 1}], B.SS_ERR_UNSUPPORTED)
    expect(call, norm_quant, [{"fwd.x": FAKE + 1}, {"fwd.residual": FAKE + 1}, {"fwd.weight": FAKE + 2}, {"fwd.bias": FAKE + 1}, {"fwd.summed": FAKE + 1},
                              {"q": FAKE + 8}, {"scale": FAKE + 2}], B.SS_ERR_ALIGN)
    expect(call, norm_quant, [{"fwd.rows": 0, "fwd.x": None, "q": None}], B.SS_OK)


def test_rms_backward_has_the_same_refusals():
    p = B.NormBwdParams()
    p.fwd.rows, p.fwd.width, p.fwd.io_dtype, p.fwd.eps, p.fwd.flags = 4, 32, B.SS_BF16, 1e-5, B.SS_NORM_RMS
    p.fwd.x = p.dout = p.dx = FAKE
    assert B.lib().ss_norm_bwd(ctypes.byref(p), None) == B.SS_ERR_NULL   # no statistics
    p.fwd.stats = FAKE
    assert B.lib().ss_norm_bwd(ctypes.byref(p), None) == B.SS_ERR_WORKSPACE


@pytest.mark.parametrize("call", [lambda: B.ss_norm_quant(t(MANY, 1)), lambda: B.ss_norm_quant(t(1, MANY), rms=True), lambda: B.ss_norm_fwd(t(MANY, 1), rms=True)])
def test_norm_sizes_beyond_32_bits(call):
    with pytest.raises(B.SsError) as e:
        call()
    assert e.value.code == B.SS_ERR_UNSUPPORTED


def test_norm_tensors_on_the_host_are_refused():
    with pytest.raises(ValueError, match="GPU"):
        B.ss_norm_quant(torch.zeros(3, 4), rms=True)
