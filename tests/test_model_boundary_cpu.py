"""What the entry points of the norms' 8-bit results, the embedding, the log probabilities and AdamW refuse, on the host, before any device call; and their structs as the C compiler lays them out."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2312_00752_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000001000   # non-null, 4096-byte aligned, never dereferenced
MANY = 2 ** 32 + 5

STRUCTS = {"ss_norm_quant_params": B.NormQuantParams, "ss_embed_params": B.EmbedParams, "ss_embed_bwd_params": B.EmbedBwdParams,
           "ss_logprob_params": B.LogprobParams, "ss_logprob_bwd_params": B.LogprobBwdParams,
           "ss_adamw_tensor": B.AdamwTensor, "ss_adamw_params": B.AdamwParams, "ss_adamw_values_params": B.AdamwValuesParams}
HEADERS = ["ss_norm.h", "ss_embed.h", "ss_logprob.h", "ss_adamw.h"]


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


# ---- embedding ----------------------------------------------------------------------------------------
def embed():
    p = B.EmbedParams()
    p.tokens, p.vocab, p.dim, p.table_dtype, p.io_dtype, p.scale = 4, 10, 32, B.SS_F32, B.SS_BF16, 1.0
    p.ids = p.table = p.out = FAKE
    return p


def embed_bwd():
    p = B.EmbedBwdParams()
    p.fwd = embed()
    p.dout = p.dtable = p.workspace = FAKE
    p.workspace_bytes = B.ss_embed_workspace_bytes(4, 10, 32)
    return p


def test_embed():
    call = B.lib().ss_embed_fwd
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, embed, [dict(ids=None), dict(table=None), dict(out=None)], B.SS_ERR_NULL)
    expect(call, embed, [dict(tokens=-1), dict(vocab=0), dict(dim=0)], B.SS_ERR_SHAPE)
    inf = float("inf")
    expect(call, embed, [dict(table_dtype=2), dict(io_dtype=-1), dict(flags=2), dict(scale=inf), dict(scale=float("nan")), dict(tokens=2 ** 31 - 1),
                         dict(vocab=2 ** 31 - 1), dict(dim=2 ** 31 - 1)], B.SS_ERR_UNSUPPORTED)
    expect(call, embed, [dict(ids=FAKE + 4), dict(ids=FAKE + 2, flags=1), dict(table=FAKE + 2), dict(out=FAKE + 1)], B.SS_ERR_ALIGN)
    expect(call, embed, [dict(tokens=0, ids=None, table=None, out=None)], B.SS_OK)
    call = B.lib().ss_embed_bwd
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, embed_bwd, [{"fwd.ids": None}, dict(dout=None), dict(dtable=None), {"fwd.tokens": 0, "dtable": None}], B.SS_ERR_NULL)
    expect(call, embed_bwd, [dict(dout=FAKE + 1), dict(dtable=FAKE + 2), dict(workspace=FAKE + 128)], B.SS_ERR_ALIGN)
    expect(call, embed_bwd, [dict(workspace=None), dict(workspace_bytes=embed_bwd().workspace_bytes - 1)], B.SS_ERR_WORKSPACE)
    assert B.ss_embed_workspace_bytes(0, 10, 32) == 0


@pytest.mark.parametrize("call", [lambda: B.ss_embed_fwd(t(MANY, dtype=torch.int64), t(3, 4)), lambda: B.ss_embed_fwd(t(3, dtype=torch.int64), t(MANY, 1)),
                                  lambda: B.ss_embed_fwd(t(3, dtype=torch.int64), t(1, MANY)), lambda: B.ss_embed_bwd(t(MANY, 1), t(MANY, dtype=torch.int32), 5),
                                  lambda: B.ss_embed_bwd(t(3, 4), t(3, dtype=torch.int32), MANY), lambda: B.ss_embed_workspace_bytes(4, 4, MANY)])
def test_embed_sizes_beyond_32_bits(call):
    with pytest.raises(B.SsError) as e:
        call()
    assert e.value.code == B.SS_ERR_UNSUPPORTED


# ---- log probabilities --------------------------------------------------------------------------------
def logprob():
    p = B.LogprobParams()
    p.rows, p.vocab, p.top, p.io_dtype, p.row_stride = 4, 20000, 5, B.SS_BF16, 20000
    for f in ("logits", "targets", "logp", "entropy", "stats", "top_logp", "top_ids", "workspace"):
        setattr(p, f, FAKE)
    p.workspace_bytes = B.ss_logprob_workspace_bytes(4, 20000, 5)
    return p


def logprob_bwd():
    p = B.LogprobBwdParams()
    p.fwd = logprob()
    p.dlogp = p.dentropy = p.dlogits = FAKE
    return p


def test_logprob():
    call = B.lib().ss_logprob_fwd
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, logprob, [{f: None} for f in ("logits", "logp", "entropy", "stats", "top_logp", "top_ids")], B.SS_ERR_NULL)
    expect(call, logprob, [dict(rows=-1), dict(vocab=0), dict(top=-1), dict(row_stride=19999)], B.SS_ERR_SHAPE)
    big = 2 ** 31 - 1
    expect(call, logprob, [dict(io_dtype=2), dict(flags=2), dict(top=65), dict(vocab=4, top=5), dict(vocab=big, row_stride=big), dict(rows=big),
                           dict(rows=2 ** 24 // 3 + 1), dict(rows=2 ** 26, vocab=2048)], B.SS_ERR_UNSUPPORTED)
    expect(call, logprob, [dict(logits=FAKE + 1), dict(targets=FAKE + 4), dict(logp=FAKE + 2), dict(entropy=FAKE + 2), dict(stats=FAKE + 1),
                           dict(top_logp=FAKE + 2), dict(top_ids=FAKE + 4), dict(workspace=FAKE + 128), dict(flags=1, targets=FAKE + 2)], B.SS_ERR_ALIGN)
    expect(call, logprob, [dict(workspace=None), dict(workspace_bytes=logprob().workspace_bytes - 1)], B.SS_ERR_WORKSPACE)
    expect(call, logprob, [dict(rows=0, logits=None, stats=None)], B.SS_OK)
    call = B.lib().ss_logprob_bwd
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, logprob_bwd, [{"fwd.logits": None}, {"fwd.stats": None}, {"fwd.entropy": None}, dict(dlogits=None)], B.SS_ERR_NULL)
    expect(call, logprob_bwd, [dict(dlogp=FAKE + 2), dict(dentropy=FAKE + 1), dict(dlogits=FAKE + 1), {"fwd.entropy": FAKE + 2}], B.SS_ERR_ALIGN)
    assert B.ss_logprob_workspace_bytes(4, 2048, 5) == 0 and B.ss_logprob_workspace_bytes(0, 20000) == 0 and B.ss_logprob_workspace_bytes(5000, 20000) == 0


@pytest.mark.parametrize("call", [lambda: B.ss_logprob_fwd(t(MANY, 4)), lambda: B.ss_logprob_fwd(t(1, MANY)), lambda: B.ss_logprob_workspace_bytes(1, MANY),
                                  lambda: B.ss_logprob_bwd(t(MANY, 4), t(2, MANY, dtype=torch.float32))])
def test_logprob_sizes_beyond_32_bits(call):
    with pytest.raises(B.SsError) as e:
        call()
    assert e.value.code == B.SS_ERR_UNSUPPORTED


# ---- AdamW --------------------------------------------------------------------------------------------
LISTS = []   # what the structs point to


def adamw(bits=32, **tensor):
    p = B.AdamwParams()
    p.tensors, p.state_bits, p.lr, p.beta1, p.beta2, p.eps, p.weight_decay = 2, bits, 1e-3, 0.9, 0.95, 1e-8, 0.1
    list_ = (B.AdamwTensor * 2)()
    for e in list_:
        e.n, e.param_dtype, e.grad_dtype = 1000, B.SS_BF16, B.SS_F32
        for f in ("param", "grad", "master", "m", "v") + (("m_scale", "v_scale") if bits == 8 else ()):
            setattr(e, f, FAKE)
    for k, v in tensor.items():
        setattr(list_[1], k, v)
    LISTS.append(list_)
    p.list = list_
    p.count = FAKE
    return p


def test_adamw():
    call = B.lib().ss_adamw_step
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, adamw, [dict(count=None), dict(list=None)], B.SS_ERR_NULL)
    expect(call, adamw, [dict(tensors=-1)], B.SS_ERR_SHAPE)
    inf, nan = float("inf"), float("nan")
    expect(call, adamw, [dict(state_bits=16), dict(lr=-1.0), dict(lr=inf), dict(lr=1e39), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=nan), dict(eps=-1.0), dict(eps=inf),
                         dict(weight_decay=-1.0), dict(weight_decay=nan)], B.SS_ERR_UNSUPPORTED)
    expect(call, adamw, [dict(count=FAKE + 2), dict(lr_device=FAKE + 1), dict(grad_scale=FAKE + 2)], B.SS_ERR_ALIGN)
    for bits in (8, 32):   # of the second tensor: nothing is launched for the first
        one = lambda code, **t: expect(call, lambda: adamw(bits, **t), [{}], code)
        for f in ("param", "grad", "m", "v") + (("m_scale", "v_scale") if bits == 8 else ()):
            one(B.SS_ERR_NULL, **{f: None})
        one(B.SS_ERR_SHAPE, n=-1)
        one(B.SS_ERR_UNSUPPORTED, n=2 ** 40 + 1)
        one(B.SS_ERR_UNSUPPORTED, param_dtype=2)
        one(B.SS_ERR_UNSUPPORTED, grad_dtype=-1)
        one(B.SS_ERR_UNSUPPORTED, param_dtype=B.SS_F32)   # with a master
        for f in ("param", "grad", "master") + (("m_scale", "v_scale") if bits == 8 else ("m", "v")):
            one(B.SS_ERR_ALIGN, **{f: FAKE + 1})


def adamw_values():
    p = B.AdamwValuesParams()
    p.n, p.with_sign, p.codes, p.scale, p.out = 1000, 1, FAKE, FAKE, FAKE
    return p


def test_adamw_values():
    call = B.lib().ss_adamw_values
    assert call(None, None) == B.SS_ERR_NULL
    expect(call, adamw_values, [dict(codes=None), dict(scale=None), dict(out=None)], B.SS_ERR_NULL)
    expect(call, adamw_values, [dict(n=-1)], B.SS_ERR_SHAPE)
    expect(call, adamw_values, [dict(n=2 ** 40 + 1), dict(with_sign=2), dict(with_sign=-1), dict(out_dtype=2)], B.SS_ERR_UNSUPPORTED)
    expect(call, adamw_values, [dict(scale=FAKE + 2), dict(out=FAKE + 2)], B.SS_ERR_ALIGN)
    expect(call, adamw_values, [dict(n=0, codes=None)], B.SS_OK)
