"""Refusals of the operators on token ids, on the host: no call here gets as far as a launch."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2605_05802_b200 as sr
from paper_2605_05802_b200 import binding, build

FAKE = 1 << 20           # never dereferenced


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def adjust(lib, x=FAKE, dtype=0, T=4, V=100, pitch=100, hist=FAKE, n_hist=10, start=FAKE, length=FAKE, prompt=None, rep=FAKE, pres=None, freq=None, bt=None, bv=None, n_bias=0, bs=None, bl=None,
           allowed=None, masks=0, mask_pitch=4, mask_row=None, out=2 * FAKE, out_pitch=100, status=None):
    return lib.sr_adjust_logits(x, dtype, T, V, pitch, hist, n_hist, start, length, prompt, rep, pres, freq, bt, bv, n_bias, bs, bl, allowed, masks, mask_pitch, mask_row, out, out_pitch, status, None)


def test_adjust_refusals(lib):
    call = lambda **k: adjust(lib, **k)
    for bad in (dict(T=-1), dict(V=0), dict(pitch=99), dict(pitch=1 << 40), dict(out_pitch=99), dict(out_pitch=1 << 40), dict(n_hist=-1), dict(n_bias=-1)):
        assert call(**bad) == sr.SR_ERR_BAD_SIZE, bad
    assert call(dtype=3) == sr.SR_ERR_BAD_DTYPE and call(dtype=-1) == sr.SR_ERR_BAD_DTYPE
    for name in ("x", "hist", "start", "length", "out"):
        assert call(**{name: None}) == sr.SR_ERR_NULL, name
    for name in ("rep", "pres", "freq"):                                  # one penalty is enough to need histories
        assert call(**{"rep": None, name: FAKE, "start": None}) == sr.SR_ERR_NULL, name
    bias = dict(bt=FAKE, bv=FAKE, bs=FAKE, bl=FAKE, n_bias=5)
    for name in ("bt", "bs", "bl"):
        assert call(**{**bias, name: None}) == sr.SR_ERR_NULL, name
    for name in ("x", "hist", "length", "prompt", "rep", "pres", "freq", "mask_row", "out", "status"):
        assert call(**{name: FAKE + 2}) == sr.SR_ERR_ALIGN, name
    for name in ("bt", "bv", "bl"):
        assert call(**{**bias, name: FAKE + 2}) == sr.SR_ERR_ALIGN, name
    assert call(start=FAKE + 4) == sr.SR_ERR_ALIGN and call(**{**bias, "bs": FAKE + 4}) == sr.SR_ERR_ALIGN
    assert call(allowed=FAKE + 1, masks=4) == sr.SR_ERR_ALIGN and call(x=FAKE + 1, dtype=1) == sr.SR_ERR_ALIGN
    mask = dict(allowed=FAKE, masks=4)
    assert call(**mask, mask_pitch=3) == sr.SR_ERR_BAD_SIZE and call(allowed=FAKE, masks=3) == sr.SR_ERR_BAD_SIZE and call(allowed=FAKE, masks=-1, mask_row=FAKE) == sr.SR_ERR_BAD_SIZE
    # neither the logits themselves nor apart from them
    assert call(out=FAKE + 4) == sr.SR_ERR_OVERLAP and call(out=FAKE + 1596) == sr.SR_ERR_OVERLAP and call(out=FAKE - 4) == sr.SR_ERR_OVERLAP
    assert call(out=FAKE, out_pitch=101) == sr.SR_ERR_OVERLAP
    assert call(T=0, x=None, hist=None, n_hist=0, start=None, length=None, rep=None, out=None) == sr.SR_OK


def test_adjust_backward_refusals(lib):
    def call(d=FAKE, dtype=0, T=4, V=100, d_pitch=100, x=3 * FAKE, pitch=100, hist=FAKE, n_hist=10, start=FAKE, length=FAKE, rep=FAKE, allowed=None, masks=0, mask_pitch=4, mask_row=None, dx=2 * FAKE,
             dx_pitch=100, status=None):
        return lib.sr_adjust_logits_backward(d, dtype, T, V, d_pitch, x, pitch, hist, n_hist, start, length, rep, allowed, masks, mask_pitch, mask_row, dx, dx_pitch, status, None)

    for bad in (dict(T=-1), dict(V=0), dict(d_pitch=99), dict(pitch=99), dict(dx_pitch=99), dict(n_hist=-1), dict(allowed=FAKE, masks=3), dict(allowed=FAKE, masks=4, mask_pitch=3)):
        assert call(**bad) == sr.SR_ERR_BAD_SIZE, bad
    assert call(dtype=7) == sr.SR_ERR_BAD_DTYPE
    for name in ("d", "x", "hist", "start", "length", "dx"):
        assert call(**{name: None}) == sr.SR_ERR_NULL, name
    for name in ("d", "x", "hist", "length", "rep", "mask_row", "dx", "status"):
        assert call(**{name: FAKE + 2}) == sr.SR_ERR_ALIGN, name
    assert call(dx=FAKE + 4) == sr.SR_ERR_OVERLAP and call(dx=3 * FAKE + 4) == sr.SR_ERR_OVERLAP and call(dx=3 * FAKE, dx_pitch=101) == sr.SR_ERR_OVERLAP
    assert call(T=0, d=None, x=None, hist=None, n_hist=0, start=None, length=None, rep=None, dx=None) == sr.SR_OK


def embed(lib, table=FAKE, td=1, V=100, D=16, tp=16, tokens=FAKE, T=4, scale=1.0, out=2 * FAKE, dtype=1, pitch=16, status=None):
    return lib.sr_embed_tokens(table, td, V, D, tp, tokens, T, scale, out, dtype, pitch, status, None)


def test_embed_refusals(lib):
    call = lambda **k: embed(lib, **k)
    for bad in (dict(T=-1), dict(V=0), dict(D=0), dict(D=(1 << 24) + 1, tp=1 << 25, pitch=1 << 25), dict(tp=15), dict(pitch=15), dict(tp=1 << 40), dict(pitch=1 << 40)):
        assert call(**bad) == sr.SR_ERR_BAD_SIZE, bad
    for td, dtype in ((3, 1), (1, 3), (1, 2), (2, 1), (1, 0), (2, 0)):
        assert call(td=td, dtype=dtype) == sr.SR_ERR_BAD_DTYPE, (td, dtype)
    for scale in (float("nan"), float("inf"), 1e39, -1e39):
        assert call(scale=scale) == sr.SR_ERR_BAD_VALUE
    for name in ("table", "tokens", "out"):
        assert call(**{name: None}) == sr.SR_ERR_NULL, name
    assert call(tokens=FAKE + 2) == sr.SR_ERR_ALIGN and call(status=FAKE + 2) == sr.SR_ERR_ALIGN and call(table=FAKE + 1) == sr.SR_ERR_ALIGN and call(out=2 * FAKE + 1) == sr.SR_ERR_ALIGN
    assert call(table=FAKE + 2, td=0) == sr.SR_ERR_ALIGN
    assert call(out=FAKE) == sr.SR_ERR_OVERLAP and call(out=FAKE + 100 * 32 - 2) == sr.SR_ERR_OVERLAP and call(out=FAKE - 4 * 32 + 2) == sr.SR_ERR_OVERLAP
    assert call(T=0, tokens=None, out=None) == sr.SR_OK


def test_embed_backward_refusals(lib):
    def call(d=2 * FAKE, dtype=1, T=4, D=16, pitch=16, tokens=FAKE, V=100, scale=1.0, table=FAKE, td=1, tp=16, acc=0, status=None, ws=3 * FAKE, wsb=1 << 20):
        return lib.sr_embed_tokens_backward(d, dtype, T, D, pitch, tokens, V, scale, table, td, tp, acc, status, ws, wsb, None)

    for bad in (dict(T=-1), dict(V=0), dict(D=0), dict(tp=15), dict(pitch=15)):
        assert call(**bad) == sr.SR_ERR_BAD_SIZE, bad
    assert call(td=2) == sr.SR_ERR_BAD_DTYPE and call(dtype=0) == sr.SR_ERR_BAD_DTYPE and call(scale=float("nan")) == sr.SR_ERR_BAD_VALUE
    for name in ("d", "tokens", "table"):
        assert call(**{name: None}) == sr.SR_ERR_NULL, name
    assert call(table=2 * FAKE) == sr.SR_ERR_OVERLAP
    need = lib.sr_embed_tokens_backward_workspace_bytes(4, 100, 16)
    assert call(ws=None) == sr.SR_ERR_WORKSPACE and call(wsb=need - 1) == sr.SR_ERR_WORKSPACE and call(ws=3 * FAKE + 8) == sr.SR_ERR_WORKSPACE
    assert call(T=0, d=None, tokens=None, acc=1) == sr.SR_OK            # nothing to add
    size = lib.sr_embed_tokens_backward_workspace_bytes
    assert size(-1, 10, 10) == 0 and size(10, 0, 10) == 0 and size(10, 10, 0) == 0 and size(10, 10, 1 << 25) == 0
    assert size(100000, 151936, 2048) >= 100000 * 16


def test_binding_refuses_what_the_library_cannot_see(lib):
    x, f, i = torch.zeros(4, 40), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: sr.sr_adjust_logits(x, out=x), lambda: sr.sr_adjust_logits_backward(x, None, d_logits=x), lambda: sr.sr_embed_tokens(x, i, out=x),
                 lambda: sr.sr_embed_tokens_backward(x, i, d_table=x, workspace=f)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    for call in (lambda: sr.sr_adjust_logits(f, out=f), lambda: sr.sr_adjust_logits(None, out=x), lambda: sr.sr_embed_tokens(f, i, out=x), lambda: sr.sr_embed_tokens_backward(None, i, d_table=x, workspace=f)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises((TypeError, ValueError)):
        sr.sr_adjust_logits(x.double(), out=x)
    with pytest.raises(TypeError):
        sr.sr_embed_tokens([1.0], i, out=x)


def test_the_header_is_plain_c(tmp_path):
    cc, inc = shutil.which("gcc") or shutil.which("cc"), os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    src = tmp_path / "tokens.c"
    src.write_text('#include "sr_tokens.h"\nint main(void) { return (int)sr_embed_tokens_backward_workspace_bytes(1, 1, 1) + SR_STATUS_BAD_INDEX + SR_DTYPE_F16; }\n')
    subprocess.run([cc, "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", inc, "-fsyntax-only", str(src)], check=True)


@pytest.mark.gpu
def test_binding_refuses_tensors_of_another_type_or_size():
    d = torch.device("cuda:0")
    x, f, i, l = torch.zeros(4, 40, device=d), torch.zeros(4, device=d), torch.zeros(4, dtype=torch.int32, device=d), torch.zeros(4, dtype=torch.int64, device=d)
    y, words, ws = torch.zeros(4, 40, device=d), torch.zeros(4, 2, dtype=torch.int32, device=d), torch.zeros(1 << 16, dtype=torch.uint8, device=d)
    hist = dict(history=i, history_start=l, history_len=i)
    sr.sr_adjust_logits(x, **hist, repetition=f + 1, allowed=words, out=y)
    for bad in (dict(history=l), dict(history_start=i), dict(history_len=l), dict(history_start=l[:3]), dict(history_len=i[:3]), dict(prompt_len=l), dict(prompt_len=i[:2]), dict(repetition=l),
                dict(repetition=f[:3]), dict(presence=i), dict(frequency=f[:1]), dict(bias_value=f, bias_token=i[:3], bias_start=l, bias_len=i), dict(bias_value=l, bias_token=i),
                dict(bias_value=f, bias_token=i, bias_start=i, bias_len=i), dict(allowed=words.long()), dict(allowed=words[:, :1]), dict(allowed=words.t()), dict(allowed=words[:3]),
                dict(allowed=words[:0], mask_row=i), dict(allowed=words, mask_row=l), dict(allowed=words, mask_row=i[:2]), dict(out=x[:3]), dict(out=x.half()), dict(out=x.cpu()), dict(out=x[:, ::2]),
                dict(status=f), dict(repetition=f.cpu())):
        with pytest.raises((TypeError, ValueError)):
            sr.sr_adjust_logits(x, **{**hist, "repetition": f + 1, "out": y, **bad})
    for bad in (dict(history_start=None), dict(bias_token=i, bias_value=f)):
        with pytest.raises(sr.SrError) as e:
            sr.sr_adjust_logits(x, **{**hist, "repetition": f + 1, "out": y, **bad})
        assert e.value.code == sr.SR_ERR_NULL
    wide = torch.zeros(200, device=d)
    with pytest.raises(sr.SrError) as e:
        sr.sr_adjust_logits(wide[:160].view(4, 40), out=wide[8:168].view(4, 40))
    assert e.value.code == sr.SR_ERR_OVERLAP
    for bad in (dict(logits=x.half()), dict(logits=x[:3]), dict(d_logits=x[:, :39]), dict(repetition=f[:3])):
        args = {"logits": x, "repetition": f + 1, "d_logits": y, **hist, **bad}
        with pytest.raises((TypeError, ValueError)):
            sr.sr_adjust_logits_backward(x, args.pop("logits"), **args)
    with pytest.raises(sr.SrError) as e:
        sr.sr_adjust_logits_backward(x, None, **hist, repetition=f + 1, d_logits=y)
    assert e.value.code == sr.SR_ERR_NULL
    for args, kind in (((x, l), TypeError), ((x, i[:3]), ValueError), ((x, torch.zeros(5, dtype=torch.int32, device=d)), ValueError), ((x[:, ::2], i), ValueError), ((x[:, :39], i), ValueError),
                       ((x.double(), i), TypeError)):
        with pytest.raises(kind):
            sr.sr_embed_tokens(*args, out=y)
    with pytest.raises(sr.SrError) as e:
        sr.sr_embed_tokens(x.half(), i, out=y)
    assert e.value.code == sr.SR_ERR_BAD_DTYPE
    with pytest.raises(sr.SrError) as e:
        sr.sr_embed_tokens_backward(x, i, d_table=y, workspace=ws[:64])
    assert e.value.code == sr.SR_ERR_WORKSPACE
    with pytest.raises(sr.SrError) as e:
        sr.sr_embed_tokens_backward(x, i, d_table=x, workspace=ws)
    assert e.value.code == sr.SR_ERR_OVERLAP
    for bad in (dict(d_table=y[:, :39]), dict(d_table=y.long()), dict(status=f)):
        with pytest.raises((TypeError, ValueError)):
            sr.sr_embed_tokens_backward(x, i, **{"d_table": y, "workspace": ws, **bad})
