"""Workspace queries and refusals of the norm, the draws and the clipping: decided on the host, before any launch (no GPU)."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

import paper_2605_26646_amd as umas
from paper_2605_26646_amd import binding

F32, BF16 = 0, 1
PLENTY = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(umas.lib_path()):
        import __graft_entry__ as g
        g.build()
    return umas.load_library()


def test_structs_match_the_header():
    assert C.sizeof(binding._Sampling) == 3 * 8 + 8 + 4 * 8 and C.sizeof(binding._Gradient) == 32 and binding.CLIP_STATS_DTYPE.itemsize == 16


def test_queries(lib):
    assert lib.umas_rms_norm_workspace_bytes(0, 64) > 0
    assert lib.umas_rms_norm_workspace_bytes(100, 2048) <= lib.umas_rms_norm_workspace_bytes(100000, 2048) == lib.umas_rms_norm_workspace_bytes(1 << 30, 2048)
    for n, d in ((-1, 64), (4, 0), (4, 16385)):
        assert lib.umas_rms_norm_workspace_bytes(n, d) == 0
    assert 0 < lib.umas_sample_logits_workspace_bytes(1, 1) < lib.umas_sample_logits_workspace_bytes(64, 151936)
    assert lib.umas_sample_logits_workspace_bytes(5000, 3001) == lib.umas_sample_logits_workspace_bytes(1 << 40, 3001)
    for n, V in ((-1, 64), (4, 0), (4, (1 << 20) + 1)):
        assert lib.umas_sample_logits_workspace_bytes(n, V) == 0
        for w in ("_min", ""):
            assert getattr(lib, "umas_sample_tokens_workspace_bytes" + w)(n, 64, V, BF16) == 0
    for dtype in (F32, BF16):
        for n, d, V in ((0, 64, 300), (1, 64, 300), (64, 2048, 151936), (700, 1024, 1000)):
            least, full = (getattr(lib, "umas_sample_tokens_workspace_bytes" + w)(n, d, V, dtype) for w in ("_min", ""))
            assert 0 < least <= full
            if n > 256:
                assert least < full
    assert lib.umas_clip_workspace_bytes(-1) == 0 < lib.umas_clip_workspace_bytes(0) <= lib.umas_clip_workspace_bytes(96) < lib.umas_clip_workspace_bytes(1000)


def call_norm(lib, **kw):
    a = {**dict(x=256, residual=None, gain=256, dtype=BF16, n=4, d=64, eps=1e-6, hidden=None, y=256, inv=None, stream=None), **kw}
    return lib.umas_rms_norm(*a.values()), lib.umas_last_error().decode()


def call_quantized(lib, **kw):
    a = {**dict(x=256, residual=None, gain=256, dtype=BF16, n=4, d=64, eps=1e-6, hidden=None, y=256, scale=256, inv=None, stream=None), **kw}
    return lib.umas_rms_norm_quantized(*a.values()), lib.umas_last_error().decode()


def call_back(lib, **kw):
    a = {**dict(dy=256, x=256, gain=256, inv=256, dhidden=None, dtype=BF16, n=4, d=64, add=0, dx=256, dgain=256, ws=256, ws_bytes=PLENTY, stream=None), **kw}
    return lib.umas_rms_norm_bwd(*a.values()), lib.umas_last_error().decode()


NORM = [(dict(dtype=7), -3, "dtype"), (dict(n=-1), -1, "negative"), (dict(d=0), -2, "d=0"), (dict(d=16392), -2, "d=16392"), (dict(d=60), -2, "d % 8"), (dict(n=1 << 31), -2, "2^31-1"),
        (dict(x=None), -1, "NULL"), (dict(gain=None), -1, "gain"), (dict(x=264), -1, "16-byte"), (dict(gain=264), -1, "16-byte")]


@pytest.mark.parametrize("call", [call_norm, call_quantized, call_back])
@pytest.mark.parametrize("kw,code,needle", NORM)
def test_shared_arguments_of_the_norm(lib, call, kw, code, needle):
    status, message = call(lib, **kw)
    assert status == code and needle in message, message


@pytest.mark.parametrize("call,kw,code,needle", [
    (call_norm, dict(eps=-1.0), -1, "eps"), (call_norm, dict(eps=math.nan), -1, "eps"), (call_norm, dict(eps=math.inf), -1, "eps"), (call_norm, dict(y=None), -1, "output"),
    (call_norm, dict(residual=512), -1, "go together"), (call_norm, dict(hidden=512), -1, "go together"), (call_norm, dict(residual=520, hidden=512), -1, "16-byte"),
    (call_norm, dict(y=264), -1, "16-byte"), (call_quantized, dict(y=None), -1, "q and scale"), (call_quantized, dict(scale=None), -1, "q and scale"),
    (call_quantized, dict(y=264), -1, "16-byte"), (call_back, dict(dy=None), -1, "dy"), (call_back, dict(inv=None), -1, "inv_rms"), (call_back, dict(dx=None), -1, "dx"),
    (call_back, dict(dgain=None), -1, "dgain"), (call_back, dict(dhidden=264), -1, "16-byte"), (call_back, dict(dx=264), -1, "16-byte"), (call_back, dict(ws=None), -4, "workspace"),
    (call_back, dict(ws=264), -4, "256-byte"), (call_back, dict(ws_bytes=256), -4, "hold")])
def test_arguments_of_the_norm(lib, call, kw, code, needle):
    status, message = call(lib, **kw)
    assert status == code and needle in message, message


SETTINGS = dict(temperature=1.0, top_p=1.0, min_p=0.0, top_k=0, temperature_of=None, top_p_of=None, min_p_of=None, top_k_of=None)


def call_logits(lib, settings=None, **kw):
    s = binding._Sampling(*{**SETTINGS, **(settings or {})}.values())
    a = {**dict(logits=256, dtype=F32, n=4, V=100, stride=100, u=256, sampling=C.addressof(s), ids=256, logp=None, logq=None, ws=256, ws_bytes=PLENTY, stream=None), **kw}
    return lib.umas_sample_logits(*a.values()), lib.umas_last_error().decode()


def call_tokens(lib, settings=None, **kw):
    s = binding._Sampling(*{**SETTINGS, **(settings or {})}.values())
    a = {**dict(H=256, W=256, dtype=BF16, n=4, d=64, V=100, rowsel=None, n_sel=4, u=256, sampling=C.addressof(s), ids=256, logp=None, logq=None, ws=256, ws_bytes=PLENTY, stream=None), **kw}
    return lib.umas_sample_tokens(*a.values()), lib.umas_last_error().decode()


@pytest.mark.parametrize("call", [call_logits, call_tokens])
@pytest.mark.parametrize("kw,code,needle", [
    (dict(dtype=7), -3, "dtype"), (dict(n=-1), -1, "negative"), (dict(V=0), -2, "positive"), (dict(V=(1 << 20) + 1, stride=1 << 21), -2, "exceeds"), (dict(u=None), -1, "u "),
    (dict(ids=None), -1, "ids"), (dict(sampling=None), -1, "sampling"), (dict(ws=None), -4, "workspace"), (dict(ws=264), -4, "256-byte"), (dict(ws_bytes=64), -4, "hold"),
    (dict(settings=dict(temperature=-0.1)), -1, "temperature"), (dict(settings=dict(temperature=math.nan)), -1, "temperature"), (dict(settings=dict(top_p=1.1)), -1, "top_p"),
    (dict(settings=dict(top_p=-0.1)), -1, "top_p"), (dict(settings=dict(top_p=math.nan)), -1, "top_p"), (dict(settings=dict(min_p=1.1)), -1, "min_p"),
    (dict(settings=dict(min_p=math.nan)), -1, "min_p"), (dict(settings=dict(top_k=-1)), -1, "top_k")])
def test_arguments_of_the_draws(lib, call, kw, code, needle):
    if call is call_tokens:
        kw = {k: v for k, v in kw.items() if k != "stride"}
    status, message = call(lib, **kw)
    assert status == code and needle in message, message


def test_arguments_of_one_draw(lib):
    for call, kw, code, needle in ((call_logits, dict(logits=None), -1, "logits"), (call_logits, dict(logits=258), -1, "aligned"), (call_logits, dict(stride=99), -1, "row_stride"),
                                   (call_tokens, dict(n_sel=3), -1, "rowsel is NULL"), (call_tokens, dict(rowsel=256, n_sel=5), -1, "exceeds n_rows"), (call_tokens, dict(d=60), -2, "d % 8"),
                                   (call_tokens, dict(H=264), -1, "16-byte")):
        status, message = call(lib, **kw)
        assert status == code and needle in message, message
    # numbers for all rows do not matter where every row has its own
    status, message = call_logits(lib, dict(temperature=-1.0, temperature_of=256, top_p=7.0, top_p_of=256, min_p=7.0, min_p_of=256, top_k=-4, top_k_of=256), ws=None)
    assert status == -4


def call_clip(lib, entries, **kw):
    g = (binding._Gradient * max(len(entries), 1))(*[binding._Gradient(*e) for e in entries])
    a = {**dict(g=C.addressof(g), n=len(entries), max_norm=1.0, stats=256, ws=256, ws_bytes=PLENTY, stream=None), **kw}
    return lib.umas_clip_gradients(*a.values()), lib.umas_last_error().decode()


@pytest.mark.parametrize("entries,kw,code,needle", [
    ([], dict(n=-1), -1, "negative"), ([], dict(n=2, g=None), -1, "gradients"), ([], dict(max_norm=0.0), -1, "max_norm"), ([], dict(max_norm=-1.0), -1, "max_norm"),
    ([], dict(max_norm=math.nan), -1, "max_norm"), ([], dict(stats=None), -1, "stats"), ([], dict(ws=None), -4, "workspace"), ([], dict(ws_bytes=8), -4, "hold"),
    ([(256, 256, 4, 7)], {}, -3, "gradient 0: dtype"), ([(256, 256, 4, F32), (512, 512, -4, F32)], {}, -1, "gradient 1: n=-4"), ([(None, 256, 4, F32)], {}, -1, "NULL"),
    ([(256, None, 4, F32)], {}, -1, "NULL"), ([(258, 258, 4, F32)], {}, -1, "aligned"), ([(257, 257, 4, BF16)], {}, -1, "aligned"),
    ([(256, 256, 4, F32), (256, 256, 4, F32)], {}, -1, "overlaps"), ([(256, 256, 100, F32), (400, 400, 4, BF16)], {}, -1, "overlaps"),
    ([(256, 1024, 100, F32), (4096, 1400, 10, F32)], {}, -1, "overlaps"), ([(256, 260, 100, F32)], {}, -1, "overlaps"), ([(4096, 256, 100, F32), (512, 2048, 4, F32)], {}, -1, "overlaps"),
    ([(256, 4096, (1 << 44) - 1, F32)], {}, -2, "too many")])
def test_arguments_of_clipping(lib, entries, kw, code, needle):
    status, message = call_clip(lib, entries, **kw)
    assert status == code and needle in message, message


def test_lists_that_do_not_overlap_get_as_far_as_the_workspace(lib):
    for entries in ([(256, 256, 4, F32), (272, 272, 4, F32)], [(256, 4096, 4, F32), (256, 8192, 4, F32)], [(256, 4096, 4, F32), (4112, 4112, 0, F32)],
                    [(None, None, 0, F32), (256, 256, 10, BF16), (276, 276, 4, BF16)]):
        assert call_clip(lib, entries, ws=None)[0] == -4


# ------------------------------------------------------------------------------------------------ the binding's own checks, on host tensors
B, F, I, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
Z = torch.zeros


def native_norm(**kw):
    a = {**dict(x=Z(6, 16, dtype=B), gain=Z(16, dtype=B), residual=None, eps=1e-6, hidden=None, y=None, inv=None), **kw}
    return binding._native().rms_norm(*a.values(), 0)


def native_quantized(**kw):
    a = {**dict(x=Z(6, 16, dtype=B), gain=Z(16, dtype=B), residual=None, eps=1e-6, hidden=None, y=None, scale=None, inv=None), **kw}
    return binding._native().rms_norm_quantized(*a.values(), 0)


def native_back(**kw):
    a = {**dict(dy=Z(6, 16, dtype=B), hidden=Z(6, 16, dtype=B), gain=Z(16, dtype=B), inv=Z(6), dhidden=None, add=False, dx=None, dgain=None, ws=None), **kw}
    return binding._native().rms_norm_bwd(*a.values(), 0)


def native_logits(**kw):
    a = {**dict(z=Z(6, 40), u=Z(6), temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, ids=None, logp=None, logq=None, ws=None), **kw}
    return binding._native().sample_logits(*a.values(), 0)


def native_tokens(**kw):
    a = {**dict(H=Z(6, 16, dtype=B), W=Z(40, 16, dtype=B), u=Z(6), rowsel=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, ids=None, logp=None, logq=None, ws=None), **kw}
    return binding._native().sample_tokens(*a.values(), 0)


def native_clip(**kw):
    a = {**dict(g=[Z(6, 4), Z(5, dtype=B)], max_norm=1.0, out=None, stats=None, ws=None), **kw}
    return binding._native().clip_gradients(*a.values(), 0)


CALLS = [native_norm, native_quantized, native_back, native_logits, native_tokens, native_clip]
WRONG = [(native_norm, dict(x=Z(6, 2, 8, dtype=B))), (native_norm, dict(x=Z(16, 6, dtype=B).T)), (native_norm, dict(gain=Z(16))), (native_norm, dict(gain=Z(15, dtype=B))),
         (native_norm, dict(residual=Z(6, 16))), (native_norm, dict(residual=Z(5, 16, dtype=B))), (native_norm, dict(hidden=Z(6, 16, dtype=B))),
         (native_norm, dict(residual=Z(6, 16, dtype=B), hidden=Z(6, 15, dtype=B))), (native_norm, dict(y=Z(6, 16))), (native_norm, dict(inv=Z(5))), (native_norm, dict(inv=Z(6, dtype=B))),
         (native_quantized, dict(y=Z(6, 16, dtype=B))), (native_quantized, dict(y=Z(6, 15).to(torch.float8_e4m3fn))), (native_quantized, dict(scale=Z(5))),
         (native_back, dict(hidden=Z(6, 16))), (native_back, dict(gain=Z(17, dtype=B))), (native_back, dict(inv=Z(7))), (native_back, dict(dhidden=Z(6, 32, dtype=B)[:, ::2])),
         (native_back, dict(dx=Z(6, 16))), (native_back, dict(dgain=Z(16, dtype=B))), (native_back, dict(add=True)), (native_logits, dict(z=Z(6, 80)[:, ::2])),
         (native_logits, dict(z=Z(1, 40).expand(6, 40))), (native_logits, dict(z=Z(40))), (native_logits, dict(u=Z(5))), (native_logits, dict(u=Z(6, dtype=torch.float64))),
         (native_logits, dict(temperature=Z(5))), (native_logits, dict(top_k=Z(6))), (native_logits, dict(top_p=Z(6, dtype=torch.float64))), (native_logits, dict(min_p=Z(6, dtype=I))),
         (native_logits, dict(ids=Z(6))), (native_logits, dict(logp=Z(5))), (native_logits, dict(logq=Z(6, dtype=B))), (native_tokens, dict(W=Z(40, 24, dtype=B))),
         (native_tokens, dict(u=Z(3), rowsel=Z(3, dtype=I))), (native_tokens, dict(temperature=Z(3), rowsel=Z(3, dtype=I))), (native_clip, dict(g=[])), (native_clip, dict(g=[Z(4, 6).T])),
         (native_clip, dict(out=[Z(6, 4)])), (native_clip, dict(out=[Z(6, 4), Z(5)])), (native_clip, dict(out=[Z(6, 4), Z(6, dtype=B)])), (native_clip, dict(stats=Z(15, dtype=U8)))]


@pytest.mark.parametrize("call,kw", WRONG)
def test_tensors_that_do_not_fit(lib, call, kw):
    with pytest.raises(ValueError, match="^(?!.*GPU)"):
        call(**kw)


@pytest.mark.parametrize("call,kw", [(native_norm, dict(x=Z(6, 16, dtype=torch.float16))), (native_norm, dict(gain=3)), (native_logits, dict(z=Z(6, 40, dtype=I))),
                                     (native_logits, dict(temperature="1")), (native_tokens, dict(rowsel=Z(3, dtype=torch.int64))), (native_clip, dict(g=5)),
                                     (native_clip, dict(g=[Z(3, dtype=torch.float16)])), (native_clip, dict(g=[1.0])), (native_clip, dict(max_norm=None))])
def test_arguments_of_other_kinds(lib, call, kw):
    with pytest.raises(TypeError):
        call(**kw)


def test_outputs_that_are_one_array(lib):
    one = Z(6)
    with pytest.raises(ValueError, match="different"):
        native_logits(logp=one, logq=one)
    x = Z(6, 16, dtype=B)
    with pytest.raises(ValueError, match="different"):
        native_norm(x=x, residual=Z(6, 16, dtype=B), hidden=x, y=x)


@pytest.mark.parametrize("call", CALLS)
def test_arrays_of_the_host(lib, call):
    with pytest.raises(ValueError, match="GPU"):
        call()


def away(*shape, dtype=F):
    return torch.empty(*shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("call,kw", [(native_norm, dict(gain=away(16, dtype=B))), (native_norm, dict(residual=away(6, 16, dtype=B))), (native_norm, dict(y=away(6, 16, dtype=B))),
                                     (native_norm, dict(inv=away(6))), (native_quantized, dict(scale=away(6))), (native_back, dict(hidden=away(6, 16, dtype=B))),
                                     (native_back, dict(inv=away(6))), (native_back, dict(dhidden=away(6, 16, dtype=B))), (native_back, dict(dgain=away(16))),
                                     (native_back, dict(ws=away(1 << 20, dtype=U8))), (native_logits, dict(u=away(6))), (native_logits, dict(temperature=away(6))),
                                     (native_logits, dict(top_k=away(6, dtype=I))), (native_logits, dict(ids=away(6, dtype=I))), (native_logits, dict(ws=away(1 << 20, dtype=U8))),
                                     (native_tokens, dict(W=away(40, 16, dtype=B))), (native_tokens, dict(rowsel=away(6, dtype=I))), (native_tokens, dict(logq=away(6))),
                                     (native_clip, dict(g=[Z(4), away(4)])), (native_clip, dict(out=[Z(6, 4), away(5, dtype=B)])), (native_clip, dict(stats=away(16, dtype=U8)))])
def test_an_array_of_another_device(lib, call, kw):
    with pytest.raises(ValueError, match="device"):
        call(**kw)


@pytest.mark.parametrize("call", [native_logits, native_tokens])
def test_draws_into_what_the_call_reads(lib, call):
    one, whole = Z(6), Z(6, dtype=I)
    for kw in (dict(u=one, logp=one), dict(u=one, logq=one), dict(temperature=one, logp=one), dict(top_p=one, logq=one), dict(min_p=one, logp=one), dict(top_k=whole, ids=whole)):
        with pytest.raises(ValueError, match="different"):
            call(**kw)


def test_statistics_of_clipping_are_aligned(lib):
    status, message = call_clip(lib, [], stats=260)
    assert status == -1 and "8-byte" in message
