"""Host-only checks of the layer operators' C ABI: sizes of workspaces and arguments that are refused before a GPU
is touched. No kernel runs here."""
import struct

import pytest

from paper_2609_36522_gb300 import abi
from paper_2609_36522_gb300 import build as pa_build

BLOCK = struct.Struct("=8id3Q9qQqQQqQQ3qQ4Q12q")  # pa_attention_t


@pytest.fixture(scope="module", autouse=True)
def _built():
    pa_build.build()


def _norm(dtype=abi.PA_F32, rows=4, cols=8, x=4096, xs=8, w=None, b=None, eps=1e-5, y=8192, ys=8, mean=None, rstd=None, count=None,
          per=1):
    return abi.pa_layer_norm(dtype, rows, cols, x, xs, w, b, eps, y, ys, mean, rstd, count, per, None)


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(cols=0), dict(eps=-1.0), dict(eps=float("inf")),
                                dict(x=None), dict(y=None), dict(x=4098), dict(w=2), dict(xs=7), dict(ys=4), dict(mean=4096),
                                dict(count=4096, per=3), dict(count=4096, per=0), dict(rows=1 << 41)])
def test_norm_refuses(kw):
    with pytest.raises(abi.PaError) as e:
        _norm(**kw)
    assert e.value.status == abi.PA_ERR_ARG and "pa_layer_norm" in str(e.value)


def test_norm_without_rows_does_nothing():
    assert _norm(rows=0, x=None, y=None) == abi.PA_OK


def test_norm_workspace():
    assert abi.pa_layer_norm_backward_workspace_bytes(-1, 8) == 0 and abi.pa_layer_norm_backward_workspace_bytes(8, 0) == 0
    few, many = (abi.pa_layer_norm_backward_workspace_bytes(n, 100) for n in (3, 10 ** 7))
    assert few % 256 == 0 and 0 < few < many < 1000 * 2 * 100 * 4

    def back(**kw):
        a = dict(dy=4096, x=8192, mean=4096, rstd=4096, dx=16384, dw=4096, db=None, ws=4096, nbytes=1 << 20)
        a.update(kw)
        return abi.pa_layer_norm_backward(abi.PA_BF16, 4, 8, a["dy"], 8, a["x"], 8, None, a["mean"], a["rstd"], a["dx"], 8, a["dw"],
                                          a["db"], None, 1, a["ws"], a["nbytes"], None)

    for kw, status in ((dict(dy=None), abi.PA_ERR_ARG), (dict(mean=None), abi.PA_ERR_ARG), (dict(dx=None), abi.PA_ERR_ARG),
                       (dict(ws=None), abi.PA_ERR_WORKSPACE), (dict(ws=4097), abi.PA_ERR_WORKSPACE),
                       (dict(nbytes=8), abi.PA_ERR_WORKSPACE)):
        with pytest.raises(abi.PaError) as e:
            back(**kw)
        assert e.value.status == status


FIELDS = ["dtype", "items", "tokens", "sources", "keys", "heads", "kv_heads", "head_dim", "scale", "q", "k", "v"]


def _block(lengths=0, mask=0, source=0, lse=65536, **kw):
    a = dict(dtype=abi.PA_BF16, items=2, tokens=3, sources=2, keys=5, heads=4, kv_heads=2, head_dim=16, scale=0.25, q=4096, k=4096,
             v=4096, out=4096, dout=4096, dq=4096, dk=4096, dv=4096, qs=(192, 64, 16), ks=(160, 32, 16))
    a.update(kw)
    return BLOCK.pack(*(a[f] for f in FIELDS), *a["qs"], *a["ks"], *a["ks"], source, 1, lengths, mask, 5, 0, a["out"], *a["qs"], lse,
                      a["dout"], a["dq"], a["dk"], a["dv"], *a["qs"], *a["qs"], *a["ks"], *a["ks"])


@pytest.mark.parametrize("kw", [dict(dtype=abi.PA_F32), dict(items=-1), dict(heads=3), dict(kv_heads=0), dict(head_dim=12),
                                dict(head_dim=264), dict(head_dim=0), dict(tokens=1 << 30), dict(items=1 << 30), dict(scale=0.0),
                                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=1e39), dict(q=0), dict(k=4104), dict(v=0),
                                dict(out=0), dict(qs=(192, 60, 16)), dict(sources=1), dict(heads=70000, kv_heads=1)])
def test_attention_refuses(kw):
    with pytest.raises(abi.PaError) as e:
        abi.pa_attention(_block(**kw), 4096, 1 << 30, None)
    assert e.value.status == abi.PA_ERR_ARG


@pytest.mark.parametrize("kw", [dict(dout=0), dict(dq=8), dict(dk=0), dict(dv=0), dict(lse=0)])
def test_attention_backward_refuses(kw):
    with pytest.raises(abi.PaError) as e:
        abi.pa_attention_backward(_block(**kw), 4096, 1 << 30, None)
    assert e.value.status == abi.PA_ERR_ARG


def test_attention_workspace():
    assert abi.pa_attention_workspace_bytes(_block(), 0) == 0
    masked = abi.pa_attention_workspace_bytes(_block(mask=4096), 0)
    assert masked >= 2 * 4 + 2 * 5 * 4 and masked % 256 == 0
    assert abi.pa_attention_workspace_bytes(_block(), 1) > 0
    for bad in (_block(head_dim=12), _block(items=-1)):
        with pytest.raises(abi.PaError):
            abi.pa_attention_workspace_bytes(bad, 0)
    for ws, nbytes in ((None, 0), (4100, 1 << 20), (4096, masked - 1)):
        with pytest.raises(abi.PaError) as e:
            abi.pa_attention(_block(mask=4096), ws, nbytes, None)
        assert e.value.status == abi.PA_ERR_WORKSPACE
    assert abi.pa_attention(_block(items=0), None, 0, None) == abi.PA_OK
    assert abi.pa_attention(_block(tokens=0), None, 0, None) == abi.PA_OK
