"""CPU tests of the head calls and of shared-prefix attention: every refused argument is
refused before anything is launched, workspace figures, and the helpers of the rotation."""
import ctypes
import math

import pytest
import torch

import paper_2106_06899_amd as tk
from paper_2106_06899_amd import layers

E_INVAL, E_NULL, E_ALIGN, E_UNSUPPORTED = -1, -2, -3, -4
FAKE = 0x10000  # aligned, never dereferenced: every call below fails validation first


def _rot(**kw):
    a = dict(positions=FAKE, freqs=FAKE, pair_axis=None, d_rot=64, axis_stride=0, batch_stride=0, token_stride=1, n_axes=1,
             position_bytes=8, adjacent=0, inverse=0)
    a.update(kw)
    return tk._Rotation(*a.values())


def _rope(rot=None, **kw):
    a = dict(x=FAKE, out=FAKE, B=1, H=2, L=5, d=64, sb=640, sh=320, sl=64)
    dtype = kw.pop("dtype", 1)
    a.update(kw)
    return tk.lib().topk_rope(*a.values(), _rot(**rot) if rot is not None else None, dtype, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), E_INVAL), (dict(H=0), E_INVAL), (dict(L=0), E_INVAL), (dict(d=0), E_INVAL), (dict(d=63), E_UNSUPPORTED),
    (dict(d=514), E_UNSUPPORTED), (dict(dtype=2), E_INVAL), (dict(x=None), E_NULL), (dict(out=None), E_NULL),
    (dict(x=FAKE + 1), E_ALIGN), (dict(out=FAKE + 2, dtype=0), E_ALIGN), (dict(sb=-1), E_INVAL), (dict(sl=1 << 40), E_INVAL),
    (dict(H=20000), E_UNSUPPORTED), (dict(B=1 << 20, L=1 << 20), E_UNSUPPORTED),
    (dict(rot=dict(d_rot=66)), E_INVAL), (dict(rot=dict(d_rot=3)), E_INVAL), (dict(rot=dict(d_rot=-2)), E_INVAL),
    (dict(rot=dict(n_axes=0)), E_INVAL), (dict(rot=dict(n_axes=5)), E_INVAL), (dict(rot=dict(positions=None)), E_NULL),
    (dict(rot=dict(freqs=None)), E_NULL), (dict(rot=dict(position_bytes=2)), E_INVAL),
    (dict(rot=dict(positions=FAKE + 4)), E_ALIGN), (dict(rot=dict(freqs=FAKE + 4)), E_ALIGN),
    (dict(rot=dict(adjacent=2)), E_INVAL), (dict(rot=dict(token_stride=-1)), E_INVAL),
    (dict(rot=dict(n_axes=2, pair_axis=bytes([0, 1] * 15 + [2, 0]))), E_INVAL),
])
def test_rope_refusals(kw, code):
    assert _rope(**kw) == code
    assert tk.lib().topk_last_error()


def _heads(name, **kw):
    a = dict(qkv=FAKE, wq=FAKE, wk=FAKE)
    outs = dict(forward=("q", "k", "v"), append=("q", "kc", "vc", "lengths"), backward=("dq", "dk", "dv", "dx", "dwq", "dwk"))[name]
    a.update({n: FAKE for n in outs})
    a.update(B=1, L=3, H=2, Hkv=1, d=64, sb=768, sl=256)
    if name == "append":
        a.update(S=10, ksb=640, ksh=640, ksl=64, vsb=640, vsh=640, vsl=64)
    a.update(norm=1, eps=1e-6)
    rot = kw.pop("rot", None)
    a.update(kw)
    fn = {"forward": "topk_qk_norm_rope", "append": "topk_qk_norm_rope_append", "backward": "topk_qk_norm_rope_backward"}[name]
    return getattr(tk.lib(), fn)(*a.values(), _rot(**rot) if rot else None, 1, None)


@pytest.mark.parametrize("form,kw,code", [(f, kw, c) for f in ("forward", "append", "backward") for kw, c in [
    (dict(Hkv=0), E_INVAL), (dict(H=0), E_INVAL), (dict(d=65), E_UNSUPPORTED), (dict(eps=-1.0), E_INVAL), (dict(eps=math.nan), E_INVAL),
    (dict(norm=2), E_INVAL), (dict(norm=0), E_INVAL), (dict(qkv=None), E_NULL), (dict(wq=FAKE + 1), E_ALIGN), (dict(sl=-1), E_INVAL),
    (dict(rot=dict(d_rot=128)), E_INVAL)]] + [
    ("forward", dict(v=None), E_NULL), ("append", dict(kc=None), E_NULL), ("append", dict(lengths=None), E_NULL),
    ("append", dict(lengths=FAKE + 2), E_ALIGN), ("append", dict(S=-1), E_INVAL), ("append", dict(vsl=-64), E_INVAL),
    ("backward", dict(dk=None), E_NULL), ("backward", dict(dx=FAKE + 1), E_ALIGN)])
def test_heads_refusals(form, kw, code):
    assert _heads(form, **kw) == code
    assert tk.lib().topk_last_error()


def _prefix(**kw):
    a = dict(Q=FAKE, pk=FAKE, pv=FAKE, k=FAKE, v=FAKE, lengths=FAKE, out=FAKE, lse=None, B=2, H=4, Hkv=2, Lq=1, P=100, S=10, d=64)
    st, causal, scale, dtype = kw.pop("strides", None), kw.pop("causal", 1), kw.pop("scale", 0.125), kw.pop("dtype", 1)
    a.update(kw)
    return tk.lib().topk_attn_prefix(*a.values(), st, causal, scale, dtype, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), E_INVAL), (dict(Lq=0), E_INVAL), (dict(P=-1), E_INVAL), (dict(S=-1), E_INVAL), (dict(H=3), E_INVAL),
    (dict(Hkv=0), E_INVAL), (dict(causal=2), E_INVAL), (dict(scale=0.0), E_INVAL), (dict(scale=math.inf), E_INVAL),
    (dict(dtype=3), E_INVAL), (dict(dtype=0), E_UNSUPPORTED), (dict(d=96), E_UNSUPPORTED), (dict(P=1 << 31), E_UNSUPPORTED),
    (dict(B=1 << 30, H=1 << 4), E_UNSUPPORTED), (dict(Q=None), E_NULL), (dict(out=None), E_NULL), (dict(pk=None), E_NULL),
    (dict(v=None), E_NULL), (dict(k=FAKE + 8), E_ALIGN), (dict(lengths=FAKE + 2), E_ALIGN), (dict(lse=FAKE + 1), E_ALIGN),
    (dict(strides=tk._PrefixStrides(6400, 64, 6400, 68)), E_ALIGN), (dict(strides=tk._PrefixStrides(6400, 1 << 26, 6400, 64)), E_UNSUPPORTED),
    (dict(strides=tk._PrefixStrides(-8, 64, 6400, 64)), E_INVAL),
])
def test_prefix_refusals(kw, code):
    assert _prefix(**kw) == code
    assert tk.lib().topk_last_error()


def test_workspace_figures():
    assert tk.attn_prefix_workspace_bytes(2, 4, 2, 1, 100, 0, 64) == 0        # one range: written at once
    assert tk.attn_prefix_workspace_bytes(2, 4, 2, 1, 0, 0, 64) == 0
    assert tk.attn_prefix_workspace_bytes(2, 4, 2, 1, 100, 10, 64) == 0
    assert tk.attn_prefix_workspace_bytes(2, 4, 2, 1, 2000, 10, 64) >= 2 * 8 * 66 * 4
    assert tk.attn_prefix_workspace_bytes(2, 4, 3, 1, 100, 10, 64) == 0       # invalid
    L = tk.lib()
    assert L.topk_qk_norm_rope_backward_workspace_bytes(8, 512, 12, 12, 64, 64, 1) >= 2 * 64 * 4
    assert L.topk_qk_norm_rope_backward_workspace_bytes(8, 512, 12, 0, 64, 64, 1) == 0
    assert L.topk_qk_norm_rope_backward_workspace_bytes(8, 512, 12, 12, 64, 66, 1) == 0


def test_frequencies_and_axes():
    f = tk.rope_frequencies(4, 100.0, device="cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(tk.rope_frequencies((2, 2), 100.0, device="cpu"), f)
    g = tk.rope_frequencies((2, 3), 100.0, restart=True, device="cpu")
    assert torch.equal(g[:2], tk.rope_frequencies(2, 100.0, device="cpu")) and torch.equal(g[2:], tk.rope_frequencies(3, 100.0, device="cpu"))
    assert tk.rope_axes((1, 2, 2)) == (0, 1, 1, 2, 2) and tk.rope_axes((1, 3, 2), interleaved=True) == (0, 1, 2, 1, 2, 1)
    with pytest.raises(ValueError):
        tk.rope_frequencies((), device="cpu")


def test_host_tensors_are_refused():
    x, p, f = torch.zeros(1, 1, 2, 64), torch.arange(2), tk.rope_frequencies(32, device="cpu")
    for call in (lambda: tk.rope(x, p, f), lambda: tk.qk_norm_rope(torch.zeros(1, 2, 192), 1, 1),
                 lambda: tk.attn_prefix(x.bfloat16(), x[0].bfloat16(), x[0].bfloat16())):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_layer_options():
    m = layers.TopkMultiheadAttention(128, 2, 8, dtype=torch.bfloat16)
    assert set(m.state_dict()) == {"qkv.weight", "qkv.bias", "out.weight", "out.bias"}  # as without the options
    m = layers.TopkMultiheadAttention(128, 2, None, causal=True, qk_norm=True, rope_theta=1e4, rope_sections=(8, 12, 12))
    assert {"q_norm", "k_norm"} < set(m.state_dict()) and "rope_bits" not in m.state_dict()
    want = tk.rope_frequencies(32, 1e4, device="cpu")
    assert torch.equal(m.to(torch.float32).rope_bits.view(torch.float64), want)
    assert m.rope_axes == (0,) * 8 + (1,) * 12 + (2,) * 12
    with pytest.raises(ValueError):
        layers.TopkMultiheadAttention(128, 2, 8, rope_theta=1e4, rope_sections=(30, 30))
    with pytest.raises(ValueError):
        layers.TopkMultiheadAttention(128, 2, 8, rope_sections=(8, 8))
    with pytest.raises(ValueError):
        layers.TopkMultiheadAttention(128, 2, 8).decode(*[torch.zeros(1, 1, 128)] * 6)


@pytest.mark.parametrize("B,H,Lq", [(1, 1, (1 << 26) + 1), (1 << 26, 2, 1), (3, 1 << 25, 1)])
def test_more_rows_than_a_launch_holds_are_refused(B, H, Lq):
    assert _prefix(B=B, H=H, Hkv=1, Lq=Lq) == E_UNSUPPORTED
    assert tk.attn_prefix_workspace_bytes(B, H, 1, Lq, 100, 10, 64) == 0


@pytest.mark.parametrize("Lq", [1, 20, 40, 80, 128, 1024])
def test_calls_without_keys_are_planned(Lq):
    for d in (64, 128):
        assert tk.attn_prefix_workspace_bytes(2, 2, 2, Lq, 0, 0, d) == 0


def _turning(**kw):
    return layers.TopkMultiheadAttention(128, 2, 8, rope_theta=1e4, rope_sections=(8, 12, 12), **kw)


def test_layers_built_without_memory():
    """Under a default device without memory, or on it by name: the frequencies are made where the weights
    are, and are there once the layer has memory, however it comes by it."""
    want = tk.rope_frequencies(32, 1e4, device="cpu")
    for named in (False, True):
        if named:
            m = _turning(device="meta")
        else:
            with torch.device("meta"):
                m = _turning()
                assert torch.equal(tk.rope_frequencies(32, 1e4, device="cpu"), want)
        assert m.qkv.weight.is_meta and m.rope_bits.is_meta
        whole = torch.nn.Sequential(m).to_empty(device="cpu")
        assert torch.equal(whole[0].rope_bits.view(torch.float64), want)
        m.load_state_dict(_turning().state_dict())
        assert torch.equal(m.rope_bits.view(torch.float64), want)
    m = _turning(device="meta")
    m.load_state_dict(_turning().state_dict(), assign=True)
    assert torch.equal(m._rotation(None, 3, torch.device("cpu"))["freqs"], want)
    before = m.rope_bits
    assert m.to(torch.float32).rope_bits is before  # (what a captured graph reads stays)


def test_layer_of_sections_without_pairs():
    """Sections of no pairs at all: nothing turns, by the default positions too."""
    m = layers.TopkMultiheadAttention(128, 2, 8, rope_theta=1e4, rope_sections=(0,))
    rot = m._rotation(None, 3, torch.device("cpu"))
    assert rot["freqs"].numel() == 0 and rot["positions"].shape == (1, 1, 3)
