"""The paged key-value cache without a GPU: the oracle's formats against torch's, page sizes, and every refusal of the entry
points (nothing is launched)."""
import ctypes as C
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2605_30010_amd as et
from oracle import kv_oracle as O
from paper_2605_30010_amd import binding as B
from paper_2605_30010_amd.build import CSRC, FLAGS, HIPCC


def test_oracle_e4m3_values_are_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3_values(), t, equal_nan=True)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_oracle_codes_are_torchs_roundings(fmt):
    """Ties (row maxima 1 and 254 / 448 times a power of two leave many) go to the even code on both sides."""
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.normal(size=(200, 64))).to(torch.bfloat16)
    x[:100] = torch.from_numpy(rng.integers(-256, 257, (100, 64)) / 256.0).to(torch.bfloat16)
    x[:50, 0], x[50:60, 0], x[60:70] = 1.0, {"int8": 254.0, "e4m3": 448.0}[fmt], 0.0
    x = x.double()
    codes, m = O.hold(x.numpy(), fmt)
    y = x * O.QMAX[fmt] / x.abs().amax(-1, keepdim=True).clamp(min=1e-30)
    ref = torch.round(y).to(torch.int8).view(torch.uint8) if fmt == "int8" else y.float().to(torch.float8_e4m3fn).view(torch.uint8)
    zero = torch.from_numpy(m == 0)[:, None]
    assert torch.equal(torch.where(zero, 0, torch.from_numpy(codes)), torch.where(zero, 0, ref))
    assert np.array_equal(m, x.abs().amax(-1).numpy())
    step = np.abs(O.stands_for(codes, m, fmt) - x.numpy()) / np.maximum(m, 1e-30)[:, None]
    # half a step: 1 / 2 of 127, and 16 of 448 where the codes are coarsest (256 to 448 in steps of 32)
    assert step.max() <= (0.5 / 127 if fmt == "int8" else 16 / 448) + 1e-12


def test_oracle_attention_is_torchs():
    rng = np.random.default_rng(4)
    q, k, v = rng.normal(size=(6, 64)), rng.normal(size=(33, 2, 64)), rng.normal(size=(33, 2, 64))
    out, mass, size = O.attend_one(q, k, v, 0.125)
    t = torch.from_numpy
    ref = torch.nn.functional.scaled_dot_product_attention(t(q)[:, None], t(k).repeat_interleave(3, 1).transpose(0, 1),
                                                           t(v).repeat_interleave(3, 1).transpose(0, 1), scale=0.125)[:, 0]
    assert np.allclose(out, ref.numpy(), atol=1e-12) and (mass >= np.abs(out)).all() and (size > 0).all()
    assert not O.attend_one(q, k[:0], v[:0], 1.0)[0].any()


def test_page_bytes():
    assert et.et_kv_page_bytes(64, 4, 128, "bf16") == 2 * 64 * 4 * 128 * 2
    assert et.et_kv_page_bytes(16, 3, 80, "int8") == et.et_kv_page_bytes(16, 3, 80, "e4m3") == 2 * 16 * 3 * (80 + 2)
    for bad in ((0, 4, 128), (8, 4, 128), (48, 4, 128), (512, 4, 128), (64, 0, 128), (64, 1025, 128), (64, 4, 72), (64, 4, 0), (64, 4, -64)):
        assert et.et_kv_page_bytes(*bad, "bf16") == 0
    assert et.load_library().et_kv_page_bytes(64, 4, 128, 3) == 0


FAKE = 4096                                              # never dereferenced: validation comes first


def cache(**kw):
    return B._KvCache(**dict(dict(data_dev=FAKE, n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, format=0), **kw))


def seqs(**kw):
    return B._KvSeqs(**dict(dict(page_table_dev=FAKE, table_stride=4, pages_per_seq=4, kv_len_dev=FAKE, n_seqs=3), **kw))


def rows_call(fn, c=None, s=None, cu=FAKE, rows=5, k=FAKE, ks=128, v=FAKE, vs=128):
    c, s = cache() if c is None else c, seqs() if s is None else s
    return fn(c and C.byref(c), s and C.byref(s), cu, rows, k, ks, v, vs, None)


def attend_call(c=None, s=None, q=FAKE, qs=256, heads=4, max_len=64, window=0, scale=0.125, ws=FAKE, ws_bytes=1 << 40, out=FAKE):
    c, s = cache() if c is None else c, seqs() if s is None else s
    return et.load_library().et_attention_paged(c and C.byref(c), s and C.byref(s), q, qs, heads, max_len, window, scale, ws, ws_bytes,
                                                out, None)


BAD_CACHES = [(dict(data_dev=None), -1), (dict(data_dev=FAKE + 8), -1), (dict(n_pages=0), -1), (dict(page_size=24), -5),
              (dict(page_size=8), -5), (dict(n_kv_heads=0), -1), (dict(n_kv_heads=2000), -1), (dict(head_dim=72), -5),
              (dict(head_dim=0), -5), (dict(format=3), -1), (dict(format=-1), -1)]
BAD_SEQS = [(dict(page_table_dev=None), -1), (dict(kv_len_dev=None), -1), (dict(n_seqs=-1), -1), (dict(pages_per_seq=0), -1),
            (dict(table_stride=3), -1), (dict(pages_per_seq=1 << 27, table_stride=1 << 27), -1)]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_refused_caches(bad, code):
    lib = et.load_library()
    assert rows_call(lib.et_kv_append, c=cache(**bad)) == code and et.et_last_error()
    assert rows_call(lib.et_kv_read, c=cache(**bad)) == code
    assert attend_call(c=cache(**bad)) == code


@pytest.mark.parametrize("bad,code", BAD_SEQS)
def test_refused_sequences(bad, code):
    lib = et.load_library()
    assert rows_call(lib.et_kv_append, s=seqs(**bad)) == code and et.et_last_error()
    assert rows_call(lib.et_kv_read, s=seqs(**bad)) == code
    assert attend_call(s=seqs(**bad)) == code


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cu=None), dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(v=FAKE + 8), dict(ks=127),
                                 dict(ks=132), dict(vs=120), dict(ks=0), dict(vs=-128)])
def test_refused_rows(bad):
    lib = et.load_library()
    for fn in (lib.et_kv_append, lib.et_kv_read):
        assert rows_call(fn, **bad) == -1 and et.et_last_error()


@pytest.mark.parametrize("bad", [dict(q=None), dict(out=None), dict(q=FAKE + 8), dict(out=FAKE + 2), dict(qs=255), dict(qs=260), dict(qs=0),
                                 dict(heads=0), dict(heads=3), dict(heads=-2), dict(max_len=0), dict(max_len=-1), dict(window=-1),
                                 dict(scale=math.nan), dict(scale=math.inf)])
def test_refused_attention(bad):
    assert attend_call(**bad) == -1 and et.et_last_error()


def test_null_descriptors_and_empty_calls():
    lib, c, s = et.load_library(), cache(), seqs()
    for fn in (lib.et_kv_append, lib.et_kv_read):
        assert fn(None, C.byref(s), FAKE, 5, FAKE, 128, FAKE, 128, None) == -1
        assert fn(C.byref(c), None, FAKE, 5, FAKE, 128, FAKE, 128, None) == -1
        assert rows_call(fn, rows=0, k=None, v=None) == 0                       # nothing to do, nothing launched
        assert rows_call(fn, s=seqs(n_seqs=0, page_table_dev=None, kv_len_dev=None)) == 0
    assert lib.et_attention_paged(None, C.byref(s), FAKE, 256, 4, 64, 0, 0.1, FAKE, 1 << 40, FAKE, None) == -1
    assert lib.et_attention_paged(C.byref(c), None, FAKE, 256, 4, 64, 0, 0.1, FAKE, 1 << 40, FAKE, None) == -1
    assert attend_call(s=seqs(n_seqs=0, page_table_dev=None, kv_len_dev=None), q=None, out=None, ws=None, ws_bytes=0) == 0


def test_binding_refuses_host_tensors():
    with pytest.raises(TypeError):
        et.KVCache(2, 16, 2, 64, data=torch.zeros((2, et.et_kv_page_bytes(16, 2, 64, "bf16")), dtype=torch.uint8))
    with pytest.raises(ValueError):
        et.KVCache(2, 16, 2, 72)
    with pytest.raises(ValueError):
        et.KVCache(0, 16, 2, 64)
    with pytest.raises(ValueError):
        et.KVCache(2, 16, 2, 64, fmt="fp8")


def test_attention_workspace():
    """Short sequences need none; the rest as much as is asked for, whatever the bound, and less is refused."""
    lib = et.load_library()
    need = lambda c, s, heads, max_len, window: lib.et_attention_paged_workspace_bytes(C.byref(c), C.byref(s), heads, max_len, window)
    c, long = cache(), seqs(pages_per_seq=1 << 20, table_stride=1 << 20)
    assert need(c, long, 4, 512, 0) == need(c, seqs(), 4, 64, 0) == 0 and need(c, long, 4, 10 ** 6, 64) == 0
    b = need(c, long, 4, 10 ** 6, 0)
    assert 0 < b <= 64 << 20 and need(c, long, 4, 2 ** 31 - 1, 0) == b
    assert need(c, long, 3, 10 ** 6, 0) == 0 and need(c, long, 4, 0, 0) == 0 and need(cache(head_dim=72), long, 4, 10 ** 6, 0) == 0
    assert attend_call(s=long, max_len=10 ** 6, ws_bytes=b - 1) == -2 and "workspace" in et.et_last_error()
    assert attend_call(s=long, max_len=10 ** 6, ws_bytes=0) == -2
    assert attend_call(s=long, max_len=10 ** 6, ws=None) == -1
    assert attend_call(s=long, max_len=10 ** 6, ws=FAKE + 4) == -1


def test_attention_of_too_much_at_once():
    assert attend_call(s=seqs(n_seqs=1 << 23), heads=4) == -1 and "2^24" in et.et_last_error()
    assert attend_call(s=seqs(n_seqs=1 << 20, pages_per_seq=1 << 20, table_stride=1 << 20), max_len=10 ** 6) == -1
    assert "2^36" in et.et_last_error()


def test_attention_kernels_keep_to_their_registers(tmp_path):
    """Two workgroups of four wavefronts share a compute unit: at most 256 registers a lane, none of them in memory."""
    run = subprocess.run([HIPCC] + FLAGS + ["--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                                            os.path.join(CSRC, "paged_attention.hip"), "-o", str(tmp_path / "paged.o")],
                         check=True, capture_output=True, text=True)
    kernels = re.findall(r"Function Name: \S*?(paged_\w+?_kernel)\S*.*?TotalSGPRs.*? VGPRs: (\d+).*? AGPRs: (\d+).*?ScratchSize \[bytes/lane\]: (\d+)",
                         run.stderr, re.S)
    assert len(kernels) == 5 * 3 * (2 + 3)
    assert all(int(v) + int(a) <= 256 and scratch == "0" for _, v, a, scratch in kernels), kernels


class _Device:
    """Stands in for torch.cuda.device and torch.cuda.stream: notes what is current."""
    current, log = 0, []

    def __init__(self, to):
        self.to = to

    def __enter__(self):
        self.was, _Device.current = _Device.current, self.to
        _Device.log.append(self.to)

    def __exit__(self, *_):
        _Device.current = self.was


class _Lib:
    """Notes under which device each entry point is called, and with which stream (its last argument)."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, _Device.current, args[-1]))
            return 64 if name.endswith("bytes") else 0
        return call


@pytest.mark.parametrize("current", [0, None])
def test_calls_run_on_the_caches_device_and_its_stream(monkeypatch, current):
    """A cache on another device than the current one: allocation and launch happen with its device current, on that device's
    stream; a stream of a third device is refused.  (Tensors without memory stand for the other device, index None.)"""
    meta = torch.device("meta")
    c = object.__new__(et.KVCache)
    c.device, c.fmt, c.head_dim, c.n_kv_heads, c._width, c._scale, c._cache, c._lib = meta, "bf16", 64, 2, 128, 0.125, None, _Lib()
    monkeypatch.setattr(B, "_current_device", lambda: _Device.current)
    monkeypatch.setattr(torch.cuda, "device", lambda d: _Device(d.index))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: _Device(s.device.index))
    monkeypatch.setattr(B, "_raw_stream", lambda d: ("stream of", d))
    _Device.current, _Device.log = current, []
    x = torch.empty((3, 128), dtype=torch.bfloat16, device=meta)
    tab, lens = torch.empty((3, 2), dtype=torch.int32, device=meta), torch.empty(3, dtype=torch.int32, device=meta)

    class Stream:
        device, cuda_stream = meta, 5

    class Other:
        device, cuda_stream = torch.device("cpu"), 6

    for extra in ({}, {"stream": Stream()}):
        c._lib.calls.clear()
        _Device.log.clear()
        c.append(x, x, tab, lens, **extra)
        c.read(tab, lens, **extra)
        c.attend(x, tab, lens, 32, **extra)
        launches = [k for k in c._lib.calls if not k[0].endswith("bytes")]
        assert [k[0] for k in launches] == ["et_kv_append", "et_kv_read", "et_attention_paged"]
        assert all(k[1] is None and k[2] == ("stream of", None) for k in launches)
        assert _Device.current == current and len(_Device.log) == (3 if extra or current == 0 else 0)
    for call in (lambda: c.append(x, x, tab, lens, stream=Other()), lambda: c.read(tab, lens, stream=Other()),
                 lambda: c.attend(x, tab, lens, 32, stream=Other())):
        with pytest.raises(ValueError):
            call()
