"""The cache in 4 bits without a GPU: the oracle's format, page sizes, launches' limits, and what is refused."""
import ctypes as C
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
from tests.test_kv_cache import BAD_SEQS, FAKE, attend_call, cache, rows_call, seqs


def test_oracle_codes_are_the_nearest_and_ties_are_even():
    """Against a search of all codes and exponents, one value at a time."""
    rng = np.random.default_rng(2)
    x = rng.integers(-64, 65, (40, 48)) / 8.0 * 2.0 ** rng.integers(-20, 20, (40, 1))
    x[3], x[4, :32], x[5, 40], x[6, 7] = 0.0, 0.0, np.inf, np.nan
    codes, exps = O.mx_hold(x)
    stand = O.mx_stands_for(codes, exps)
    assert codes.shape == (40, 24) and exps.shape == (40, 2)
    for r in range(40):
        for i, block in enumerate((slice(0, 32), slice(32, 48))):
            b, e = x[r, block], int(exps[r, i]) - 127
            if not np.isfinite(b).all():
                assert e == 128 and np.isnan(stand[r, block]).all()
                continue
            m = np.abs(b).max()
            assert m <= 7 * 2.0 ** e and (m > 7 * 2.0 ** (e - 1) or e == -125)
            for v, s in zip(b, stand[r, block]):
                far = np.abs(np.abs(v) / 2.0 ** e - O.MX_GRID)
                best = np.flatnonzero(far == far.min())
                want = best[best % 2 == 0][0] if len(best) > 1 else best[0]
                assert s == np.sign(v) * O.MX_GRID[want] * 2.0 ** e, (v, s, e)
    assert O.mx_hold(np.array([-0.0] * 32))[0].tolist() == [0x88] * 16


def test_oracle_exponents_at_their_limits():
    for top, e in ((7.0, 0), (7.03125, 1), (3.5, -1), (3.515625, 0), (2.0 ** -133, -125), (1.75 * 2.0 ** -123, -125), (1.7578125 * 2.0 ** -123, -124),
                   (3.3895313892515355e38, 125), (0.0, -125)):
        codes, exps = O.mx_hold(np.array([top] + [0.0] * 31))
        assert int(exps[0]) - 127 == e, (top, exps)
    assert O.mx_stands_for(*O.mx_hold(np.array([3.3895313892515355e38] * 32)))[0] == 6 * 2.0 ** 125


def test_page_bytes():
    for page, kv, d, row in ((64, 4, 128, 68), (16, 3, 80, 43), (32, 1, 64, 34), (256, 8, 256, 136), (16, 2, 96, 51)):
        assert et.et_kv_page_bytes(page, kv, d, "mxfp4") == 2 * page * kv * row and et.et_kv_page_bytes(page, kv, d, "mxfp4") % 16 == 0
    for bad in ((0, 4, 128), (8, 4, 128), (512, 4, 128), (64, 0, 128), (64, 1025, 128), (64, 4, 72)):
        assert et.et_kv_page_bytes(*bad, "mxfp4") == 0
    assert et.load_library().et_kv_page_bytes(64, 4, 128, 5) == 0


@pytest.mark.parametrize("bad,code", [(dict(data_dev=None), -1), (dict(data_dev=FAKE + 8), -1), (dict(n_pages=0), -1), (dict(page_size=24), -5),
                                      (dict(n_kv_heads=0), -1), (dict(head_dim=72), -5), (dict(format=5), -1), (dict(format=3), -1)])
def test_refused_caches(bad, code):
    lib, c = et.load_library(), cache(**dict(dict(format=B.ET_KV_MXFP4), **bad))
    assert rows_call(lib.et_kv_append, c=c) == code and et.et_last_error()
    assert rows_call(lib.et_kv_read, c=c) == code and attend_call(c=c) == code


@pytest.mark.parametrize("bad,code", BAD_SEQS)
def test_refused_sequences(bad, code):
    lib, c = et.load_library(), cache(format=B.ET_KV_MXFP4)
    assert rows_call(lib.et_kv_append, c=c, s=seqs(**bad)) == code and rows_call(lib.et_kv_read, c=c, s=seqs(**bad)) == code
    assert attend_call(c=c, s=seqs(**bad)) == code


def test_workspace_and_empty_calls():
    lib, c, long = et.load_library(), cache(format=B.ET_KV_MXFP4), seqs(pages_per_seq=1 << 20, table_stride=1 << 20)
    need = lambda max_len: lib.et_attention_paged_workspace_bytes(C.byref(c), C.byref(long), 4, max_len, 0)
    assert need(512) == 0 and 0 < need(10 ** 6) <= 64 << 20
    assert attend_call(c=c, s=long, max_len=10 ** 6, ws_bytes=need(10 ** 6) - 1) == -2 and attend_call(c=c, s=long, max_len=10 ** 6, ws=None) == -1
    none = seqs(n_seqs=0, page_table_dev=None, kv_len_dev=None)
    assert attend_call(c=c, s=none, q=None, out=None, ws=None, ws_bytes=0) == 0
    assert rows_call(lib.et_kv_append, c=c, s=none) == 0 and rows_call(lib.et_kv_read, c=c, rows=0, k=None, v=None) == 0


def test_attention_kernels_keep_to_their_registers(tmp_path):
    """Two workgroups of four wavefronts share a compute unit: at most 256 registers a lane, none of them in memory."""
    run = subprocess.run([HIPCC] + FLAGS + ["--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                                            os.path.join(CSRC, "paged_attention_mxfp4.hip"), "-o", str(tmp_path / "paged.o")],
                         check=True, capture_output=True, text=True)
    kernels = re.findall(r"Function Name: \S*?(paged_\w+?_kernel)\S*.*?TotalSGPRs.*? VGPRs: (\d+).*? AGPRs: (\d+).*?ScratchSize \[bytes/lane\]: (\d+)",
                         run.stderr, re.S)
    assert len(kernels) >= 5
    assert all(int(v) + int(a) <= 256 and scratch == "0" for _, v, a, scratch in kernels), kernels
