"""The paged cache without a GPU: the header, the library's and the binding's refusals, the oracle against torch's own conversions."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2502_14477_amd as esa
from oracle import paged_oracle as orc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, ODD = 4096, 4104            # never dereferenced: every call below fails validation, or has nothing to do


def test_header_is_plain_c_and_its_symbols_are_exported():
    path = os.path.join(ROOT, "include", "esa_paged.h")
    for lang, std in (("c", "-std=c99"), ("c++", "-std=c++11")):
        r = subprocess.run(["gcc", "-x", lang, std, "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only", path], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
    names = sorted(set(re.findall(r"ESA_API\s+[\w\s\*]+?\b(esa_\w+)\s*\(", open(path).read())))
    assert names == sorted(esa.PAGED_EXPORTS)
    raw = ctypes.CDLL(esa.lib_path())
    for n in names:
        assert hasattr(raw, n), n


def test_the_structures_are_laid_out_as_in_c(tmp_path):
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    names = {"esa_paged_cache": [f[0] for f in esa.PagedCache._fields_], "esa_paged_batch": [f[0] for f in esa.PagedBatch._fields_]}
    lines = "".join('printf("%%zu ", sizeof(%s));' % t + "".join('printf("%%zu ", offsetof(%s, %s));' % (t, f) for f in fields) for t, fields in names.items())
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "esa_paged.h"\nint main(void) { %s return 0; }' % lines)
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for t in (esa.PagedCache, esa.PagedBatch):
        want += [ctypes.sizeof(t)] + [getattr(t, f[0]).offset for f in t._fields_]
    assert got == want


def batch(**kw):
    d = dict(cu=FAKE, start=FAKE, pages=FAKE, pages_ld=8, n_tok=4, n_seq=2, max_pages=8)
    return esa.PagedBatch(**{**d, **kw})


def cache(**kw):
    d = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, page_stride=2 * 64 * 128, head_stride=64 * 128, tok_stride=128, n_pages=16, page_size=64,
             h_kv=2, d=128, dtype=esa.ESA_E4M3)
    return esa.PagedCache(**{**d, **kw})


def append(b=None, c=None, k=FAKE, ldk=256, v=FAKE, ldv=256, q=FAKE, ldq=512, h=4, out_q=FAKE, ldoq=512, base=5e5, dtype=1):
    return esa.lib.esa_append_paged(k, ldk, v, ldv, q, ldq, h, out_q, ldoq, ctypes.byref(b or batch()), ctypes.byref(c or cache()), base, dtype, None)


def attend(b=None, c=None, q=FAKE, ldq=512, h=4, l_i=1 << 40, l_l=0, idx=None, n_sel=0, idx_ld=0, scale=0.1, cap=0.0, out=2 * FAKE, ldo=512, lse=None,
           dtype=1, ws=FAKE, ws_bytes=1 << 40):
    return esa.lib.esa_attend_paged(q, ldq, h, ctypes.byref(b or batch()), ctypes.byref(c or cache()), l_i, l_l, idx, n_sel, idx_ld, scale, cap, out, ldo,
                                    lse, dtype, ws, ws_bytes, None)


COMMON = [
    ("dtype", dict(dtype=7), -2), ("cache of another type", dict(c=cache(dtype=0)), -2), ("unknown cache type", dict(c=cache(dtype=9)), -2),
    ("head size", dict(c=cache(d=48)), -2), ("head size 0", dict(c=cache(d=0)), -2), ("page size", dict(c=cache(page_size=48)), -2),
    ("page size 256", dict(c=cache(page_size=256)), -2), ("no pages", dict(c=cache(n_pages=0)), -1), ("no heads", dict(c=cache(h_kv=0)), -1),
    ("negative tokens", dict(b=batch(n_tok=-1)), -1), ("negative sequences", dict(b=batch(n_seq=-1)), -1), ("no table", dict(b=batch(max_pages=0)), -1),
    ("overlapping table", dict(b=batch(pages_ld=7)), -1), ("heads no multiple", dict(h=3), -1), ("no heads of queries", dict(h=0), -1),
    ("too many positions", dict(b=batch(max_pages=1 << 25, pages_ld=1 << 25)), -1), ("too many tokens", dict(b=batch(n_tok=1 << 30)), -1),
    ("null cu", dict(b=batch(cu=None)), -1), ("null start", dict(b=batch(start=None)), -1), ("null pages", dict(b=batch(pages=None)), -1),
    ("odd cu", dict(b=batch(cu=FAKE + 2)), -1), ("null cache", dict(c=cache(k=None)), -1), ("odd cache", dict(c=cache(v=ODD)), -1),
    ("no scales", dict(c=cache(k_scale=None)), -1), ("no value scales", dict(c=cache(v_scale=None)), -1),
    ("stride of no whole 16 bytes", dict(c=cache(tok_stride=136, head_stride=64 * 136, page_stride=128 * 136)), -1),
    ("tokens overlap", dict(c=cache(tok_stride=64)), -1), ("heads overlap", dict(c=cache(head_stride=128)), -1),
    ("pages overlap", dict(c=cache(page_stride=64 * 128)), -1), ("nowhere for queries", dict(out=None), -1),
    ("odd queries", dict(q=ODD), -1), ("queries' rows overlap", dict(ldq=256), -1), ("odd row stride", dict(ldq=516), -1),
]


@pytest.mark.parametrize("name,change,code", COMMON, ids=[c[0] for c in COMMON])
def test_both_calls_refuse(name, change, code):
    as_append = dict(change)
    if "out" in as_append:
        as_append["out_q"] = as_append.pop("out")
    assert append(**as_append) == code
    assert attend(**change) == code
    assert b"esa_attend_paged" in esa.lib.esa_last_error()


def test_append_refuses():
    for change in (dict(k=None), dict(v=None), dict(k=ODD), dict(ldk=128), dict(ldv=252), dict(base=-1.0), dict(base=float("nan")), dict(base=0.0),
                   dict(ldoq=520), dict(ldoq=1024, ldq=512)):
        assert append(**change) == -1, change
        assert b"esa_append_paged" in esa.lib.esa_last_error()


def test_both_refuse_more_rows_than_they_count():
    assert append(b=batch(n_tok=1 << 26)) == -1 and attend(b=batch(n_tok=1 << 26)) == -1
    assert b"2^28" in esa.lib.esa_last_error()


def test_append_refuses_keys_and_values_in_one_place():
    there = dict(v=2 * FAKE, v_scale=2 * FAKE)
    for c in (cache(**{**there, "v": FAKE}), cache(**{**there, "v_scale": FAKE})):
        assert append(c=c) == -1
        assert b"one place" in esa.lib.esa_last_error()


def test_attend_refuses():
    for change in (dict(scale=0.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")),
                   dict(l_i=-1), dict(l_l=-1), dict(n_sel=-1), dict(n_sel=4, idx=None, idx_ld=4), dict(n_sel=4, idx=FAKE + 2, idx_ld=4),
                   dict(n_sel=4, idx=FAKE, idx_ld=3), dict(out=FAKE), dict(lse=FAKE + 2), dict(ldo=500)):
        assert attend(**change) == -1, change
    for change in (dict(ws=None), dict(ws=ODD), dict(ws_bytes=0)):
        assert attend(**change) == -3, change


def test_attend_refuses_caps_that_its_arithmetic_cannot_hold():
    for change in (dict(cap=4097.0), dict(cap=1e-38, scale=1.0), dict(scale=2e38)):
        assert attend(**change) == -1, change


def test_nothing_to_do():
    for b in (batch(n_tok=0, cu=None, start=None, pages=None), batch(n_seq=0, cu=None, start=None, pages=None)):
        assert append(b=b, k=None, v=None, q=None, out_q=None) == 0
        assert attend(b=b, q=None, out=None, ws=None, ws_bytes=0) == 0


def tensors(**kw):
    t = dict(k=torch.zeros(5, 2, 64, dtype=torch.bfloat16), v=torch.zeros(5, 2, 64, dtype=torch.bfloat16), q=torch.zeros(5, 4, 64, dtype=torch.bfloat16),
             cu=torch.tensor([0, 2, 5], dtype=torch.int32), start=torch.zeros(2, dtype=torch.int32), pages=torch.zeros(2, 3, dtype=torch.int32),
             k_cache=torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16), v_cache=torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16), k_scale=None, v_scale=None, idx=None)
    t.update(kw)
    return t


def f8(*shape):
    return torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e4m3fn)


BAD = [
    ("64-bit offsets", dict(cu=torch.tensor([0, 2, 5]))), ("offsets of other sequences", dict(cu=torch.tensor([0, 5], dtype=torch.int32))),
    ("table of other sequences", dict(pages=torch.zeros(3, 3, dtype=torch.int32))), ("table of one dimension", dict(pages=torch.zeros(2, dtype=torch.int32))),
    ("strided offsets", dict(cu=torch.zeros(6, dtype=torch.int32)[::2])), ("transposed table", dict(pages=torch.zeros(3, 2, dtype=torch.int32).t())),
    ("value cache of another shape", dict(v_cache=torch.zeros(6, 2, 32, 64, dtype=torch.bfloat16))),
    ("value cache in another order", dict(v_cache=torch.zeros(6, 16, 2, 64, dtype=torch.bfloat16).transpose(1, 2))),
    ("value cache of another type", dict(v_cache=torch.zeros(6, 2, 16, 64))), ("caches of another type", dict(k_cache=torch.zeros(6, 2, 16, 64), v_cache=torch.zeros(6, 2, 16, 64))),
    ("caches of another head size", dict(k_cache=torch.zeros(6, 2, 16, 32, dtype=torch.bfloat16), v_cache=torch.zeros(6, 2, 16, 32, dtype=torch.bfloat16))),
    ("8 bits without scales", dict(k_cache=f8(6, 2, 16, 64), v_cache=f8(6, 2, 16, 64))),
    ("scales beside the storage type", dict(k_scale=torch.zeros(6, 2, dtype=torch.uint8), v_scale=torch.zeros(6, 2, dtype=torch.uint8))),
    ("scales of another pool", dict(k_cache=f8(6, 2, 16, 64), v_cache=f8(6, 2, 16, 64), k_scale=torch.zeros(5, 2, dtype=torch.uint8), v_scale=torch.zeros(5, 2, dtype=torch.uint8))),
    ("scales of another type", dict(k_cache=f8(6, 2, 16, 64), v_cache=f8(6, 2, 16, 64), k_scale=torch.zeros(6, 2), v_scale=torch.zeros(6, 2))),
    ("queries whose heads lie apart", dict(q=torch.zeros(5, 8, 64, dtype=torch.bfloat16)[:, ::2])), ("queries of two dimensions", dict(q=torch.zeros(5, 256, dtype=torch.bfloat16))),
]


@pytest.mark.parametrize("name,change", BAD, ids=[b[0] for b in BAD])
def test_binding_refuses_what_does_not_fit(name, change):
    t = tensors(**change)
    common = (t["cu"], t["start"], t["pages"], t["k_cache"], t["v_cache"], t["k_scale"], t["v_scale"])
    for call in (lambda: esa.esa_append_paged(t["k"], t["v"], *common, q=t["q"], rope_base=5e5), lambda: esa.esa_attend_paged(t["q"], *common)):
        with pytest.raises(AssertionError, match=r"cu|n\[|k\.|ks|f8|s\[|size|scalar_type"):
            call()


def test_binding_refuses_host_memory_and_unknown_types():
    t = tensors()
    common = (t["cu"], t["start"], t["pages"], t["k_cache"], t["v_cache"])
    with pytest.raises(AssertionError, match="GPU"):
        esa.esa_append_paged(t["k"], t["v"], *common)
    with pytest.raises(AssertionError, match="GPU"):
        esa.esa_attend_paged(t["q"], *common)
    with pytest.raises(esa.EsaError):
        esa.esa_attend_paged(t["q"].half(), *common)
    with pytest.raises(esa.EsaError):
        esa.esa_append_paged(t["k"].half(), t["v"].half(), *common)
    with pytest.raises(esa.EsaError):
        esa.esa_append_paged(t["k"], t["v"], *common, rope_base=-1.0)
    for bad in (dict(v=t["v"][:4]), dict(v=t["v"].float()), dict(k=torch.zeros(5, 1, 64, dtype=torch.bfloat16)), dict(q=t["q"][:4]), dict(q=t["q"].float())):
        with pytest.raises(AssertionError):
            esa.esa_append_paged(bad.get("k", t["k"]), bad.get("v", t["v"]), *common, q=bad.get("q"), rope_base=5e5)
    for bad in (torch.zeros(2, 4, dtype=torch.int64), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)):
        with pytest.raises(AssertionError):
            esa.esa_attend_paged(t["q"], *common, l_i=4, l_l=4, idx=bad)
    with pytest.raises(AssertionError):
        esa.esa_attend_paged(t["q"], *common, out=torch.zeros(5, 4, 64))


def test_oracle_rounds_to_e4m3_as_torch_does():
    x = torch.cat((torch.linspace(-460, 460, 20001), torch.linspace(-0.05, 0.05, 20001), torch.tensor(orc.e4m3_table()[:127]).float()))
    x = torch.cat((x, (x[1:] + x[:-1]) / 2)).clamp(-448, 448)
    assert np.array_equal(orc.to_e4m3(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())
    assert np.array_equal(orc.e4m3_table()[:127], torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())


def test_oracle_scale_covers_and_is_smallest():
    for amax in (0.0, 1e-45, 2.0 ** -91, 1.0, 1.75, 1.7500001, 448.0, 448.1, 3e38):
        byte = orc.scale_byte(amax)
        assert byte in (27, 239) or amax <= 448 * 2.0 ** (byte - 127) and amax > 448 * 2.0 ** (byte - 128)
