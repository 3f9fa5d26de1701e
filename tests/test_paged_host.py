"""What the calls on a paged cache refuse, checked on the host: nothing is launched, so no GPU is needed."""
import ctypes
import os
import re
import subprocess
import sys

import pytest
import torch

import __graft_entry__
from paper_2608_27514_b200 import binding as B

P = 4096  # an address that is never read


@pytest.fixture(scope="module")
def lib():
    __graft_entry__.build()
    return B.lib()


def cache(**kw):
    c = B.tsd_paged_cache()
    f = dict(k_pages=P, v_pages=P, page_stride=(64 * 4 * 128, 4 * 128, 128), k_scale=None, v_scale=None, page_table=P, table_stride=20, batch=2,
             n_pages=40, page_size=64, max_pages=20, n_kv_heads=4, head_dim=128, dtype=B.TSD_BF16)
    f.update(kw)
    for name, v in f.items():
        if name == "page_stride":
            c.page_stride[:] = v
        else:
            setattr(c, name, v)
    return c


BAD_CACHES = [(dict(k_pages=None), B.TSD_ERR_INVALID_ARG), (dict(page_table=None), B.TSD_ERR_INVALID_ARG), (dict(v_pages=P + 8), B.TSD_ERR_INVALID_ARG),
              (dict(batch=0), B.TSD_ERR_INVALID_ARG), (dict(n_pages=0), B.TSD_ERR_INVALID_ARG), (dict(max_pages=0), B.TSD_ERR_INVALID_ARG),
              (dict(page_size=0), B.TSD_ERR_INVALID_ARG), (dict(page_size=48), B.TSD_ERR_UNSUPPORTED), (dict(page_size=4), B.TSD_ERR_UNSUPPORTED),
              (dict(page_size=2048), B.TSD_ERR_UNSUPPORTED), (dict(max_pages=1 << 25, table_stride=1 << 25), B.TSD_ERR_INVALID_ARG),
              (dict(table_stride=19), B.TSD_ERR_INVALID_ARG), (dict(head_dim=96), B.TSD_ERR_UNSUPPORTED), (dict(dtype=3), B.TSD_ERR_UNSUPPORTED),
              (dict(k_scale=P), B.TSD_ERR_INVALID_ARG), (dict(page_stride=(32768, 512, 64)), B.TSD_ERR_INVALID_ARG),
              (dict(page_stride=(32768, 516, 128)), B.TSD_ERR_INVALID_ARG), (dict(page_stride=(-32768, 512, 128)), B.TSD_ERR_INVALID_ARG)]


def token(lib, c, **kw):
    f = dict(Hq=28, dtype=B.TSD_BF16, q=P, qb=28 * 128, qh=128, lens=None, out=P, ob=28 * 128, oh=128, lse=None, scale=0.1, ws=P, ws_bytes=1 << 24)
    f.update(kw)
    return lib.tsd_paged_attention(ctypes.byref(c), f["Hq"], f["dtype"], f["q"], f["qb"], f["qh"], f["lens"], f["out"], f["ob"], f["oh"], f["lse"],
                                   f["scale"], f["ws"], f["ws_bytes"], None, None)


def test_bad_caches_are_refused_everywhere(lib):
    layout = B.make_layout(2, 4, 32, 1280, 28, 4, 128, B.TSD_BF16)
    for kw, code in BAD_CACHES:
        c = cache(**kw)
        assert token(lib, c) == code, kw
        assert lib.tsd_paged_attention_workspace_bytes(ctypes.byref(c), 28) == 0
        assert lib.tsd_verify_attention_paged_workspace_bytes(ctypes.byref(layout), ctypes.byref(c), 0) == 0
        assert append(lib, cache=c) == code, kw
        assert verify(lib, layout, c) in (B.TSD_ERR_INVALID_ARG, B.TSD_ERR_UNSUPPORTED), kw
    # a pool of one page, or one head, has no use for that stride
    one = cache(n_pages=1, n_kv_heads=1, page_stride=(0, 128, 0))
    assert lib.tsd_paged_attention_workspace_bytes(ctypes.byref(one), 7) > 0


def test_token_refusals(lib):
    c = cache()
    need = lib.tsd_paged_attention_workspace_bytes(ctypes.byref(c), 28)
    assert need > 0 and lib.tsd_paged_attention_workspace_bytes(ctypes.byref(c), 30) == 0
    assert lib.tsd_paged_attention_workspace_bytes(None, 28) == 0
    for kw, code in [(dict(Hq=30), B.TSD_ERR_INVALID_ARG), (dict(Hq=0), B.TSD_ERR_INVALID_ARG), (dict(q=None), B.TSD_ERR_INVALID_ARG),
                     (dict(out=None), B.TSD_ERR_INVALID_ARG), (dict(scale=float("nan")), B.TSD_ERR_INVALID_ARG), (dict(dtype=2), B.TSD_ERR_UNSUPPORTED),
                     (dict(dtype=B.TSD_F32), B.TSD_ERR_UNSUPPORTED), (dict(q=P + 4), B.TSD_ERR_INVALID_ARG), (dict(out=P + 4), B.TSD_ERR_INVALID_ARG),
                     (dict(qh=64), B.TSD_ERR_INVALID_ARG), (dict(qb=28 * 128 + 4), B.TSD_ERR_INVALID_ARG), (dict(ob=-8), B.TSD_ERR_INVALID_ARG),
                     (dict(ws=None), B.TSD_ERR_INVALID_ARG), (dict(ws=P + 4), B.TSD_ERR_INVALID_ARG), (dict(ws_bytes=need - 1), B.TSD_ERR_WORKSPACE)]:
        assert token(lib, c, **kw) == code, kw
    assert token(lib, cache(dtype=B.TSD_F32)) == B.TSD_ERR_UNSUPPORTED              # bf16 queries over an fp32 cache


class append_args(ctypes.Structure):
    _fields_ = [("cache", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in ("batch", "n_blocks", "n_rows", "n_q_heads", "n_kv_heads", "head_dim", "dtype")] \
        + [(n, ctypes.c_void_p) for n in ("block", "n_new", "first_slot", "positions", "inv_freq")] \
        + [(n, ctypes.c_int32) for n in ("rotary_dim", "interleaved")] + [(n, ctypes.c_void_p) for n in ("k", "v", "q")] \
        + [(n, ctypes.c_int64 * 3) for n in ("kv_stride", "q_stride")] + [(n, ctypes.c_void_p) for n in ("k_out", "q_out")] \
        + [(n, ctypes.c_int64 * 3) for n in ("k_out_stride", "q_out_stride")] + [("status", ctypes.c_void_p)]


def append(lib, **kw):
    a = append_args()
    f = dict(cache=cache(), batch=2, n_blocks=3, n_rows=32, n_q_heads=28, n_kv_heads=4, head_dim=128, dtype=B.TSD_BF16, inv_freq=P, rotary_dim=128, k=P,
             v=P, q=P, q_out=P, kv_stride=(96 * 512, 512, 128), q_stride=(96 * 3584, 3584, 128), q_out_stride=(96 * 3584, 3584, 128),
             k_out_stride=(96 * 512, 512, 128))
    f.update(kw)
    keep = f["cache"]
    for name, v in f.items():
        if name == "cache":
            a.cache = None if v is None else ctypes.addressof(v)
        elif name.endswith("stride"):
            getattr(a, name)[:] = v
        else:
            setattr(a, name, v)
    rc = lib.tsd_append_paged_kv(ctypes.byref(a), None)
    del keep
    return rc


def test_append_refusals(lib):
    assert lib.tsd_append_paged_kv(None, None) == B.TSD_ERR_INVALID_ARG
    bad, no = B.TSD_ERR_INVALID_ARG, B.TSD_ERR_UNSUPPORTED
    for kw, code in [(dict(batch=-1), bad), (dict(batch=1), bad), (dict(n_blocks=0), bad), (dict(n_rows=-1), bad), (dict(n_kv_heads=2), bad),
                     (dict(head_dim=64), bad), (dict(head_dim=96), no), (dict(dtype=2), no), (dict(dtype=B.TSD_F32), no), (dict(rotary_dim=-16), bad),
                     (dict(rotary_dim=144), bad), (dict(rotary_dim=24), no), (dict(inv_freq=None), bad), (dict(k=None), bad), (dict(v=None), bad),
                     (dict(q=None), bad), (dict(q_out=None), bad), (dict(n_q_heads=0), bad), (dict(k=P + 2), bad), (dict(q_out=P + 4), bad),
                     (dict(k_out=P + 8), bad), (dict(kv_stride=(96 * 512, 512, 64)), bad), (dict(kv_stride=(96 * 512, 516, 128)), bad),
                     (dict(q_stride=(-8, 3584, 128)), bad), (dict(k_out=P, k_out_stride=(96 * 512, 512, 4)), bad),
                     (dict(batch=70000, cache=cache(batch=70000), n_rows=40000, n_blocks=1), no)]:
        assert append(lib, **kw) == code, kw
    for kw in (dict(n_rows=0), dict(batch=0, cache=None)):                              # nothing to do, nothing launched
        assert append(lib, **kw) == B.TSD_OK, kw


def verify(lib, layout, c, **kw):
    N = layout.n_branches * layout.rows_per_branch
    f = dict(mask=P, q=P, scale=0.1, ws=None, ws_bytes=0, flags=0, qs=(N * 3584, 3584, 128), ds=(N * 512, 512, 128), k=P, out=P)
    f.update(kw)
    return lib.tsd_verify_attention_paged(ctypes.byref(layout), f["mask"], f["q"], *f["qs"], ctypes.byref(c), f["k"], P, *f["ds"], f["out"], *f["qs"],
                                          None, f["scale"], f["ws"], f["ws_bytes"], f["flags"], None, None)


def test_verify_refusals(lib):
    layout = B.make_layout(2, 4, 32, 1280, 28, 4, 128, B.TSD_BF16)
    bad, no = B.TSD_ERR_INVALID_ARG, B.TSD_ERR_UNSUPPORTED
    need = lambda c, l=layout, flags=0: lib.tsd_verify_attention_paged_workspace_bytes(ctypes.byref(l), ctypes.byref(c), flags)
    assert need(cache()) == 0
    for c, flags in ((cache(), B.TSD_ATTN_FORCE_SIMT), (cache(dtype=B.TSD_E4M3, k_scale=P, v_scale=P), 0)):
        n = need(c, flags=flags)
        assert n == 2 * 2 * 1280 * 4 * 128 * 2
        assert verify(lib, layout, c, flags=flags) == bad                                # no workspace
        assert verify(lib, layout, c, flags=flags, ws=P, ws_bytes=n - 1) == B.TSD_ERR_WORKSPACE
        assert verify(lib, layout, c, flags=flags, ws=P + 4, ws_bytes=n) == bad
        assert verify(lib, layout, c, flags=flags, ws=P, ws_bytes=n, mask=None) == bad
    for l in (B.make_layout(1, 4, 32, 1280, 28, 4, 128, 1), B.make_layout(2, 4, 32, 1281, 28, 4, 128, 1), B.make_layout(2, 4, 32, 1280, 28, 2, 128, 1),
              B.make_layout(2, 4, 32, 1280, 28, 4, 64, 1)):
        assert verify(lib, l, cache()) == bad
    assert verify(lib, B.make_layout(2, 4, 32, 1280, 28, 4, 128, 0), cache()) == no      # an fp32 pass over bf16 pages
    assert verify(lib, layout, cache(dtype=B.TSD_F32)) == no
    for kw in (dict(mask=None), dict(q=None), dict(out=None), dict(k=None), dict(q=P + 4), dict(scale=float("nan")), dict(qs=(1, 3584, 128)),
               dict(ds=(128 * 512, 512, 64))):
        assert verify(lib, layout, cache(), **kw) == bad, kw


def test_descriptions_of_host_tensors_are_refused(lib):
    pages = torch.zeros((4, 8, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.make_paged_cache(pages, pages, torch.zeros((1, 4), dtype=torch.int32))


def test_results_that_would_meet_and_sizes_at_the_limit(lib):
    # a stride of 0 is for what is read only; the largest cache leaves the kernels room to count behind its last token
    bad = B.TSD_ERR_INVALID_ARG
    assert token(lib, cache(), ob=0) == bad and token(lib, cache(), ob=64) == bad
    for kw in (dict(q_out_stride=(0, 3584, 128)), dict(q_out_stride=(96 * 3584, 0, 128)), dict(k_out=P, k_out_stride=(96 * 512, 0, 128))):
        assert append(lib, **kw) == bad, kw
    need = lambda **kw: lib.tsd_paged_attention_workspace_bytes(ctypes.byref(cache(**kw)), 28)
    assert need(page_size=1024, max_pages=(1 << 21) - 4, table_stride=1 << 21) > 0
    assert need(page_size=1024, max_pages=(1 << 21) - 3, table_stride=1 << 21) == 0
    assert need(page_size=8, max_pages=(1 << 28) - 512, table_stride=1 << 28) > 0
    assert need(page_size=8, max_pages=(1 << 28) - 511, table_stride=1 << 28) == 0


def test_what_a_block_hands_on_is_read_behind_a_barrier():
    # A warp without chunks comes to the joining functions at once: in front of their first block barrier they may look at nothing that
    # another warp writes to shared memory.  Read in the source, since on a GPU the window is too narrow to be met.
    csrc = os.path.join(os.path.dirname(os.path.abspath(B.__file__)), "csrc", "tsd_paged_attention.cu")
    with open(csrc) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    for name in ("join_cluster", "join_parts"):
        body = code.split("void %s(" % name, 1)[1].split("\n}\n", 1)[0].split("{", 1)[1]
        before, barrier, _ = body.partition("__syncthreads();")
        assert barrier and not re.search(r"\bsh\.", before), name


@pytest.mark.parametrize("table", ["none", "of another version"])
def test_a_torch_without_an_exchange_table_has_the_other_calls(lib, table):
    # only the calls on a paged cache read tensors through that table; in a process of its own, since the module keeps what it was given
    code = """
import ctypes, sys, torch
from paper_2608_27514_b200 import binding as B
B.lib()
from paper_2608_27514_b200 import _tsd_native as N
other = (ctypes.c_uint32 * 32)(2, 0)  # a header of version 2
new = ctypes.pythonapi.PyCapsule_New
new.restype, new.argtypes = ctypes.py_object, [ctypes.c_void_p, ctypes.c_char_p, ctypes.c_void_p]
table = None if sys.argv[1] == "none" else new(ctypes.addressof(other), b"dlpack_exchange_api", None)
N.setup(lambda: 0, lambda device: 0, torch.float32, torch.bfloat16, B.TsdError, torch.Tensor, table)
B._native = N
try:
    B.tsd_build_branch_mask(B.make_layout(0, 1, 32, 0, 1, 1, 128, B.TSD_BF16), None, None, torch.zeros(64, dtype=torch.uint8))
    raise SystemExit("an empty layout was taken")
except B.TsdError as e:
    assert e.code == B.TSD_ERR_INVALID_ARG, e
x = torch.zeros((1, 1, 1, 64))
for call in (lambda: B.tsd_append_paged_kv(None, x, None), lambda: B.tsd_paged_attention(None, x, None, x),
             lambda: B.tsd_verify_attention_paged(None, None, x, None, x, x, x)):
    try:
        call()
        raise SystemExit("a call on a paged cache was made without the table")
    except RuntimeError as e:
        assert "exchange table" in str(e), e
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(B.__file__)))
    done = subprocess.run([sys.executable, "-c", code, table], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
