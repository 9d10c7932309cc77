"""Refusals of the 8-bit paged cache's calls, from the host's checks, and its plain forms.  No GPU needed."""
import ctypes as C

import pytest
import torch

import paged8_util as p8
import paper_2510_11958_amd as pkg
from test_paged_host import APPEND, ATTENTION, P, cache, refused

E4M3 = dict(dtype=3, k_scale=P, v_scale=P, scale_stride=0)


@pytest.mark.parametrize("in_cache, word", [
    (dict(dtype=2), "dtype"), (dict(dtype=4), "dtype"), (dict(dtype=-1), "dtype"), (dict(k_scale=None), "k_scale"), (dict(v_scale=None), "v_scale"), (dict(k_scale=P + 8), "aligned"),
    (dict(v_scale=P + 1), "aligned"), (dict(scale_stride=16), "scale_stride"), (dict(scale_stride=40), "scale_stride"), (dict(scale_stride=-32), "scale_stride"),
    (dict(page_stride=2 * 16 * 64 + 8), "page_stride"), (dict(page_stride=2 * 16 * 64 - 16), "page_stride"), (dict(head_dim=96), "head_dim"), (dict(k=P + 8), "aligned"),
])
def test_a_bad_8_bit_cache_is_refused(in_cache, word):
    lib = pkg.load_library()
    c = cache()
    for k, v in dict(E4M3, **in_cache).items():
        setattr(c, k, v)
    refused(lib.dmtd_paged_append(C.byref(c), *APPEND.values(), None), word)
    refused(lib.dmtd_paged_attention(C.byref(c), *ATTENTION.values(), None), word)
    refused(lib.dmtd_paged_read(C.byref(c), *READ.values(), None), word)
    assert lib.dmtd_paged_workspace_bytes(C.byref(c)) == 0


READ = dict(slots=P, n=4, k_out=P, v_out=P, ldo=128)


@pytest.mark.parametrize("dtype", [0, 1, 3])
@pytest.mark.parametrize("args, word", [
    (dict(slots=None), "slots"), (dict(slots=P + 4), "slots"), (dict(n=-1), "n must"), (dict(n=1 << 30), "n must"), (dict(n=(1 << 26) + 1), "n must"), (dict(k_out=None), "k_out"), (dict(v_out=None), "v_out"),
    (dict(k_out=P + 8), "k_out"), (dict(v_out=P + 4), "v_out"), (dict(ldo=120), "ldo"), (dict(ldo=132), "ldo"), (dict(ldo=1 << 25), "ldo"),
])
def test_paged_read_refuses(dtype, args, word):
    c = cache(dtype=dtype)
    c.k_scale = c.v_scale = P
    refused(pkg.load_library().dmtd_paged_read(C.byref(c), *dict(READ, **args).values(), None), word)


def test_a_null_cache_is_refused():
    refused(pkg.load_library().dmtd_paged_read(None, *READ.values(), None), "null")


def test_a_context_of_8_bit_weights_is_refused():
    cfg = pkg.ModelConfig(2, 64, 4, 2, 64, 128, 100, max_seq_len=32).to_c(0)
    assert pkg.load_library().dmtd_workspace_bytes(C.byref(cfg)) > 0
    cfg.dtype = 3
    assert pkg.load_library().dmtd_workspace_bytes(C.byref(cfg)) == 0


def test_the_plain_form_of_the_codes():
    """Against torch's own conversion, at every code's border: halves between neighbours go to the even one, and rows of one value take the least power of two."""
    every = torch.arange(0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    x = torch.cat([every, (every[1:] + every[:-1]) / 2, (every[1:] + every[:-1]) / 2 * (1 + 2.0 ** -20), torch.tensor([448.0], dtype=torch.float64)])
    x = torch.cat([x, -x])[None]
    e = p8.scale_bytes(x)
    assert e.tolist() == [127]
    q, b = p8.codes(x, e)
    want = x.float().to(torch.float8_e4m3fn)
    assert torch.equal(q.float(), want.float()) and torch.equal(b, want.view(torch.uint8))
    rows = torch.tensor([[448.0], [448.0 * (1 + 2.0 ** -23)], [224.0], [224.1], [0.0], [1e-40], [3e38], [2.0 ** -111 * 448]], dtype=torch.float64)
    assert p8.scale_bytes(rows).tolist() == [127, 128, 126, 127, 16, 16, 247, 16]
    _, e, v = p8.stored(torch.randn(50, 128, dtype=torch.float64, generator=torch.Generator().manual_seed(0)))
    assert torch.equal(v, v.bfloat16().double())                      # bf16 holds what is stored
