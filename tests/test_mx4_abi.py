"""CPU-side checks of normalised heads and the 4-bit cache: host-checkable argument errors and sizes.  No compute call is made here."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2506_07311_amd as pa
from paper_2506_07311_amd import binding
from tests import mx4_reference as ref

INVALID, UNSUPPORTED, SMALL = 1, 2, 3
i32, i64, f32, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
P, NULL = ctypes.c_void_p(0x4000), ctypes.c_void_p(0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2506_07311_amd import build
        build.build()
    return binding.load_library()


def desc(**kw):
    d = dict(records=0x1000, page_stride=8 * 2176, head_stride=2176, num_pages=4, page_size=16, num_kv_heads=8, head_dim=128)
    d.update(kw)
    return binding._Mx4Desc(**d)


def plain(**kw):
    d = dict(k_cache=0x1000, v_cache=0x2000, page_stride=16 * 8 * 128, token_stride=8 * 128, head_stride=128, num_pages=4, page_size=16,
             num_kv_heads=8, head_dim=128, dtype=1)
    d.update(kw)
    return binding._Desc(**d)


def tokens(**kw):
    t = dict(q=0x4000, q_out=0x4000, k_new=0x4000, v_new=0x4000, rope_positions=0x4000, inv_freq=0x4000, q_weight=0x4000, k_weight=0x4000,
             seq_ids=0x4000, positions=0x4000, block_table=0x4000, num_q_heads=32, T=3, batch=2, max_blocks=4, axes=1, rotary_dim=128, norm_q=1,
             norm_k=1, weight_dtype=1, eps=1e-6, mscale=1.0)
    t.update(kw)
    return binding._NormRope(**t)


def call(fn, args, **change):
    assert set(change) <= set(args), change
    args = dict(args, **change)
    return fn(*(ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args.values()))


def test_record_sizes(lib):
    assert pa.pa_mx4_record_bytes(16, 128) == 2176 and pa.pa_mx4_record_bytes(64, 64) == 4352 and pa.pa_mx4_record_bytes(32, 256) == 8704
    for page, d in ((8, 128), (24, 128), (0, 64), (-16, 64), (16, 96), (16, 80), (16, 0), (16, 512), (1 << 30, 128)):
        assert pa.pa_mx4_record_bytes(page, d) == 0
    with pytest.raises(pa.PagedAttnError):
        pa.pa_mx4_cache(4, 16, 2, 96, device="cpu")


def test_norm_rope_append_refusals(lib):
    bad_tokens = (dict(T=-1), dict(rotary_dim=7), dict(rotary_dim=130), dict(rotary_dim=-2), dict(q=0), dict(q_out=0), dict(k_new=0),
                  dict(v_new=0), dict(num_q_heads=0), dict(rope_positions=0), dict(inv_freq=0), dict(inv_freq=0x4004), dict(seq_ids=0),
                  dict(positions=0), dict(block_table=0), dict(batch=0), dict(max_blocks=0), dict(mscale=float("nan")), dict(axes=0),
                  dict(axes=3), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(weight_offset=float("nan")),
                  dict(q_stride=4088), dict(q_out_stride=4088), dict(k_stride=1016), dict(v_stride=-1024), dict(q_stride=8192))
    odd_tokens = (dict(k_stride=1028), dict(v_stride=1025), dict(k_new=0x4008), dict(q_weight=0x4004), dict(k_weight=0x4008),
                  dict(weight_dtype=2), dict(weight_dtype=7))
    for fn, first in ((lib.paged_norm_rope_append, dict(cache=plain())), (lib.paged_norm_rope_append_mx4, dict(cache=desc(), dtype=i32(1)))):
        a = dict(first, tokens=tokens(), stream=NULL)
        for bad in bad_tokens:
            assert call(fn, a, tokens=tokens(**bad)) == INVALID, bad
        for odd in odd_tokens:
            assert call(fn, a, tokens=tokens(**odd)) == UNSUPPORTED, odd
        assert call(fn, a, tokens=NULL) == INVALID and call(fn, a, cache=NULL) == INVALID
        assert call(fn, a, tokens=tokens(T=0)) == 0 and call(fn, a, tokens=tokens(q=0, q_out=0, k_new=0, v_new=0)) == 0
    a = dict(cache=plain(), tokens=tokens(), stream=NULL)
    assert call(lib.paged_norm_rope_append, a, cache=plain(page_size=12)) == INVALID
    assert call(lib.paged_norm_rope_append, a, cache=plain(head_dim=100)) == UNSUPPORTED


BAD_CACHES = (dict(records=0), dict(num_pages=0), dict(num_kv_heads=0), dict(head_dim=0), dict(page_size=0), dict(page_size=24),
              dict(head_stride=2160), dict(page_stride=0), dict(page_stride=-2176), dict(page_stride=16))
ODD_CACHES = (dict(head_dim=96), dict(page_size=8), dict(records=0x1008), dict(page_stride=8 * 2176 + 8), dict(head_stride=2184))


def test_cache_refusals(lib):
    append = dict(cache=desc(), dtype=i32(1), k=P, v=P, ids=P, pos=P, T=i32(3), table=P, batch=i32(2), max_blocks=i32(4), stream=NULL)
    gather = dict(cache=desc(), dtype=i32(1), k=P, v=P, rows=i32(9), table=P, first=NULL, lens=P, cu=P, batch=i32(2), max_blocks=i32(4), max_len=i32(64),
                  stream=NULL)
    for fn, a in ((lib.paged_kv_append_mx4, append), (lib.paged_kv_gather_mx4, gather), (lib.paged_attention_mx4, attention_args())):
        for bad in BAD_CACHES:
            assert call(fn, a, cache=desc(**bad)) == INVALID, bad
        for odd in ODD_CACHES:
            assert call(fn, a, cache=desc(**odd)) == UNSUPPORTED, odd
        assert call(fn, a, cache=NULL) == INVALID and call(fn, a, dtype=i32(3)) == UNSUPPORTED
    for bad in (dict(T=i32(-1)), dict(k=NULL), dict(v=NULL), dict(ids=NULL), dict(pos=NULL), dict(table=NULL), dict(batch=i32(0)),
                dict(max_blocks=i32(0)), dict(batch=i32(-1))):
        assert call(lib.paged_kv_append_mx4, append, **bad) == INVALID, bad
    assert call(lib.paged_kv_append_mx4, append, k=ctypes.c_void_p(0x4008)) == UNSUPPORTED
    assert call(lib.paged_kv_append_mx4, append, T=i32(0)) == 0
    for bad in (dict(k=NULL), dict(v=NULL), dict(lens=NULL), dict(cu=NULL), dict(table=NULL), dict(batch=i32(-1)), dict(max_blocks=i32(0)),
                dict(max_len=i32(-1)), dict(rows=i32(-1))):
        assert call(lib.paged_kv_gather_mx4, gather, **bad) == INVALID, bad
    assert call(lib.paged_kv_gather_mx4, gather, v=ctypes.c_void_p(0x4004)) == UNSUPPORTED
    assert call(lib.paged_kv_gather_mx4, gather, batch=i32(0)) == 0 and call(lib.paged_kv_gather_mx4, gather, max_len=i32(0)) == 0
    assert call(lib.paged_kv_gather_mx4, gather, rows=i32(0)) == 0


def test_calls_of_more_threads_than_a_launch_has(lib):
    for fn, first in ((lib.paged_norm_rope_append, dict(cache=plain())), (lib.paged_norm_rope_append_mx4, dict(cache=desc(), dtype=i32(1)))):
        for T in (1 << 25, (1 << 31) - 1):
            assert call(fn, dict(first, tokens=tokens(T=T), stream=NULL)) == UNSUPPORTED
    append = dict(cache=desc(), dtype=i32(1), k=P, v=P, ids=P, pos=P, T=i32(1 << 25), table=P, batch=i32(2), max_blocks=i32(4), stream=NULL)
    assert call(lib.paged_kv_append_mx4, append) == UNSUPPORTED
    gather = dict(cache=desc(), dtype=i32(1), k=P, v=P, rows=i32((1 << 31) - 1), table=P, first=NULL, lens=P, cu=P, batch=i32(1 << 10),
                  max_blocks=i32(1 << 14), max_len=i32(1 << 18), stream=NULL)
    assert call(lib.paged_kv_gather_mx4, gather) == UNSUPPORTED
    assert call(lib.paged_kv_gather_mx4, gather, rows=i32((1 << 27) - 7)) == UNSUPPORTED


def attention_args():
    return dict(cache=desc(), dtype=i32(1), q=P, out=P, lse=NULL, cu=P, total=i32(6), max_q=i32(3), table=P, lens=P, batch=i32(2), hq=i32(32),
                max_blocks=i32(4), max_len=i32(64), scale=f32(0.1), ws=ctypes.c_void_p(0x10000), bytes=size(1 << 40), stream=NULL)


def test_attention_refusals(lib):
    a, fn = attention_args(), lib.paged_attention_mx4
    for bad in (dict(total=i32(-1)), dict(max_q=i32(-1)), dict(q=NULL), dict(out=NULL), dict(cu=NULL), dict(table=NULL), dict(lens=NULL),
                dict(batch=i32(-1)), dict(hq=i32(12)), dict(hq=i32(0)), dict(max_blocks=i32(3)), dict(max_len=i32(-1)),
                dict(scale=f32(float("nan"))), dict(ws=ctypes.c_void_p(0x10010))):
        assert call(fn, a, **bad) == INVALID, bad
    for bad in (dict(q=ctypes.c_void_p(0x4008)), dict(out=ctypes.c_void_p(0x4004))):
        assert call(fn, a, **bad) == UNSUPPORTED, bad
    assert call(fn, a, ws=NULL) == SMALL and call(fn, a, bytes=size(16)) == SMALL
    assert call(fn, a, batch=i32(0)) == 0 and call(fn, a, total=i32(0)) == 0 and call(fn, a, max_q=i32(0)) == 0
    # bounds whose places pass 31 bits
    assert call(fn, a, batch=i32(1 << 10), total=i32(1 << 24), max_q=i32(1 << 24), max_len=i32(1 << 30), max_blocks=i32(1 << 26)) == UNSUPPORTED


def test_workspace_bound(lib):
    for args in ((1, 8, 8, 64, 5, 5, 128), (64, 32, 8, 128, 300, 8, 32768), (0, 8, 8, 64, 0, 0, 0), (16, 64, 8, 256, 256, 16, 131072)):
        n = pa.paged_attention_mx4_workspace_bytes(*args)
        assert n > 0 and n % 256 == 0
    # a bound on a sequence's queries beyond all queries asks for nothing more
    assert pa.paged_attention_mx4_workspace_bytes(4, 32, 8, 128, 9, 9, 5000) == pa.paged_attention_mx4_workspace_bytes(4, 32, 8, 128, 9, 10 ** 9, 5000)


def test_binding_refuses_host_tensors_and_odd_records(lib):
    cache = torch.zeros(2, 2, 2176, dtype=torch.uint8)
    with pytest.raises(pa.PagedAttnError):
        binding.mx4_desc(cache, 128)
    q = torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(pa.PagedAttnError):
        pa.paged_kv_append_mx4(cache, q, q, q, q, q)


def test_the_reference_rounds_as_defined():
    """The tests' own definition, by the nearest of all values: each block's scale by its largest magnitude, ties to even mantissas."""
    x = np.array([[0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.001, 7.99, -0.25, -5.0, 0.26, 6.0] + [0.0] * 18])
    codes, scales = ref.quantised(x)
    assert scales.tolist() == [[127]]
    assert codes[0, :14].tolist() == [0, 0, 2, 2, 4, 4, 6, 6, 7, 7, 8, 14, 1, 7]
    for a in (1.0, 3.9, 4.0, 2.0 ** -140, 2.0 ** 127):
        _, s = ref.quantised(np.array([[a] + [0.0] * 31]))
        assert s[0, 0] == max(int(np.floor(np.log2(a))) - 2, -127) + 127
    for bad in (np.inf, -np.inf, np.nan):
        codes, s = ref.quantised(np.array([[bad] + [1.0] * 31]))
        assert s[0, 0] == 255 and (codes == 0).all()
