"""The 4-bit cache without a GPU: sizes, refusals of the C entry points and of the binding, and its oracle's own pins."""
import ctypes

import numpy as np
import pytest

import kv4_oracle as O
from paper_2404_18911_amd import binding as B


def _cache(**over):
    c = B.kg_kv4_cache(4096, 4 * 64 * 160, 8, 64, 4, 128, 2, 5, 4096, 4096)
    for k, v in over.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [dict(pool_dev=None), dict(pool_dev=4104), dict(page_stride=4 * 64 * 160 - 16), dict(page_stride=4 * 64 * 160 + 8), dict(n_pages=0),
              dict(page_tokens=8), dict(page_tokens=256), dict(page_tokens=48), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=96),
              dict(n_seqs=0), dict(n_seqs=4097), dict(max_pages=0), dict(max_pages=1 << 30), dict(page_table_dev=None), dict(len_dev=None)]


def test_page_bytes():
    L = B.lib()
    assert L.kg_op_kv4_page_bytes(128, 128, 32) == 32 * 128 * 160
    assert L.kg_op_kv4_page_bytes(64, 16, 1) == 16 * 80
    for bad in ((96, 64, 1), (128, 8, 1), (128, 256, 1), (128, 48, 1), (128, 64, 0), (128, 64, 1025), (0, 0, 0)):
        assert L.kg_op_kv4_page_bytes(*bad) == 0, bad


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(bad):
    L, c, ok = B.lib(), _cache(**bad), _cache()
    p = 1 << 20
    assert L.kg_op_kv4_append(c, 0, p, 512, p, 512, p, 1, None) == B.KG_EINVAL
    assert L.kg_op_kv4_read(c, 0, p, 512, 2 * p, 512, p, 1, None) == B.KG_EINVAL
    assert L.kg_op_kv4_work_bytes(c, 1, 4, 100) == 0
    assert L.kg_op_kv4_attention(c, 0, p, 512, 4, p, 1, 100, 0.1, 2 * p, 512, None, None, p, 1 << 40, None) == B.KG_EINVAL
    assert L.kg_op_kv4_evict(c, ok, 8, 0, 0, p, 2 * p, p, None) == B.KG_EINVAL
    assert L.kg_op_kv4_evict(ok, c, 8, 0, 0, p, 2 * p, p, None) == B.KG_EINVAL


def test_append_and_read_refusals():
    L, c, p = B.lib(), _cache(), 1 << 20
    for fn in (L.kg_op_kv4_append, L.kg_op_kv4_read):
        good = [c, 1, p, 512, 2 * p, 512, p, 3, None]
        for i, v in ((0, None), (1, 3), (1, -1), (2, None), (2, p + 1), (3, 511), (3, -512), (3, 1 << 45), (3, 1 << 62), (4, None), (4, p + 1), (5, 100), (6, None), (7, -1)):
            a = list(good)
            a[i] = v
            assert fn(*a) == B.KG_EINVAL, (i, v)
        assert fn(c, 1, None, 0, None, 0, p, 0, None) == B.KG_OK          # no rows: nothing to do
    assert L.kg_op_kv4_read(c, 0, p, 512, p + 4, 512, p, 2, None) == B.KG_EINVAL        # k and v share memory


def test_attention_refusals():
    L, c, p = B.lib(), _cache(), 1 << 20
    n = L.kg_op_kv4_work_bytes(c, 3, 8, 100)
    assert n >= 3 * 8 * 4
    #       0  1  2   3    4  5  6  7    8      9     10    11    12    13 14 15
    good = [c, 0, p, 1024, 8, p, 3, 100, 0.125, 2 * p, 1024, None, None, p, n, None]
    for i, v in ((0, None), (1, 3), (2, None), (2, p + 2), (3, 1023), (4, 0), (4, 6), (4, 1028), (5, None), (6, -1), (7, 0), (7, (1 << 30) + 1),
                 (8, float("nan")), (8, float("inf")), (9, None), (9, 2 * p + 1), (9, p + 4), (9, p), (10, 1000), (11, p), (13, None), (13, p + 4)):
        a = list(good)
        a[i] = v
        assert L.kg_op_kv4_attention(*a) == B.KG_EINVAL, (i, v)
    a = list(good)
    a[14] = n - 1
    assert L.kg_op_kv4_attention(*a) == B.KG_ENOSPC
    a = list(good)
    a[11], a[12] = p + 64, p                    # weights_in and weights_out share memory and are not the same
    assert L.kg_op_kv4_attention(*a) == B.KG_EINVAL
    for bad in ((-1, 8, 100), (1, 0, 100), (1, 6, 100), (1, 8, 0)):
        assert L.kg_op_kv4_work_bytes(c, *bad) == 0
    a = list(good)
    a[2] = a[9] = None
    a[6] = 0
    assert L.kg_op_kv4_attention(*a) == B.KG_OK     # no rows and no weights: nothing to do


def test_evict_refusals():
    L, src, dst, p = B.lib(), _cache(), _cache(max_pages=2), 1 << 20
    good = [src, dst, 100, 4, 32, p, 2 * p, 3 * p, None]
    for i, v in ((2, 0), (3, -1), (4, -1), (3, 101), (4, 97), (5, None), (6, None), (6, p + 128), (7, None)):
        a = list(good)
        a[i] = v
        assert L.kg_op_kv4_evict(*a) == B.KG_EINVAL, (i, v)
    a = list(good)
    a[2] = 129                                      # more than two pages of 64
    assert L.kg_op_kv4_evict(*a) == B.KG_ENOSPC
    for over in (dict(head_dim=64), dict(n_kv_heads=2), dict(n_seqs=3)):
        a = list(good)
        a[1] = _cache(**over)
        assert L.kg_op_kv4_evict(*a) == B.KG_EINVAL, over


def test_binding_refuses_what_is_not_on_a_gpu():
    import torch
    z = torch.zeros
    with pytest.raises(ValueError):
        B.Kv4Cache(z(1 << 20, dtype=torch.uint8), z(1, 2, dtype=torch.int32), z(1, dtype=torch.int32), 4, 128, 64)
    with pytest.raises(ValueError):
        B.Kv4Cache(z(1 << 20, dtype=torch.uint8), z(1, 2, dtype=torch.int32), z(1, dtype=torch.int32), 4, 96, 64)
    with pytest.raises(ValueError):
        B.Kv4Cache(z(1 << 20, dtype=torch.uint8), z(1, 2, dtype=torch.int32), z(1, dtype=torch.int32), 4, 128, 64, page_stride=100)


def test_oracle_quantisation_by_hand():
    """Levels 0..15 come back exactly, a border goes to the even level, constants and small groups hold their value."""
    x = np.zeros((4, 32), np.float32)
    x[0, :16] = np.arange(16) - 3.0
    x[0, 16:] = -3.0
    x[1] = x[0]
    x[1, 16:20] = [-2.5, -1.5, -0.5, 11.5]      # 0.5, 1.5, 2.5, 14.5 steps above the least
    x[2] = 7.25
    x[3, 0] = np.nan
    n, s, m = O.quantise(x)
    assert list(s[:3, 0]) == [1, 1, 0] and list(m[:3, 0]) == [-3, -3, 7.25] and np.isnan(s[3, 0])
    assert (O.values((n, s, m))[0] == x[0]).all() and (O.values((n, s, m))[2] == 7.25).all() and np.isnan(O.values((n, s, m))[3]).all()
    assert list(n[1, 0, 16:20]) == [0, 2, 2, 14]
    r = np.random.default_rng(0).standard_normal((64, 128)).astype(np.float32)
    n, s, m = O.quantise(r)
    v = O.values((n, s, m))
    # half a step, and what the roundings of s and m to fp16 move the ends by
    assert (np.abs(v - r) <= np.repeat(s / 2 + 15 * s * 2.0 ** -11 + np.abs(m) * 2.0 ** -11, 32, axis=1)).all()


def test_oracle_bytes_of_a_page_do_not_overlap():
    for D, T, H in ((64, 16, 2), (128, 32, 1)):
        seen = set()
        for h in range(H):
            for t in range(T):
                o = O.token_offsets(H, D, T, h, t)
                assert len(o) == D * 5 // 4 and not (o & seen)
                seen |= o
        assert seen == set(range(H * T * D * 5 // 4))


def test_oracle_eviction_by_hand():
    w = np.array([9, 1, 5, 5, 0, 5, 2, 7, 0, 0], float)
    assert list(O.evict(w, 10, 5, 1, 2)) == [0, 2, 7, 8, 9]
    assert list(O.evict(w, 10, 6, 1, 2)) == [0, 2, 3, 7, 8, 9]
    assert list(O.evict(w, 4, 5, 1, 2)) == [0, 1, 2, 3]
    w[4] = np.nan
    assert list(O.evict(w, 10, 4, 0, 0)) == [0, 2, 4, 7]


@pytest.mark.parametrize("head_dim", [64, 128])
def test_calls_beyond_a_launch_are_refused(head_dim):
    """A launch has fewer than 2^32 threads: such a call is an error of its arguments, found before anything runs."""
    L, p, far = B.lib(), 1 << 20, 1 << 46
    c, n = _cache(head_dim=head_dim), (1 << 32) * 8 // head_dim      # head_dim / 8 threads a row and head
    w = 4 * head_dim
    assert L.kg_op_kv4_append(c, 1, p, w, far, w, p, n, None) == B.KG_EINVAL
    assert L.kg_op_kv4_read(c, 1, p, w, far, w, p, n, None) == B.KG_EINVAL
    # weights: 256 threads for 128 tokens of a sequence and head, 2^24 such blocks
    c = _cache(head_dim=head_dim, n_kv_heads=1024, n_seqs=16, max_pages=1 << 11, page_stride=1024 * 64 * head_dim * 5 // 4)
    work = L.kg_op_kv4_work_bytes(c, 0, 1024, 1 << 17)
    assert L.kg_op_kv4_attention(c, 0, None, 0, 1024, p, 0, 1 << 17, 0.1, None, 0, None, far, p, work, None) == B.KG_EINVAL


@pytest.mark.parametrize("kept", [(1 << 20) + 64, (1 << 21) + 64])
def test_evict_refuses_kept_tokens_over_the_weights(kept):
    L, src, dst, p = B.lib(), _cache(), _cache(max_pages=2), 1 << 20
    assert L.kg_op_kv4_evict(src, dst, 100, 4, 32, p, 2 * p, kept, None) == B.KG_EINVAL
