"""What lserve_sparse_decode_tree refuses, on the host and before anything is launched; its workspace."""
import ctypes

import pytest
import torch

import paper_2502_14866_amd as L
from paper_2502_14866_amd import binding as B

i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
i64 = lambda *s: torch.zeros(s, dtype=torch.int64)  # noqa: E731
f16 = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
pool = f16(8, 2, 64, 128)


def _kv(**kw):
    return L.PagedKV(**{**dict(k_pool=pool, v_pool=pool, stats=None, page_table=i32(2, 4), seq_lens=i32(4)[:2]), **kw})


def _args(**kw):
    a = dict(desc=L.AttnDesc(4, 2, [1, 0]), kv=_kv(), q=f16(8, 4, 128), k_new=f16(8, 2, 128), v_new=f16(8, 2, 128), cu_new=i32(4)[:3],
             max_new_per_seq=4, out=f16(8, 4, 128), lse_out=torch.zeros(8, 4), tree_mask=i64(8, 1), positions=i32(8),
             sel_pages=i32(2, 2, 4), sel_count=i32(2, 2), sel_seq_len=i32(2), workspace=torch.zeros(16, dtype=torch.uint8), stream=0)
    a.update(kw)
    return a


def _code(**kw):
    with pytest.raises(B.LserveError) as e:
        L.lserve_sparse_decode_tree(**_args(**kw))
    return e.value.code


@pytest.mark.parametrize("bad,code", [
    (dict(), -3), (dict(workspace=None), -3), (dict(max_new_per_seq=0), -1), (dict(max_new_per_seq=9), -1),
    (dict(tree_mask=None), -1), (dict(positions=None), -1), (dict(sel_pages=None), -1), (dict(sel_count=None), -1), (dict(sel_seq_len=None), -1),
    (dict(k_new=None), -1), (dict(v_new=None), -1), (dict(sel_pages=i32(2, 2, 0)), -1),
    (dict(kv=_kv(k_pool=None)), -1), (dict(kv=_kv(v_pool=None)), -1), (dict(kv=_kv(kv_bits=5)), -1), (dict(kv=_kv(pool_heads=1)), -1),
    (dict(kv=_kv(k_pool_stream=pool, v_pool_stream=pool)), -1),  # a ring without its table
    (dict(desc=L.AttnDesc(4, 2, [1, 0], page_size=32)), -2), (dict(desc=L.AttnDesc(4, 2, [1, 0], sm_scale=-1.0)), -1),
    (dict(q=f16(1100, 4, 128), k_new=f16(1100, 2, 128), v_new=f16(1100, 2, 128), out=f16(1100, 4, 128), lse_out=None,
          tree_mask=i64(1100, 18), positions=i32(1100), max_new_per_seq=1025), -2),
    (dict(q=f16(128, 4, 128), k_new=f16(128, 2, 128), v_new=f16(128, 2, 128), out=f16(128, 4, 128), lse_out=None,
          tree_mask=i64(128, 1), positions=i32(128), max_new_per_seq=65), -1),  # a second word is missing
    (dict(positions=i32(12)[1:9]), -1), (dict(tree_mask=i64(9, 1)[1:]), -1),  # misaligned
])
def test_refused(bad, code):
    assert _code(**bad) == code


@pytest.mark.parametrize("bad", [
    dict(q=f16(8, 128, 4).transpose(1, 2)), dict(q=torch.zeros((8, 4, 128), dtype=torch.bfloat16)), dict(k_new=f16(7, 2, 128)),
    dict(out=f16(7, 4, 128)), dict(lse_out=torch.zeros(7, 4)), dict(lse_out=f16(8, 4)), dict(tree_mask=i32(8, 1)), dict(tree_mask=i64(7, 1)),
    dict(positions=i64(8)), dict(cu_new=i32(2)), dict(sel_count=i32(2, 1)), dict(sel_seq_len=i32(1)), dict(kv=_kv(seq_lens=i32(1))),
    dict(kv=_kv(k_pool=pool.float())),
])
def test_tensors_that_do_not_fit(bad):
    with pytest.raises(ValueError):
        L.lserve_sparse_decode_tree(**_args(**bad))


def test_a_stride_without_a_selection():
    lib, a = L.load_library(), _args()
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    assert lib.lserve_sparse_decode_tree(a["desc"].c(), a["kv"].c(), p(a["q"]), p(a["k_new"]), p(a["v_new"]), p(a["cu_new"]), None, 0, None,
                                         None, None, None, 4, 8, 4, p(a["out"]), None, p(a["workspace"]), ctypes.c_size_t(16), None) == -1


def test_workspace():
    d = L.AttnDesc(32, 8, [1] * 4 + [0] * 4)
    need = L.lserve_tree_workspace_bytes(d, 16, 256, 16, 513, 64)
    assert 0 < need <= 64 << 20
    assert L.lserve_tree_workspace_bytes(d, 4096, 4096, 1, 100) == 0  # so many lists that none is cut
    for bad in ((0, 16, 4, 8), (4, 0, 4, 8), (4, 16, 0, 8), (4, 16, 17, 8), (4, 2000, 1025, 8), (4, 16, 4, 0), (65536, 65536, 1, 8), (4, 16, 4, 8, -1)):
        assert L.lserve_tree_workspace_bytes(d, *bad) == 0
    assert L.lserve_tree_workspace_bytes(L.AttnDesc(32, 8, [0] * 8, page_size=32), 4, 16, 4, 8) == 0
    # a workspace that fits a batch of short sequences does not fit one of long ones: the call says so
    a = _args(workspace=torch.zeros(L.lserve_tree_workspace_bytes(L.AttnDesc(4, 2, [1, 0]), 2, 8, 4, 4, 4) - 1, dtype=torch.uint8))
    with pytest.raises(B.LserveError) as e:
        L.lserve_sparse_decode_tree(**a)
    assert e.value.code == -3
