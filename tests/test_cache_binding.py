"""The Python side of the cache and norm calls on the host: what reaches the C
ABI, and that a refusal names what is wrong (no GPU: the library is replaced by
a recorder, or the call ends at the tensors' device)."""
import pytest
import torch

import paper_2609_23153_amd as sa
import test_abi_operators as T


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 16 if name.endswith("_size") else 0
        return call


@pytest.fixture
def recorded(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(sa, "library", lambda: lib)
    monkeypatch.setattr(sa, "_stream", lambda t: 0)
    return lib.calls


def test_append_takes_rows_without_a_table(recorded):
    args = T.cache_args()
    rows = torch.zeros(6, dtype=torch.int32)
    assert sa.sparse_attn_cache_append(**args, rope_row=rows) is None
    q = torch.zeros(6, 8, 128, dtype=torch.bfloat16)
    assert sa.sparse_attn_cache_append(**args, rope_row=rows, q=q, q_out=q) is q
    for name, a in recorded:
        assert name == "sparse_attn_cache_append"
        assert a[3] is None and a[4] == a[5] == 0      # no table
    assert recorded[1][1][7] == recorded[1][1][8] == q.data_ptr()


@pytest.mark.parametrize("rows", [torch.zeros(5, dtype=torch.int32), torch.zeros(6, dtype=torch.int64),
                                  torch.zeros(12, dtype=torch.int32)[::2]])
def test_rows_without_a_table_are_checked_alike(recorded, rows):
    with pytest.raises(ValueError, match="rope_row"):
        sa.sparse_attn_cache_append(**T.cache_args(), rope_row=rows)
    assert not recorded


def norm_args():
    return dict(x=torch.zeros(4, 8)), dict(dy=torch.zeros(4, 8), x=torch.zeros(4, 8),
                                           mean=torch.zeros(4), rstd=torch.ones(4))


def test_tensors_off_the_gpu_are_refused():
    # nothing may reach a kernel with a host address
    args = T.cache_args()
    fwd, bwd = norm_args()
    q = torch.zeros(6, 8, 128, dtype=torch.bfloat16)
    pool = {n: t for n, t in args.items() if n not in ("k", "v")}
    for call, kw in ((sa.sparse_attn_cache_append, args), (sa.sparse_attn_fwd_cache, dict(pool, q=q)),
                     (sa.sparse_attn_layer_norm, fwd), (sa.sparse_attn_layer_norm_bwd, bwd),
                     (sa.sparse_attn_quant_rows_fp8, dict(x=q[:, 0]))):
        with pytest.raises(ValueError, match="on a GPU"):
            call(**kw)


@pytest.mark.parametrize("bad", T.BAD_CACHE_TENSORS)
def test_refusals_of_the_cache_name_the_tensor(recorded, bad):
    # (by their own checks: the device is looked at last)
    args = T.cache_args()
    args.update(bad)
    with pytest.raises(ValueError, match="|".join(bad)):
        sa.sparse_attn_cache_append(**args)
    del args["k"], args["v"]
    with pytest.raises(ValueError, match="|".join(bad)):
        sa.sparse_attn_fwd_cache(torch.zeros(6, 8, 128, dtype=torch.bfloat16), **args)
    assert not [c for c in recorded if not c[0].endswith("_size")]


def test_a_pool_without_key_heads_and_scalars_are_refused(recorded):
    args = T.cache_args()
    none = dict(args, k8=args["k8"][:, :0], v8=args["v8"][:, :0], sk=args["sk"][:, :0], sv=args["sv"][:, :0])
    q = torch.zeros(6, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="k8"):
        sa.sparse_attn_cache_append(**dict(none, k=args["k"][:, :0], v=args["v"][:, :0], q=q))
    with pytest.raises(ValueError, match="k8"):
        sa.sparse_attn_fwd_cache(q, **{n: t for n, t in none.items() if n not in ("k", "v")})
    with pytest.raises(ValueError, match="k must be"):
        sa.sparse_attn_cache_append(**dict(args, k=args["k"][0, 0, 0]))
    assert not recorded
