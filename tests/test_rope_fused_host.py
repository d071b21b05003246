"""The layer's permutation and the paged cache's store with norms and rotations, without a GPU: plans that fit each other, arguments, refusals."""
import pytest
import torch

from paper_2512_24086_amd import rf2

AT = 0x10000
needs_no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="with a device the calls that are in order would be launched on made-up addresses")


def layer(**over):
    return rf2.Plan(**dict(dict(batch=2, heads=4, head_dim=64, T=3, H=8, W=8, block=64, sparsity=0.5, sink_frames=1, text_tokens=5), **over))


def rope(**over):
    return rf2.RopePlan(**dict(dict(heads=4, kv_heads=4, head_dim=64, axis_dims=(16, 24, 24)), **over))


def permute_code(p, r, **over):
    names = ("q", "k", "v", "pos", "pos_batch", "wq", "wk", "wq_text", "wk_text", "qp", "kp", "vp", "qbar", "kbar")
    a = dict({n: AT for n in names}, pos_batch=0)
    a.update(over)
    return rf2.lib().rf2_permute_rope(p._h if p else None, r._h if r else None, *(a[n] for n in names), None)


@needs_no_device
@pytest.mark.parametrize("over", [dict(), dict(wq_text=None, wk_text=None), dict(qbar=None, kbar=None), dict(pos_batch=591)], ids=str)
def test_permutations_in_order_reach_the_device(over):
    assert permute_code(layer(), rope(), **over) == rf2.RF2_ERR_HIP


@needs_no_device
def test_permutations_without_a_norm_or_positions():
    plain = dict(wq=None, wk=None, wq_text=None, wk_text=None)
    assert permute_code(layer(), rope(norm=rf2.RF2_NORM_NONE), **plain) == rf2.RF2_ERR_HIP
    assert permute_code(layer(), rope(norm=rf2.RF2_NORM_NONE)) == rf2.RF2_ERR_INVALID_ARG
    assert permute_code(layer(), rope(norm=rf2.RF2_NORM_NONE), **dict(plain, wk_text=AT, wq_text=AT)) == rf2.RF2_ERR_INVALID_ARG
    assert permute_code(layer(), rope(axis_dims=()), pos=None) == rf2.RF2_ERR_HIP


@needs_no_device
@pytest.mark.parametrize("over", [dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(wq=None), dict(wk=None), dict(wq_text=None), dict(wk_text=None),
                                  dict(qp=None), dict(kp=None), dict(vp=None), dict(qbar=None), dict(kbar=None), dict(q=AT + 8), dict(k=AT + 2), dict(v=AT + 4),
                                  dict(pos=AT + 2), dict(wq=AT + 8), dict(wk_text=AT + 2), dict(qp=AT + 8), dict(kp=AT + 8), dict(vp=AT + 8), dict(qbar=AT + 2),
                                  dict(kbar=AT + 1), dict(pos_batch=-1), dict(pos_batch=2 ** 33)], ids=str)
def test_permutations_that_are_refused(over):
    assert permute_code(layer(), rope(), **over) == rf2.RF2_ERR_INVALID_ARG


@needs_no_device
@pytest.mark.parametrize("over", [dict(heads=8), dict(kv_heads=2), dict(head_dim=128), dict(dtype=torch.float16)], ids=str)
def test_plans_that_do_not_fit_a_layer(over):
    assert permute_code(layer(), rope(**over)) == rf2.RF2_ERR_INVALID_ARG


def test_no_plan():
    assert permute_code(None, rope()) == permute_code(layer(), None) == rf2.RF2_ERR_INVALID_ARG
    assert store_code(None, rope(kv_heads=2)) == store_code(cache(), None) == rf2.RF2_ERR_INVALID_ARG


def cache(**over):
    return rf2.PagedPlan(**dict(dict(heads=4, kv_heads=2, head_dim=64, page=32, n_pages=9, max_seqs=3, max_pages=4, max_tokens=40), **over))


def store_code(p, r, **over):
    names = ("n_tokens", "q", "q_stride", "k", "k_stride", "v", "v_stride", "pos", "wq", "wk", "slots", "n_live", "k_cache", "v_cache", "q_out", "q_out_stride")
    a = dict({n: AT for n in names}, n_tokens=7, q_stride=256, k_stride=128, v_stride=128, q_out_stride=256)
    a.update(over)
    return rf2.lib().rf2_paged_store_rope(p._h if p else None, r._h if r else None, *(a[n] for n in names), None)


@needs_no_device
@pytest.mark.parametrize("over", [dict(), dict(n_live=None), dict(n_tokens=40), dict(n_tokens=1, q_stride=0, k_stride=0, v_stride=0, q_out_stride=0),
                                  dict(n_tokens=0, q=None, k=None, v=None, pos=None, wq=None, wk=None, slots=None, q_out=None), dict(q_stride=2 ** 36, v_stride=512)], ids=str)
def test_stores_in_order_reach_the_device(over):
    assert store_code(cache(), rope(kv_heads=2), **over) == rf2.RF2_ERR_HIP


@needs_no_device
@pytest.mark.parametrize("over", [dict(n_tokens=-1), dict(n_tokens=41), dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(wq=None), dict(wk=None), dict(slots=None),
                                  dict(k_cache=None), dict(v_cache=None), dict(q_out=None), dict(q=AT + 8), dict(k=AT + 2), dict(v=AT + 8), dict(pos=AT + 1), dict(wq=AT + 4),
                                  dict(wk=AT + 8), dict(slots=AT + 2), dict(n_live=AT + 1), dict(k_cache=AT + 8), dict(v_cache=AT + 4), dict(q_out=AT + 8), dict(q_stride=248),
                                  dict(q_stride=260), dict(k_stride=120), dict(k_stride=132), dict(v_stride=0), dict(v_stride=-128), dict(q_out_stride=192),
                                  dict(q_out_stride=257), dict(q_stride=2 ** 37), dict(k_stride=2 ** 62), dict(q_out_stride=2 ** 40)], ids=str)
def test_stores_that_are_refused(over):
    assert store_code(cache(), rope(kv_heads=2), **over) == rf2.RF2_ERR_INVALID_ARG


@needs_no_device
@pytest.mark.parametrize("over", [dict(heads=2), dict(kv_heads=4), dict(head_dim=128), dict(dtype=torch.float16)], ids=str)
def test_plans_that_do_not_fit_a_cache(over):
    assert store_code(cache(), rope(**dict(dict(kv_heads=2), **over))) == rf2.RF2_ERR_INVALID_ARG
    fits = dict(dict(kv_heads=2), **over)
    same = {k: v for k, v in fits.items() if k != "axis_dims"}
    assert store_code(cache(**same), rope(**fits), q_stride=1024, k_stride=1024, v_stride=1024, q_out_stride=1024) == rf2.RF2_ERR_HIP


@needs_no_device
def test_more_windows_than_a_grid_holds():
    p, r = cache(heads=512, kv_heads=512, max_tokens=1 << 20, n_pages=1 << 10), rope(heads=512, kv_heads=512)
    wide = dict(q_stride=512 * 64, k_stride=512 * 64, v_stride=512 * 64, q_out_stride=512 * 64)
    assert store_code(p, r, n_tokens=524256, **wide) == rf2.RF2_ERR_HIP
    assert store_code(p, r, n_tokens=524288, **wide) == rf2.RF2_ERR_UNSUPPORTED


class NoStream:
    cuda_stream = 0


@pytest.mark.parametrize("change", ["q", "q type", "q strides", "k", "v", "pos", "qp", "kp", "vp", "qbar", "kbar type", "no weight", "text weight"])
def test_tensors_of_a_layer_that_the_binding_refuses(change):
    p, r = layer(text_tokens=0), rope()
    r.device = -1
    n, bf = 192, torch.bfloat16
    t = {x: torch.zeros(2, 4, n, 64, dtype=bf) for x in "qkv"}
    t.update({k: v for k, v in p.alloc("cpu").items() if k in ("qp", "kp", "vp", "qbar", "kbar")}, pos=torch.zeros(n, 3, dtype=torch.int32), wq=torch.ones(64, dtype=bf),
             wk=torch.ones(64, dtype=bf), wq_text=None, wk_text=None)
    t.update({"q": dict(q=t["q"][:1]), "q type": dict(q=t["q"].half()), "q strides": dict(q=torch.zeros(4, 2, n, 64, dtype=bf).transpose(0, 1)), "k": dict(k=t["k"][:, :3]),
              "v": dict(v=t["v"][:, :, :8].contiguous()), "pos": dict(pos=torch.zeros(n + 1, 3, dtype=torch.int32)), "qp": dict(qp=t["qp"][:1]), "kp": dict(kp=t["kp"][:1]),
              "vp": dict(vp=t["vp"].float()), "qbar": dict(qbar=t["qbar"][:1]), "kbar type": dict(kbar=t["kbar"].to(bf)), "no weight": dict(wq=None),
              "text weight": dict(wq_text=torch.ones(32, dtype=bf), wk_text=torch.ones(64, dtype=bf))}[change])
    with pytest.raises(ValueError):
        p.rf2_permute_rope(r, t["q"], t["k"], t["v"], t["pos"], t["qp"], t["kp"], t["vp"], t["qbar"], t["kbar"], t["wq"], t["wk"], t["wq_text"], t["wk_text"], stream=NoStream)


@pytest.mark.parametrize("change", ["q", "k", "v", "v strides", "pos", "slots", "k_cache", "v_cache", "q_out", "q_out strides", "cu_new", "no cu_new", "no weight"])
def test_tensors_of_a_cache_that_the_binding_refuses(change):
    p, r = cache(), rope(kv_heads=2)
    p.device = r.device = -1
    bf, n = torch.bfloat16, 7
    t = {x: torch.zeros(n, h, 64, dtype=bf) for x, h in (("q", 4), ("k", 2), ("v", 2), ("q_out", 4))}
    t.update(pos=torch.zeros(n, 3, dtype=torch.int32), slots=torch.zeros(n, dtype=torch.int32), k_cache=torch.zeros(p.info.cache_elements, dtype=bf),
             v_cache=torch.zeros(p.info.cache_elements, dtype=bf), cu_new=torch.zeros(3, dtype=torch.int32), wq=torch.ones(64, dtype=bf), wk=torch.ones(64, dtype=bf))
    t.update({"q": dict(q=t["q"][:6]), "k": dict(k=t["k"].float()), "v": dict(v=t["v"][:, :1]), "v strides": dict(v=torch.zeros(n, 64, 2, dtype=bf).transpose(1, 2)),
              "pos": dict(pos=t["pos"][:, :2].contiguous()), "slots": dict(slots=t["slots"].long()), "k_cache": dict(k_cache=t["k_cache"][:-1]),
              "v_cache": dict(v_cache=t["v_cache"].half()), "q_out": dict(q_out=t["q_out"][:, :2]), "q_out strides": dict(q_out=torch.zeros(4, n, 64, dtype=bf).transpose(0, 1)),
              "cu_new": dict(cu_new=t["cu_new"].long()), "no cu_new": dict(cu_new=t["cu_new"][:0]), "no weight": dict(wk=None)}[change])
    with pytest.raises(ValueError):
        p.rf2_paged_store_rope(r, t["q"], t["k"], t["v"], t["pos"], t["slots"], t["k_cache"], t["v_cache"], t["q_out"], t["wq"], t["wk"], t["cu_new"], stream=NoStream)
