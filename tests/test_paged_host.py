"""The paged cache's entry points without a GPU: configurations, arguments and their refusals."""
import ctypes as C

import pytest
import torch

from paper_2512_24086_amd import rf2

GOOD = dict(heads=8, kv_heads=2, head_dim=64, page=64, n_pages=10, max_seqs=4, max_pages=5, max_tokens=32)


def make(**over):
    return rf2.PagedPlan(**dict(GOOD, **over))


@pytest.mark.parametrize("bad", [dict(heads=0), dict(kv_heads=0), dict(heads=7), dict(heads=-8, kv_heads=-2), dict(n_pages=0), dict(max_seqs=0),
                                 dict(max_pages=0), dict(max_tokens=0), dict(max_tokens=-1), dict(causal=2), dict(scale=-1.0), dict(scale=float("nan")),
                                 dict(scale=float("inf"))], ids=str)
def test_invalid_configurations(bad):
    with pytest.raises(rf2.Rf2Error) as e:
        make(**bad)
    assert e.value.code == rf2.RF2_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(head_dim=96), dict(head_dim=0), dict(page=16), dict(page=48), dict(page=512), dict(heads=514), dict(max_seqs=4097),
                                 dict(max_tokens=(1 << 20) + 1), dict(n_pages=(1 << 24) + 1), dict(max_pages=(1 << 18) + 1),
                                 dict(max_seqs=4096, max_pages=(1 << 18) + 1, page=32)], ids=str)
def test_unsupported_configurations(bad):
    with pytest.raises(rf2.Rf2Error) as e:
        make(**bad)
    assert e.value.code == rf2.RF2_ERR_UNSUPPORTED


@pytest.mark.parametrize("scale, fine", [(2.0 ** 127, True), (2.3e38, True), (2.4e38, False), (3.4e38, False)])
def test_a_scale_is_finite_in_the_exponent_of_two_as_well(scale, fine):
    if fine:
        make(scale=scale).close()
        return
    with pytest.raises(rf2.Rf2Error) as e:
        make(scale=scale)
    assert e.value.code == rf2.RF2_ERR_INVALID_ARG


def test_a_type_that_is_none_of_the_two():
    with pytest.raises(ValueError):
        make(dtype=torch.float32)
    cfg = rf2.rf2_paged_config(8, 2, 64, 64, 10, 4, 5, 32, 2, 1, 0.0)
    h = C.c_void_p(0)
    assert rf2.lib().rf2_paged_plan_create(C.byref(cfg), C.byref(h)) == rf2.RF2_ERR_INVALID_ARG and not h


@pytest.mark.parametrize("over", [dict(), dict(head_dim=128, page=32), dict(heads=40, kv_heads=40), dict(heads=512, kv_heads=512), dict(heads=3, kv_heads=1), dict(max_seqs=256),
                                  dict(max_seqs=257), dict(max_seqs=4096)], ids=str)
def test_sizes(over):
    p = make(**over)
    c = p.cfg
    assert p.info.cache_elements == c.n_pages * c.kv_heads * c.page * c.head_dim
    survey = 16 * (c.max_seqs + 1) if c.max_seqs > 256 else 0
    assert survey < p.info.workspace_bytes <= 1024 * (2 * 128 * (c.head_dim + 2) * 4 + 16 * 32) + 32 + survey
    buf = p.alloc("cpu")
    assert buf["k_cache"].numel() == buf["v_cache"].numel() == p.info.cache_elements
    assert buf["free_pages"].tolist() == list(range(c.n_pages - 1, -1, -1)) and buf["n_free"].item() == c.n_pages
    p.close()
    p.close()


def test_null_arguments():
    lib = rf2.lib()
    bad = rf2.RF2_ERR_INVALID_ARG
    assert lib.rf2_paged_plan_create(None, None) == bad and lib.rf2_paged_plan_info(None, None) == bad
    assert lib.rf2_paged_plan_destroy(None) == rf2.RF2_OK
    none = [None] * 11
    assert lib.rf2_paged_append(None, 1, 1, *none) == bad
    assert lib.rf2_paged_release(None, 1, *none[:9]) == bad
    assert lib.rf2_paged_store(None, 1, None, 0, None, 0, *none[:4]) == bad
    assert lib.rf2_paged_attn(None, 1, 1, None, 0, *none[:9]) == bad
    p = make()
    assert lib.rf2_paged_append(p._h, 1, 1, *none) == bad
    assert lib.rf2_paged_release(p._h, 1, *none[:9]) == bad
    assert lib.rf2_paged_store(p._h, 1, None, 128, None, 128, *none[:4]) == bad
    assert lib.rf2_paged_attn(p._h, 1, 1, None, 512, *none[:9]) == bad


def calls(p, n_seqs=2, n_tokens=8, at=0x10000, **over):
    """The four calls' codes with plausible addresses, some of them replaced; none of them reaches a launch here."""
    lib = rf2.lib()
    ptr = {n: at for n in ("seq_len", "new_len", "free", "n_free", "table", "len_out", "free_out", "cu", "slots", "status", "done", "k", "v", "kc", "vc",
                           "q", "ws", "o", "lse")}
    stride = dict(q_stride=512, k_stride=128, v_stride=128)
    ptr.update({k: v for k, v in over.items() if k in ptr})
    stride.update({k: v for k, v in over.items() if k in stride})
    g = ptr.get
    return (lib.rf2_paged_append(p._h, n_seqs, n_tokens, g("seq_len"), g("new_len"), g("free"), g("n_free"), g("table"), g("len_out"), g("free_out"),
                                 g("cu"), g("slots"), g("status"), None),
            lib.rf2_paged_release(p._h, n_seqs, g("done"), g("seq_len"), g("table"), g("free"), g("n_free"), g("len_out"), g("free_out"), g("status"), None),
            lib.rf2_paged_store(p._h, n_tokens, g("k"), stride["k_stride"], g("v"), stride["v_stride"], g("slots"), g("kc"), g("vc"), None),
            lib.rf2_paged_attn(p._h, n_seqs, n_tokens, g("q"), stride["q_stride"], g("kc"), g("vc"), g("table"), g("seq_len"), g("cu"), g("ws"), g("o"),
                               g("lse"), None))


# name of what is replaced, its value, and which of (append, release, store, attn) refuse it
@pytest.mark.parametrize("over, refuse", [
    (dict(n_seqs=-1), "ar-t"), (dict(n_seqs=5), "ar-t"), (dict(n_tokens=-1), "a-st"), (dict(n_tokens=33), "a-st"),
    (dict(seq_len=0), "ar-t"), (dict(new_len=0), "a---"), (dict(free=0), "ar--"), (dict(n_free=0), "ar--"), (dict(table=0), "ar-t"),
    (dict(len_out=0), "ar--"), (dict(free_out=0), "ar--"), (dict(cu=0), "a--t"), (dict(slots=0), "a-s-"), (dict(status=0), "ar--"), (dict(done=0), "-r--"),
    (dict(k=0), "--s-"), (dict(v=0), "--s-"), (dict(kc=0), "--st"), (dict(vc=0), "--st"), (dict(q=0), "---t"), (dict(ws=0), "---t"), (dict(o=0), "---t"),
    (dict(q=0x10008), "---t"), (dict(k=0x10002), "--s-"), (dict(vc=0x10008), "--st"), (dict(ws=0x10004), "---t"), (dict(o=0x10008), "---t"),
    (dict(slots=0x10002), "a-s-"), (dict(lse=0x10001), "---t"), (dict(cu=0x10003), "a--t"),
    (dict(q_stride=504), "---t"), (dict(q_stride=516), "---t"), (dict(k_stride=120), "--s-"), (dict(v_stride=130), "--s-"), (dict(q_stride=-512), "---t"),
], ids=str)
def test_arguments_are_checked_before_the_device(over, refuse):
    if torch.cuda.is_available():
        pytest.skip("with a device the calls that are in order would be launched on made-up addresses")
    p = make()
    p_over = {k: v for k, v in over.items() if k in ("n_seqs", "n_tokens")}
    rest = {k: (v or None) if isinstance(v, int) and v == 0 else v for k, v in over.items() if k not in p_over}
    for code, name, mark in zip(calls(p, **p_over, **rest), "arst", refuse):
        if mark == name:
            assert code == rf2.RF2_ERR_INVALID_ARG, (name, code)
        else:
            assert code == rf2.RF2_ERR_HIP, (name, code)        # (everything else is in order: there is no device)


def test_more_rows_than_a_grid_has_room_for():
    p = make(heads=512, kv_heads=512, max_tokens=1 << 20)
    for n in (1 << 20, (1 << 20) - 31):
        assert rf2.lib().rf2_paged_store(p._h, n, 0x10000, 512 * 64, 0x10000, 512 * 64, 0x10000, 0x10000, 0x10000, None) == rf2.RF2_ERR_UNSUPPORTED


def test_without_a_device_nothing_computes():
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    p = make()
    assert set(calls(p)) == {rf2.RF2_ERR_HIP}
    buf, step = p.alloc("cpu"), p.alloc_step(4, 8, "cpu")
    q = torch.zeros(8, 8, 64, dtype=torch.bfloat16)
    with pytest.raises((rf2.Rf2Error, RuntimeError, AssertionError)):
        p.rf2_paged_attn(q, buf["k_cache"], buf["v_cache"], buf["block_table"], buf["seq_len"], step["cu_new"], buf["workspace"], step["o"],
                         stream=type("S", (), {"cuda_stream": 0}))


@pytest.mark.parametrize("what", ["shape", "dtype", "heads", "channels", "contiguous", "cache", "workspace", "ints"])
def test_the_binding_checks_tensors(what):
    p = make()
    p.device = -1                            # (of tensors in host memory)
    buf, step = p.alloc("cpu"), p.alloc_step(4, 8, "cpu")
    t = dict(q=torch.zeros(8, 8, 64, dtype=torch.bfloat16), k_cache=buf["k_cache"], v_cache=buf["v_cache"], block_table=buf["block_table"],
             seq_len=buf["seq_len"], cu_new=step["cu_new"], workspace=buf["workspace"], o=step["o"])
    if what == "shape":
        t["q"] = t["q"].view(8, 4, 128)
    elif what == "dtype":
        t["q"] = t["q"].half()
    elif what == "heads":
        t["q"] = torch.zeros(8, 16, 64, dtype=torch.bfloat16)[:, ::2]
    elif what == "channels":
        t["q"] = torch.zeros(8, 64, 8, dtype=torch.bfloat16).transpose(1, 2)
    elif what == "contiguous":
        t["o"] = torch.zeros(8, 64, 8, dtype=torch.bfloat16).transpose(1, 2)
    elif what == "cache":
        t["k_cache"] = t["k_cache"][:5]
    elif what == "workspace":
        t["workspace"] = t["workspace"][16:]
    else:
        t["seq_len"] = t["seq_len"].long()
    with pytest.raises(ValueError):
        p.rf2_paged_attn(**t)
