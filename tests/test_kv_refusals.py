"""What the paged cache and its attention refuse before a device is touched."""
import pytest
import torch


@pytest.fixture(scope="module")
def hx():
    import __graft_entry__ as entry
    entry.build()
    import paper_2605_16637_b200 as mod
    return mod


def parts(layers=2, pages=6, tokens=4, heads=2, dim=64, seqs=3, columns=5, dtype=torch.bfloat16):
    k = torch.zeros(layers, pages, tokens, heads, dim, dtype=dtype)
    return dict(k=k, v=torch.zeros_like(k), ref=torch.zeros(pages, dtype=torch.int32),
                table=torch.full((seqs, columns), -1, dtype=torch.int32), length=torch.zeros(seqs, dtype=torch.int32))


def test_a_described_cache(hx):
    c = hx.KvCache(**parts())
    assert (c.c.n_pages, c.c.page_tokens, c.c.max_seqs, c.c.max_pages, c.c.n_layers, c.c.head_dim) == (6, 4, 3, 5, 2, 64)
    assert c.work.numel() == hx.HX_KV_WORK(6, 3)
    assert c.with_tables(c.ref.clone(), c.table.clone(), c.length.clone()).work is c.work
    one = parts(layers=1, pages=1)
    one["k"], one["v"] = one["k"].as_strided(one["k"].shape, (3, 5, 128, 64, 1)), one["v"].as_strided(one["v"].shape, (3, 5, 128, 64, 1))
    assert hx.KvCache(**one).c.page_stride == 4 * 128                 # strides of single elements mean nothing


def test_strided_layers_and_pages(hx):
    both = torch.zeros(6, 2, 2, 4, 2, 64, dtype=torch.float16)        # [pages, keys or values, layers, tokens, heads, dim]
    p = parts(dtype=torch.float16)
    p["k"], p["v"] = both[:, 0].transpose(0, 1), both[:, 1].transpose(0, 1)
    c = hx.KvCache(**p)
    assert (c.c.layer_stride, c.c.page_stride) == (512, 4 * 512)


@pytest.mark.parametrize("change, fragment", [
    (lambda p: p.update(v=p["v"][:, :5]), "agree"),
    (lambda p: p.update(v=p["v"].half()), "agree"),
    (lambda p: p.update(k=p["k"][0], v=p["v"][0]), "agree"),
    (lambda p: p.update(k=p["k"].transpose(2, 3), v=p["v"].transpose(2, 3)), "contiguous"),
    (lambda p: p.update(k=p["k"].double(), v=p["v"].double()), "float16"),
    (lambda p: p.update(k=p["k"][..., :4].contiguous()[:, :, :, :1].contiguous(), v=p["v"][..., :4].contiguous()[:, :, :, :1].contiguous()), "multiple of 16"),
    (lambda p: p.update(k=p["k"][:0], v=p["v"][:0]), "at least one"),
    (lambda p: p.update(ref=p["ref"][:5]), "ref"),
    (lambda p: p.update(ref=p["ref"].long()), "ref"),
    (lambda p: p.update(table=p["table"].long()), "table"),
    (lambda p: p.update(table=p["table"].t()), "table"),
    (lambda p: p.update(table=p["table"][0]), "columns"),
    (lambda p: p.update(table=torch.zeros(16385, 1, dtype=torch.int32), length=torch.zeros(16385, dtype=torch.int32)), "16384"),
    (lambda p: p.update(length=p["length"][:2]), "length"),
    (lambda p: p.update(work=torch.zeros(3, dtype=torch.int32)), "HX_KV_WORK"),
    (lambda p: p.update(k=torch.zeros(2 * 6 * 512 + 1, dtype=torch.bfloat16)[1:].view(2, 6, 4, 2, 64)), "aligned"),
])
def test_caches_that_are_refused(hx, change, fragment):
    p = parts()
    change(p)
    with pytest.raises(hx.HxError) as e:
        hx.KvCache(**p)
    assert e.value.code == -1 and fragment in str(e.value)


@pytest.mark.parametrize("change, fragment", [
    (dict(n_pages=0), "at least one"), (dict(page_tokens=0), "at least one"), (dict(max_pages=-1), "at least one"),
    (dict(n_pages=1 << 29), "2^31"), (dict(max_pages=1 << 20, page_tokens=1 << 11), "2^31"), (dict(max_pages=(1 << 20) + 1), "2^20"),
    (dict(n_layers=1025), "1024"), (dict(n_kv_heads=1 << 15), "2^20"), (dict(dtype=9), "type"), (dict(page_stride=508), "16 bytes"),
    (dict(page_stride=256), "overlap"), (dict(layer_stride=256), "overlap"), (dict(k=0), "NULL"), (dict(work=0), "NULL"),
])
def test_descriptions_that_are_refused(hx, change, fragment):
    c = hx.KvCache(**parts()).c
    for name, value in change.items():
        setattr(c, name, value)
    with pytest.raises(hx.HxError) as e:
        hx.hx_kv_check(c)
    assert e.value.code == -1 and fragment in str(e.value)


def test_no_cache_is_refused(hx):
    with pytest.raises(hx.HxError):
        hx.hx_kv_check(None)


def test_every_call_refuses_a_missing_handle(hx):
    c = hx.KvCache(**parts()).c
    calls = [lambda: hx.hx_kv_fork(None, c, None, None, None, 0), lambda: hx.hx_kv_free(None, c, None, 0),
             lambda: hx.hx_kv_grow(None, c, None, None, 0), lambda: hx.hx_kv_copy(None, c, c, None, None, 0),
             lambda: hx.hx_kv_compact(None, c, None, None), lambda: hx.hx_kv_report(None, c, 0),
             lambda: hx.hx_kv_write(None, c, 0, None, None, 0, None, None, 0, 0, None, 0),
             lambda: hx.hx_attend_window(None, c, 0, None, None, None, 0, 0, 0, 0),
             lambda: hx.hx_attend_tree(None, c, 0, None, None, None, 0, None, None, 0, 1)]
    for call in calls:
        with pytest.raises(hx.HxError) as e:
            call()
        assert e.value.code == -1


@pytest.mark.parametrize("dtype, dim, heads, q_heads, fragment", [
    (torch.float32, 64, 2, 2, "F16 and BF16"), (torch.bfloat16, 80, 2, 2, "64, 96 or 128"), (torch.bfloat16, 64, 2, 3, "times"),
    (torch.bfloat16, 64, 2, 0, "times"), (torch.float16, 128, 1, 129, "times"),
])
def test_heads_that_attention_refuses(hx, dtype, dim, heads, q_heads, fragment):
    with pytest.raises(hx.HxError) as e:
        hx.hx_attend_work(hx.KvCache(**parts(dtype=dtype, dim=dim, heads=heads)).c, q_heads)
    assert fragment in str(e.value)


def test_scratch_does_not_depend_on_the_batch(hx):
    c = hx.KvCache(**parts(dim=128))
    assert 0 < c.attend_bytes(2) == c.attend_bytes(16) < 1 << 27
