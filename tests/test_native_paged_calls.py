"""The native half of the binding on the calls of a paged cache: what it takes gives what the ctypes half gives."""
import pytest
import torch

from paged_cases import Cache, ints, normal
from paper_2603_15619_amd import binding
from test_native_cache_calls import Half


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
def test_paged_calls_give_the_same_results_as_through_ctypes(monkeypatch, mx):
    g = torch.Generator().manual_seed(2)
    t = lambda *s: normal(g, *s).cuda()
    lens = [50, 0, 1, 33]
    c = Cache(2, 16, 64, lens, mx=mx)
    Q, K, V, Kd, Vd, lengths = t(4, 6, 64), t(4, 2, 9, 64), t(4, 2, 9, 64), t(4, 2, 3, 64), t(4, 2, 3, 64), ints(lens)
    bounds = t(c.n_pages, 2, 2, 64)

    def calls():
        a = {n: x.clone() if x is not None else None for n, x in c.args().items()}
        b = bounds.clone()
        r = [x.view(torch.uint8) for x in binding.moda_page_append(K, V, **a, lengths=lengths, counts=ints([9, 0, 1, 5]), Kbounds=b)]
        out = tuple(torch.zeros(4, 2, 20, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        r += binding.moda_page_read(**a, lengths=lengths, first=30, out=out)
        chosen = torch.zeros(4, 2, 3, dtype=torch.int32, device="cuda")
        r.append(binding.moda_page_select(Q, b, a["page_table"], 3, 16, lengths=lengths, first=0, recent=2, T=48, out=chosen))
        r += binding.moda_attn_decode_paged(Q, **a, Kdepth=Kd, Vdepth=Vd, lengths=lengths, selected=chosen, T=48, depth_count=2, scale=0.3)
        r += binding.moda_attn_decode_paged(Q, **a, lengths=lengths)
        torch.cuda.synchronize()
        return r + [b]

    takes = Half(binding._native())
    monkeypatch.setattr(binding, "_native_module", takes)
    native = calls()
    assert takes.taken == ["page_append", "page_read", "page_select", "paged", "paged"]
    monkeypatch.setattr(binding, "_native_module", Half(None))
    for x, y in zip(native, calls()):
        assert torch.equal(x.isnan(), y.isnan()) and torch.equal(torch.nan_to_num(x), torch.nan_to_num(y))


def test_paged_calls_decline_what_is_not_plain():
    m = binding._native()
    t, i = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 3, dtype=torch.int32)
    assert m.page_append(t, t, t, t, i, *[None] * 5) is None  # host tensors
    assert m.page_read(t, t, i, None, 0, None, None, t, t) is None
    assert m.page_select(t[0], t, i, 1, 16, None, 1, 0, None, i, None) is None
    assert m.paged(t[0], t, t, i, *[None] * 12) is None
    assert m.page_append() is None and m.page_read(1) is None and m.page_select(1, 2) is None and m.paged(3) is None
    with pytest.raises(TypeError):
        m.init_pages(1)
    with pytest.raises(ValueError):
        m.init_pages(0, 1, 1, 1, 1, 1)
