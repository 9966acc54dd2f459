"""The native half of the binding on the calls of a shared or bounded cache: what it takes gives what the ctypes half gives."""
import pytest
import torch

from paper_2603_15619_amd import binding


class Half:
    """The native half (None: one that declines everything), with the names of the calls that it took."""

    def __init__(self, native):
        self.native, self.taken = native, []

    def __getattr__(self, name):
        def call(*a):
            r = getattr(self.native, name)(*a) if self.native else None
            if r is not None:
                self.taken.append(name)
            return r

        return call


@pytest.mark.gpu
def test_cache_calls_give_the_same_results_as_through_ctypes(monkeypatch):
    g = torch.Generator().manual_seed(2)
    t = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    Q, K, V, Kp, Vp, Kd, Vd = t(4, 6, 64), t(4, 2, 50, 64), t(4, 2, 50, 64), t(2, 2, 70, 64), t(2, 2, 70, 64), t(4, 2, 3, 64), t(4, 2, 3, 64)
    Qt, W = t(4, 6, 50, 64), torch.rand(4, 2, 50, generator=g).cuda()
    _, LSE = binding.moda_attn_fwd(Qt, K, V)

    def calls():
        r = list(binding.moda_attn_decode_shared(Q, Kp, Vp, K, V, Kd, Vd, ints(70, 3), ints(50, 0, 1, 33), T=49, depth_count=2, scale=0.3))
        r += binding.moda_attn_decode_shared(Q, Kp, Vp, None, None)
        r += binding.moda_attn_decode_weights(Q, K, V, W, lengths=ints(50, 0, 1, 33), weights_out=torch.zeros_like(W))
        r += binding.moda_attn_decode_weights(Q, K, V)
        r.append(binding.moda_attn_weights(Qt, K, LSE, window=7, lengths=ints(50, 0, 1, 33)))
        c = [x.clone() for x in (K, V, W)]
        r += binding.moda_cache_evict(*c, 20, 5, lengths=ints(50, 0, 1, 33)) + tuple(c)
        torch.cuda.synchronize()
        return r

    takes = Half(binding._native())
    monkeypatch.setattr(binding, "_native_module", takes)
    native = calls()
    assert takes.taken == ["shared"] * 4 + ["weights", "evict"]
    monkeypatch.setattr(binding, "_native_module", Half(None))
    for x, y in zip(native, calls()):
        assert torch.equal(x, y)


def test_cache_calls_decline_what_is_not_plain():
    m = binding._native()
    t = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    assert m.shared(t[0], None, None, t, t, *[None] * 13) is None      # host tensors
    assert m.weights(t, t, t, 0, True, None, None, None, t, None) is None
    assert m.evict(t, t, t, None, None, t, t, t, None, t, t, 1, 0, 16, None) is None
    assert m.shared() is None and m.weights(1) is None and m.evict(1, 2) is None
    with pytest.raises(TypeError):
        m.init_cache(1)
    with pytest.raises(ValueError):
        m.init_cache(0, 1, 1, 1, 1, 1)
