"""Sampling settings given as numbers that fp32 does not hold."""
import pytest
import torch

import paper_2506_05632_b200 as gls
from paper_2506_05632_b200 import binding


@pytest.mark.parametrize("value", [1e39, 1e300, 10 ** 50, 10 ** 400, -1e39], ids=["1e39", "1e300", "10^50", "10^400", "-1e39"])
def test_an_inverse_temperature_beyond_fp32_is_not_infinite(value):
    """Infinity is a setting of its own (the most likely token); finite numbers beyond the range are refused like those within fp32."""
    with pytest.raises(gls.GlsError):
        binding._setting(binding._Sampling(), "inv_temp", value, torch.float32, (1, 1, 1), 0)


def test_numbers_that_are_taken():
    s = binding._Sampling()
    for name, value, want in (("inv_temp", float("inf"), float("inf")), ("inv_temp", 0.5, 0.5), ("inv_temp", 3, 3.0), ("inv_temp", True, 1.0),
                              ("top_p", 1e300, float("inf")), ("min_p", 0.25, 0.25)):
        binding._setting(s, name, value, torch.float32, (1, 1, 1), 0)
        assert getattr(s, name) == want


@pytest.mark.parametrize("name", ["inv_temp", "top_p", "min_p"])
def test_a_setting_with_a_tangent(name):
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(torch.ones(1), torch.ones(1))
        with pytest.raises(gls.GlsError, match="forward-mode"):
            gls.sample_tokens(torch.zeros(1, 1, 1, 8), torch.zeros(1, 1, 1), **{name: dual})


@pytest.mark.gpu
@pytest.mark.parametrize("value", [1e39, 1e300, 10 ** 50, 10 ** 400], ids=["1e39", "1e300", "10^50", "10^400"])
def test_calls_with_it(gls, monkeypatch, value):
    """By the compiled calls and by the general way."""
    x, u = torch.zeros((1, 1, 2, 50), device="cuda"), torch.full((1, 1, 2), 0.9, device="cuda")
    for _ in range(2):
        with pytest.raises(gls.GlsError):
            gls.sample_tokens(x, u, inv_temp=value)
        assert gls.sample_tokens(x, u, inv_temp=float("inf"))["tokens"].tolist() == [[[0, 0]]]
        monkeypatch.setattr(binding, "_calls", binding._GeneralWay())
