"""Tensors that decoder.py's layer operators have to refuse, or take as they are (no GPU): the calls that launch kernels are
replaced by ones that note their arguments."""
import pytest
import torch

from paper_1911_08076_gb300 import decoder, ifq
from test_layer_decoder_host import calls   # noqa: F401 (a fixture)


def test_expanded_rows_are_refused(calls):   # noqa: F811
    """A row stride of 0 means dense to the calls: they would read past the one row that there is."""
    w, pair = decoder.Weights4(torch.randn(24, 40), group=32), decoder.Weights4(torch.randn(24, 40), torch.randn(24, 40), group=32)
    del calls[:]
    x = torch.zeros(1, 40, dtype=torch.bfloat16)
    overlapping = torch.zeros(80, dtype=torch.bfloat16).as_strided((6, 40), (8, 1))
    for bad in (x.expand(6, 40), overlapping):
        with pytest.raises(ValueError):
            w.matmul(bad)
        with pytest.raises(ValueError):
            pair.gate(bad)
    with pytest.raises(ValueError):
        decoder.token_scores(torch.zeros(1, 50).expand(7, 50))
    with pytest.raises(ValueError):
        decoder.token_scores(torch.zeros(80).as_strided((6, 40), (8, 1)))
    with pytest.raises(ValueError):
        decoder.token_scores(torch.zeros(1, 50), torch.zeros((), dtype=torch.int64).expand(2))
    assert calls == []
    # one row has no stride, and no rows neither
    w.matmul(x.expand(1, 40))
    decoder.token_scores(torch.zeros(1, 50).expand(1, 50))
    w.matmul(x.expand(0, 40))
    assert [a[0].x_stride for n, a in calls if n == "ifq_w4_matmul"] == [0, 0] and calls[1][1][0].stride == 0


def test_the_stride_of_one_row_does_not_matter(calls):   # noqa: F811
    w = decoder.Weights4(torch.randn(24, 40), group=32)
    wide = torch.zeros(6, 44, dtype=torch.bfloat16)
    w.matmul(wide[:1, :40])
    assert calls[-1][0] == "ifq_w4_matmul" and calls[-1][1][0].m == 1 and calls[-1][1][0].x_stride == 0
    with pytest.raises(ValueError):
        w.matmul(wide[:2, :40])


def test_tensors_of_other_devices_are_refused(calls, monkeypatch):   # noqa: F811
    """The calls take addresses: one of another device than the current one, or of the host, is not the kernels' to read."""
    w, pair = decoder.Weights4(torch.randn(24, 40), group=32), decoder.Weights4(torch.randn(24, 40), torch.randn(24, 40), group=32)
    del calls[:]
    x, weight, logits = torch.zeros(6, 40, dtype=torch.bfloat16), torch.ones(40, dtype=torch.bfloat16), torch.zeros(6, 50)
    for call in (lambda: w.matmul(x.to("meta")), lambda: pair.gate(x.to("meta")),
                 lambda: w.matmul(x, torch.zeros(6, 24, dtype=torch.bfloat16, device="meta")),
                 lambda: decoder.rms_norm(x, weight.to("meta")), lambda: decoder.rms_norm(x, weight, 1e-5, x.to("meta")),
                 lambda: decoder.token_scores(logits, torch.zeros(6, dtype=torch.int64, device="meta"))):
        with pytest.raises(ValueError):
            call()
    assert calls == []

    class On:
        def __init__(self, device):
            self.device = torch.device(device)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    decoder._check_devices(On("cuda:1"), None, On("cuda:1"))
    for bad in (("cuda:0", "cuda:0"), ("cuda:1", "cuda:0"), ("cuda:1", "cpu")):
        with pytest.raises(ValueError):
            decoder._check_devices(*map(On, bad))
