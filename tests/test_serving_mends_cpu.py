"""What the decoder's host side must not refuse, lose or slow down, on the CPU."""
import pytest
import torch

from paper_2606_09508_amd import binding as eb
from paper_2606_09508_amd import prefill as pf


@pytest.mark.parametrize("n,kernel", [(8192, True), (8193, False)])
def test_more_adapters_than_the_kernel_takes(monkeypatch, n, kernel):
    """The tensor operations stand in, to bf16's rounding of fp32 sums."""
    calls = []
    monkeypatch.setattr(pf, "_kernel_device", lambda dev: dev.type == "cpu")
    monkeypatch.setattr(eb, "adapter_plan", lambda *a: calls.append("plan"))
    monkeypatch.setattr(eb, "adapter_add", lambda *a: calls.append("add"))
    monkeypatch.setattr(eb, "adapter_add_workspace_bytes", lambda *a: 16)
    g = torch.Generator().manual_seed(n)
    t = eb.Adapters((torch.randn((n, 8, 16), generator=g) * 0.1).bfloat16(),
                    (torch.randn((n, 8, 8), generator=g) * 0.1).bfloat16())
    layers = [{"wq": torch.zeros((16, 8), dtype=torch.bfloat16)}]
    assert pf.check_adapters([{"wq": t}], layers) == n
    index = [n - 1, -1, 5]
    own = pf.BatchAdapters([{"wq": t}], n, torch.tensor(index, dtype=torch.int32), 3)
    h = torch.randn((1, 3, 16), generator=g).bfloat16()
    y = torch.randn((1, 3, 8), generator=g).bfloat16()
    got, = own.layer(0)(h, ("wq",), [y.clone()])
    assert calls == (["plan", "add"] if kernel else [])
    if not kernel:
        want = y.double().clone()
        for s, i in enumerate(index):
            if i >= 0:
                want[0, s] += t.b[i].double() @ (t.a[i].double() @ h[0, s].double())
        assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()
