"""The token operators on tensors whose rows share memory or are not equally
far apart: refused, nothing read or written."""
import pytest

from paper_2108_02416_amd import aspis

from _helpers import device

pytestmark = pytest.mark.gpu

KINDS = ["float32", "bfloat16", "float16"]


def _views(x):
    """Views of x [4, 8] that hold 12 or 400 rows by their shape."""
    return [x.view(4, 1, 8).expand(4, 3, 8), x.view(4, 1, 8).expand(4, 100, 8),
            x.view(1, 4, 8).expand(3, 4, 8), x[:1].expand(12, 8), x[:, :1].unsqueeze(1).expand(4, 3, 1)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("which", range(5))
def test_rows_that_share_memory_are_refused(which, kind):
    import torch
    x = torch.arange(32.0, device=device()).view(4, 8).to(getattr(torch, kind))
    view, before = _views(x)[which], x.clone()
    n, d = view.shape[:-1].numel(), view.shape[-1]
    tokens = torch.zeros(n, dtype=torch.int64, device=device())
    v, plain = torch.ones(n, device=device()), view.contiguous()
    calls = [
        lambda: aspis.embed(plain.view(n, d), tokens, out=view),
        lambda: aspis.embed_workspace(view, tokens, 5),
        lambda: aspis.embed_grad(view, tokens, 5),
        lambda: aspis.embed_grad(plain, tokens, n, out=view),
        lambda: aspis.dropout(view, 0.5, 1), lambda: aspis.dropout(plain, 0.5, 1, out=view),
        lambda: aspis.dropout(plain, 0.5, 1, residual=view),
        lambda: aspis.policy_workspace(view), lambda: aspis.token_logps(view, tokens),
        lambda: aspis.policy_loss(view, tokens, v, v, v),
        lambda: aspis.policy_loss(plain, tokens, v, v, v, grad=view),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(aspis.AspisError, match="equally far apart"):
            call()
            raise AssertionError(i)
    assert torch.equal(x, before)


def test_an_incoming_gradient_made_contiguous_is_taken():
    """What a mean over positions sends back, which is expanded."""
    import torch
    x = torch.randn((4, 8), generator=torch.Generator().manual_seed(1)).to(device())
    grad = x.unsqueeze(1).expand(4, 100, 8)
    tokens = (torch.arange(400, device=device()) // 100).view(4, 100)
    got = aspis.embed_grad(grad.contiguous(), tokens, 5)
    # 99 additions of a number to itself, half a step each
    assert ((got[:4] - 100 * x).abs() <= 101 * 2.0 ** -24 * 100 * x.abs()).all()
    assert (got[4] == 0).all()


def test_series_of_rows_in_several_dimensions():
    """Rows equally far apart through all leading dimensions, some of size 1."""
    import torch
    buf = torch.randn((3, 1, 4, 13), generator=torch.Generator().manual_seed(2)).to(device())
    x = buf[..., 2:10]
    assert aspis._tensors().layout(x) == (12, 8, 13)
    want = aspis.dropout(x.contiguous(), 0.3, 9, offset=5)
    assert torch.equal(aspis.dropout(x, 0.3, 9, offset=5), want)
