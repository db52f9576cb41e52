"""Forward-mode tangents and the query-tower operators, on the GPU: refused, not
dropped; without tangents a call at a forward-mode level gives what it gives
elsewhere."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2609_16175_amd as boa

pytestmark = pytest.mark.gpu


def calls():
    g = torch.Generator("cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    labels = torch.randint(40, (5,), generator=g, device="cuda")
    return [(boa.linear, [r(5, 24), r(16, 24), r(16), r(5, 16)], {}),
            (boa.linear, [r(70, 24), r(16, 24), r(16), r(70, 16)], dict(activation="gelu")),
            (lambda h, p, b: boa.softmax_xent(h, p, labels, b), [r(5, 24), r(40, 24), r(40)], {}),
            (lambda h, p, b: boa.softmax_xent(h, p, labels, b, reduction="none"), [r(5, 24), r(40, 24), r(40)], {}),
            (boa.layer_norm, [r(5, 24), r(24), r(24)], {}),
            (lambda x, f, g: boa.block_norm(x, f, g)[1], [r(5, 24), r(5, 24), r(24)], {})]


@pytest.mark.parametrize("at", range(6))
def test_tangents(at):
    f, args, kw = calls()[at]
    want = f(*args, **kw)
    with forward_ad.dual_level():
        torch.testing.assert_close(f(*args, **kw), want, rtol=2.0 ** -20, atol=2.0 ** -20)
        for i in range(len(args)):
            dual = [forward_ad.make_dual(t, torch.ones_like(t)) if k == i else t for k, t in enumerate(args)]
            with pytest.raises(NotImplementedError, match="forward mode"):
                f(*dual, **kw)
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward mode"):
                f(*dual, **kw)
