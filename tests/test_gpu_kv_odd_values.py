"""An infinity or NaN in one element of V: rows that see the token get no finite number in that element, whatever its weight, and
nothing else changes by a bit."""
import pytest
import torch

from kv_common import KvCase, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("q_scale", [1.5, 300.0])                 # 300: most weights are zero in 32 bits
@pytest.mark.parametrize("rows,n,dim,window", [(1, 3000, 128, 0), (6, 700, 64, 0), (6, 700, 128, 90), (150, 700, 128, 0), (150, 2500, 64, 0),
                                               (150, 700, 128, 300), (40, 700, 200, 0)])
def test_one_element_of_v(bad, q_scale, rows, n, dim, window):
    make = lambda: KvCase([rows], [n], 4, 2, dim, seed=rows + dim, q_scale=q_scale)                     # noqa: E731
    want, want_lse = attend(make().device(), dim ** -0.5, True, window)
    for token in (0, 10, n - rows, n - 1 - rows // 2, n - 1):
        case = make()
        case.v5[0, case.table[0, token // 16], 1, token % 16, 5] = bad
        out, lse = attend(case.device(), dim ** -0.5, True, window)
        at = torch.arange(n - rows, n, device="cuda")
        sees = (at >= token) & ((at < token + window) if window else True)
        hit = torch.zeros((rows, 4, dim), dtype=torch.bool, device="cuda")
        hit[:, 2:, 5] = sees[:, None]                              # heads 2 and 3 share key/value head 1
        assert not torch.isfinite(out.view(rows, 4, dim)[hit]).any()
        assert torch.equal(out.view(rows, 4, dim)[~hit], want.view(rows, 4, dim)[~hit])
        assert torch.equal(lse, want_lse)
