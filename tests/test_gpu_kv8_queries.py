"""Attention over 8-bit records with queries and open keys that are not
finite: what the softmax of such logits is, whichever tokens there are."""
import kv8_ref as ref
import numpy as np
import pytest
from test_gpu_kv8 import SCALE, Stored, attend, host, ss  # noqa: F401 -- ss is the fixture

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("blk", [8, 16, 32])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("held", [1, 3])
def test_infinite_queries_over_open_tokens(ss, blk, sign, held):  # noqa: F811
    """Logits that are all +inf, all -inf or of both signs have no softmax: NaN,
    over open tokens alone too, and for no other head; without a token 0."""
    rng = np.random.default_rng(blk + held)
    s = Stored(rng, blk, 0, [held, 2 * blk + held, 2 * blk, 0], 2, 4)
    s.open_k[..., 40] = sign * ref.bf16(1 + np.abs(s.open_k[..., 40]))
    s.q[:, 1, 40], s.q[:, 6, 40], s.q[:, 7, 9] = np.inf, -np.inf, np.nan
    s.to_device()
    out = host(attend(ss, s, None, 3, with_open=True))
    want = np.zeros((4, 8), bool)
    want[:3, [1, 6, 7]] = True
    assert np.array_equal(np.isnan(out), np.broadcast_to(want[:, :, None], out.shape))
    assert (out[3] == 0).all()
    s.q[:, [1, 6, 7]] = 0  # the other heads by the formula
    for b in range(3):
        for g in range(2):
            k, v = s.tokens(b, g, range(3), int(s.len[b]) % blk)
            plain, bound = ref.attention(s.q[b, 4 * g:4 * g + 4].astype(np.float64), k, v, SCALE)
            heads = [h for h in range(4) if not want[b, 4 * g + h]]
            assert (np.abs(out[b, 4 * g:4 * g + 4] - plain) <= bound)[heads].all()


@pytest.mark.parametrize("blk", [8, 16, 32])
def test_open_keys_of_minus_infinite_logits(ss, blk):  # noqa: F811
    """An open token whose logit is -inf counts as none; one of +inf makes its heads NaN."""
    rng = np.random.default_rng(blk)
    s = Stored(rng, blk, 1, [2 * blk + 3, 3, 1, 2 * blk + 1], 2, 4)
    s.q = np.abs(s.q)
    s.open_k[0, :, 1, 5], s.open_k[1, :, 0, 5], s.open_k[2, :, 0, 5] = -np.inf, -np.inf, -np.inf
    s.open_k[3, 0, 0, 5] = np.inf
    s.to_device()
    out = host(attend(ss, s, None, 3, with_open=True)).astype(np.float64)
    assert (out[2] == 0).all() and np.isnan(out[3, :4]).all()
    for b, gone in ((0, 1), (1, 0)):
        for g in range(2):
            k, v = s.tokens(b, g, range(3), int(s.len[b]) % blk)
            keep = np.arange(len(k)) != s.nblk[b] * blk + gone
            plain, bound = ref.attention(s.q[b, 4 * g:4 * g + 4].astype(np.float64), k[keep], v[keep], SCALE)
            assert (np.abs(out[b, 4 * g:4 * g + 4] - plain) <= bound).all(), (b, g)
