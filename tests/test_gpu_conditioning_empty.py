"""The conditioning block where nothing is retained, or there is nothing to attend to."""
import pytest
import torch

from test_gpu_conditioning import IMAGES, TOKENS, H, HK, D, GROUPS, inputs, u  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("empty", ["tokens", "states"])
def test_block_without_tokens_or_states(u, empty, dtype):  # noqa: F811
    from paper_2609_23169_gb300.conditioning import ConditioningBlock
    mask, x, states, cu, key_mask, w, dy = inputs(dtype)
    if empty == "tokens":
        mask = torch.zeros_like(mask)
    else:
        states, cu, key_mask = states[:0], torch.zeros_like(cu), key_mask[:0]
    block = ConditioningBlock(IMAGES, TOKENS, H, HK, D, GROUPS)
    status = u.status_word()
    y = block.forward(mask, x, states, cu, w, key_mask, status)
    dx, dstates, g = block.backward(dy, status)
    u.check_status(status)
    assert torch.equal(y, x) and torch.equal(dx, dy) and dstates.shape == states.shape and not dstates.any()
    for t, ref in zip((g.gamma, g.beta, g.wq, g.wkv, g.wo), (w.gamma, w.beta, w.wq, w.wkv, w.wo)):
        assert t.shape == ref.shape and not t.any()


def test_scatter_and_compaction_of_no_rows(u):  # noqa: F811
    """Empty lists of rows have no row size to compare."""
    x = torch.randn(6, 24, device="cuda")
    y = x.clone()
    idx = torch.empty(0, dtype=torch.int32, device="cuda")
    u.ut_fg_scatter(idx, 0, [x[:0]], [y], u.UT_BG_KEEP)
    assert torch.equal(x, y)
    u.ut_fg_scatter(idx, 0, [x[:0]], [y], u.UT_BG_ZERO)
    assert not y.any()
    status = u.status_word()
    _, n, (out,) = u.ut_fg_compact(torch.zeros(6, dtype=torch.uint8, device="cuda"), [x], capacity=0, status=status)
    u.check_status(status)
    assert int(n) == 0 and out.shape == (0, 24)
