"""What a segment's gradient may depend on."""
import pytest
import torch

from test_gpu_xattn import cu_tensor, inputs, u  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,kv_heads,d", [(8, 2, 64), (4, 4, 128)])
def test_short_prompts_beside_long_ones(u, heads, kv_heads, d, dtype):  # noqa: F811
    """dQ of a segment, to the bit, is the one that it gets alone, whatever the lengths beside it."""
    lq, lk = [200, 90, 33, 300], [10, 1000, 77, 128]
    q, k, v, dout = inputs(lq, lk, heads, kv_heads, d, dtype, seed=d)
    how = dict(cu_q=cu_tensor(lq), cu_k=cu_tensor(lk))
    out, lse = u.ut_xattn_fwd(q, k, v, **how)
    dq = u.ut_xattn_bwd(q, k, v, out, lse, dout, **how)[0]
    for s in range(len(lq)):
        a, b = sum(lq[:s]), sum(lk[:s])
        rows, keys = slice(a, a + lq[s]), slice(b, b + lk[s])
        alone = u.ut_xattn_bwd(q[rows], k[keys], v[keys], out[rows], lse[:, rows].contiguous(), dout[rows])[0]
        assert torch.equal(dq[rows], alone), s
