"""Keys of the 4-bit append whose products with the norm's weights are past fp32 (GPU): the
definition's 64 bits hold them, and words and grids equal the oracle's, bit for bit.  Norms of fp32
would need squares below 2^128; these run in 64 bits, where bf16 values cannot leave the range."""

import numpy as np
import pytest
import torch

from oracle import lowbit_ref as low
from oracle import target_ref as ref
from paper_2607_04244_amd import qlin

from test_kv4 import HEAD, Cache, bits, f64, i32, rand, words_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [3, 650])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, True), (48, False), (0, False)])
@pytest.mark.parametrize("x,w", [(120, 0), (120, 12), (126, 30), (100, 100), (-100, -40), (-60, -90), (0, 0)])
def test_keys_and_weights_of_all_sizes(x, w, rot, interleaved, rows):
    """Keys of about 2^x and weights of about 2^w, whose product goes from 2^-150 to 2^200: keys of
    size 2^w are stored."""
    k = (rand(1, (rows, 2 * HEAD)).double().clamp(-1.9, 1.9) * 2.0 ** x).to(torch.bfloat16)
    wk = ((1 + rand(2, (HEAD,), 0.2)).double() * 2.0 ** w).to(torch.bfloat16)
    assert torch.isfinite(k).all() and torch.isfinite(wk).all()
    v = rand(3, (rows, 2 * HEAD))
    freq = 1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))
    c = Cache("heads", [rows + 7], 2, 4)
    qlin.norm_rope_append_kv4(v.cuda(), k.cuda(), v.cuda(), c.dev, i32([0, rows]), i32([rows + 7]), k_norm=wk.cuda(), eps=0.0,
                              inv_freq=freq.cuda() if rot else None, interleaved=interleaved)
    torch.cuda.synchronize()
    for m in range(rows):
        y = low.to_bf16(ref.rotate(ref.norm(f64(k[m]).reshape(2, HEAD), f64(wk), 0.0), 7 + m, freq.numpy(), interleaved))
        assert np.isfinite(y).all()
        codes, step, offset = low.lay_on_grid(y)
        assert torch.equal(c.dev[0][0, :, 7 + m].cpu(), words_of(codes)), m
        assert torch.equal(bits(c.dev[1][0, :, 7 + m]), bits(torch.from_numpy(np.stack([step, offset], -1)).to(torch.bfloat16))), m
