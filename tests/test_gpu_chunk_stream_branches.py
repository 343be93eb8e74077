"""ChunkStream's branches and residuals meet in fp32, whoever keeps the page tables.

The biases after the branches lift the residual to 256 and 512 and bring it back, and norms do not
see a bias that all columns share: the result is that of the plain block, if nothing is rounded
to fewer bits on the way.  fp32 has steps of 2^-14 below 1024, far below the bars (those of
test_gpu_chunk_stream_device.py); a branch rounded to bf16 has steps of 2 at 256 and of 4 at 512, where the
results are of size 1."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from synth import generate as G                    # noqa: E402
from test_gpu_chunk_stream_device import F32, W, bf, cond_kv, reference   # noqa: E402


@pytest.fixture(scope="module")
def ec():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_02474_gb300 import echocache
    return echocache


@pytest.mark.parametrize("tables", ["host", "device", "modulated"])
def test_branches_are_not_rounded(ec, tables):
    import torch
    from paper_2608_02474_gb300.pipeline import ChunkStream
    weights = [G.block_weights(W, l) for l in range(2)]
    for w in weights:
        w["bo"], w["boc"], w["b2"] = (np.full(W.D, b, F32) for b in (256, 256, -512))
    cond, x = G.random_rows(20, W.D, seed=3), G.random_rows(60, W.D, seed=4)
    st = ChunkStream([ec.DeviceBlock.from_host(w, np.zeros((1, W.D), F32)) for w in weights], W.H, W.d, 24, n_pages=6,
                     cond_pages=2, page_tokens=16, kind=ec.CACHE_BF16, device_tables=tables != "host")
    mods = np.zeros((2, 6, W.D), F32)
    mods[:, [2, 5]] = 1                                 # gates
    st.open(5, cond_kv(ec, weights, cond))
    got = []
    for lo, hi in ((0, 24), (24, 60)):
        m = {5: torch.from_numpy(mods).cuda()} if tables == "modulated" else None
        got.append(st.step({5: bf(x[lo:hi])}, m)[5].float().cpu().numpy())
    assert ec.echo_get_device_error() == 0
    y = np.concatenate(got)
    ref = reference(G.to_bf16_values(x), weights, [G.to_bf16_values(cond)] * 2, 24, "bf16", False, None)
    rel = np.abs(y - ref).max(axis=1) / np.abs(ref).max(axis=1)
    mean = np.abs(y - ref).sum() / np.abs(ref).sum()
    assert rel.max() <= 2e-2 and mean <= 5e-3, (rel.max(), mean)
