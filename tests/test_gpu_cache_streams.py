"""A model on a stream of the caller's: workspaces that are outgrown there."""

import numpy as np
import pytest
import torch

from paper_2606_09061_amd import model as M

pytestmark = pytest.mark.gpu

CFG = M.ModelConfig(hidden=256, layers=2, hq=4, hkv=2, head_dim=64, inter=512, vocab=1024)
FORWARD = {"all keys": {}, "groups": dict(groups=[(0, 3, 300)]), "budget": dict(budget=5)}


@pytest.mark.parametrize("how", [*FORWARD, "verify"])
def test_an_outgrown_workspace_stays_while_its_stream_is_busy(how):
    """The model and its workspaces belong to the default stream, which must not get
    their memory again while another stream, behind 100 large products, has the
    iteration that used them ahead of it."""
    m = M.Model(CFG, max_seqs=4, max_seq_len=2048, max_tokens=64, seed=3, fill_caches=True,
                page_bounds=True, lm_head=how == "verify")   # (its row indexes are a waiting copy)
    dev, side = m.dev, torch.cuda.Stream(m.dev)
    big = torch.zeros(8192, 8192, dtype=torch.bfloat16, device=dev)
    product = torch.empty_like(big)
    rows = np.array([(0, 400, 1, 401), (1, 1500, 1, 1501), (2, 1300, 1, 1301)], np.int32)
    tokens = torch.zeros(3, dtype=torch.int32, device=dev)
    parents = torch.full((3,), -1, dtype=torch.int32, device=dev)

    def run():
        if how == "verify":
            m.verify(rows, tokens, parents, stream=side)
        else:
            m.forward(rows, stream=side, **FORWARD[how])

    side.wait_stream(torch.cuda.current_stream(dev))
    run()                                         # (loads the kernels, too)
    torch.cuda.synchronize()
    want = m.x[:3].clone()
    m.ws, m.ws_gemm = (torch.empty(256, dtype=torch.uint8, device=dev) for _ in range(2))
    side.wait_stream(torch.cuda.current_stream(dev))
    old = {m.ws.data_ptr(), m.ws_gemm.data_ptr()}
    with torch.cuda.stream(side):
        for _ in range(100):
            torch.mm(big, big, out=product)
    run()
    assert m.ws.numel() > 256
    new = [torch.empty(256, dtype=torch.uint8, device=dev) for _ in range(4000)]
    grown = old - {m.ws.data_ptr(), m.ws_gemm.data_ptr()}
    busy = not side.query()
    torch.cuda.synchronize()
    assert busy and grown and not grown & {t.data_ptr() for t in new}
    assert torch.equal(m.x[:3], want)
