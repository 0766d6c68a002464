"""A caller's workspace of the calls on the 8-bit cache and on log probabilities is written by the GPU: it has to be dense memory of the
current device, as the other tensors of a call."""
import pytest
import torch

from paper_2605_23163_amd import binding as bd


class On:
    """Stands in for a tensor on device `index`."""
    def __init__(self, index, dense=True):
        self.index, self.dense = index, dense

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return self.dense


def test_place_and_layout():
    bd._check_workspace(None, 0)
    bd._check_workspace(On(0), 0)
    bd._check_workspace(On(3), 3)
    for w, dev in ((On(1), 0), (On(0), 1), (On(0, False), 0), (torch.empty(256, dtype=torch.uint8), 0)):
        with pytest.raises(ValueError, match="workspace"):
            bd._check_workspace(w, dev)


@pytest.mark.gpu
def test_calls_refuse_host_and_spread_memory():
    import paper_2605_23163_amd as F
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")
    q, b, batch = z(2, 8, 8, 64), z(2, 8, 2, 64), F.fdd_quant_prefix(4096, 2, 64, batch=2)
    for t in batch:
        t.view(torch.uint8).fill_(0)
    p = F.QuantPrefix(*(t[0] for t in batch))
    logits, tokens = z(2, 8, 152064), z(2, 8, dtype=torch.int32)
    calls = ((lambda ws: F.fdd_block_attn_quant(q, p, 4096, b, b, workspace=ws), F.fdd_block_attn_quant_workspace(q, p, 4096, b, b)),
             (lambda ws: F.fdd_block_attn_quant_batched(torch.stack([q, q]), batch, 4096, torch.stack([b, b]), torch.stack([b, b]), workspace=ws),
              F.fdd_block_attn_quant_batched_workspace(torch.stack([q, q]), batch, 4096, torch.stack([b, b]), torch.stack([b, b]))),
             (lambda ws: F.fdd_token_logprobs(logits, tokens, top=3, workspace=ws), F.fdd_token_logprobs_workspace(logits, top=3)))
    for call, need in calls:
        assert need > 0
        for ws in (torch.empty(need, dtype=torch.uint8), torch.empty(need, dtype=torch.uint8, pin_memory=True), z(1, dtype=torch.uint8).expand(need),
                   z(2 * need, dtype=torch.uint8)[::2]):
            with pytest.raises(ValueError, match="workspace"):
                call(ws)
        call(z(need, dtype=torch.uint8))
    torch.cuda.synchronize()
