"""The stream that a block's contribution waits for, on the CPU: a stand-in for
a stream, and a block whose results are there only once it has been waited for."""
import torch

from paper_2205_11048_amd import worker


class _Stream:
    """Does its pending work when it is waited for."""

    def __init__(self, work):
        self.work, self.cuda_stream = work, 7

    def synchronize(self):
        self.work()


def _block(monkeypatch):
    block = object.__new__(worker.EmbeddingBlock)
    block._words = torch.tensor([9, 0])
    block.num_unique, block.err = block._words[:1], block._words[1:].view(torch.int32)[:1]
    block.flat, block.unique_ids, block.rows = torch.zeros(4), torch.arange(10), torch.zeros((10, 2))
    block.list = block.norm = block.workspace = block.coef = None
    block.max_norm, block._stream = 1.0, None
    monkeypatch.setattr(worker, "gba_clip_grads", lambda *a, **kw: None)
    return block


def test_the_contribution_waits_for_the_steps_stream(monkeypatch):
    block = _block(monkeypatch)
    block.clip(stream=_Stream(lambda: block.num_unique.fill_(4)))
    flat, ids, rows = block.contribution()
    assert ids.tolist() == [0, 1, 2, 3] and rows.shape == (4, 2)


def test_the_contribution_waits_for_the_stream_it_is_given(monkeypatch):
    block = _block(monkeypatch)
    block.clip(stream=_Stream(lambda: block.num_unique.fill_(4)))
    assert block.contribution(stream=_Stream(lambda: block.num_unique.fill_(2)))[1].tolist() == [0, 1]
