"""The workspace that a call of the shared prefix's attention allocates is its stream's (no GPU needed; see
test_binding_streams)."""
import pytest
import torch

from paper_2608_10362_amd import binding
from tests.test_binding_streams import CURRENT, SIDE, Memory, Stream, _kv, stand_in  # noqa: F401


@pytest.mark.parametrize("stream,handle", [(None, CURRENT), (Stream(SIDE), SIDE)], ids=["current", "given"])
def test_a_calls_own_memory_belongs_to_its_stream(stand_in, stream, handle):  # noqa: F811
    q = torch.ones(2, 1, 1, 32)
    binding.specdec_attention_shared(_kv(), _kv(), 0, q, torch.ones(2, 1, 1, 32), stream=stream)
    assert [s for _, s in stand_in.launched] == [handle]
    assert Memory.made and all(m.of == handle for m in Memory.made)
