"""What the binding allocates for a call on a given stream comes from that
stream's memory: memory of another stream could be handed out again, by that
stream's next allocation, while the call still writes it.  No GPU needed: the
library and torch's allocator are stand-ins that record."""
import contextlib

import pytest
import torch

from paper_2608_10362_amd import binding

CURRENT, SIDE = 1, 2  # stream handles


class Stream:
    def __init__(self, handle):
        self.cuda_stream, self.waited = handle, []

    def wait_stream(self, other):
        self.waited.append(other.cuda_stream)


class Memory:
    """Stands for a device tensor: the stream it was allocated for, and those it is recorded on."""
    made = []

    def __init__(self, shape, stream, dtype):
        self.shape, self.of, self.dtype, self.recorded = shape, stream, dtype, set()
        Memory.made.append(self)

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return 1 << 30

    def record_stream(self, stream):
        self.recorded.add(stream.cuda_stream)


class Library:
    """Every entry point succeeds; sizes are 256; the stream of each launch is kept."""
    def __init__(self):
        self.launched = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes") or name.endswith("_fp8"):
                if not name.startswith("specdec_kv_init"):
                    return 256
            if name == "specdec_kv_state_count":
                return 12
            self.launched.append((name, args[-1]))
            return 0
        return call


@pytest.fixture
def stand_in(monkeypatch):
    now = [CURRENT]

    @contextlib.contextmanager
    def on(stream):
        was, now[0] = now[0], (now[0] if stream is None else stream.cuda_stream)
        yield
        now[0] = was

    lib = Library()
    Memory.made = []
    monkeypatch.setattr(binding, "lib", lambda: lib)
    monkeypatch.setattr(binding, "_stream", lambda s: now[0] if s is None else s.cuda_stream)
    for name in ("_dev", "_on_current", "_same_device"):
        monkeypatch.setattr(binding, name, lambda *a, **k: 0)
    make = lambda shape, dtype=None, device=None, **k: Memory(shape, now[0], dtype)  # noqa: E731
    for name in ("empty", "zeros"):
        monkeypatch.setattr(torch, name, make)
    monkeypatch.setattr(torch, "empty_like", lambda t: Memory(t.shape, now[0], t.dtype))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream(now[0]))
    return lib


def _kv():
    kv = binding.KVCache.__new__(binding.KVCache)
    kv.kv, kv.data = binding.KV(), torch.ones(1)
    kv.kv.batch, kv.kv.n_kv_heads, kv.kv.head_dim, kv.kv.dtype = 2, 1, 32, binding.SPECDEC_FP8
    return kv


F, I = torch.ones(4, dtype=torch.float32), torch.ones(4, dtype=torch.int32)
CALLS = {
    "attention": lambda s: binding.specdec_attention(_kv(), 0, torch.ones(2, 1, 1, 32), torch.ones(2, 1, 1, 32), stream=s),
    "sample_logits": lambda s: binding.specdec_sample_logits(torch.ones(2, 8), out=torch.ones(2, dtype=torch.int32), stream=s),
    "accept": lambda s: binding.specdec_accept(1, 1, 4, 1, 0.0, F, None, I, 1, None, 0, 0, I, I, stream=s),
    "read_context": lambda s: _kv().read_context(0, 0, 0, 3, stream=s),
}


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("stream,handle", [(None, CURRENT), (Stream(SIDE), SIDE)], ids=["current", "given"])
def test_a_calls_own_memory_belongs_to_its_stream(stand_in, call, stream, handle):
    CALLS[call](stream)
    assert [s for _, s in stand_in.launched] == [handle]
    assert Memory.made and all(m.of == handle for m in Memory.made)
    if call == "read_context":  # (what goes back to the caller is kept for the caller's stream too)
        assert all(m.recorded >= {CURRENT} or m.of == CURRENT for m in Memory.made)


class Waits(Library):
    """Keeps what the launch stream had waited for at each launch."""
    def __init__(self, stream):
        super().__init__()
        self.stream, self.before = stream, []

    def __getattr__(self, name):
        call = super().__getattr__(name)

        def noted(*args):
            if not name.endswith("_bytes"):
                self.before.append((name, list(self.stream.waited)))
            return call(*args)
        return noted


@pytest.mark.parametrize("fp8", [False, True], ids=["KVCache", "Fp8KVCache"])
def test_a_caches_set_up_waits_for_what_made_its_memory(stand_in, monkeypatch, fp8):
    """The buffers are the current stream's (which may still have work in memory it hands
    out again, and zeroes the state): a set-up on another stream comes after that."""
    side = Stream(SIDE)
    lib = Waits(side)
    monkeypatch.setattr(binding, "lib", lambda: lib)
    model = binding.Model.__new__(binding.Model)
    model.workspace, model.n_layers, model.handle, model.max_rows = torch.ones(1), 1, 0, 16
    model.desc = binding.ModelDesc()
    (binding.Fp8KVCache if fp8 else binding.KVCache)(model, 1, 64, stream=side)
    init = [w for name, w in lib.before if name.startswith("specdec_kv_init")]
    assert init == [[CURRENT]]
    assert all(m.of == CURRENT for m in Memory.made)
