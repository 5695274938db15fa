"""Which stream a cache call runs on, decided on the host (no GPU needed: torch's streams are stood in for)."""
import types

import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402


class _Streams:
    """torch.cuda's streams as far as the binding uses them; ExternalStream takes 0 for no handle and makes a stream of its own."""

    def __init__(self, monkeypatch):
        self.current = ["current"]
        monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: ("default", device))
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda at, device=None: ("external", at, device) if at else ("pool", device))
        monkeypatch.setattr(torch.cuda, "stream", self._entered)

    def _entered(self, s):
        outer = self

        class On:
            def __enter__(self):
                outer.current.append(s)

            def __exit__(self, *a):
                outer.current.pop()
        return On()


@pytest.mark.parametrize("stream,want", [(0, ("default", "cuda:0")), (4096, ("external", 4096, "cuda:0")), (None, "current")])
def test_calls_run_on_the_stream_that_they_are_given(monkeypatch, stream, want):
    streams, seen = _Streams(monkeypatch), []
    t = types.SimpleNamespace(is_cuda=True, device="cuda:0", numel=lambda: 3)
    ints = tuple(types.SimpleNamespace() for _ in range(5))

    def attention(*args):
        seen.append((streams.current[-1], args[14]))
        return "out"

    def assign(*args):
        seen.append((streams.current[-1], args[6]))
        return (0,) + ints

    monkeypatch.setattr(S, "_kv", types.SimpleNamespace(attention=attention, assign=assign))
    S.kv_attention(t, t, t, t, t, t, 1, 9, stream=stream)
    S.kv_attention(t, t, t, t, t, t, 1, 9, workspace=t, stream=stream)
    S.kv_assign(t, t, t, t, 16, 8, stream=stream)
    assert seen == [(want, None)] * 3


@pytest.mark.parametrize("stream", [0, 4096])
def test_a_given_stream_and_host_tensors_are_refused(stream):
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        S.kv_assign(z, z, torch.zeros(4, 2, dtype=torch.int32), z, 16, 8, stream=stream)
    k, cache = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        S.kv_attention(k, cache, cache, torch.zeros(1, 2, dtype=torch.int32), z[:2], z[:1], 1, 1, stream=stream)
