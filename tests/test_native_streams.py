"""Where the decoder's convenience call allocates."""
import contextlib

import pytest

from paper_2609_16874_amd import native

torch = pytest.importorskip("torch")


class Stream:
    cuda_stream = 77


@pytest.mark.parametrize("given", [True, False])
def test_outputs_are_allocated_on_the_stream_that_decodes(given, monkeypatch):
    streams, seen = [], []

    @contextlib.contextmanager
    def on(stream):
        streams.append(stream)
        yield
        streams.pop()

    def new_outputs(device="cuda", score=False):
        seen.append(streams[-1] if streams else None)
        return dict.fromkeys(("centroids", "num_centroids", "labels", "score_map"))

    d = object.__new__(native.Decoder)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(d, "new_outputs", new_outputs)
    monkeypatch.setattr(d, "decode", lambda *a: native.CPE_ERR_INVALID_ARG)
    stream = Stream() if given else None
    with pytest.raises(native.CpeError):
        d.run(torch.zeros(1), torch.zeros(1), 0.5, 1.0, stream=stream)
    assert seen == [stream]


@pytest.mark.gpu
def test_decoding_on_a_side_stream_while_the_current_one_is_busy():
    import numpy as np

    from paper_2609_16874_amd import synth
    f = synth.make_frame(0)
    spec = f.spec
    fx, fy = spec.freqs()
    dec = native.Decoder(spec.H, spec.W, spec.n_freq, spec.dtype, fx, fy, spec.bins, spec.bins)
    emb, fg = torch.from_numpy(f.emb).cuda(), torch.from_numpy(f.fg).cuda()
    want = dec.run(emb, fg, spec.fg_threshold, 0.5)
    side, a = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(8):
        b = a @ a       # the current stream is busy
    scrap = torch.empty((spec.H, spec.W), dtype=torch.int32, device="cuda").fill_(7)
    del scrap, b
    got = dec.run(emb, fg, spec.fg_threshold, 0.5, stream=side)
    assert got["K"] == want["K"] and np.array_equal(got["labels"], want["labels"])
    assert np.array_equal(got["centroids"], want["centroids"])
    dec.close()
