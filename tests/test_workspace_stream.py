"""A workspace that a call makes for itself is gone when the call returns, with its work still queued: it has to belong to the stream
that the work was given, or the next tensor of the current stream would lie in it."""

import contextlib
import re

import pytest

torch = pytest.importorskip("torch")


def test_the_workspace_belongs_to_the_stream(monkeypatch):
    from paper_2605_29986_amd import binding
    entered = []

    @contextlib.contextmanager
    def stream_context(stream):
        entered.append(stream)
        yield
        entered.append(None)

    made = []
    empty = torch.empty

    def recorded(*args, **kwargs):
        made.append(entered[-1] if entered else None)
        return empty(*args, **kwargs)

    monkeypatch.setattr(torch.cuda, "stream", stream_context)
    monkeypatch.setattr(torch, "empty", recorded)
    side = object()
    assert binding._workspace(1000, "cpu", side).numel() == 1000 and binding._workspace(3, "cpu", None).numel() == 256
    assert made == [side, None] and entered == [side, None]


def test_every_call_says_which():
    from paper_2605_29986_amd import binding
    calls = re.findall(r"(?<!def )_workspace\((.*)\)", open(binding.__file__).read())
    calls = [c for c in calls if "nbytes" not in c]
    assert len(calls) >= 7 and all(re.search(r", stream\)?( if need else None)?$", c) for c in calls), calls


@pytest.mark.gpu
def test_calls_on_a_busy_stream_keep_their_workspace():
    """The side stream is behind by some products; what the current stream writes meanwhile does not reach the calls' workspaces."""
    import paper_2605_29986_amd as lib
    gen = torch.Generator(device="cuda").manual_seed(0)
    h = torch.randn((300, 256), device="cuda", generator=gen).bfloat16()
    w = (torch.randn((3000, 256), device="cuda", generator=gen) * 0.1).bfloat16()
    t = torch.randint(0, 3000, (300,), device="cuda", generator=gen).int()
    g = torch.randn((300,), device="cuda", generator=gen)
    codes, scales = lib.cfgzip_mx4_quantize(w)
    half = h.half()
    a = torch.randn((4096, 4096), device="cuda", generator=gen)
    loss, lse = lib.cfgzip_head_loss(h, w, t)
    want = [loss, lse, *lib.cfgzip_head_loss_grad(h, w, t, lse, g), lib.cfgzip_mx4_logits(half, codes, scales)]
    out = [torch.zeros_like(x) for x in want]
    raw = lib.load_library()
    sizes = [raw.cfgzip_head_loss_workspace_bytes(300, 3000, 256, 2), raw.cfgzip_head_loss_grad_workspace_bytes(300, 3000, 256, 2),
             raw.cfgzip_mx4_logits_workspace_bytes(2, 300, 3000, 256, 2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            a @ a
    lib.cfgzip_head_loss(h, w, t, loss=out[0], lse=out[1], stream=side)
    lib.cfgzip_head_loss_grad(h, w, t, lse, g, grad_hidden=out[2], grad_weight=out[3], stream=side)
    lib.cfgzip_mx4_logits(half, codes, scales, logits=out[4], stream=side)
    over = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda.synchronize()
    for x, y in zip(out, want):
        assert torch.equal(x, y)
    assert all(bool((x == 255).all()) for x in over)
