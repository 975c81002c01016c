"""What a call of the norm and rotation takes from its arguments, and leaves in them."""
import threading

import pytest
import torch

import paper_2502_01941_b200 as skv
from paper_2502_01941_b200 import binding
from test_norm_rope_gpu import Layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2502_01941_b200.build import build_library
    build_library()
    c = skv.Context(0)
    yield c
    c.close()


@pytest.fixture(params=["module", "ctypes"])
def way(request, monkeypatch):
    assert binding._native is not None or skv.lib()
    if request.param == "ctypes":
        monkeypatch.setattr(binding, "_native", None)


def test_the_description_is_read_only(ctx, way):
    """One description serves calls on tensors of other strides and other tables."""
    layers = [Layer(2, 1, 8, 2, 64, 30, 5, 3, 20, 32, fused=fused, given=given) for fused, given in ((True, False), (False, True), (True, True))]
    rope = layers[0].rope
    before = bytes(rope)
    for s in layers:
        s.rope = rope
        s.run(ctx)
        assert bytes(rope) == before
        s.check()
    bad = layers[0]
    bad.table = bad.table[:, :3].contiguous()
    with pytest.raises(ValueError, match="cos_sin"):
        bad.run(ctx)
    assert bytes(rope) == before


def test_threads_share_a_description(way):
    """Two threads with a context and a stream each, one description, tensors of different strides and tables of different lengths."""
    rope = skv.make_rope(rows=40, rot=64, first=2)
    errors = []

    def work(seed):
        try:
            torch.cuda.set_device(0)
            c, stream = skv.Context(0), torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for i in range(60):
                    s = Layer(2, 1, 8, 2, 64, 50, 9, 2, 40, 64, fused=bool(seed), given=bool(seed), seed=i)
                    s.rope = rope
                    s.eps = rope.eps
                    s.run(c)
                    stream.synchronize()
                    s.check()
            c.close()
        except BaseException as e:                          # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors[0]


def test_positions_are_those_of_every_prompt_and_row(ctx, way):
    """One row of positions for all prompts is not expanded: it is refused, as is any other number of them."""
    s = Layer(2, 1, 8, 2, 64, 50, 9, 2, 40, 64, given=True)
    good = s.positions
    for bad in (good[:1], good[0], good[:, :39].contiguous(), torch.cat([good, good[:1]]), good[:0]):
        s.positions = bad
        with pytest.raises(ValueError, match="positions"):
            s.run(ctx)
    for bad in ([0] * 80, good.long(), good.float()):
        s.positions = bad
        with pytest.raises(TypeError, match="positions"):
            s.run(ctx)
    for same in (good, good.flatten()):
        s.positions = same
        s.K.fill_(7), s.V.fill_(7), s.Qwin.fill_(7)
        s.run(ctx)
        s.positions = good
        s.check()
