"""What the binding of the token-movement calls passes on when an argument is left out.  No GPU: a recorder stands in for the library."""
import pytest
import torch

from paper_2506_08027_b200 import binding as B


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name,) + args) or 0


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(B, "lib", lambda: r)
    monkeypatch.setattr(B, "_stream_for", lambda stream, *tensors: 5)
    return r


TOKENS, TOP_K, ROWS, COLS, EXPERTS = 3, 2, 256, 32, 4


def tensors():
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)
    return dict(dy=torch.zeros(TOKENS, COLS, dtype=torch.bfloat16), src=torch.zeros(ROWS, COLS), row_of=ints(TOKENS, TOP_K), slot_of=ints(ROWS),
                weights=torch.zeros(TOKENS, TOP_K), group_offsets=ints(EXPERTS + 1), d_src=torch.zeros(ROWS, COLS), d_weights=torch.zeros(TOKENS, TOP_K))


@pytest.mark.parametrize("without", [(), ("weights",), ("src", "d_weights"), ("d_src", "slot_of"), ("d_src", "group_offsets"), ("d_src", "slot_of", "group_offsets"),
                                     ("d_src", "slot_of", "group_offsets", "weights")])
def test_either_gradient_alone_needs_only_its_own_arrays(recorder, without):
    t = tensors()
    for name in without:
        t[name] = None
    B.mxfp8_moe_combine_grad(**t)
    at = {k: None if v is None else v.data_ptr() for k, v in t.items()}
    assert recorder.calls == [("mxfp8_moe_combine_grad", at["dy"], B.BF16, TOKENS, COLS, at["src"], B.FP32, ROWS, at["row_of"], at["slot_of"], TOP_K, at["weights"],
                               at["group_offsets"], 1 if t["group_offsets"] is None else EXPERTS, at["d_src"], at["d_weights"], 5)]


def test_the_gradient_refuses_arrays_that_do_not_agree(recorder):
    def call(**other):
        B.mxfp8_moe_combine_grad(**{**tensors(), **other})
    for wrong in (dict(src=torch.zeros(ROWS, COLS + 1)), dict(d_src=torch.zeros(ROWS + 128, COLS)), dict(d_src=torch.zeros(ROWS, COLS, dtype=torch.bfloat16)),
                  dict(slot_of=torch.zeros(ROWS - 1, dtype=torch.int32)), dict(row_of=torch.zeros(TOKENS + 1, TOP_K, dtype=torch.int32), weights=None, d_weights=None),
                  dict(src=None, d_weights=None, d_src=torch.zeros(ROWS, COLS + 1)), dict(src=None, d_src=None),
                  dict(src=None, d_weights=None, slot_of=torch.zeros(ROWS + 1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call(**wrong)
    for wrong in (dict(weights=torch.zeros(TOKENS, TOP_K + 1)), dict(d_weights=torch.zeros(TOKENS, TOP_K, dtype=torch.float64)),
                  dict(slot_of=torch.zeros(ROWS, dtype=torch.int64)), dict(group_offsets=torch.zeros(EXPERTS + 1))):
        with pytest.raises(TypeError):
            call(**wrong)
    assert recorder.calls == []
