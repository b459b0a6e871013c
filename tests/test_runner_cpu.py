"""The path over buffers, with a stand-in for the library: which of its calls the buffers' form asks for."""
import types

import pytest

from paper_2609_34555_b200.irq import CudaNormal
from paper_2609_34555_b200.runner import RecallPath


class Calls:
    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        return lambda *args, **kw: self.made.append(name)


def buffers(**kw):
    names = ("pool", "block_table", "slot_block", "slot_stamp", "digest", "sel_slots", "sel_blocks", "sel_count", "recall_list", "recall_count")
    return types.SimpleNamespace(**dict.fromkeys(names), **kw)


@pytest.mark.parametrize("kw,suffix", [(dict(), ""), (dict(kv_bits=16), ""), (dict(kv_bits=4), "_kv4")])
def test_calls_by_the_form_of_the_blocks(kw, suffix):
    """Buffers of a program's own, which say nothing of their form, hold bf16 blocks."""
    path = object.__new__(RecallPath)
    path.pi = Calls()
    buf = buffers(**kw)
    path.recall(0, buf, None, None, None)
    path.append(0, 1, buf, None, None, None, None)
    path.attention(0, buf, None, None, None)
    assert path.pi.made == [{"": "recall_gather_scatter"}.get(suffix, "recall_kv4"), {"": "append_kv"}.get(suffix, "append_kv4"), "sparse_decode_attn" + suffix]
    normal = object.__new__(CudaNormal)
    normal.pi, normal.buf, normal.q, normal.ctx, normal.out, normal.stream = Calls(), buf, None, None, None, None
    normal.torch = types.SimpleNamespace(cuda=types.SimpleNamespace(Event=lambda: types.SimpleNamespace(record=lambda stream: None)))
    normal.enqueue_attention(0)
    assert normal.pi.made == ["sparse_decode_attn" + suffix]
