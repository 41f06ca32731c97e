"""CPU-only checks of the block's operators at the ends of what their arguments can hold."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def e2f():
    import paper_2501_19216_amd as e
    return e


@pytest.fixture(scope="module")
def ctx(e2f):
    c = e2f.e2f_create(0, None)
    yield c
    c.close()


def test_cutoffs_and_caps_without_a_reciprocal(e2f, ctx):
    need = ctypes.c_size_t(0)

    def call(cutoff=5.0, cap=10.0):
        prm = e2f.AttentionParams(4, 4, 8, 32, cutoff, 0.3, cap, 0, 0, 0)
        size = e2f.lib.e2f_attention_backward_workspace_size(ctx.handle, ctypes.byref(prm), 10, 30, ctypes.byref(need))
        p = [ctypes.c_void_p((i + 1) << 20) for i in range(9)]
        forward = e2f.lib.e2f_attention_forward(ctx.handle, ctypes.byref(prm), p[0], None, p[1], p[2], 10, p[3], p[4],
                                                p[5], 30, p[6], p[7], None)
        assert forward == (e2f.E2F_EDEVICE if size == e2f.E2F_OK else size)
        return size

    for tiny in (2.0 ** -149, 2.0 ** -126, 2.0 ** -101):
        assert call(cap=tiny) == e2f.E2F_EINVAL and call(cutoff=tiny) == e2f.E2F_EINVAL
    assert call(cap=2.0 ** -100, cutoff=2.0 ** -100) == e2f.E2F_OK and call(cap=0.0) == e2f.E2F_OK
    assert call(cap=3e38, cutoff=3e38) == e2f.E2F_OK


def test_bindings_do_not_take_sizes_modulo_two_to_the_32(e2f, ctx):
    # tensors without memory: the call ends before their addresses are taken
    import torch
    meta = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="meta")  # noqa: E731
    many = 2 ** 32 + 4
    edges = dict(row_ptr=meta(many + 1, dtype=torch.int64), col_idx=meta(8, dtype=torch.int32))
    assert meta(1).get_device() == ctx.device
    for call in (lambda: e2f.e2f_transpose_graph(ctx, many, **edges),
                 lambda: e2f.e2f_attention_forward(ctx, meta(many, 3), **edges, cutoff=5.0, heads=4),
                 lambda: e2f.e2f_attention_forward(ctx, meta(1, 3), meta(2, dtype=torch.int64), edges["col_idx"], 5.0,
                                                   q=meta(1, many, 2), k=meta(1, many, 2)),
                 lambda: e2f.e2f_attention_forward(ctx, meta(1, 3), meta(2, dtype=torch.int64), edges["col_idx"], 5.0,
                                                   rbf_w=meta(4, many)),
                 lambda: e2f.e2f_attention_backward(ctx, meta(many, 3), **edges, cutoff=5.0, alpha=meta(8, 4),
                                                    lse=meta(many, 4), grad_alpha=meta(8, 4), heads=4),
                 lambda: e2f.e2f_block_norm_forward(ctx, meta(many, 4), 0, pre_w=meta(1, 4)),
                 lambda: e2f.e2f_block_norm_forward(ctx, meta(1, many), 0, pre_w=meta(1, many)),
                 lambda: e2f.e2f_block_norm_backward(ctx, meta(many, 4), meta(many, 2), 0, pre_w=meta(1, 4))):
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_capture_is_asked_of_the_context_s_device(e2f, monkeypatch):
    # two devices, as torch shows them: the current one, and one whose current stream is being captured
    import types

    import torch
    state = dict(current=0, capturing=1)

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, state["current"] = state["current"], self.index

        def __exit__(self, *a):
            state["current"] = self.before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: state["current"])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state["current"] == state["capturing"])
    monkeypatch.setattr(torch.cuda, "device", Device)
    for current in (0, 1):
        for device in (0, 1):
            state["current"] = current
            own = types.SimpleNamespace(device=device, stream_workspaces={})
            ask = lambda: e2f._workspace(own, None, 10, torch.device("cpu"), types.SimpleNamespace(value=7))  # noqa: E731
            if device == state["capturing"]:
                with pytest.raises(ValueError, match="capture"):
                    ask()
                assert not own.stream_workspaces
            else:
                assert ask().numel() >= 10
            assert state["current"] == current
