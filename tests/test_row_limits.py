"""The row operators at the ends of what their arguments can say, without a GPU: stand-ins of tensors whose addresses are never read."""
import pytest
import torch

import paper_2605_05802_amd as sr

MANY = 1 << 32                         # its low 32 bits are 0: no rows


class Stub:
    """What the binding asks a tensor for."""
    is_cuda = True
    nbytes = 1 << 40

    def __init__(self, *shape, dtype=torch.float32):
        self.shape, self.dtype = torch.Size(shape), dtype

    def numel(self):
        return self.shape.numel()

    def stride(self, d=None):
        s = [1]
        for n in self.shape[:0:-1]:
            s.insert(0, s[0] * n)
        return tuple(s) if d is None else s[d]

    def dim(self):
        return len(self.shape)

    def data_ptr(self):
        return 4096 * (1 + id(self) % 997)

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0


@pytest.fixture
def on_any_device(monkeypatch):
    monkeypatch.setattr(sr, "_launch_on", lambda *a: 0)


def f(*shape, dtype=torch.float32):
    return Stub(*shape, dtype=dtype)


def i4(n):
    return Stub(n, dtype=torch.int32)


WS = Stub(1 << 20, dtype=torch.uint8)
BEYOND = {
    "embed, tokens": lambda: sr.sr_embed(f(10, 1), i4(MANY), f(MANY, 1)),
    "embed, vocabulary": lambda: sr.sr_embed(f(MANY + 10, 1), i4(0), f(0, 1)),
    "embed, just beyond": lambda: sr.sr_embed(f(10, 1), i4(1 << 31), f(1 << 31, 1)),
    "embed_grad, tokens": lambda: sr.sr_embed_grad(f(MANY, 1), i4(MANY), f(10, 1), WS, accumulate=True),
    "embed_grad, vocabulary": lambda: sr.sr_embed_grad(f(0, 1), i4(0), f(MANY + 10, 1), WS, accumulate=True),
    "dropout, rows": lambda: sr.sr_dropout(f(MANY, 1), f(MANY, 1), sr.Dropout(0.1, 1)),
    "dropout, columns": lambda: sr.sr_dropout(f(0, MANY + 4), f(0, MANY + 4), sr.Dropout(0.1, 1)),
    "add_norm, rows": lambda: sr.sr_add_norm(f(MANY, 1), f(1), f(MANY, 1)),
    "add_norm_grad, rows": lambda: sr.sr_add_norm_grad(f(MANY, 1), f(MANY, 1), f(MANY), f(1), None, d_x=f(MANY, 1)),
}


@pytest.mark.parametrize("call", BEYOND)
def test_sizes_that_32_bits_do_not_hold_are_refused(on_any_device, call):
    """Not taken modulo 2^32: 2^32 + 5 rows are no call of five."""
    with pytest.raises(sr.SrError, match=r"2\*\*31 - 1") as e:
        BEYOND[call]()
    assert e.value.status == sr.SR_E_LIMIT


@pytest.fixture
def without_a_stream(monkeypatch):
    monkeypatch.setattr(sr, "_stream", lambda stream: 0)


f8 = lambda n: Stub(n, dtype=torch.float64)
BEYOND_BEFORE = {                      # the entry points of the update step and of the gate
    "grpo_loss, groups": lambda: sr.sr_grpo_loss(f8(MANY * 2), f(MANY * 2), 2, 1e-6, f(MANY * 2), f8(MANY), f8(1)),
    "grpo_loss_static, groups": lambda: sr.sr_grpo_loss_static(f8(MANY * 2), f(MANY * 2), 2, 1e-6, f(MANY * 2), f8(1)),
    "policy_loss, rows": lambda: sr.sr_policy_loss(f(MANY, 2), i4(MANY), i4(2), f(MANY), f(1), f(4), WS),
    "policy_loss, vocabulary": lambda: sr.sr_policy_loss(f(1, MANY + 2), i4(1), i4(2), f(1), f(1), f(4), WS),
    "policy_loss, sequences": lambda: sr.sr_policy_loss(f(1, 2), i4(1), i4(MANY + 2), f(1), f(MANY + 1), f(4), WS),
    "preference_loss, rows": lambda: sr.sr_preference_loss(f(MANY, 2), i4(MANY), i4(3), f(4), WS),
    "gate_batch, groups": lambda: sr.sr_gate_batch(Stub(MANY + 1, 2, 1, dtype=torch.int32), [1], 0.5, i4(MANY + 1)),
    "gate_batch, stride": lambda: sr.sr_gate_batch(Stub(1, 2, MANY + 1, dtype=torch.int32), [1], 0.5, i4(1)),
    "gate_batch_antidiag, groups": lambda: sr.sr_gate_batch_antidiag(Stub(MANY + 1, 2, 1, dtype=torch.int32), [1], 0.5, i4(MANY + 1)),
    "signals_batch, groups": lambda: sr.sr_signals_batch(Stub(MANY + 1, 2, 1, dtype=torch.int32), [1], 0.5, 0.0, f(1)),
}


class NothingCalled:
    def __getattr__(self, name):
        if name == "sr_strerror":
            return sr._lib.sr_strerror
        return lambda *a: sr.SR_OK     # what it was given has gone through ints already, or would have


@pytest.mark.parametrize("call", BEYOND_BEFORE)
def test_sizes_that_32_bits_do_not_hold_are_refused_by_the_losses_and_the_gate(without_a_stream, monkeypatch, call):
    sr.lib()
    monkeypatch.setattr(sr, "lib", NothingCalled)
    with pytest.raises(sr.SrError, match=r"2\*\*31 - 1") as e:
        BEYOND_BEFORE[call]()
    assert e.value.status == sr.SR_E_LIMIT


def test_chunks_that_32_bits_do_not_hold_are_refused(without_a_stream, monkeypatch):
    sr.lib()
    monkeypatch.setattr(sr, "lib", NothingCalled)
    c = sr.Context.__new__(sr.Context)
    c._h = 0
    tokens = Stub(1, MANY + 3, dtype=torch.int32)
    for call in (lambda: c.sr_prefill_chunk(tokens, False), lambda: c.sr_score_chunk(tokens)):
        with pytest.raises(sr.SrError, match=r"2\*\*31 - 1"):
            call()


@pytest.mark.parametrize("options", [dict(eps=None), dict(eps="1e-6"), dict(scale_block=1 << 40), dict(scale_block=-(1 << 40)), dict(scale_block=32.5)])
def test_numbers_that_the_norm_s_structure_does_not_hold_are_refused(on_any_device, options):
    with pytest.raises(sr.SrError, match="eps|scale") as e:
        sr.sr_add_norm(f(4, 64), f(64), f(4, 64), **options)
    assert e.value.status == sr.SR_E_ARG


@pytest.mark.parametrize("call", [lambda d: sr.sr_add_norm(f(4, 64), f(64), f(4, 64), dropout=d),
                                  lambda d: sr.sr_add_norm_grad(f(4, 64), f(4, 64), f(4), f(64), None, d_x=f(4, 64), dropout=d)])
@pytest.mark.parametrize("dropout", [0.1, True, "0.1", (0.1, 7)])
def test_the_norms_take_a_dropout_for_a_mask_and_nothing_else(on_any_device, call, dropout):
    with pytest.raises(sr.SrError, match="a Dropout expected"):
        call(dropout)


def test_a_torch_without_its_private_functions(monkeypatch):
    """The current device and the stream's handle by way of torch's public functions, as in the other entry points."""
    device, handle = sr._device_calls(object())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: type("Stream", (), {"cuda_stream": 4000 + device}))
    assert device is torch.cuda.current_device and handle(3) == 4003


@pytest.mark.gpu
def test_calls_by_way_of_public_functions(monkeypatch):
    table, tokens = torch.randn(9, 16, device="cuda"), torch.tensor([3, -1, 8], dtype=torch.int32, device="cuda")
    out = [torch.empty(3, 16, device="cuda") for _ in range(2)]
    sr.sr_embed(table, tokens, out[0])
    device, handle = sr._device_calls(object())
    monkeypatch.setattr(sr, "_current_device", device)
    monkeypatch.setattr(sr, "_current_handle", handle)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sr.sr_embed(table, tokens, out[1])
    side.synchronize()
    assert torch.equal(out[0], out[1])
