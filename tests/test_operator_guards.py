"""Host-side guards of the operators around the expert layer, on the CPU: what must be refused before a kernel could race on it."""
import ctypes

import pytest
import torch

from paper_2603_06626_b200 import binding as B

OK, INVALID = 0, -1
A = 1 << 20           # stands for a device address: the layout is host arithmetic


def _layout(*tensors):
    """Code of the layout of (param, grad, elements, param type, grad type) tuples."""
    desc = (B.AdamwTensor * len(tensors))(*[B.AdamwTensor(p, g, n, 0.0, pt, gt) for p, g, n, pt, gt in tensors])
    return B.load_library().grouter_adamw_layout_host(desc, len(tensors), ctypes.byref(B.AdamwLayout()), None)


def test_adamw_refuses_parameters_that_share_memory():
    far = A + (1 << 16)
    one = (A, far, 100, B.F32, B.F32)
    assert _layout(one, (A, far + 4096, 100, B.F32, B.F32)) == INVALID                  # the same tensor twice
    assert _layout(one, (A + 396, far + 4096, 8, B.F32, B.F32)) == INVALID              # its last element
    assert _layout(one, (A - 32, far + 4096, 9, B.F32, B.F32)) == INVALID               # its first
    assert _layout((A, far, 10 ** 6, B.BF16, B.F32), (A + 4000, A, 0, B.F32, B.F32), (A + 8000, 1 << 40, 2, B.F32, B.F32)) == INVALID   # inside a long one
    assert _layout(one, (A + 400, far + 4096, 8, B.F32, B.F32)) == OK                   # next to each other
    assert _layout(one, (A, far, 0, B.F32, B.F32)) == OK                                # an empty tensor has no memory


def test_adamw_refuses_a_parameter_over_a_gradient_that_others_read():
    far = A + (1 << 16)
    assert _layout((A, far, 100, B.F32, B.F32), (far + 200, far + 4096, 8, B.F32, B.F32)) == INVALID      # over another tensor's gradient
    assert _layout((A, A + 4, 100, B.F32, B.F32)) == INVALID                                              # over its own, shifted
    assert _layout((A, A - 8, 100, B.BF16, B.BF16)) == INVALID
    assert _layout((A, A, 100, B.F32, B.F32)) == OK                                                       # an element reads what it writes
    assert _layout((A, A, 100, B.BF16, B.F32), (A + 200, far, 4, B.BF16, B.BF16)) == INVALID              # its gradient goes on behind it
    assert _layout((A, far, 100, B.F32, B.F32), (A + 400, far, 100, B.F32, B.F32)) == OK                  # a gradient that two of them read


def test_the_binding_refuses_a_gradient_of_another_type_in_its_parameters_memory(monkeypatch):
    monkeypatch.setattr(B, "_device_index", lambda dev: 0)
    p, g = torch.zeros(64), torch.zeros(64)
    B.AdamW([p], [g])
    with pytest.raises(B.GrouterError):
        B.AdamW([p, p], [g, torch.zeros(64)])
    flat = torch.zeros(96)
    with pytest.raises(B.GrouterError):
        B.AdamW([flat[:64], flat[32:]], [g, g])
    half = g.view(torch.bfloat16)
    with pytest.raises(ValueError):
        B.AdamW([half[:64]], [g])
    with pytest.raises(ValueError):
        B.AdamW([g], [half[:64]])


def test_threads_that_make_a_devices_first_call_together_share_one_status_word(monkeypatch):
    """The second of two words would be freed while a kernel may still set a bit in it."""
    import threading
    import time
    started = threading.Barrier(4)
    made = []

    def zeros(*shape, **kw):
        time.sleep(0.05)                       # long enough for every other thread to come by
        made.append(torch.empty(1, dtype=torch.int32))
        return made[-1]

    monkeypatch.setattr(B, "_status_words", {})
    monkeypatch.setattr(B.torch, "zeros", zeros)
    monkeypatch.setattr(B.torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(B.torch.cuda, "synchronize", lambda index: None)
    got = [None] * 4

    def first_call(i):
        started.wait()
        got[i] = B._status_word(0)

    threads = [threading.Thread(target=first_call, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(made) == 1 and all(w is made[0] for w in got)


def test_a_status_word_is_shared_only_once_it_is_zeroed(monkeypatch):
    """Another thread's call must not get the word between its creation and the end of the zeroing."""
    monkeypatch.setattr(B, "_status_words", {})
    monkeypatch.setattr(B.torch, "zeros", lambda *shape, **kw: torch.empty(1, dtype=torch.int32))
    monkeypatch.setattr(B.torch.cuda, "is_current_stream_capturing", lambda: False)
    seen = []
    monkeypatch.setattr(B.torch.cuda, "synchronize", lambda index: seen.append(B._status_words.get(0)))
    B._status_word(0)
    assert seen == [None] and B._status_words[0] is not None


def test_adamw_keeps_no_history_of_parameters_that_require_gradients(monkeypatch):
    import copy
    monkeypatch.setattr(B, "_device_index", lambda dev: 0)
    p = [torch.nn.Parameter(torch.randn(5, 7).bfloat16()), torch.nn.Parameter(torch.randn(40).bfloat16())]
    opt = B.AdamW(p, [torch.zeros(5, 7), torch.zeros(40)])
    for t in (opt.master, opt.m, opt.v):
        assert not t.requires_grad and t.is_leaf and t.grad_fn is None
    assert torch.equal(copy.deepcopy(opt.master)[64:104], p[1].detach().float()) and (opt.master.numpy()[35:64] == 0).all()


class _Word:
    """A status word on which another thread's kernel sets a bit right after it has been read."""

    def __init__(self, before, after):
        self.value, self.after = before, after

    def item(self):
        seen, self.value = self.value, self.value | self.after
        return seen

    def zero_(self):
        self.value = 0

    def bitwise_and_(self, keep):
        self.value &= keep


def test_a_check_clears_only_the_bits_that_it_reports(monkeypatch):
    word = _Word(0, 2)
    monkeypatch.setattr(B, "_device_index", lambda dev: 0)
    monkeypatch.setattr(B, "_status_words", {0: word})
    monkeypatch.setattr(B.torch.cuda, "synchronize", lambda index: None)
    B.check_status()                                     # nothing had been found
    assert word.value == 2
    word.after = 1
    with pytest.raises(B.GrouterError) as e:
        B.check_status()
    assert e.value.code == -7 and word.value == 1        # the wait that ran out is reported, the id that came after is not lost
    word.after = 0
    with pytest.raises(B.GrouterError) as e:
        B.check_status()
    assert e.value.code == -6 and word.value == 0


def test_the_block_says_what_its_sizes_have_to_be():
    from paper_2603_06626_b200.block import RoutedBlock
    for name in ("T", "d", "ffn", "E", "hidden"):
        sizes = dict(T=64, d=64, ffn=64, E=8, k=2, hidden=64)
        sizes[name] += 4
        with pytest.raises(ValueError, match=f"^{name}: a multiple of 8"):
            RoutedBlock(**sizes)


def test_losses_without_ids_are_not_held_to_the_ids_limits():
    """E up to 1024: the limit of 256 is that of 8-bit ids, and none are given here."""
    def bal(idx, E, T=0):
        return B.load_library().grouter_balance_loss(A, E, B.F32, idx, B.IDX_U8, None, A, A, None, B.NORM_SOFTMAX, T, E, 1, 0.1, 0.1, None, None, A, None,
                                                     None, None)
    assert bal(None, 256) == OK and bal(None, 257) == OK and bal(None, 1024) == OK
    assert bal(A, 257) == -3 and bal(None, 1025) == -3


def test_the_block_checks_its_batch_before_a_kernel_reads_it():
    """The plan and the layer take addresses: a shorter batch would be read past its end."""
    from paper_2603_06626_b200.block import RoutedBlock
    block = object.__new__(RoutedBlock)
    block.T, block.d, block.status = 64, 32, torch.zeros(1, dtype=torch.int32)
    for call, name in ((block.forward, "x"), (block.backward, "dout")):
        for bad in (torch.zeros(56, 32), torch.zeros(72, 32), torch.zeros(64, 24)):
            with pytest.raises(ValueError, match=f"^{name}: shape"):
                call(bad.bfloat16())
        with pytest.raises(TypeError, match=f"^{name}: torch.bfloat16"):
            call(torch.zeros(64, 32))
        with pytest.raises(ValueError, match=f"^{name}: a contiguous"):
            call(torch.zeros(32, 64, dtype=torch.bfloat16).t())


def test_a_check_of_a_given_word_waits_for_that_words_device(monkeypatch):
    waited = []
    monkeypatch.setattr(B, "_device_index", lambda dev: dev.index if dev.index is not None else 5)
    monkeypatch.setattr(B.torch.cuda, "synchronize", lambda index: waited.append(index))
    B.check_status(status=torch.zeros(1, dtype=torch.int32))       # stands for one on another device than the default, cuda:0
    assert waited == [5]
