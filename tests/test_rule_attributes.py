"""A rule's attributes set anew between calls, and a rule that calls share: every call passes on what the rule holds then. The tensors
are stand-ins, of which nothing but their descriptions is read."""
import pytest

torch = pytest.importorskip("torch")


class Stand:
    is_cuda = True

    def __init__(self, n, at, dtype=torch.int32, gpu=0):
        self.shape, self.at, self.dtype, self.gpu = (n,), at, dtype, gpu

    def dim(self):
        return 1

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at

    def get_device(self):
        return self.gpu


def test_an_attention_rule_follows_its_attributes():
    from paper_2605_30852_amd.cache import AttentionRule
    r = AttentionRule(cap=5.0, window=3, slopes=Stand(8, 64, torch.float32), first=Stand(7, 128), open_lens=Stand(2, 256))
    c = r.check(7, 2, 8, 0)
    assert (c.cap, c.window, c.slopes, c.first, c.open_lens) == (5.0, 3, 64, 128, 256)
    r.cap, r.window, r.slopes, r.first, r.open_lens = 6.0, 0, None, Stand(9, 512), Stand(3, 1024)
    c = r.check(9, 3, 8, 0)
    assert (c.cap, c.window, c.slopes, c.first, c.open_lens) == (6.0, 0, None, 512, 1024)
    r.first.at = 2048  # other storage in the same tensor
    assert r.check(9, 3, 8, 0).first == 2048
    for name, bad in (("cap", -1.0), ("cap", float("nan")), ("window", -1), ("window", 1 << 31), ("first", Stand(8, 512)),
                      ("first", Stand(9, 512, torch.int64)), ("open_lens", Stand(3, 512, gpu=1)), ("slopes", Stand(8, 512))):
        old = getattr(r, name)
        setattr(r, name, bad)
        with pytest.raises(ValueError):
            r.check(9, 3, 8, 0)
        setattr(r, name, old)
    r.check(9, 3, 8, 0)


def test_a_head_rule_follows_its_attributes():
    from paper_2605_30852_amd.cache import HeadRule
    r = HeadRule(q_gain=Stand(64, 64, torch.float32), eps=1e-5)
    c = r.check(64, 0, 32)
    assert (c.q_gain, c.k_gain, c.rot, c.interleaved) == (64, None, 32, 0)
    r.q_gain, r.k_gain, r.eps, r.interleaved = None, Stand(64, 128, torch.float32), 0.5, True
    c = r.check(64, 0, 32)
    assert (c.q_gain, c.k_gain, c.eps, c.rot, c.interleaved) == (None, 128, 0.5, 32, 1)
    r.k_gain = Stand(128, 128, torch.float32)
    with pytest.raises(ValueError):
        r.check(64, 0, 32)


def test_calls_of_other_widths_have_structs_of_their_own():
    """Another thread's call may come behind whatever a call writes into the rule that both use."""
    from paper_2605_30852_amd.cache import HeadRule

    class Shared(HeadRule):
        here = False

        def __setattr__(self, name, value):
            super().__setattr__(name, value)
            if Shared.here:
                Shared.here = False
                self.check(128, 0, 128)

    r = Shared()
    kept = r.check(128, 0, 128)
    Shared.here = True
    assert r.check(128, 0, 64).rot == 64
    Shared.here = False
    assert kept.rot == 128
