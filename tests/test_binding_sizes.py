"""CPU checks that the binding refuses sizes past the C arguments' 32 bits, before
anything is called (stand-ins for tensors that no machine here holds)."""
import math

import pytest
import torch

PAST = [2 ** 31, 2 ** 32, 2 ** 32 + 5]


class Big:
    """A contiguous device tensor by what the binding asks it."""

    def __init__(self, *shape, dtype=torch.int32):
        self.shape, self.dtype = shape, dtype
        self.nbytes = 1 << 60

    def numel(self):
        return math.prod(self.shape)

    def dim(self):
        return len(self.shape)

    def data_ptr(self):
        return 16


@pytest.fixture
def api(monkeypatch):
    from paper_2506_01979_amd import api as A

    def called(*a):
        raise AssertionError("a call went to the library")
    for name in ("sb_count_tokens", "sb_count_step", "sb_linear_pack", "sb_linear_quantized", "sb_shape_logits"):
        monkeypatch.setattr(A.lib, name, called)
    monkeypatch.setattr(A, "_need", lambda *a: None)
    monkeypatch.setattr(A, "_stream_on", lambda *a: 0)
    return A


@pytest.mark.parametrize("n", PAST)
def test_sizes_past_32_bits_are_refused(api, n):
    ok, big, res = Big(64), Big(n), Big(300)
    f32 = torch.float32
    for call in (lambda: api.sb_count_tokens(big, ok), lambda: api.sb_count_tokens(big, ok, accumulate=False),
                 lambda: api.sb_count_tokens(ok, big), lambda: api.sb_count_step(big, res, ok),
                 lambda: api.sb_count_step(ok, res, big), lambda: api.sb_linear_pack(Big(n, 8), ok),
                 lambda: api.sb_linear_pack(Big(8, n), ok),
                 lambda: api.sb_linear_quantized(ok, Big(n, 8, dtype=f32), Big(n, 8, dtype=f32), ok),
                 lambda: api.sb_linear_quantized(ok, Big(4, n, dtype=f32), Big(4, 8, dtype=f32), ok),
                 lambda: api.sb_linear_quantized(ok, Big(4, 8, dtype=f32), Big(4, n, dtype=f32), ok),
                 lambda: api.sb_shape_logits(api.LogitRules(), ok, [-1], Big(1, n), Big(1, n), 1.0, ok, ok),
                 lambda: api.LogitRules(mask=Big(2, n)),
                 lambda: api.sb_linear_packed_bytes(n, 8), lambda: api.sb_linear_workspace_bytes(8, n, 1),
                 lambda: api.sb_shape_workspace_bytes(n, 1)):
        with pytest.raises(ValueError):
            call()
