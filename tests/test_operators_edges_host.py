"""Host side of the learner-side operators where it meets more than one device or stream; nothing here needs a GPU."""
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_11125_b200", "csrc")


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def test_nothing_of_a_device_is_kept_for_the_process():
    """What a call asks of the runtime (attributes it sets, blocks that fit) holds for the device it was asked on. A variable of static
    storage that is initialised by such a call would hand the first device's answer to a handle on another."""
    for name in ("operators.cu", "layer_norm.cuh", "ns_small.cuh", "ffn_tokens.cuh", "tc_product.cuh", "operand_prep.cuh", "ops_common.cuh"):
        for line in re.findall(r"\bstatic\b[^;{]*=[^;]*;", _code(name)):
            assert not re.search(r"\bcuda[A-Z]\w*\s*\(|\bresident\s*\(|\bo->", line), "%s: %s" % (name, line.strip())
    # and the limit that the layer norm's backward pass needs is raised where a handle is made
    create = _code("operators.cu").split("int scalecom_ops_create(")[1].split("void scalecom_ops_destroy(")[0]
    for kind in ("float", "__half", "__nv_bfloat16"):
        assert "ln_attributes<%s>()" % kind in create


class _Elsewhere:
    """A stand-in for a CUDA tensor of device `dev`: what the binding looks at, and an address that nothing may follow."""
    def __init__(self, dev, *shape, dtype=torch.float32):
        self.dev, self.shape, self.dtype, self.is_cuda = dev, torch.Size(shape), dtype, dev >= 0

    def get_device(self):
        return self.dev

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def stride(self):
        return tuple(torch.Size(self.shape[i + 1:]).numel() for i in range(len(self.shape)))

    def unsqueeze(self, _):
        return _Elsewhere(self.dev, 1, *self.shape, dtype=self.dtype)

    def data_ptr(self):
        return 256


def _calls(ops):
    """name, call, its tensors by name"""
    r, w, h = 4, 8, 6
    v = lambda *s: lambda dev: _Elsewhere(dev, *s)      # noqa: E731
    yield ops.layer_norm, dict(x=v(r, w), gamma=v(w), beta=v(w), y=v(r, w), mean=v(r), rstd=v(r)), dict(eps=1e-5)
    yield ops.layer_norm_backward, dict(dy=v(r, w), x=v(r, w), gamma=v(w), mean=v(r), rstd=v(r), dx=v(r, w), dgamma=v(w), dbeta=v(w)), {}
    block = dict(x=v(r, w), w_gate=v(h, w), w_up=v(h, w), w_down=v(w, h), saved=v(2, r, h))
    yield ops.gated_ffn, dict(block, y=v(r, w)), {}
    yield ops.gated_ffn_backward, dict(block, dy=v(r, w), dx=v(r, w), dw_gate=v(h, w), dw_up=v(h, w), dw_down=v(w, h)), {}
    yield ops.orthogonalise, dict(update=v(r, w), out=v(r, w)), {}


def test_a_tensor_of_another_device_is_refused():
    """The handle's kernels would follow its address on their own device."""
    from paper_2104_11125_b200.operators import Operators
    ops, reached = Operators.__new__(Operators), []
    ops._h, ops._device = None, 1
    for name in ("layer_norm", "layer_norm_backward", "gated_ffn", "gated_ffn_backward", "orthogonalise"):
        setattr(ops, "_" + name, lambda *a: reached.append(a) or 0)
    for call, tensors, more in _calls(ops):
        here = {k: make(1) for k, make in tensors.items()}
        del reached[:]
        call(**here, **more)
        assert len(reached) == 1
        for k, make in tensors.items():
            for dev in (0, -1):
                with pytest.raises(TypeError):
                    call(**dict(here, **{k: make(dev)}), **more)
        assert len(reached) == 1
