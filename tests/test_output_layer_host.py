"""The boundary of layer norm, the 8-bit blocks of 128 and the loss against a teacher without a GPU: argument structs are the header's, NULL
handles and arguments answer with an error code, tensors that do not fit are refused before anything is called, and the
64-bit references have the properties they are defined by."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import output_layer_ref as O
import paper_1801_04928_b200 as lf
from operators_ref import D

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = ("lf_layer_norm_args", "lf_layer_norm_backward_args", "lf_pack_blocks_args", "lf_product_blocks_args", "lf_distill_args")


def test_binding_structs_are_the_headers(tmp_path):
    lines = ['printf("LF_DISTILL_MAX_TOP %d\\n", LF_DISTILL_MAX_TOP);']
    for name in STRUCTS:
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in getattr(lf, name)._fields_]
    src = tmp_path / "offsets.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "leapfrog.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    exe = tmp_path / "offsets"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    said = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(said["LF_DISTILL_MAX_TOP"]) == lf.LF_DISTILL_MAX_TOP
    for name in STRUCTS:
        cls = getattr(lf, name)
        assert int(said[name]) == ctypes.sizeof(cls), name
        for f, _ in cls._fields_:
            assert int(said[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)


def test_null_handles_and_arguments():
    for name, args in (("lf_layer_norm", "lf_layer_norm_args"), ("lf_layer_norm_backward", "lf_layer_norm_backward_args"),
                       ("lf_pack_blocks", "lf_pack_blocks_args"), ("lf_pack_tiles", "lf_pack_blocks_args"),
                       ("lf_product_blocks", "lf_product_blocks_args"), ("lf_distill", "lf_distill_args"), ("lf_distill_backward", "lf_distill_args")):
        assert getattr(lf, name)(None, getattr(lf, args)()) == lf.LF_ENULL, name
        assert getattr(lf, name)(None, None) == lf.LF_ENULL, name


def test_tensors_that_do_not_fit():
    """The native module refuses with a text that names the argument; the entry point is not reached (its address here is no function)."""
    from paper_1801_04928_b200 import _marshal as m
    x, v, i = torch.zeros(4, 136), torch.zeros(136), torch.zeros(4, 3, dtype=torch.int32)
    q, s = torch.zeros(4, 144, dtype=torch.uint8)[:, :136], torch.zeros(2, 4)

    def refused(name, argument, *a):
        status, text = getattr(m, name)(1, 1, *a, 0)
        assert status == lf.LF_EINVAL and f"argument {argument}" in text, text
    refused("layer_norm", "x", x, v, None, x, None, None, None, None, None, None, 1e-5)            # on the host
    refused("layer_norm", "x", x.double(), v, None, x, None, None, None, None, None, None, 1e-5)
    refused("layer_norm", "x", v, v, None, x, None, None, None, None, None, None, 1e-5)
    refused("layer_norm", "x", None, v, None, x, None, None, None, None, None, None, 1e-5)
    refused("layer_norm_backward", "dy", x, x, v, v, v, x, None, None, None)
    refused("pack_blocks", "x", x, q, s, None, None)
    refused("pack_tiles", "x", x.to_sparse(), q, s, None, None)
    refused("product_blocks", "a", q, s, q, s, x, None, None)
    refused("product_blocks", "d", q, s, q, s, 3, None, None)
    refused("distill", "z", x, i, torch.zeros(4, 3), v, None, None, None, 1.0)
    refused("distill_backward", "index", x, torch.zeros(4, dtype=torch.int32), torch.zeros(4, 3), None, v, None, x, 1.0)
    with pytest.raises(TypeError):
        m.distill(1, 1, x, i)
    with pytest.raises(TypeError):
        m.distill(1, 1, x, i, torch.zeros(4, 3), v, None, None, None, "warm", 0)


def test_reference_of_the_blocks():
    g = torch.Generator().manual_seed(3)
    v = torch.randn(140, 300, generator=g, dtype=D) * torch.exp2(torch.randint(-120, 100, (140, 1), generator=g).to(D))
    for tiles in (False, True):
        q, s = O.pack(v, tiles)
        got, scale = O.values(q, s, tiles), O.spread(s, 140, 300, tiles)
        assert s.shape == ((2, 3) if tiles else (3, 140))
        assert bool((torch.frexp(s)[0] == 0.5).all())
        assert bool((v.abs() <= 448 * scale).all())
        assert bool(((got - v).abs() <= 2.0 ** -4 * v.abs() + 2.0 ** -10 * scale).all())
        # no smaller scale would do
        small = s / 2
        fits = v.abs() <= 448 * O.spread(small, 140, 300, tiles)
        for j in range(3):
            b = fits[:, j * 128:(j + 1) * 128]
            assert bool((~b[:128].all() if tiles else ~b.all(1)).all())


def test_reference_of_the_loss_is_its_definition():
    """p ln(p / q) written out for one token, a gradient by autograd, and the loss of a student that agrees."""
    g = torch.Generator().manual_seed(5)
    z, tau = torch.randn(2, 6, generator=g, dtype=D), 1.5
    index, value = torch.tensor([[4, 1, -1], [0, 2, 5]], dtype=torch.int32), torch.randn(2, 3, generator=g)
    w = torch.tensor([0.5, 2.0])
    (loss, lse, dz), _ = O.distill(z, index, value, w, tau)
    e = [math.exp(value[0, k].item() / tau) for k in range(2)]
    q = [math.exp(v / tau) for v in z[0].tolist()]
    want = sum(e[k] / sum(e) * math.log(e[k] / sum(e) / (q[i] / sum(q))) for k, i in ((0, 4), (1, 1)))
    assert abs(loss[0].item() - 0.5 * tau ** 2 * want) < 1e-12 and abs(lse[0].item() - math.log(sum(q))) < 1e-12
    zz = z.clone().requires_grad_(True)
    grad, = torch.autograd.grad(O.distill(zz, index, value, w, tau)[0][0].sum(), zz)
    assert (grad - dz).abs().max() < 1e-12
    agree = torch.full((1, 6), -math.inf, dtype=D)
    agree[0, index[1].long()] = value[1].to(D)
    assert abs(O.distill(agree, index[1:], value[1:], w[1:], 1.0)[0][0].item()) < 1e-12


def test_reference_of_the_norm_gradient():
    g = torch.Generator().manual_seed(6)
    h, dy, gain = torch.randn(5, 16, generator=g), torch.randn(5, 16, generator=g), torch.randn(16, generator=g)
    leaves = [t.to(D).requires_grad_(True) for t in (h, gain, torch.zeros(16))]
    y = O.layer_norm(*leaves)[3]
    want = torch.autograd.grad((y * dy).sum(), leaves)
    _, m, r, _ = O.layer_norm(h, gain, None)
    got, _ = O.layer_norm_backward(dy, h, gain, m[:, 0], r[:, 0])
    for a, b in zip(got, want):
        assert (a - b).abs().max() < 1e-12


def test_shared_arrays_that_are_read_in_vectors_are_aligned():
    """An array in shared memory promises its element's alignment and no more: one that is accessed 8 or 16 bytes at a time says so."""
    wide = {"uint4": 16, "int4": 16, "float4": 16, "uint2": 8, "int2": 8, "float2": 8}
    own = {"float4": 16, "uint4": 16, "float2": 8, "uint2": 8, "unsigned long long": 8, "double": 8}
    csrc, seen = os.path.join(ROOT, "paper_1801_04928_b200", "csrc"), 0
    for name in sorted(os.listdir(csrc)):
        text = open(os.path.join(csrc, name)).read()
        # a name may be declared in several kernels: the least promise of a file counts
        promised = {}
        for align, kind, array in re.findall(r"__shared__\s+(?:__align__\((\d+)\)\s+)?((?:unsigned long long|unsigned char|\w+))\s+(\w+)\[", text):
            has = max(int(align or 1), own.get(kind, 4 if kind in ("float", "int", "unsigned") else 1))
            promised[array] = min(has, promised.get(array, 1024))
        for kind, array in re.findall(r"reinterpret_cast<(?:const\s+)?(\w+)\s*\*>\(\s*&?(\w+)", text):
            if kind in wide and array in promised:
                seen += 1
                assert promised[array] >= wide[kind], f"{name}: {array} promises {promised[array]} bytes and is accessed as {kind}"
    assert seen >= 5


class _Recorder:
    """Stands in for the operators: keeps the tensors that each call is given."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*a, **k):
            self.calls.append((name, [t for t in (*a, *k.values()) if isinstance(t, torch.Tensor)]))
        return call


def _steps(layer, tokens, width, vocab, sizes, backward=True):
    z, x = torch.zeros(tokens, vocab), torch.zeros(tokens, width)
    index, value, loss = torch.zeros(tokens, 2, dtype=torch.int32), torch.zeros(tokens, 2), torch.zeros(tokens)
    for m in sizes:
        layer.forward(x[:m], x[:m], z[:m], keep=backward)
        if backward:
            layer.backward(z[:m], index[:m], value[:m], loss[:m], x[:m])


def test_output_layer_keeps_buffers_for_its_tokens_once(monkeypatch):
    from paper_1801_04928_b200.output_layer import OutputLayer
    made, empty = [], torch.empty

    def counted(*a, **k):
        made.append(empty(*a, **k))
        return made[-1]
    monkeypatch.setattr(torch, "empty", counted)

    def bytes_for(sizes, backward=True):
        made.clear()
        ops = _Recorder()
        _steps(OutputLayer(ops, 40, 72, 264, device="cpu"), 40, 72, 264, sizes, backward)
        return sum(t.untyped_storage().nbytes() for t in made), ops
    most, _ = bytes_for([40])
    for sizes in (range(40, 0, -1), [*range(1, 41), *range(1, 41)]):
        got, ops = bytes_for(sizes)
        assert got == most, (got, most)
    # every view is what the operators take: scales contiguous, rows of bytes 16 bytes apart or a multiple, from a 16-byte boundary
    for name, ts in ops.calls:
        for t in ts:
            if t.dtype == torch.uint8:
                assert t.stride(1) == 1 and t.stride(0) % 16 == 0 and t.data_ptr() % 16 == 0, name
            elif t.dim() == 2 and t.dtype == torch.float32:
                assert t.is_contiguous(), name
    # tokens without a backward pass have no use for the gradient's forms: z's in 8 bits, both ways, and u's turned
    gradient = (40 * 272 + 264 * 48 + 72 * 48) + 4 * (3 * 40 + 264 + 72)
    assert bytes_for([1, 40], backward=False)[0] == most - gradient
    layer = OutputLayer(_Recorder(), 40, 72, 264, device="cpu")
    with pytest.raises(ValueError):
        layer.forward(torch.zeros(41, 72), torch.zeros(41, 72), torch.zeros(41, 264), keep=False)
