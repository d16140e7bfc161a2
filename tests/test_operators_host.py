"""The layer operators' boundary without a GPU: the binding's argument structs are the header's, NULL handles and
arguments answer with an error code, and the 64-bit reference of the 8-bit form has the properties it is defined by."""
import ctypes
import os
import re
import subprocess
import sys
import textwrap

import pytest
import torch

import operators_ref as R
import paper_1801_04928_b200 as lf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = ("lf_linear_args", "lf_linear_grad_x_args", "lf_linear_grad_w_args", "lf_rms_norm_args", "lf_rms_norm_backward_args", "lf_ops_stats")


def test_binding_structs_are_the_headers(tmp_path):
    lines = []
    for name in STRUCTS:
        cls = getattr(lf, name)
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "offsets.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "leapfrog.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    exe = tmp_path / "offsets"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    said = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for name in STRUCTS:
        cls = getattr(lf, name)
        assert int(said[name]) == ctypes.sizeof(cls), name
        for f, _ in cls._fields_:
            assert int(said[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)


def test_constants_are_the_headers():
    text = open(os.path.join(ROOT, "include", "leapfrog.h")).read()
    for name in ("LF_F32", "LF_BF16", "LF_F16", "LF_ACT_NONE", "LF_ACT_SILU", "LF_ACT_GELU", "LF_FORM_STREAM", "LF_FORM_SPLIT", "LF_FORM_PAIRS"):
        assert int(re.search(rf"\b{name} = (\d+)", text).group(1)) == getattr(lf, name), name


def test_null_handles_and_arguments():
    for name in ("lf_linear", "lf_linear_grad_x", "lf_linear_grad_w", "lf_rms_norm", "lf_rms_norm_backward"):
        args = getattr(lf, name + "_args")()
        assert getattr(lf, name)(None, args) == lf.LF_ENULL, name
    assert lf.lf_pack8(None, 0, 1, 8, 16, 0, 16, 16) == lf.LF_ENULL
    assert lf.lf_unpack8(None, 0, 3, 1, 8, 16, 16, 16, 0) == lf.LF_ENULL
    assert lf.lf_act_backward(None, 0, 3, 1, 8, 16, 0, 16, 16, 16, 0) == lf.LF_ENULL
    for f in (lf.lf_ops_sync, lf.lf_ops_destroy):
        assert f(None) == lf.LF_ENULL
    assert lf.lf_ops_set_stream(None, None) == lf.LF_ENULL
    assert lf.lf_ops_set_option(None, lf.LF_OPT_WITHHOLD, 1) == lf.LF_ENULL
    assert lf.lf_ops_last_cuda_error(None) == 0


def test_workspace_and_create():
    fixed = lf.lf_ops_workspace(0, 0)
    assert fixed > 0 and lf.lf_ops_workspace(-1, 8) == lf.LF_EINVAL
    assert lf.lf_ops_workspace(8192, 16384) == fixed + 8192 * 16384 * 2
    assert lf.lf_ops_workspace(3, 8) >= fixed + 48
    rc, h = lf.lf_ops_create(fixed - 1)
    assert rc == lf.LF_EINVAL and not h.value
    if not torch.cuda.is_available():
        rc, h = lf.lf_ops_create(fixed)
        assert rc == lf.LF_ECUDA and not h.value
        with pytest.raises(lf.LeapfrogError):
            lf.Operators()


def test_layer_activations_are_no_network_option():
    # LF_ACT_NONE, SILU and GELU belong to the layer operators; a network context is not offered them
    assert {lf.LF_ACT_SIGMOID, lf.LF_ACT_TANH, lf.LF_ACT_RELU} == {0, 1, 2}
    assert {lf.LF_ACT_NONE, lf.LF_ACT_SILU, lf.LF_ACT_GELU} == {3, 4, 5}


def test_reference_of_the_eight_bit_form():
    g = torch.Generator().manual_seed(3)
    v = torch.randn(40, 72, generator=g, dtype=R.D) * torch.exp2(torch.randint(-130, 110, (40, 1), generator=g).to(R.D))
    v[3] = 0
    q, s = R.pack8(v.float())
    v = v.float().to(R.D)
    e = R.columns(s, 72).to(R.D) - 127
    back = R.unpack8(q, s)
    assert bool((v.abs() <= 448 * torch.exp2(e)).all())
    assert bool(((back - v).abs() <= 2.0 ** -4 * v.abs() + 2.0 ** -10 * torch.exp2(e)).all())
    assert bool((s[3] == 0).all()) and bool((back[3] == 0).all())
    # the scale is the smallest one: half of it would not hold the group's maximum
    pad = torch.zeros(40, 96, dtype=R.D)
    pad[:, :72] = v
    amax = pad.view(40, 3, 32).abs().amax(-1)
    assert bool(((amax > 224 * torch.exp2(s.to(R.D) - 127)) | (s == 0)).all())


@pytest.mark.parametrize("kind", [R.NONE, R.SILU, R.GELU, R.SIGMOID, R.TANH, R.RELU])
def test_reference_derivatives_by_differences_and_their_bounds(kind):
    z = torch.linspace(-12, 12, 4001, dtype=R.D) + 1e-3
    h = 1e-6
    d = R.act_prime(z, kind)
    fd = (R.act(z + h, kind) - R.act(z - h, kind)) / (2 * h)
    assert (d - fd).abs().max().item() < 1e-7
    assert d.abs().max().item() <= R.LIP1[kind]


def _without_gpu(code):
    """Run `code` in a process of its own, with `o` an Operators that has no handle: calls end at their checks of tensors."""
    head = """
        import torch, paper_1801_04928_b200 as lf
        from paper_1801_04928_b200 import _marshal
        o = object.__new__(lf.Operators)
        o._h, o._a, o._m, o._device = None, 0, _marshal, 0
        def refused(f, *a, **k):
            try:
                f(*a, **k)
            except lf.LeapfrogError as e:
                assert e.status == lf.LF_EINVAL, e
                return str(e)
            raise AssertionError("not refused")
    """
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(head) + textwrap.dedent(code)], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr[-3000:])


@pytest.mark.parametrize("make", ["m.to_sparse()", "m.to_sparse_csr()", "torch.nested.nested_tensor([m, m[:2]])",
                                  "torch.nested.nested_tensor([m, m[:2]], layout=torch.jagged)", "m.to(torch.float32).to_mkldnn()"])
def test_tensors_without_plain_memory_are_refused_and_do_not_end_the_process(make):
    _without_gpu(f"""
        import warnings
        warnings.simplefilter("ignore")
        m, byte = torch.ones(4, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.uint8)
        odd, gain = {make}, torch.ones(8)
        calls = [(o.linear, odd, m, m), (o.linear, m, odd, m), (o.linear, m, m, odd), (o.linear_grad_x, odd, m, m), (o.linear_grad_x, m, odd, m),
                 (o.linear_grad_w, odd, m), (o.linear_grad_w, m, odd), (o.rms_norm, odd, gain, m), (o.rms_norm_backward, m, odd, gain, m),
                 (o.pack8, odd, byte, byte), (o.unpack8, byte, byte, odd), (o.act_backward, odd, byte, byte, m)]
        for f, *a in calls:
            assert "argument" in refused(f, *a)
    """)


def test_activations_beyond_an_int_are_refused():
    _without_gpu("""
        m, byte = torch.ones(4, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.uint8)
        for act in (2 ** 32, 2 ** 32 + 3, -2 ** 32, 2 ** 31, -2 ** 31 - 1, 2 ** 64, -2 ** 80):
            for f, *a in ((o.linear, m, m, m), (o.linear_grad_x, m, m, m), (o.linear_grad_w, m, m), (o.unpack8, byte, byte, m), (o.act_backward, m, byte, byte, m)):
                assert "argument act: out of range" in refused(f, *a, act=act)
        try:
            o.linear(m, m, m, act="gelu")
        except TypeError:
            pass
        else:
            raise AssertionError("a text is no activation")
    """)


def test_the_library_is_built_without_torch(monkeypatch, tmp_path, capsys):
    import importlib.util
    from paper_1801_04928_b200 import build
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert not os.path.exists(build.MARSHAL) and "torch not found" in capsys.readouterr().err


def test_the_tensor_module_is_rebuilt_for_another_torch(monkeypatch, tmp_path):
    import importlib.util
    import types
    from paper_1801_04928_b200 import build
    home, runs = tmp_path / "torch", []
    home.mkdir()
    (home / "version.py").write_text("__version__ = '1'")

    def compiler(cmd, **kw):
        runs.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: types.SimpleNamespace(origin=str(home / "__init__.py")))
    monkeypatch.setattr(build, "OBJ", str(tmp_path))
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(build.subprocess, "run", compiler)
    build._build_marshal(False)
    build._build_marshal(False)
    assert len(runs) == 1
    (home / "version.py").write_text("__version__ = '2'")
    build._build_marshal(False)
    build._build_marshal(False)
    assert len(runs) == 2 and str(home / "lib") in runs[1]


def test_workspace_beyond_any_call_is_refused():
    assert lf.lf_ops_workspace(1 << 30, 1 << 24) == lf.lf_ops_workspace(0, 0) + (1 << 55)
    for tokens, n_in in (((1 << 30) + 1, 8), (8, (1 << 24) + 8), (1 << 40, 1 << 24), (1 << 62, 2), (1 << 32, 1 << 31), (8, -1)):
        assert lf.lf_ops_workspace(tokens, n_in) == lf.LF_EINVAL
