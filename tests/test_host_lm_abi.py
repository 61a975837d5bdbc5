"""The language-model operators' structs as the C compiler lays them out, and refusals that need no GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = ["rgc_token_scores", "rgc_distill", "rgc_sequence", "rgc_recurrence", "rgc_recurrence_grads"]


def test_structs_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    from paper_1808_04357_amd import binding
    lines = []
    for name in STRUCTS:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in getattr(binding, name)._fields_]
    lines += ['printf("%s %%d\\n", %s);' % (c, c) for c in ("RGC_F32", "RGC_BF16", "RGC_F16", "RGC_TOP_MAX", "RGC_RECURRENCE_CHUNK")]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "%s"\nint main(void) {\n%s\nreturn 0;\n}\n'
                   % (os.path.join(ROOT, "include", "rgc.h"), "\n".join(lines)))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-o", str(tmp_path / "layout"), str(src)], check=True)
    told = dict(l.split() for l in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.splitlines())
    for name in STRUCTS:
        struct = getattr(binding, name)
        assert ctypes.sizeof(struct) == int(told[name])
        for f, _ in struct._fields_:
            assert getattr(struct, f).offset == int(told["%s.%s" % (name, f)]), (name, f)
    for c in ("RGC_F32", "RGC_BF16", "RGC_F16", "RGC_TOP_MAX", "RGC_RECURRENCE_CHUNK"):
        assert getattr(binding, c) == int(told[c])


def test_no_context_is_refused_before_any_gpu_call():
    from paper_1808_04357_amd import binding, build
    if not os.path.exists(binding.library_path()):
        build.build(force=True)
    lib = binding.load_library()
    assert lib.rgc_token_logprobs(None, ctypes.byref(binding.rgc_token_scores()), None) == -1
    assert lib.rgc_token_logprobs_backward(None, ctypes.byref(binding.rgc_token_scores()), None, None, None, 0, None) == -1
    assert lib.rgc_distill_loss(None, ctypes.byref(binding.rgc_distill()), None) == -1
    assert lib.rgc_gated_recurrence(None, ctypes.byref(binding.rgc_recurrence()), None) == -1
    assert lib.rgc_gated_recurrence_backward(None, ctypes.byref(binding.rgc_recurrence()), ctypes.byref(binding.rgc_recurrence_grads()), None) == -1


def test_descriptors_check_shapes_types_and_strides_on_the_host():
    import torch
    import paper_1808_04357_amd as rgc
    z, t = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32)
    assert rgc.TokenScores(z, t, logprob=torch.zeros(4)).desc.row_stride == 10
    assert rgc.TokenScores(torch.zeros(4, 16)[:, :10]).desc.row_stride == 16
    assert rgc.Recurrence(z[None], z[None], z[None]).desc.x.step_stride == 10
    for make in (lambda: rgc.TokenScores(z.t()), lambda: rgc.TokenScores(z, t.long()), lambda: rgc.TokenScores(z.int()),
                 lambda: rgc.Distillation(z, t, t), lambda: rgc.Recurrence(z, z, z), lambda: rgc.Recurrence(z[None], z[None].half(), z[None])):
        with pytest.raises(rgc.RgcError) as e:
            make()
        assert e.value.status == -1
