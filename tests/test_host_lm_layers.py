"""The structs of the embedding and of the state space layer's operators as the C compiler lays them out, and what is refused without a GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = ["rgc_embedding", "rgc_convolution", "rgc_convolution_grads", "rgc_scan", "rgc_scan_grads"]
CONSTANTS = ["RGC_TAPS_MAX", "RGC_SCAN_CHUNK", "RGC_SCAN_STATES_MAX"]


def test_structs_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    from paper_1808_04357_amd import binding
    lines = []
    for name in STRUCTS:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in getattr(binding, name)._fields_]
    lines += ['printf("%s %%d\\n", %s);' % (c, c) for c in CONSTANTS]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "%s"\nint main(void) {\n%s\nreturn 0;\n}\n' % (os.path.join(ROOT, "include", "rgc.h"), "\n".join(lines)))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-o", str(tmp_path / "layout"), str(src)], check=True)
    told = dict(l.split() for l in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.splitlines())
    for name in STRUCTS:
        struct = getattr(binding, name)
        assert ctypes.sizeof(struct) == int(told[name])
        for f, _ in struct._fields_:
            assert getattr(struct, f).offset == int(told["%s.%s" % (name, f)]), (name, f)
    for c in CONSTANTS:
        assert getattr(binding, c) == int(told[c])


def test_no_context_is_refused_before_any_gpu_call():
    from paper_1808_04357_amd import binding, build
    if not os.path.exists(binding.library_path()):
        build.build(force=True)
    lib = binding.load_library()
    new = {name: ctypes.byref(getattr(binding, name)()) for name in STRUCTS}
    assert lib.rgc_embed_tokens(None, new["rgc_embedding"], None) == -1
    assert lib.rgc_embed_tokens_backward(None, new["rgc_embedding"], None, 0, None, 0x10, None) == -1
    assert lib.rgc_causal_convolution(None, new["rgc_convolution"], None) == -1
    assert lib.rgc_causal_convolution_backward(None, new["rgc_convolution"], new["rgc_convolution_grads"], None) == -1
    assert lib.rgc_selective_scan(None, new["rgc_scan"], None) == -1
    assert lib.rgc_selective_scan_backward(None, new["rgc_scan"], new["rgc_scan_grads"], None) == -1


def test_descriptors_check_shapes_types_and_strides_on_the_host():
    import torch
    import paper_1808_04357_amd as rgc
    z, t = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32)
    assert rgc.Embedding(z, t, torch.zeros(4, 10).half()).desc.out_stride == 10
    assert rgc.Embedding(torch.zeros(7, 16)[:, :10], t, z).desc.table_stride == 16
    s = torch.zeros(2, 6, 8)
    c = rgc.Convolution(s, torch.zeros(8, 3), torch.zeros(6, 2, 8).transpose(0, 1), silu=True, before=torch.zeros(2, 2, 8))
    assert (c.desc.y.batch_stride, c.desc.y.step_stride, c.desc.taps, c.desc.silu) == (8, 16, 3, 1)
    n = rgc.Scan(s, s, torch.zeros(8, 5), torch.zeros(2, 6, 10), torch.zeros(2, 6, 10), s, groups=2, softplus=True, states=torch.zeros(2, 1, 8, 5))
    assert (n.desc.states, n.desc.groups, n.desc.softplus) == (5, 2, 1)
    for make in (lambda: rgc.Embedding(z.t(), t, z), lambda: rgc.Embedding(z, t.long(), z), lambda: rgc.Embedding(z, t, z[:, :9]), lambda: rgc.Embedding(z, t[:3], z), lambda: rgc.Convolution(s, z, s),
                 lambda: rgc.Convolution(s, torch.zeros(8, 3).half(), s), lambda: rgc.Convolution(s, torch.zeros(8, 3), s, before=torch.zeros(2, 3, 8)), lambda: rgc.Convolution(s[0], torch.zeros(8, 3), s[0]),
                 lambda: rgc.Scan(s, s, torch.zeros(8, 5), torch.zeros(2, 6, 5), torch.zeros(2, 6, 4), s), lambda: rgc.Scan(s, s, torch.zeros(8, 5), torch.zeros(2, 6, 10), torch.zeros(2, 6, 10), s, groups=3),
                 lambda: rgc.Scan(s, s.half(), torch.zeros(8, 5), torch.zeros(2, 6, 5), torch.zeros(2, 6, 5), s), lambda: rgc.ScanGrads(n, s, s, s, torch.zeros(8, 5), torch.zeros(2, 6, 10), torch.zeros(2, 6, 9)),
                 lambda: rgc.ScanGrads(n, s, s, s, torch.zeros(8, 5), torch.zeros(2, 6, 10), torch.zeros(2, 6, 10), dgate=s)):
        with pytest.raises(rgc.RgcError) as e:
            make()
        assert e.value.status == -1
