"""The operators' C structs, and refusals that need no GPU: nothing of a bad call reaches one."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2512_21835_amd as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layout_matches_the_header(tmp_path):
    structs = [("stage_batch", P.StageBatch), ("stage_cache", P.StageCache), ("stage_append_args", P.StageAppendArgs),
               ("stage_window_args", P.StageWindowArgs), ("stage_adapter_args", P.StageAdapterArgs)]
    lines, want = ['#include <stdio.h>', '#include <stddef.h>', '#include "stage_ops.h"', 'int main(void) {'], []
    for cname, py in structs:
        lines.append(f'printf("%zu\\n", sizeof({cname}));')
        want.append(ctypes.sizeof(py))
        for f in py._fields_:
            lines.append(f'printf("%zu\\n", offsetof({cname}, {f[0]}));')
            want.append(getattr(py, f[0]).offset)
    (tmp_path / "l.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")])
    assert [int(x) for x in subprocess.check_output([str(tmp_path / "l")]).decode().split()] == want


@pytest.mark.parametrize("name", ["stage_norm_rope_append", "stage_window_attention", "stage_adapter_add",
                                  "stage_window_workspace", "stage_adapter_workspace"])
def test_null_and_empty_arguments_are_refused(name):
    L = P.lib()
    more = {"stage_norm_rope_append": (None,), "stage_window_workspace": (ctypes.byref(ctypes.c_int64()),),
            "stage_adapter_workspace": (ctypes.byref(ctypes.c_int64()),)}.get(name, (None, 0, None))
    assert getattr(L, name)(None, *more) == P.STAGE_EINVAL
    kind = {"stage_norm_rope_append": P.StageAppendArgs, "stage_adapter_add": P.StageAdapterArgs,
            "stage_adapter_workspace": P.StageAdapterArgs}.get(name, P.StageWindowArgs)
    assert getattr(L, name)(ctypes.byref(kind()), *more) == P.STAGE_EINVAL


def test_tensors_of_the_host_are_refused():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        P.stage_adapter_add(x, x, x, torch.zeros(1, 4, 8).bfloat16(), torch.zeros(1, 8, 4).bfloat16(), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        P.stage_batch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32), 1, 1)


def test_packed_arguments_are_the_structs():
    """Each field of a packed call is where the structure has it."""
    from paper_2512_21835_amd import ops
    assert ops._BATCH.size == ctypes.sizeof(P.StageBatch)
    batch = P.StageBatch.from_buffer_copy(ops._BATCH.pack(*range(1, 8)))
    assert [getattr(batch, n) for n, _ in P.StageBatch._fields_] == list(range(1, 8))
    for packed, kind in ((ops._APPEND, P.StageAppendArgs), (ops._WINDOW, P.StageWindowArgs), (ops._ADAPTER, P.StageAdapterArgs)):
        assert packed.size == ctypes.sizeof(kind)
        values = list(range(11, 11 + 40))
        args = kind.from_buffer_copy(packed.pack(*[bytes(batch) if packed is not ops._ADAPTER and i == 1 else values[i]
                                                   for i in range(len(packed.unpack(bytes(packed.size))))]))
        flat = []
        for n, _ in kind._fields_:
            v = getattr(args, n)
            if isinstance(v, ctypes.Array):
                flat += list(v)
            elif isinstance(v, P.StageCache):
                flat += [getattr(v, m) for m, _ in P.StageCache._fields_]
            elif isinstance(v, P.StageBatch):
                assert bytes(v) == bytes(batch)
                flat.append(values[len(flat)])
            else:
                flat.append(v)
        assert flat == values[:len(flat)]
