"""What the tests of the operators around the attention share."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# A handle's memory, all zero: the argument checks come first, then the look at the current device, which fails on a machine
# without one (HOOK_ATTN_ERR_CUDA).  Never passed where a device exists.
_handle_memory = ctypes.create_string_buffer(256)
FAKE_HANDLE = ctypes.addressof(_handle_memory)
no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="passes addresses that no device may see")


def struct_fields(name):
    """Field names of a struct of the header, in order."""
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hook_attn.h")).read(), flags=re.S)
    body = text[:text.index("} %s;" % name)]
    body = body[body.rindex("typedef struct {") + len("typedef struct {"):]
    fields = []
    for decl in body.split(";"):
        names = decl.split(",")
        if decl.strip():
            fields += [re.sub(r"\[.*", "", n.split()[-1].lstrip("*")) for n in names]
    return fields
