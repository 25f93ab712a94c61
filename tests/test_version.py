"""The library says which header its argument structs are of.  They have no size field, so a struct that changes without the major number would be
read beyond what an older program passes."""
import ctypes as C
import os
import shutil
import subprocess

from paper_2502_02789_amd import binding as sp
from tests.test_cache_args import ROOT

# bytes of the structs of major version 3
SIZES = dict(sp_score_args=184, sp_pool_select_args=96, sp_gather_args=96, sp_cache_append_args=256, sp_cache_read_args=208, sp_attend_args=272,
             sp_verify_args=152)


def test_major_version_and_the_structs_it_stands_for(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc") or "/opt/rocm/llvm/bin/clang"
    lines = ["printf(\"%s %%zu\\n\", sizeof(%s));" % (n, n) for n in SIZES]
    (tmp_path / "sizes.c").write_text("#include <stdio.h>\n#include \"specprefill.h\"\nint main(void) { %s printf(\"version %%d\\n\", SP_VERSION); return 0; }\n" % " ".join(lines))
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), "sizes.c", "-o", "sizes"], cwd=tmp_path, check=True)
    got = dict(line.split() for line in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.splitlines())
    version = int(got.pop("version"))
    assert sp.sp_version() == version and version // 10000 == 3
    assert {k: int(v) for k, v in got.items()} == SIZES
    for cls, name in ((sp.ScoreArgs, "sp_score_args"), (sp.PoolSelectArgs, "sp_pool_select_args"), (sp.GatherArgs, "sp_gather_args"),
                      (sp.CacheAppendArgs, "sp_cache_append_args"), (sp.CacheReadArgs, "sp_cache_read_args"), (sp.AttendArgs, "sp_attend_args"),
                      (sp.VerifyArgs, "sp_verify_args")):
        assert C.sizeof(cls) == SIZES[name]
