"""The library reads no environment variable: a program may set some while another of its threads calls it."""
import subprocess

import paper_2605_05888_amd as hub


def test_the_library_does_not_read_the_environment():
    hub.load_library()
    r = subprocess.run(["nm", "-D", "--undefined-only", hub.lib_path()], capture_output=True, text=True, check=True)
    names = {line.split()[-1].split("@")[0] for line in r.stdout.splitlines() if line.strip()}
    assert "hipLaunchKernel" in names  # (the list is the library's)
    assert not names & {"getenv", "secure_getenv", "environ", "setenv", "putenv"}
