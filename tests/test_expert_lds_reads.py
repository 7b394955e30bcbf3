"""The gradient of the experts' weights, as test_lds_reads.py has it for the products: its K loops, too, read fragments by inline assembly and wait for
them by count."""
import subprocess

from test_lds_reads import kernels, reads_in_flight
from test_store_instructions import gfx950_code_objects, objdump


def test_no_register_is_used_with_an_lds_read_into_it_under_way(tmp_path):
    seen = {"expert_gradient_kernel": 0, "expert_gradient_thin_kernel": 0}
    for i, code_object in enumerate(gfx950_code_objects()):
        if not any(name.encode() in code_object for name in seen):
            continue
        path = tmp_path / ("%d.co" % i)
        path.write_bytes(code_object)
        p = subprocess.run([objdump(), "-d", "--mcpu=gfx950", str(path)], stdout=subprocess.PIPE, text=True, check=True)
        for name, code in kernels(p.stdout.splitlines()).items():
            kind = [k for k in seen if k in name]
            if kind:
                bad, reads = reads_in_flight(code)
                assert not bad, (name, bad[:5])
                assert reads > 4, name
                seen[kind[0]] += 1
    assert min(seen.values()) >= 1, seen
