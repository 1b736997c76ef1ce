"""A paged layer is refused while another device is current than the one its pages are on (a kernel there could not read them)."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import torch, warnings
warnings.simplefilter("ignore")
from paper_2605_12825_b200 import build
if {fallback}:
    build.native_path = lambda: "/nonexistent"
from paper_2605_12825_b200 import binding as b
assert b._native.__name__.endswith("._marshal" if {fallback} else "._native")
z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
i = lambda *s: z(*s, dt=torch.int32)
pages, q, kv, slots = z(4, 2, 16, 64), z(1, 1, 4, 64), z(1, 1, 2, 64), z(1, 1, dt=torch.int64)
layer = b.make_paged_layer(pages, pages.clone(), i(1, 4), i(1), 4, 1)
ws = b.new_workspace(b.orthrus_paged_attend_workspace_bytes(layer))
calls = [lambda: b.orthrus_paged_ar_attend(layer, q, torch.empty_like(q), ws), lambda: b.orthrus_paged_diffusion_attend(layer, q, torch.empty_like(q), ws),
         lambda: b.orthrus_paged_kv_write(layer, slots, kv, kv), lambda: b.orthrus_rope_paged_kv_write(layer, slots, q, kv, kv, 1e4, torch.empty_like(q)),
         lambda: b.orthrus_paged_commit_len(layer, i(1))]
assert layer.device == torch.cuda.current_device()
for call in calls:
    call()
layer.device += 1                       # as if the device had been changed after the layer was made
n0 = b.orthrus_launch_count()
for call in calls:
    try:
        call()
    except ValueError as e:
        assert "current device" in str(e), e
    else:
        raise SystemExit("not refused")
assert b.orthrus_launch_count() == n0
layer.device = None                     # a descriptor that was filled by hand
for call in calls:
    call()
assert b.orthrus_read_status(ws) == 0
print("refused")
"""


@pytest.mark.parametrize("fallback", [False, True])
def test_a_layer_of_another_device_is_refused(fallback):
    r = subprocess.run([sys.executable, "-c", CODE.format(fallback=fallback)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "refused" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
