"""Kernels with more than 64 KB of dynamic LDS are allowed it on every device that they are launched on, not only on a process's first one.
The calls of the HIP runtime that a launch makes are replaced by ones that keep a record (a small library, preloaded into a child
interpreter), so that this runs without a GPU and with as many devices as one likes."""
import os
import subprocess
import sys
import textwrap

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RECORDER = r"""
#include <stddef.h>
#include <stdint.h>
typedef struct { uint32_t x, y, z; } dim3_t;
static int device;
static dim3_t grid, block;
static size_t lds;
static void* stream;
struct entry { const void* kernel; int device; int64_t bytes; };
static struct entry allowed[4096], launched[4096];
static int n_allowed, n_launched;
void recorder_device(int d) { device = d; }
int recorder_entries(int which, struct entry* out) {
  int n = which ? n_launched : n_allowed;
  for (int i = 0; i < n; ++i) out[i] = (which ? launched : allowed)[i];
  return n;
}
int hipGetDevice(int* d) { *d = device; return 0; }
int hipFuncSetAttribute(const void* f, int attribute, int value) {
  (void)attribute;
  if (n_allowed < 4096) allowed[n_allowed++] = (struct entry){f, device, value};
  return 0;
}
int __hipPushCallConfiguration(dim3_t g, dim3_t b, size_t l, void* s) { grid = g; block = b; lds = l; stream = s; return 0; }
int __hipPopCallConfiguration(dim3_t* g, dim3_t* b, size_t* l, void** s) { *g = grid; *b = block; *l = lds; *s = stream; return 0; }
int hipLaunchKernel(const void* f, dim3_t g, dim3_t b, void** args, size_t l, void* s) {
  (void)g; (void)b; (void)args; (void)s;
  if (n_launched < 4096) launched[n_launched++] = (struct entry){f, device, (int64_t)l};
  return 0;
}
int hipGetLastError(void) { return 0; }
int hipMemcpyAsync(void* to, const void* from, size_t n, int kind, void* s) { (void)to; (void)from; (void)n; (void)kind; (void)s; return 0; }
int hipEventRecord(void* e, void* s) { (void)e; (void)s; return 0; }
"""

CHILD = textwrap.dedent("""
    import ctypes, os, sys
    sys.path.insert(0, %(root)r)
    from paper_2605_15250_amd import binding as B
    rec = ctypes.CDLL(%(recorder)r)
    class entry(ctypes.Structure):
        _fields_ = [("kernel", ctypes.c_void_p), ("device", ctypes.c_int), ("bytes", ctypes.c_int64)]
    def entries(which):
        e = (entry * 4096)()
        return [(x.kernel, x.device, x.bytes) for x in e[:rec.recorder_entries(which, e)]]
    A = 0x10000
    def shape(batch=2, h_q=32, g=8, d_h=128, d_v=0, s_q=1):
        return B.make_shape(batch, h_q, g, d_h, 512, 64, s_q, B.GQLA_BF16, 0.0, d_v)
    def cache(groups, max_pages=64, batch=2):
        return B.make_cache(A, A, None, 64, max_pages, max_pages * batch, groups)
    def decode(sh, lens, path, call, units=256, chunk=0):
        plan = B.gqla_plan_create(sh, lens, 64, units, path, chunk)
        n = B.gqla_plan_workspace_bytes(plan)
        B.lib().gqla_plan_upload(plan, A, n, None)
        call(plan, n)
        B.gqla_plan_destroy(plan)
    def run():
        for d_h, d_v in ((128, 0), (192, 256)):
            for h_q, g, s_q, lens, units, chunk in ((32, 8, 1, [1000, 70], 256, 0), (128, 4, 2, [300, 70], 256, 0), (16, 1, 2, [900, 65], 256, 0),
                                                     (32, 8, 1, [900, 640], 2, 4)):
                sh, c = shape(h_q=h_q, g=g, d_h=d_h, d_v=d_v, s_q=s_q), cache(g)
                decode(sh, lens, B.GQLA_PATH_GQA, lambda p, n: B.gqla_decode_gqa(sh, p, A, A, c, A, None, A, n, stream=0), units, chunk)
                decode(sh, lens, B.GQLA_PATH_GQA, lambda p, n: B.gqla_decode_gqa_fp8_blocks(sh, p, A, A, c, A, None, A, n, stream=0), units, chunk)
                if d_h == 128:
                    decode(sh, lens, B.GQLA_PATH_GQA, lambda p, n: B.gqla_decode_gqa_fp8(sh, p, A, A, c, 1.0, 1.0, A, None, A, n, stream=0), units, chunk)
            for h_q, batch in ((32, 2), (128, 2), (128, 256), (96, 256), (20, 40)):
                sh, c = shape(batch=batch, h_q=h_q, g=4, d_h=d_h, d_v=d_v), cache(0, batch=batch)
                lens = [4000] * batch
                decode(sh, lens, B.GQLA_PATH_ABSORB, lambda p, n: B.gqla_decode_absorb(sh, p, A, A, c, A, A, None, A, n, stream=0))
                decode(sh, lens, B.GQLA_PATH_ABSORB, lambda p, n: B.gqla_decode_absorb_fp8(sh, p, A, A, c, 1.0, A, A, None, A, n, stream=0))
                B.gqla_absorb_query(sh, A, A, A, stream=0)
                if h_q * (d_v or d_h) %% 256 == 0:
                    B.gqla_output_projection(sh, 4096, A, A, A, A, 1 << 40, stream=0)
            sh = shape(g=8, d_h=d_h, d_v=d_v)
            for total in (5, 4000):
                B.gqla_attend_gqa_fp8_blocks(sh, A, total, A, A, cache(8), A, None, A, 1 << 40, stream=0)
            B.gqla_expand_cache(sh, cache(0), A, A, 0, 8, cache(8), A, 1 << 40, stream=0)
            B.gqla_compress_cache(sh, cache(8), A, cache(0), stream=0)
    for device in (0, 1, 0, 70):
        rec.recorder_device(device)
        run()
    allowed = {}
    for kernel, device, size in entries(0):
        allowed[kernel, device] = max(size, allowed.get((kernel, device), 0))
    need = {(kernel, device, size) for kernel, device, size in entries(1) if size > 65536}
    assert len({k for k, _, _ in need}) >= 12 and {d for _, d, _ in need} == {0, 1, 70}, need
    missing = [x for x in need if allowed.get(x[:2], 0) < x[2]]
    assert not missing, "%%d of %%d launches with more LDS than their device allows: %%s" %% (len(missing), len(need), missing[:4])
    print("kernels:", len({k for k, _, _ in need}))
""")


def test_every_device_is_asked(tmp_path):
    from paper_2605_15250_amd import binding as B
    B.lib()
    source, recorder = tmp_path / "recorder.c", str(tmp_path / "librecorder.so")
    source.write_text(RECORDER)
    built = subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-o", recorder, str(source)], capture_output=True, text=True)
    assert built.returncode == 0, built.stderr
    env = dict(os.environ)
    env["LD_PRELOAD"] = recorder + ((":" + env["LD_PRELOAD"]) if env.get("LD_PRELOAD") else "")
    r = subprocess.run([sys.executable, "-c", CHILD % {"root": ROOT, "recorder": recorder}], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "kernels:" in r.stdout
