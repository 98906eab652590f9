"""No C++ exception leaves a C entry: an allocation that fails is a status."""
import os
import subprocess
import textwrap

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIBDIR = os.path.join(ROOT, "paper_2608_23834_amd", "_lib")


def test_rope_create_without_memory(tmp_path):
    """Every allocation of the table's size fails while kv_rope_create runs.  (The table's address is a
    placeholder: without a device the copy there is refused.)"""
    src = tmp_path / "t.cpp"
    src.write_text(textwrap.dedent("""\
        #include <cstdio>
        #include <cstdlib>
        #include <new>
        extern "C" {
        struct desc { int head_dim, rot_dim, n_axes, interleaved; double scale; const double* f; const unsigned char* axis;
                      void* table; size_t bytes; };
        int kv_rope_create(const desc*, void**);
        }
        static bool armed = false;
        void* operator new(size_t n) {
          if (armed && n == 128 * 16) throw std::bad_alloc();
          if (void* p = malloc(n)) return p;
          throw std::bad_alloc();
        }
        void operator delete(void* p) noexcept { free(p); }
        void operator delete(void* p, size_t) noexcept { free(p); }
        int main() {
          static double f[128];
          for (double& x : f) x = 1.0;
          desc d = {256, 256, 1, 0, 1.0, f, nullptr, (void*)(1 << 20), 128 * 16};
          void* r = nullptr;
          armed = true;
          const int st = kv_rope_create(&d, &r);
          armed = false;
          printf("status %d\\n", st);
          return st != 0 && r == nullptr ? 0 : 1;
        }
        """))
    exe = tmp_path / "t"
    subprocess.run(["g++", "-O1", "-rdynamic", str(src), "-o", str(exe), os.path.join(LIBDIR, "libminimakv.so"),
                    f"-Wl,-rpath,{LIBDIR}:/opt/rocm/lib", "-Wl,-rpath-link,/opt/rocm/lib"], check=True, timeout=60)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60, env={**os.environ, "HIP_VISIBLE_DEVICES": "-1"})
    assert r.returncode == 0 and "status" in r.stdout, (r.returncode, r.stdout, r.stderr)
