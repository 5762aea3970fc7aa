// Host-side print of the CTAs that an attention call over the 8-bit cache launches (runtime faked): built once per kernel,
// with SOURCE the file and CALL its launcher.  Reads "B H H_kv D keys n tree f32 max_ctas" lines, prints the CTAs of the
// attention kernel, 0 where the launcher leaves the call to another.
#include "fake_cudart.cuh"

#include SOURCE

int main() {
  alignas(16) static unsigned char buffer[64];
  int B, H, Hkv, D, keys, n, tree, f32, most;
  while (std::scanf("%d %d %d %d %d %d %d %d %d", &B, &H, &Hkv, &D, &keys, &n, &tree, &f32, &most) == 9) {
    glide::Kv8AttnArgs a{};
    a.q = a.kt = a.vt = buffer;
    a.K = a.V = buffer;
    a.Ke = a.Ve = reinterpret_cast<const int8_t*>(buffer);
    a.kv_len = reinterpret_cast<const int*>(buffer);
    a.parent = tree ? a.kv_len : nullptr;
    a.out = a.ws = buffer;
    a.B = B;
    a.H = H;
    a.Hkv = Hkv;
    a.D = D;
    a.S_cap = a.max_kv_len = keys;
    a.nq = n;
    a.dtype = f32;
    a.scale = 0.1f;
    a.max_ctas = most;
    fake::launches.clear();
    const cudaError_t e = glide::CALL(a, nullptr);
    if (e != cudaSuccess && e != cudaErrorNotSupported) return 1;
    std::printf("%u\n", fake::launches.empty() ? 0u : fake::launches[0].grid);
  }
  return 0;
}
