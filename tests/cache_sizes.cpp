// The attention's workspace size over the ends of its arguments' ranges, with
// csrc/cache.cpp compiled in: any overflow ends the program.
#include "../paper_2606_03113_amd/csrc/cache.cpp"

#include <climits>
#include <cstdio>

namespace lede {
hipError_t launch_cache_plan(const CachePlanArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_cache_append(int, const CacheRowsArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_cache_read(int, const CacheRowsArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_cache_attention(int, const CacheAttnArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_logprobs(int, const LogprobsArgs&, hipStream_t) { return hipSuccess; }
}  // namespace lede

int main() {
  const int heads[][2] = {{1, 1}, {64, 8}, {65536, 1}, {65536, 1024}, {1024, 1024}, {INT_MAX, INT_MAX}, {INT_MAX, 1}};
  size_t most = 0;
  for (int seqs : {1, 100, 8191, 65535, 65536, INT_MAX})
    for (const auto& h : heads)
      for (int rows : {0, 1, INT_MAX})
        for (int max_new : {0, 1, 40, 1000, INT_MAX})
          for (int max_kv : {0, 1, 100000, INT_MAX})
            for (int hd : {0, 64, 96, 128})
              for (int dtype : {0, 1}) {
                const size_t n = lede_op_cache_attention_bytes(dtype, seqs, rows, h[0], h[1], hd, max_new, max_kv);
                if (n && (hd % 64 || !hd || seqs > 65535 || h[0] > 65536 || h[1] > 1024)) return 1;
                most = n > most ? n : most;
              }
  std::printf("largest workspace %zu\n", most);
  return most < (1ull << 30) ? 0 : 2;
}
