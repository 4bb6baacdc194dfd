/* Beside host_cudart.c, and before it: a count of clusters that can be made to fail, which leaves an error with the
 * runtime as a real one does, and the address of a device symbol. */
static int g_fail, g_none, g_last;
static int g_word;

void host_clusters_set(int fail, int none) { g_fail = fail, g_none = none; }
int cudaOccupancyMaxActiveClusters(int* n, const void* f, const void* cfg) {
  (void)f, (void)cfg;
  *n = g_fail ? -7 : g_none ? 0 : 76;
  if (g_fail) g_last = 1;
  return g_last;
}
int cudaGetLastError(void) {
  const int e = g_last;
  g_last = 0;
  return e;
}
int cudaGetSymbolAddress(void** p, const void* symbol) {
  (void)symbol;
  *p = &g_word;
  return 0;
}
