#include <ATen/ATen.h>
#include <stdexcept>
#include <iostream>
using at::Tensor;
[[noreturn]] void value_error(const std::string& w) { throw std::runtime_error(w); }
struct Rows { int64_t rows, cols, ld; };
Rows rows_of(const Tensor& t, const char* name) {
  const auto size = t.sizes();
  const auto stride = t.strides();
  const int64_t n = t.dim();
  if (n == 0) value_error(std::string(name) + " needs at least one dimension");
  Rows r{1, size[n - 1], size[n - 1]};
  for (int64_t i = 0; i < n - 1; ++i) r.rows *= size[i];
  if (r.rows == 0 || r.cols == 0) return r;
  if (r.cols > 1 && stride[n - 1] != 1) value_error(std::string(name) + ": the elements of a row must be contiguous");
  int64_t span = 0;  // what one step of the dimension to the left has to be
  bool known = false;  // whether a dimension has given the row distance (0 too: an expanded one repeats its rows, and is refused)
  for (int64_t i = n - 2; i >= 0; --i) {
    if (size[i] == 1) continue;
    if (!known) r.ld = stride[i];
    else if (stride[i] != span) value_error(std::string(name) + ": no single distance leads from row to row (make it contiguous)");
    known = true;
    span = stride[i] * size[i];
  }
  if (r.ld < r.cols) value_error(std::string(name) + ": rows overlap");
  return r;
}
int main() {
  struct { std::vector<int64_t> size, stride; } cases[] = {{{4,512,768},{768,0,1}}, {{4,512,768},{0,768,1}}, {{4,512,768},{0,0,1}}, {{4,3,8},{24,8,1}}, {{4,1,8},{8,0,1}},
    {{1,4,8},{0,8,1}}, {{4,8},{0,1}}, {{4,3,8},{32,8,1}}, {{4,3,2,8},{0,16,8,1}}, {{4,3,2,8},{48,0,8,1}}, {{4,3,2,8},{48,16,0,1}}, {{4,1},{0,1}}, {{2,3,1},{3,1,1}}, {{5,4,1},{0,1,1}}};
  for (auto& c : cases) {
    Tensor t = at::empty_strided(c.size, c.stride);
    int64_t have = t.storage().nbytes() / 4;
    try { Rows r = rows_of(t, "t"); int64_t last = (r.rows - 1) * r.ld + r.cols;
      std::cout << t.sizes() << t.strides() << " rows " << r.rows << " ld " << r.ld << " reads up to " << last << " of " << have << (last > have ? "  OUT OF STORAGE" : "") << (( r.rows-1)*r.ld+r.cols < t.numel() ? " WRONG" : "") << "\n";
    } catch (std::exception& e) { std::cout << t.sizes() << t.strides() << " refused: " << e.what() << "\n"; }
  }
}
