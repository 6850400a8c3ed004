// Reads calls from stdin, one a line: "NAME arguments...", pointers as numbers.  Prints a
// line for each: the code, how many launches it made, and the message (none: "-").
#include <cstdint>
#include <cstdlib>
#include <iostream>
#include <functional>
#include <map>
#include <sstream>
#include <string>
#include <tuple>
#include <type_traits>

#include "sa.h"

extern int sa_stub_page_launches;

template <class T>
T read_arg(std::istream& in) {
  std::string s;
  in >> s;
  if constexpr (std::is_pointer_v<T>)
    return reinterpret_cast<T>(static_cast<uintptr_t>(std::strtoull(s.c_str(), nullptr, 0)));
  else if constexpr (std::is_floating_point_v<T>)
    return static_cast<T>(std::strtod(s.c_str(), nullptr));
  else if constexpr (std::is_unsigned_v<T>)
    return static_cast<T>(std::strtoull(s.c_str(), nullptr, 0));
  else
    return static_cast<T>(std::strtoll(s.c_str(), nullptr, 0));
}

template <class R, class... A>
std::function<unsigned long long(std::istream&)> call(R (*f)(A...)) {
  return [f](std::istream& in) {
    std::tuple<A...> args{read_arg<A>(in)...};  // braces: read in order
    return static_cast<unsigned long long>(std::apply(f, args));
  };
}

int main() {
  const std::map<std::string, std::function<unsigned long long(std::istream&)>> calls = {
      {"sa_pages_reserve", call(sa_pages_reserve)},
      {"sa_pages_write", call(sa_pages_write)},
      {"sa_pages_fork", call(sa_pages_fork)},
      {"sa_pages_free", call(sa_pages_free)},
      {"sa_pages_compact", call(sa_pages_compact)},
      {"sa_pages_copy", call(sa_pages_copy)},
      {"sa_prefix_attention", call(sa_prefix_attention)},
      {"sa_prefix_attention_workspace", call(sa_prefix_attention_workspace)}};
  std::string line;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    std::string name;
    in >> name;
    sa_stub_page_launches = 0;
    const unsigned long long r = calls.at(name)(in);
    const char* text = sa_last_error();
    std::cout << r << " " << sa_stub_page_launches << " " << (*text ? text : "-") << std::endl;
  }
  return 0;
}
