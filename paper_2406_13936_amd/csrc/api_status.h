// How entry points outside abs_api.hip report: the thread's last error (abs_last_error(NULL)) and the status of a caught exception.
#pragma once
#include <string>
#include "../../include/abs.h"

namespace absk {

abs_status set_error(abs_status st, const std::string &msg);
abs_status exception_status() noexcept;      // inside a catch block

}  // namespace absk
